"""CPU checks of what the engine plans and refuses for paged caches and sampling filters."""
import pytest

from paper_2609_21704_amd.configs import CONFIGS
from paper_2609_21704_amd.engine import Engine, cache_bytes, placement


def test_pools_take_their_pages():
    cfg = CONFIGS[2]
    rows = placement(cfg, 1 << 40, 4, 1024, 4)["bytes"]["planned"]
    pool = placement(cfg, 1 << 40, 4, 1024, 4, pages=17)["bytes"]["planned"]
    # five caches: the direct decoder's, and a parent's and a draft's for each of the two drafts
    assert rows - pool == 5 * (cache_bytes(cfg, cfg.layers, 4, 1024) - cache_bytes(cfg, cfg.layers, 1, 17 * 64))
    less = placement(cfg, 1 << 40, 4, 1024, 4, pages=17, draft_cache="q4")["bytes"]["planned"]
    assert pool - less == 2 * (cache_bytes(cfg, cfg.layers, 1, 17 * 64) - cache_bytes(cfg, cfg.layers, 1, 17 * 64, "q4"))


@pytest.mark.parametrize("bad,match", [(dict(pages=0), "paged caches"), (dict(pages=4, chains=2), "paged caches"),
                                       (dict(pages=4, capacity=100), "paged caches"), (dict(top_p=-0.1), "top_p"),
                                       (dict(min_p=float("nan")), "min_p"), (dict(top_k=1.5), "top_k")])
def test_refusals(bad, match):
    """Before anything is sized, built or asked of a device."""
    with pytest.raises(ValueError, match=match):
        Engine(CONFIGS[0], "cpu", free_bytes=1, **bad)
