"""CPU checks of the cache formats that the engine plans for."""
import pytest

from paper_2609_21704_amd.configs import CONFIGS
from paper_2609_21704_amd.engine import Engine, cache_bytes, placement


def test_sizes():
    cfg = CONFIGS[2]
    heads = 2 * 3 * cfg.kv_heads * 128  # layers, rows, kv heads, positions: a key and a value each
    assert cache_bytes(cfg, 2, 3, 128) == heads * 512 and cache_bytes(cfg, 2, 3, 128, "q4") == heads * 144
    big = placement(cfg, 1 << 40, 4, 1024, 4)["bytes"]["planned"]
    less = placement(cfg, 1 << 40, 4, 1024, 4, draft_cache="q4")["bytes"]["planned"]
    assert big - less == 2 * (cache_bytes(cfg, cfg.layers, 4, 1024) - cache_bytes(cfg, cfg.layers, 4, 1024, "q4"))


def test_unknown_formats_are_refused():
    """Before anything is sized, built or asked of a device."""
    cfg = CONFIGS[0]
    with pytest.raises(ValueError, match="'f16' or 'q4'"):
        cache_bytes(cfg, 1, 1, 64, "q8")
    with pytest.raises(ValueError, match="'f16' or 'q4'"):
        placement(cfg, 1 << 40, 1, 64, 2, draft_cache="int4")
    with pytest.raises(ValueError, match="draft_cache must be"):
        Engine(cfg, "cpu", draft_cache="int4")
