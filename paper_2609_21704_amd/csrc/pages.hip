// The bookkeeping of paged caches (which sequence holds which pages) and the copies of pages.
//   pages_reserve_kernel   rows take the pages they lack
//   pages_trim_kernel      rows give pages back
//   pages_fork_kernel      rows share the pages of others
//   pages_compact_kernel, pages_remap_kernel   the used pages move to the lowest ids
//   page_copy_kernel       page contents, in all layers
// There is no list of free pages: a page is free where refs is 0, and the lowest free ids are found by a scan of refs.
// Giving pages back is then a count per page, which no order of execution changes, and there is no list to be left in
// disorder.  The scan runs only when pages are needed (a sequence needs one every 64 tokens) and ends once it has found
// enough; the calls are bound by their launch and a few dependent round trips to memory.
#include "sq_device.hpp"
#include "sq_internal.hpp"

namespace sq {
namespace {

constexpr int32_t kNoPages = 32, kBadPage = 64, kBadFork = 128;  // the SQ_DEV_* values of the C header
constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kIds = 16;  // page ids a thread looks at in one step of a scan

__device__ __forceinline__ void flag(int32_t* status, int32_t bit) {
  if (status) atomicOr(status, bit);
}

// Exclusive prefix sum over the workgroup in thread order; total: the workgroup's sum.  Every thread calls it.
__device__ __forceinline__ int block_scan(int v, int* sh, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int o = __shfl_up(x, d, kWave);
    x += lane >= d ? o : 0;
  }
  if (lane == 63) sh[w] = x;
  __syncthreads();
  int base = 0, t = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    base += i < w ? sh[i] : 0;
    t += sh[i];
  }
  __syncthreads();
  total = t;
  return base + x - v;
}

// Calls f(id, rank) for the ids in [from, to) with is(refs[id]), of which `rank` lower ones there are, and returns how many
// were found; stops after the step in which there are `enough`.
template <class P, class F>
__device__ __forceinline__ int pick_ids(const int32_t* refs, int from, int to, int enough, int* sh, P is, F f) {
  int found = 0;
  for (int base = from; base < to && found < enough; base += kThreads * kIds) {  // uniform
    const int id0 = base + (int)threadIdx.x * kIds;
    int x[kIds];
#pragma unroll
    for (int i = 0; i < kIds; ++i) x[i] = refs[id0 + i < to ? id0 + i : to - 1];
    uint32_t set = 0;
#pragma unroll
    for (int i = 0; i < kIds; ++i) set |= (id0 + i < to && is(x[i]) ? 1u : 0u) << i;
    int total;
    int rank = found + block_scan(__builtin_popcount(set), sh, total);
    while (set) {
      const int i = __builtin_ctz(set);
      set &= set - 1;
      f(id0 + i, rank++);
    }
    found += total;
  }
  return found;
}

// The pages that positions below `n` take, at most one more than INT32 pages can hold.
__device__ __forceinline__ int64_t pages_for(int64_t n) { return n <= 0 ? 0 : (n + kPage - 1) / kPage; }

// The lowest free ids, up to `most` of them, to list (device memory of the workgroup's own); how many there are.
__device__ __forceinline__ int free_ids(const int32_t* refs, int pages, int most, int32_t* list, int* sh) {
  const int found = pick_ids(refs, 0, pages, most, sh, [](int n) { return n <= 0; },
                             [&](int id, int rank) {
                               if (rank < most) list[rank] = id;
                             });
  __syncthreads();
  return found < most ? found : most;
}

__global__ __launch_bounds__(kThreads) void pages_reserve_kernel(PageState p, const int32_t* __restrict__ pos_base,
                                                                 int ahead, int32_t* __restrict__ list,
                                                                 int32_t* __restrict__ status) {
  __shared__ int sh[kWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int cap = p.pages + 1;  // more than there are
  // pages that row s lacks; -1: a row that cannot be served
  auto lacks = [&](int s, int& held) -> int {
    held = 0;
    if (s >= p.b) return 0;
    const int pos = pos_base[s];
    held = p.held[s];
    if (pos < 0) return 0;
    if (held < 0 || held > p.width) return -2;
    const int64_t want = pages_for((int64_t)pos + ahead);
    if (want <= held) return 0;
    if (want > p.width) return -1;
    return want - held < cap ? (int)(want - held) : cap;
  };
  int total = 0;
  for (int s0 = 0; s0 < p.b; s0 += kThreads) {
    int held, t;
    const int d = lacks(s0 + tid, held);
    if (d == -1) flag(status, kNoPages);
    if (d == -2) flag(status, kBadPage);
    block_scan(d > 0 ? d : 0, sh, t);
    total = total + t < cap ? total + t : cap;  // (at most 2^30 a step)
  }
  if (total == 0) return;
  const int found = free_ids(p.refs, p.pages, total, list, sh);
  int before = 0;
  for (int s0 = 0; s0 < p.b; s0 += kThreads) {
    const int s = s0 + tid;
    int held, t;
    const int d = lacks(s, held);
    const int at = before + block_scan(d > 0 ? d : 0, sh, t);
    before = before + t < cap ? before + t : cap;
    const bool served = d > 0 && at + d <= found;
    if (d > 0 && !served) flag(status, kNoPages);
    // a few pages by the row's own thread, many (a prompt) by its wavefront
    constexpr int kFew = 4;
    if (served && d <= kFew) {
      for (int i = 0; i < d; ++i) {
        const int id = list[at + i];
        p.table[(int64_t)s * p.width + held + i] = id;
        p.refs[id] = 1;
      }
    }
    uint64_t many = __ballot(served && d > kFew);
    while (many) {
      const int l = __builtin_ctzll(many);
      many &= many - 1;
      const int ls = __shfl(s, l), lh = __shfl(held, l), ld = __shfl(d, l), la = __shfl(at, l);
      for (int i = lane; i < ld; i += kWave) {
        const int id = list[la + i];
        p.table[(int64_t)ls * p.width + lh + i] = id;
        p.refs[id] = 1;
      }
    }
    if (served) p.held[s] = held + d;
  }
}

// A wavefront a row.
__global__ __launch_bounds__(256) void pages_trim_kernel(PageState p, const int32_t* __restrict__ keep,
                                                         int32_t* __restrict__ status) {
  const int s = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (s >= p.b) return;
  const int n = keep[s], held = p.held[s];
  if (n < 0) return;
  if (held < 0 || held > p.width) {
    if (lane == 0) flag(status, kBadPage);
    return;
  }
  const int first = (int)pages_for(n);
  if (first >= held) return;
  int32_t* row = p.table + (int64_t)s * p.width;
  for (int i = first + lane; i < held; i += kWave) {
    const int id = row[i];
    row[i] = -1;
    if ((uint32_t)id < (uint32_t)p.pages)
      atomicSub(&p.refs[id], 1);
    else
      flag(status, kBadPage);
  }
  if (lane == 0) p.held[s] = first;
}

__global__ __launch_bounds__(kThreads) void pages_fork_kernel(PageState p, const int32_t* __restrict__ parent,
                                                              const int32_t* __restrict__ child,
                                                              const int32_t* __restrict__ length, int n,
                                                              int32_t* __restrict__ src, int32_t* __restrict__ dst,
                                                              int32_t* __restrict__ count, int32_t* __restrict__ list,
                                                              int32_t* __restrict__ status) {
  __shared__ int sh[kWaves];
  __shared__ __align__(16) int sc[kThreads];  // child
  __shared__ int sp[kThreads], sl[kThreads], sr[kThreads];  // parent, length (0: no fork), fresh page
  const int tid = threadIdx.x, lane = tid & 63;
  const bool mine = tid < n;
  const int pa = mine ? parent[tid] : -1, ch = mine ? child[tid] : -1, len = mine ? length[tid] : 0;
  sc[tid] = ch;
  __syncthreads();
  bool ok = mine && ch >= 0;
  const bool asked = ok;
  if (ok) ok = ch < p.b && pa >= 0 && pa < p.b && pa != ch;
  if (ok) {
    const int hp = p.held[pa];
    ok = p.held[ch] == 0 && hp > 0 && hp <= p.width && len >= 1 && len <= (int64_t)hp * kPage;
  }
  const int before = __any(ok) ? n : 0;  // (wavefronts without a pair need not look)
  for (int j = 0; j < before; j += 4) {  // (the same words for all; past n they are -1)
    const int4 c = *reinterpret_cast<const int4*>(&sc[j]);
    if ((j < tid && c.x == ch) || (j + 1 < tid && c.y == ch) || (j + 2 < tid && c.z == ch) || (j + 3 < tid && c.w == ch))
      ok = false;
  }
  if (asked && !ok) flag(status, kBadFork);
  const bool part = ok && len % kPage != 0;
  int total;
  const int rank = block_scan(part ? 1 : 0, sh, total);
  const int found = total ? free_ids(p.refs, p.pages, total, list, sh) : 0;
  if (part && rank >= found) {
    ok = false;
    flag(status, kNoPages);
  }
  sp[tid] = pa;
  sl[tid] = ok ? len : 0;
  sr[tid] = ok && part ? list[rank] : -1;
  __syncthreads();
  // a wavefront a pair, four of its pairs' loads in flight
  constexpr int kPairs = 4;
  for (int i0 = tid >> 6; i0 < n; i0 += kPairs * kWaves) {
    int full[kPairs], most = 0;
#pragma unroll
    for (int x = 0; x < kPairs; ++x) {
      const int i = i0 + x * kWaves;
      full[x] = i < n ? sl[i] / kPage : 0;  // (sl 0: nothing)
      most = full[x] > most ? full[x] : most;
    }
    for (int e = lane; e < most; e += kWave) {
      int id[kPairs];
#pragma unroll
      for (int x = 0; x < kPairs; ++x)
        if (e < full[x]) id[x] = p.table[(int64_t)sp[i0 + x * kWaves] * p.width + e];
#pragma unroll
      for (int x = 0; x < kPairs; ++x) {
        if (e >= full[x]) continue;
        p.table[(int64_t)sc[i0 + x * kWaves] * p.width + e] = id[x];
        if ((uint32_t)id[x] < (uint32_t)p.pages)
          atomicAdd(&p.refs[id[x]], 1);
        else
          flag(status, kBadPage);
      }
    }
  }
  if (ok) {  // a thread a pair
    const int full = len / kPage;
    if (part) {
      p.table[(int64_t)ch * p.width + full] = sr[tid];
      p.refs[sr[tid]] = 1;
    }
    p.held[ch] = full + (part ? 1 : 0);
  }
  if (ok && part) {  // (those that got a page are the first of those that needed one)
    src[rank] = p.table[(int64_t)pa * p.width + len / kPage];
    dst[rank] = sr[tid];
  }
  if (tid == 0) *count = found;
}

// to[id] for the ids from `used` on: where their pages went.
__global__ __launch_bounds__(kThreads) void pages_compact_kernel(PageState p, int32_t* __restrict__ src,
                                                                 int32_t* __restrict__ dst, int32_t* __restrict__ count,
                                                                 int32_t* __restrict__ used, int32_t* __restrict__ to) {
  __shared__ int sh[kWaves];
  const int all = p.pages + 1;  // (no scan ends early)
  auto held = [](int n) { return n > 0; };
  const int u = pick_ids(p.refs, 0, p.pages, all, sh, held, [](int, int) {});
  pick_ids(p.refs, 0, u, all, sh, [](int n) { return n <= 0; }, [&](int id, int rank) { dst[rank] = id; });
  const int n = pick_ids(p.refs, u, p.pages, all, sh, held, [&](int id, int rank) { src[rank] = id; });
  for (int i = u + threadIdx.x; i < p.pages; i += kThreads) to[i] = i;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads) {  // as many free ids below u as used ones from u on
    const int a = src[i], b = dst[i];
    to[a] = b;
    p.refs[b] = p.refs[a];
    p.refs[a] = 0;
  }
  if (threadIdx.x == 0) {
    *count = n;
    *used = u;
  }
}

__global__ __launch_bounds__(256) void pages_remap_kernel(PageState p, const int32_t* __restrict__ used,
                                                          const int32_t* __restrict__ to, int32_t* __restrict__ status) {
  const int u = *used;
  const int s = blockIdx.x;
  const int held = p.held[s];
  if (held < 0 || held > p.width) {
    if (threadIdx.x == 0 && blockIdx.y == 0) flag(status, kBadPage);
    return;
  }
  int32_t* row = p.table + (int64_t)s * p.width;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < held; i += gridDim.y * 256) {
    const int id = row[i];
    if ((uint32_t)id >= (uint32_t)p.pages)
      flag(status, kBadPage);
    else if (id >= u)
      row[i] = to[id];
  }
}

// A workgroup copies 16 KB pieces of pages, four loads of 16 bytes a thread in flight.
constexpr int64_t kPiece = 16384;

__global__ __launch_bounds__(256) void page_copy_kernel(uint8_t* __restrict__ pool, int layers, int pages,
                                                        int64_t page_bytes, const int32_t* __restrict__ src,
                                                        const int32_t* __restrict__ dst,
                                                        const int32_t* __restrict__ count, int most,
                                                        int32_t* __restrict__ status) {
  int n = *count;
  n = n < 0 ? 0 : (n > most ? most : n);
  const int64_t pieces = (page_bytes + kPiece - 1) / kPiece, units = (int64_t)n * layers * pieces;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t pl = unit / pieces, piece = unit - pl * pieces;
    const int l = (int)(pl / n), i = (int)(pl - (int64_t)l * n);
    const int a = src[i], b = dst[i];
    if ((uint32_t)a >= (uint32_t)pages || (uint32_t)b >= (uint32_t)pages) {
      if (l == 0 && piece == 0 && threadIdx.x == 0) flag(status, kBadPage);
      continue;
    }
    if (a == b) continue;
    const int64_t off = piece * kPiece, left = page_bytes - off;
    const uint8_t* from = pool + ((int64_t)l * pages + a) * page_bytes + off;
    uint8_t* to = pool + ((int64_t)l * pages + b) * page_bytes + off;
    u32x4 v[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int64_t at = 4096 * x + 16 * (int)threadIdx.x;
      if (at < left) v[x] = *reinterpret_cast<const u32x4*>(from + at);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int64_t at = 4096 * x + 16 * (int)threadIdx.x;
      if (at < left) *reinterpret_cast<u32x4*>(to + at) = v[x];
    }
  }
}

hipError_t page_list(const PageState& p, hipStream_t stream, int32_t** list) {
  void* ws = nullptr;
  const hipError_t e = workspace((size_t)p.pages * sizeof(int32_t), stream, &ws);
  *list = static_cast<int32_t*>(ws);
  return e;
}

}  // namespace

hipError_t launch_pages_reserve(const PageState& p, const int32_t* pos_base, int ahead, int32_t* status,
                                hipStream_t stream) {
  int32_t* list;
  const hipError_t e = page_list(p, stream, &list);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(kThreads), 0, stream, p, pos_base, ahead, list, status);
  return hipGetLastError();
}

hipError_t launch_pages_trim(const PageState& p, const int32_t* keep, int32_t* status, hipStream_t stream) {
  hipLaunchKernelGGL(pages_trim_kernel, dim3((p.b + 3) / 4), dim3(256), 0, stream, p, keep, status);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PageState& p, const int32_t* parent, const int32_t* child, const int32_t* length, int n,
                             int32_t* src, int32_t* dst, int32_t* count, int32_t* status, hipStream_t stream) {
  int32_t* list;
  const hipError_t e = page_list(p, stream, &list);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_fork_kernel, dim3(1), dim3(kThreads), 0, stream, p, parent, child, length, n, src, dst, count,
                     list, status);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PageState& p, int32_t* src, int32_t* dst, int32_t* count, int32_t* used,
                                int32_t* status, hipStream_t stream) {
  int32_t* to;
  const hipError_t e = page_list(p, stream, &to);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(kThreads), 0, stream, p, src, dst, count, used, to);
  const int slices = p.width > 256 * 16 ? 16 : (p.width + 255) / 256;
  hipLaunchKernelGGL(pages_remap_kernel, dim3(p.b, slices), dim3(256), 0, stream, p, used, to, status);
  return hipGetLastError();
}

hipError_t launch_page_copy(void* pool, int layers, int pages, int64_t page_bytes, const int32_t* src, const int32_t* dst,
                            const int32_t* count, int n, int32_t* status, hipStream_t stream) {
  const int64_t units = (int64_t)n * layers * ((page_bytes + kPiece - 1) / kPiece);
  const int64_t most = (int64_t)cu_count() * 8;
  hipLaunchKernelGGL(page_copy_kernel, dim3((unsigned)(units < most ? units : most)), dim3(256), 0, stream,
                     static_cast<uint8_t*>(pool), layers, pages, page_bytes, src, dst, count, n, status);
  return hipGetLastError();
}

}  // namespace sq
