// Entries (sequences) of a decode state to entries of another: fork, reorder, join, free.
//
// Copies of whole arrays, bound by memory.  Each array of a unit is a number of rows (the history's w, else one) of which the
// slots that both sides have are copied; a CTA moves 16 KB, eight 16-byte words a thread requested before the first is stored.  (CTAs
// of 256 threads: 8 entries of 32 x 2049 slots 82.6 us as well, but 256 units of 8-head 4-bit entries 14.5 and 13.0 us; 512 threads 18.2.)
// Entries that take the same source are written by the first of them, from one read.  (Each by itself, one prompt of 32 x 2049 slots
// into eight samples: 60 us, so 53.8; 304 MB.)
#include "cache_copy.cuh"

namespace vatp {
namespace {

constexpr int CC_THREADS = 128;

__global__ void __launch_bounds__(CC_THREADS)
cache_copy_kernel(const __grid_constant__ CopyPlan plan, int batch, int heads, int from_batch, int from_cap, int from_budget, int cap, int budget, int in_place, const int32_t* src_of,
                  vatp_cache a, vatp_cache c, int32_t* dev_status) {
  const int unit = blockIdx.x / plan.ctas, b = unit / heads, head = unit - b * heads, tid = threadIdx.x, lane = tid & 31;
  int cta = blockIdx.x - unit * plan.ctas;
  const bool first = cta == 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int src = src_of[b];
  if (src == VATP_SEQ_KEEP || (in_place && src == b)) return;
  if (src == VATP_SEQ_FREE) {
    if (first) {
      for (int s = tid; s < cap; s += CC_THREADS) c.pos[(int64_t)unit * cap + s] = -1;
      if (tid == 0) { c.len[unit] = 0; c.free_slot[unit] = 0; c.next_pos[unit] = 0; c.last_slot[unit] = -1; }
    }
    return;
  }
  // an entry of the same arrays may be read only if nobody writes it; an entry of more tokens than the target's budget does not fit
  bool fits = src >= 0 && src < from_batch;
  if (fits && in_place) {
    const int there = src_of[src];
    fits = there == src || there == VATP_SEQ_KEEP;
  }
  const int v = fits ? src * heads + head : 0;
  if (fits && from_budget > budget) fits = a.len[v] <= budget;
  if (!fits) {
    if (tid == 0 && dev_status) atomicExch(dev_status, (int)VATP_ERR_INVALID_ARG);
    return;
  }
  // bit i: entry e0 + i takes this source too (an entry that is its own source within one state stays)
  auto takers = [&](int e0) {
    const int e = e0 + lane;
    return __ballot_sync(0xffffffffu, e < batch && src_of[e] == src && !(in_place && e == src));
  };
  const int e_first = b & ~31;
  for (int e0 = 0; e0 < e_first; e0 += 32)
    if (takers(e0)) return;
  const unsigned same = takers(e_first);
  if (same & ((1u << (b & 31)) - 1u)) return;
  // f(u) for every unit that takes unit v of the source, this one first
  auto each = [&](auto f) {
    unsigned rest = same;
    for (int e0 = e_first;;) {
      for (; rest; rest &= rest - 1) f((e0 + __ffs((int)rest) - 1) * heads + head);
      e0 += 32;
      if (e0 >= batch) break;
      rest = takers(e0);
    }
  };
  if (first)
    each([&](int u) {
      for (int s = from_cap + tid; s < cap; s += CC_THREADS) c.pos[(int64_t)u * cap + s] = -1;
      if (tid == 0) copy_unit_words(a, v, c, u);
    });
  copy_words<CC_THREADS>(plan, cta, v, each);
}

}  // namespace

cudaError_t launch_cache_copy(int units, int heads, int from_batch, int from_budget, int budget, const CacheArray* arrays, int n, const int32_t* src_of,
                              bool in_place, const vatp_cache& a, const vatp_cache& c, int32_t* dev_status, cudaStream_t st) {
  const int fc = cache_capacity(from_budget), tc = cache_capacity(budget);
  CopyPlan plan;
  if (!make_copy_plan(&plan, arrays, n, false, fc, tc, CC_THREADS) || (int64_t)units * plan.ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  DependentLaunch dl(dim3((unsigned)(units * plan.ctas)), dim3(CC_THREADS), 0, st);
  return cudaLaunchKernelEx(&dl.cfg, cache_copy_kernel, plan, units / heads, heads, from_batch, fc, from_budget, tc, budget, in_place ? 1 : 0, src_of, a, c, dev_status);
}

}  // namespace vatp
