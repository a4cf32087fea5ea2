// Entries (sequences) of a decode state to entries of another: fork, reorder, join, free; and the state that goes with rows whose
// form is converted.
//
// Copies of whole arrays, bound by memory.  Each array of a unit is a number of rows (the history's w, else one) of which the
// slots that both sides have are copied; a CTA moves 16 KB, eight 16-byte words a thread requested before the first is stored.  (CTAs
// of 256 threads: 8 entries of 32 x 2049 slots 82.6 us as well, but 256 units of 8-head 4-bit entries 14.5 and 13.0 us; 512 threads 18.2.)
// Entries that take the same source are written by the first of them, from one read.  (Each by itself, one prompt of 32 x 2049 slots
// into eight samples: 60 us, so 53.8; 304 MB.)
#include "vatp_internal.cuh"

namespace vatp {
namespace {

constexpr int CC_THREADS = 128, CC_WORDS = 8, CC_CTA = CC_THREADS * CC_WORDS;      // 16-byte words of a CTA

struct CopyPart {
  const uint4* from;
  uint4* to;
  int rows, words;              // per unit; of a row that both sides have
  int from_row, to_row;         // words from one row to the next
  int ctas;                     // of a unit
};
struct CopyPlan {
  CopyPart part[MAX_CACHE_ARRAYS];
  int parts, ctas;              // of a unit, over all parts
};

__global__ void __launch_bounds__(CC_THREADS)
cache_copy_kernel(const __grid_constant__ CopyPlan plan, int batch, int heads, int from_batch, int from_cap, int cap, int budget, int in_place, const int32_t* src_of,
                  vatp_cache a, vatp_cache c, int32_t* dev_status) {
  const int unit = blockIdx.x / plan.ctas, b = unit / heads, head = unit - b * heads, tid = threadIdx.x, lane = tid & 31;
  int cta = blockIdx.x - unit * plan.ctas;
  const bool first = cta == 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int src = src_of ? src_of[b] : b;
  if (src == VATP_SEQ_KEEP || (src_of && in_place && src == b)) return;
  if (src == VATP_SEQ_FREE) {
    if (first) {
      for (int s = tid; s < cap; s += CC_THREADS) c.pos[(int64_t)unit * cap + s] = -1;
      if (tid == 0) { c.len[unit] = 0; c.free_slot[unit] = 0; c.next_pos[unit] = 0; c.last_slot[unit] = -1; }
    }
    return;
  }
  // an entry of the same arrays may be read only if nobody writes it; an entry of more tokens than the target's budget does not fit
  bool fits = src >= 0 && src < from_batch;
  if (fits && src_of && in_place) {
    const int there = src_of[src];
    fits = there == src || there == VATP_SEQ_KEEP;
  }
  const int v = fits ? src * heads + head : 0;
  if (fits && from_cap > cap) fits = a.len[v] <= budget;
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
  unsigned same = 0;
  if (src_of) {
    for (int e0 = 0; e0 < e_first; e0 += 32)
      if (takers(e0)) return;
    same = takers(e_first);
    if (same & ((1u << (b & 31)) - 1u)) return;
  }
  // f(u) for every unit that takes unit v of the source, this one first
  auto each = [&](auto f) {
    f(unit);
    if (!src_of) return;
    unsigned rest = same & ~(1u << (b & 31));
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
      if (tid == 0) {
        // (a conversion leaves words that both states share alone)
        if (u != v || c.len != a.len) c.len[u] = a.len[v];
        if (u != v || c.free_slot != a.free_slot) c.free_slot[u] = a.free_slot[v];
        if (u != v || c.next_pos != a.next_pos) c.next_pos[u] = a.next_pos[v];
        if (u != v || c.last_slot != a.last_slot) c.last_slot[u] = a.last_slot[v];
      }
    });
  for (int i = 0; i < plan.parts; ++i) {
    const CopyPart& p = plan.part[i];
    if (cta >= p.ctas) { cta -= p.ctas; continue; }
    const uint4* from = p.from + (int64_t)v * p.rows * p.from_row;
    const int64_t total = (int64_t)p.rows * p.words, w0 = (int64_t)cta * CC_CTA + tid;
    uint4 x[CC_WORDS];
    int64_t at[CC_WORDS];
#pragma unroll
    for (int k = 0; k < CC_WORDS; ++k) {
      const int64_t w = w0 + k * CC_THREADS;
      at[k] = -1;
      if (w < total) {
        const int64_t r = p.rows == 1 ? 0 : w / p.words, col = w - r * p.words;
        at[k] = r * p.to_row + col;
        x[k] = load_behind_wait(from + r * p.from_row + col);
      }
    }
    each([&](int u) {
      uint4* to = p.to + (int64_t)u * p.rows * p.to_row;
#pragma unroll
      for (int k = 0; k < CC_WORDS; ++k)
        if (at[k] >= 0) __stcs(to + at[k], x[k]);      // (streamed past L2's older lines: one into eight 57.4 us without)
    });
    return;
  }
}

}  // namespace

cudaError_t launch_cache_copy(int units, int heads, int from_batch, int from_budget, int budget, const CacheArray* arrays, int n, const int32_t* src_of,
                              bool in_place, const vatp_cache& a, const vatp_cache& c, int32_t* dev_status, cudaStream_t st) {
  const int fc = cache_capacity(from_budget), tc = cache_capacity(budget), both = fc < tc ? fc : tc;
  CopyPlan plan = {};
  for (int i = 0; i < n; ++i) {
    if (!src_of && arrays[i].from == arrays[i].to) continue;       // (shared by both states)
    CopyPart& p = plan.part[plan.parts++];
    p.from = static_cast<const uint4*>(arrays[i].from);
    p.to = static_cast<uint4*>(arrays[i].to);
    p.rows = arrays[i].rows;
    // (capacities are multiples of eight slots and a slot has at least four bytes)
    if ((int64_t)(fc > tc ? fc : tc) * arrays[i].slot_bytes > 0x7fffffffll) return cudaErrorInvalidValue;
    p.words = both * arrays[i].slot_bytes / 16;
    p.from_row = fc * arrays[i].slot_bytes / 16;
    p.to_row = tc * arrays[i].slot_bytes / 16;
    const int64_t ctas = ((int64_t)p.rows * p.words + CC_CTA - 1) / CC_CTA;
    if (ctas > 0x7fffffffll - plan.ctas) return cudaErrorInvalidValue;
    p.ctas = (int)ctas;
    plan.ctas += p.ctas;
  }
  if (!plan.ctas) plan.ctas = 1;                                   // (the unit's words alone)
  if ((int64_t)units * plan.ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  DependentLaunch dl(dim3((unsigned)(units * plan.ctas)), dim3(CC_THREADS), 0, st);
  return cudaLaunchKernelEx(&dl.cfg, cache_copy_kernel, plan, units / heads, heads, from_batch, fc, tc, budget, in_place ? 1 : 0, src_of, a, c, dev_status);
}

}  // namespace vatp
