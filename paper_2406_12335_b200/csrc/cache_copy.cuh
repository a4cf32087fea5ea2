// Copies of the arrays of decode states, as part of a kernel: entry for entry in cache_copy.cu, the state that goes along with rows
// whose form is converted in pack_q4.cu.
#pragma once
#include "vatp_internal.cuh"

namespace vatp {

constexpr int CC_WORDS = 8;     // 16-byte words of a thread, requested before the first is stored

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

// The arrays' first `from_cap` and `cap` slots side by side, by CTAs of `threads`; shared: leave out arrays that are the same on both
// sides.  False where a count does not fit into 32 bits.
inline bool make_copy_plan(CopyPlan* plan, const CacheArray* arrays, int n, bool shared, int from_cap, int cap, int threads) {
  const int both = from_cap < cap ? from_cap : cap;
  *plan = CopyPlan{};
  for (int i = 0; i < n; ++i) {
    if (shared && arrays[i].from == arrays[i].to) continue;
    CopyPart& p = plan->part[plan->parts++];
    if ((int64_t)(from_cap > cap ? from_cap : cap) * arrays[i].slot_bytes > 0x7fffffffll) return false;
    p.from = static_cast<const uint4*>(arrays[i].from);
    p.to = static_cast<uint4*>(arrays[i].to);
    p.rows = arrays[i].rows;
    // (capacities are multiples of eight slots and a slot has at least four bytes)
    p.words = both * arrays[i].slot_bytes / 16;
    p.from_row = from_cap * arrays[i].slot_bytes / 16;
    p.to_row = cap * arrays[i].slot_bytes / 16;
    const int64_t ctas = ((int64_t)p.rows * p.words + threads * CC_WORDS - 1) / (threads * CC_WORDS);
    if (ctas > 0x7fffffffll - plan->ctas) return false;
    p.ctas = (int)ctas;
    plan->ctas += p.ctas;
  }
  return true;
}

inline bool unit_words_apart(const vatp_cache& a, const vatp_cache& c) {
  return a.len != c.len || a.free_slot != c.free_slot || a.next_pos != c.next_pos || a.last_slot != c.last_slot;
}

// CTA `cta` of a unit: its words of unit v on one side to every unit that each(f) calls f with on the other.
template <int THREADS, typename Each>
__device__ __forceinline__ void copy_words(const CopyPlan& plan, int cta, int v, Each each) {
  for (int i = 0; i < plan.parts; ++i) {
    const CopyPart& p = plan.part[i];
    if (cta >= p.ctas) { cta -= p.ctas; continue; }
    const uint4* from = p.from + (int64_t)v * p.rows * p.from_row;
    const int64_t total = (int64_t)p.rows * p.words, w0 = (int64_t)cta * THREADS * CC_WORDS + threadIdx.x;
    uint4 x[CC_WORDS];
    int64_t at[CC_WORDS];
#pragma unroll
    for (int k = 0; k < CC_WORDS; ++k) {
      const int64_t w = w0 + k * THREADS;
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
        if (at[k] >= 0) __stcs(to + at[k], x[k]);      // (streamed past L2's older lines: one entry into eight 57.4 us without)
    });
    return;
  }
}

// the words of unit v of `a` that say how many tokens it has and where the next one goes, to unit u of `c` (one thread; words that both
// states share are left alone)
__device__ __forceinline__ void copy_unit_words(const vatp_cache& a, int v, const vatp_cache& c, int u) {
  if (u != v || c.len != a.len) c.len[u] = a.len[v];
  if (u != v || c.free_slot != a.free_slot) c.free_slot[u] = a.free_slot[v];
  if (u != v || c.next_pos != a.next_pos) c.next_pos[u] = a.next_pos[v];
  if (u != v || c.last_slot != a.last_slot) c.last_slot[u] = a.last_slot[v];
}

}  // namespace vatp
