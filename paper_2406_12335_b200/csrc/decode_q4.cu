// Decode step on a cache whose rows are held in 4 bits: append (quantised), attend (Eq. 1), indicator update (Eq. 2 / Eq. 3),
// importance (Eq. 4), release of the lowest-importance unprotected slot.
//
// With the values lo_ig + sc_ig code_ic of row i, group g and channel c:
//   s_i = scale * sum_g ( sc_ig * sum_{c in g} q_c code_ic + lo_ig * sum_{c in g} q_c ),   p = softmax(s)
//   o_c = sum_i p_i lo_ig + sum_i (p_i sc_ig) code_ic
// The sums over codes run on the warp-level tensor-core path, the rest in fp32.  How depends on the query heads of a unit:
//   * one head (INT; mma.sync m16n8k32 in 8-bit integers, 32-bit sums): a byte of a row is lo + 16 hi, its upper half 16 hi after one AND,
//     so the rows' words are operands as they are and unpacking is an instruction per eight codes.  The other operand has eight
//     columns for one head: q is a 25-bit integer (a power of two takes the largest below 2^25), and lo q_lo + hi q_hi =
//     byte * q_lo + upper half / 16 * (q_hi - 16 q_lo), each factor as four signed digits of 8 bits in columns of their own, two groups
//     side by side.  p_i sc_ig is an integer below 2^29 in four unsigned digits.  All products are exact; a fp32 q loses 2^-25 of the
//     largest, p sc 2^-29 of the warp's largest;
//   * several heads (m16n8k16 in fp16, 32-bit sums; two columns for each head): a code in bits 6-9 of a 16-bit word IS the fp16 number
//     code * 2^-18 (subnormal): unpacking is a shift and an AND per two codes; the constant factor goes into the result.  The tensor
//     cores align such a product by its nominal exponent of -14 and cut off what lies 24 bits below the largest of a sum, hence not
//     bits 0-3 and 4-7, where an AND alone would do: beside a channel of q that is 125 times the others logits were then off by 1.1e-5 to
//     1.5e-5, so by 3e-6.
//     The other operand's magnitude does not matter: q is scaled by a power of two per head, p_i sc_ig by one per warp and head that the
//     largest of them determines.  p_i sc_ig and a q of 32 bits are a high half and a remainder, 2^-22 (with p_i sc_ig in one fp16, 2^-12,
//     one bf16 output in six came out a step away from the nearest; now one in fifty at most.  Both together cost 5 to 10 %: 16 units x 4002
//     slots, four heads, 9.6 -> 10.3 us per step; 128 x 2049, eight heads, 29.5 -> 32.5); a bf16 q fits one fp16 down to
//     2^-28 of the head's largest channel, below that it is off by 2^-38 of that channel at most;
//   * rows are stored so that the 8 or 16 bytes a lane takes hold the channels it needs in an MMA operand, of every group.
// A unit is split over a thread-block cluster; the slots of a CTA over eight or sixteen warps, 32 at a time.
//   * An item of K or of V is 32 consecutive rows, two bulk copies (codes, parameters) into the warp's ring in shared memory.  Those
//     of K, as many as the ring holds, are requested before the launch ahead has finished (after it: 256 units x 1639 slots 16.9 -> 17.9 us);
//     the one row that it may have appended since (last_slot) is patched in.  The first of V go out while q and the state words are under
//     way: what stands before the wait delays the CTAs that start last, when others of the launch ahead have just left their SMs.
//   * A warp keeps its own softmax: its maximum, sum and partial output, without a barrier between the two products.
//   * One more warp takes the incoming token, which is no part of any item: it quantises and stores the rows and is a partial of its own.
//   * The CTA joins its partials, the cluster those of its CTAs by st.async into the partners' shared memory; every CTA then updates the
//     indicators of its own slots, and every warp sends its eviction candidate to rank 0.
// What bounds it (one head, d 128): instructions and their latency, not memory.  An item's two products are 645 instructions of a warp
// (110 of them requests) for 5 KB, and a step has some 1000 more per warp that do not depend on its length.  32 units x 2049 slots: 6.3 us
// per step in a chain of steps, of which the time between launches takes 0.7, q 0.85, two items' K 0.8, V 1.25, joining partials, CTAs and candidates
// 2.6; 256 units x 1639: 16.7 us, 4.4 TB/s.  Not faster: a warp that requests all rings' items; three CTAs an SM (72 registers spill); p sc of the next
// item formed while this one's products run (spills with eight warps in pairs: 18.7 -> 21.5 us; without spills 6.74 -> 6.97).
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "known_counts.h"
#include "q4.cuh"

namespace cg = cooperative_groups;

namespace vatp {
namespace {

constexpr int Q4_TILE = 16;            // slots of an MMA tile
constexpr int Q4_ROWS = 32;            // slots of a warp at a time: an item of its ring
constexpr int Q4_SPLIT = 16;           // CTAs of a unit at most
constexpr int Q4_HEADS = 8;            // query heads of a unit at most (columns of the MMA tiles)
constexpr int Q4_EXTRA = 8;            // slots beyond the tiles that the last warp takes at most
constexpr int Q4_DEPTH = 8;            // items in a warp's ring at most
constexpr int Q4_FLUSH = 64 * Q4_ROWS;      // 255 * 15 * 257 * 2048 < 2^31
constexpr int Q4_NO_J = -1000000;           // exponent of p sc before the first slot
constexpr float Q4_LOG2E = 1.4426950408889634f;
constexpr unsigned long long Q4_NO_KEY = ~0ull;

__device__ __forceinline__ uint32_t s32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(s32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// bounded wait (about a second): false when what the barrier counts never arrived
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  if (bar_try(bar, parity)) return true;
  uint64_t t0, t1;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  while (!bar_try(bar, parity)) {
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
    if (t1 - t0 > 1000000000ull) return false;
  }
  return true;
}
// global -> shared bulk copy; dst, src and bytes are multiples of 16
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// address of `addr` (this CTA's shared memory) in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void send(uint32_t addr, float a, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(addr), "r"(__float_as_uint(a)), "r"(bar) : "memory");
}
__device__ __forceinline__ void send2(uint32_t addr, float a, float b, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];"
               ::"r"(addr), "r"(__float_as_uint(a)), "r"(__float_as_uint(b)), "r"(bar) : "memory");
}
__device__ __forceinline__ void send4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d), "r"(bar) : "memory");
}
// D (16x8, fp32) += A (16x16, fp16, row) * B (16x8, fp16, col)
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D (16x8, int32) = A (16x32, u8, row) * B (32x8, s8 or u8, col) + C
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, int c) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(c));
}
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_u8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.u8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// one lane of the warp
__device__ __forceinline__ bool elected() {
  uint32_t p;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^e, exactly; 2^127 beyond that, 0 below the normal numbers
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)min(max(e + 127, 0), 254) << 23); }
__device__ __forceinline__ float max_of(float x) {      // over the warp
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
// NV values of every lane summed over the lanes that agree in what lies below LOW: lane l gets the sum of v[l / (32 / NV)] in v[0].
// (Lanes halve the values between them as they go: 16 values take 16 shuffles, of which an SM does one per cycle, instead of 80.)
template <int NV, int LOW> __device__ __forceinline__ void sum_over(float (&v)[NV], int lane) {
  int o = 16;
#pragma unroll
  for (int half = NV / 2; half > 0; half /= 2, o /= 2) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < half; ++i) v[i] = (up ? v[i + half] : v[i]) + __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + half], o);
  }
#pragma unroll
  for (; o >= LOW; o /= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// past L1: what the launch ahead has stored since this CTA requested the row early
__device__ __forceinline__ uint32_t load_fresh(const uint32_t* p) {
  uint32_t x;
  asm volatile("ld.global.cg.u32 %0, [%1];" : "=r"(x) : "l"(p));
  return x;
}
template <int N> __device__ __forceinline__ void words_of(const unsigned char* p, uint32_t (&w)[N]) {      // from shared memory
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x; w[1] = x.y;
  } else {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  }
}

// eight consecutive channels of q as they lie in memory, and as floats
template <typename T> struct Raw8 {
  uint4 r[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) r[k] = load_behind_wait(reinterpret_cast<const uint4*>(p) + k);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
      const uint32_t w[4] = {r[k].x, r[k].y, r[k].z, r[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
          x[4 * k + i] = __uint_as_float(w[i]);
        } else {
          x[2 * i] = __uint_as_float(w[i] << 16);
          x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
      }
    }
  }
};
// four consecutive channels of a new row
__device__ __forceinline__ void load_new(const __nv_bfloat16* p, float (&x)[4]) {
  const uint2 r = *reinterpret_cast<const uint2*>(p);
  x[0] = __uint_as_float(r.x << 16); x[1] = __uint_as_float(r.x & 0xffff0000u);
  x[2] = __uint_as_float(r.y << 16); x[3] = __uint_as_float(r.y & 0xffff0000u);
}
__device__ __forceinline__ void load_new(const float* p, float (&x)[4]) {
  const float4 r = load_behind_wait(reinterpret_cast<const float4*>(p));
  x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
}
__device__ __forceinline__ void to_out(float* p, float x) { *p = x; }
__device__ __forceinline__ void to_out(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }

struct __align__(16) Q4Candidate {      // eviction candidate of a CTA, sent to rank 0 (key Q4_NO_KEY: none)
  unsigned long long key;
  int slot, pos;
};
// eviction order as one integer: lower importance first, among equals the higher position first
__device__ __forceinline__ unsigned long long q4_evict_key(float I, int pos) {
  return ((unsigned long long)__float_as_uint(I) << 32) | (unsigned)(0x7fffffff - pos);
}
__device__ __forceinline__ unsigned long long min_key(unsigned long long key) {
  const unsigned h = (unsigned)(key >> 32), mh = __reduce_min_sync(0xffffffffu, h);
  const unsigned ml = __reduce_min_sync(0xffffffffu, h == mh ? (unsigned)key : 0xffffffffu);
  return ((unsigned long long)mh << 32) | ml;
}

// GT: 1 - one query head per cache; 4 - two to four, the columns of the second product are the heads' high halves and then the
// remainders; 8 - five to eight, a column a head and two products.
// Dynamic shared memory: rings [WARPS][depth][item], which take the warps' partial outputs in the end | the last partial [G][HD] |
// slices received [2 G HD at most] | logits [G][ld].
template <int HD> constexpr int q4_item = Q4_ROWS * (HD / 2 + HD / 8);      // bytes of an item: codes, then parameters

// ALONE: one CTA on an SM (eight warps then have 128 registers and more instead of 96: 32 units x 2049 slots 7.3 -> 6.8 us).
template <typename T, int HD, bool WINDOWED, int GT, int WARPS, bool ALONE>
__global__ void __launch_bounds__(WARPS * 32 + 32, ALONE ? 1 : 2)
decode_q4_kernel(int G_arg, int split, int chunk, int ld, int depth, int B, int cap, int F, int R, int w, int norm, float scale_log2, vatp_cache_q4 c, const T* q_new,
                 const T* k_new, const T* v_new, T* out, int32_t* evicted, int32_t* dev_status) {
  constexpr int WORKERS = WARPS * 32, THREADS = WORKERS + 32;   // warps that take slots, and one more
  constexpr int NG = HD / 32, KW = HD / 32, VW = HD / 64;       // groups of a row; 32-bit words of a lane in a K row and a V row
  constexpr bool INT = GT == 1;                                 // products in integers (see the top)
  constexpr int KP = INT ? NG / 2 : NG;                         // parameter words of a lane per K row
  constexpr int CODES = HD / 2, PARAMS = NG * 4, ITEM = q4_item<HD>;      // bytes of a row's codes and parameters, of an item
  constexpr bool Q_REST = sizeof(T) == 4;                       // q has a remainder beyond its high half
  constexpr int XC = GT > 4 ? 16 : 8;                           // columns of the second product's operand: see x_col
  constexpr int N = GT > 4 ? 1 : 2;                             // tiles a warp works on at a time (with eight heads: registers)
  constexpr int PG = N == 2 ? NG : VW;                          // groups of a lane where p sc is formed: a slot or half of one
  constexpr int XS = INT ? NG * 4 * 2 * Q4_TILE : N * NG * XC * Q4_TILE * 2;      // bytes of a warp's second operand
  constexpr int CODE_EXP = 18;                                  // a code in bits 6-9 stands for code * 2^-CODE_EXP
  auto codes0 = [](uint32_t x) { return x << 6 & 0x03c003c0u; };      // the four codes of a 16-bit word
  auto codes1 = [](uint32_t x) { return x << 2 & 0x03c003c0u; };
  auto codes2 = [](uint32_t x) { return x >> 2 & 0x03c003c0u; };
  auto codes3 = [](uint32_t x) { return x >> 6 & 0x03c003c0u; };
  const int G = GT == 1 ? 1 : G_arg;
  // high half and remainder of head h: neighbours, i.e. in one lane's accumulators, or eight columns apart (two products)
  auto x_col = [](int h, int low) { return GT > 4 ? h + 8 * low : 2 * h + low; };
  extern __shared__ __align__(128) unsigned char dyn[];
  const int ring_bytes = depth * ITEM;                          // of a warp
  float* new_o = reinterpret_cast<float*>(dyn + WARPS * ring_bytes);
  float* xo = new_o + G * HD;                                   // slices of partial outputs received [split][G][slice]
  float* logit_s = xo + 2 * G * HD;
  // the second product's operand, [tile][group][column][slot] of fp16 or [group][digit][tile][slot] of bytes; slot s of a tile
  // stands at 4 (s mod 4) + s / 4
  __shared__ __align__(16) unsigned char xs[WARPS][XS];
  __shared__ float part_m[WARPS + 1][GT], part_l[WARPS + 1][GT], part_lo[WARPS][GT][NG];
  __shared__ float2 ex_ml[Q4_SPLIT][GT];                                // per rank and head: maximum of its logits, sum of exp2(s - m)
  __shared__ float fr_s[Q4_SPLIT][GT], all_m[GT], all_inv[GT], new_norm_s;
  __shared__ Q4Candidate cand[Q4_SPLIT * WARPS];                     // in rank 0
  __shared__ __align__(8) uint64_t full[WARPS][Q4_DEPTH], k_done, ex_bar, cand_bar;

  const int rank = split > 1 ? (int)cg::this_cluster().block_rank() : 0;
  const int tid = threadIdx.x, lane = tid & 31, wid = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int r8 = lane >> 2, t4 = lane & 3;
  const int u = blockIdx.x / split;
  const int slice_log2 = (HD == 128 ? 7 : 6) - (31 - __clz(split)), slice = 1 << slice_log2;      // channels of the output that rank r < HD / slice writes
  const bool writes = rank * slice < HD;
  // this CTA's slots of the unit: those of the tiles, and in the last CTA up to Q4_EXTRA more (see launch_gt)
  const int s0 = min(rank * chunk, cap), rows_alloc = min(chunk, cap - s0), rows_all = rank == split - 1 ? cap - s0 : rows_alloc;
  const int64_t base = (int64_t)u * cap + s0;
  if (tid < WARPS * Q4_DEPTH) bar_init(&full[0][tid], 1);
  if (tid == WORKERS) {
    bar_init(&k_done, WARPS + 1);
    bar_init(&ex_bar, 1);
    bar_init(&cand_bar, 1);
  }
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  if (tid == WORKERS) {
    bar_expect(s32(&ex_bar), (uint32_t)(8 * G * split + (writes ? 4 * G * slice * split : 0)));
    if (rank == 0) bar_expect(s32(&cand_bar), (uint32_t)(split * WARPS * sizeof(Q4Candidate)));
  }
  if (!INT && wid < WARPS)      // (columns without a head stay 0)
    for (int i = lane; i < XS / 4; i += 32) reinterpret_cast<uint32_t*>(xs[wid])[i] = 0u;
  __syncthreads();
  // Another CTA's shared memory may only be written once that CTA runs and its barriers are armed: everyone arrives here and
  // waits (long since satisfied) just before the first remote store.
  if (split > 1) cluster_arrive_release();

  bool bad = false;                      // this thread's wait ran out: it no longer waits, the results are void
  const unsigned char* kc = static_cast<const unsigned char*>(c.state.k_cache) + base * CODES;
  const unsigned char* vc = static_cast<const unsigned char*>(c.state.v_cache) + base * CODES;
  const unsigned char* kp = static_cast<const unsigned char*>(c.k_params) + base * PARAMS;
  const unsigned char* vp = static_cast<const unsigned char*>(c.v_params) + base * PARAMS;
  unsigned char* ring = dyn + (size_t)wid * ring_bytes;
  // This warp's items: rows 32 (wid + WARPS j) ..; n of them among the first `rows` slots.  Item j < n of its ring holds rows of K, item
  // n + j of V.
  auto items_in = [&](int rows) { return max(rows - wid * Q4_ROWS + WARPS * Q4_ROWS - 1, 0) / (WARPS * Q4_ROWS); };
  auto item_row = [&](int j) { return (wid + WARPS * j) * Q4_ROWS; };
  const uint32_t ring_a = s32(ring), full_a = s32(&full[wid < WARPS ? wid : 0][0]);
  auto request = [&](int j, int n, int slot) {      // one lane: item j into ring slot `slot`
    const bool is_v = j >= n;
    const unsigned r0 = item_row(is_v ? j - n : j), rows = min(Q4_ROWS, rows_alloc - (int)r0);      // (a multiple of eight)
    const uint32_t bar = full_a + 8 * slot, dst = ring_a + slot * ITEM;
    bar_expect(bar, rows * (CODES + PARAMS));
    bulk_load(dst, (is_v ? vc : kc) + (uint64_t)r0 * CODES, rows * CODES, bar);
    bulk_load(dst + Q4_ROWS * CODES, (is_v ? vp : kp) + (uint64_t)r0 * PARAMS, rows * PARAMS, bar);
  };
  const int n_alloc = wid < WARPS ? items_in(rows_alloc) : 0, early = min(depth, n_alloc), ahead = min(depth, 2 * n_alloc);
  if (elected())
    for (int j = 0; j < early; ++j) request(j, n_alloc, j);
  __syncwarp();

  // Nothing but K rows is read before the previous launch has completed.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int len_m = c.state.len[u], fs_m = c.state.free_slot[u], t = c.state.next_pos[u], ls = c.state.last_slot[u];
  // q for the B operand of K q^T, requested along with the words above.  Lane (n = r8, t4): channels 8 t4 .. 8 t4 + 7 of groups of its column.
  // INT: columns 0 - 3 are the four digits of group 0 (then of group 2), columns 4 - 7 of group 1 (3).  Else: column n is head n.
  constexpr int QG = INT ? NG / 2 : NG;      // (INT: every second group)
  Raw8<T> q_raw[QG];
  if (wid < WARPS) {
    const T* qp = q_new + ((int64_t)u * G + (INT ? 0 : min(r8, G - 1))) * HD + 32 * (INT ? r8 >> 2 : 0) + 8 * t4;
#pragma unroll
    for (int g = 0; g < QG; ++g) q_raw[g].load(qp + (INT ? 64 : 32) * g);
    // the ring's first items of V, while these loads are under way
    if (elected())
      for (int j = early; j < ahead; ++j) request(j, n_alloc, j);
    __syncwarp();
  }

  if (wid == WARPS) {
    // ---- the last warp: the incoming token.  Lane l < HD / 4 has channels 4 l .. 4 l + 3.
    float kv[2][4], qv[GT][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      kv[0][e] = kv[1][e] = 0.f;
#pragma unroll
      for (int h = 0; h < GT; ++h) qv[h][e] = 0.f;
    }
    if (lane < HD / 4) {
      load_new(k_new + (int64_t)u * HD + 4 * lane, kv[0]);
      load_new(v_new + (int64_t)u * HD + 4 * lane, kv[1]);
#pragma unroll
      for (int h = 0; h < GT; ++h)
        if (h < G) load_new(q_new + ((int64_t)u * G + h) * HD + 4 * lane, qv[h]);
    }
    const int len = min(max(len_m, 0), cap - 1), fs_local = min(max(fs_m, 0), cap - 1) - s0;
    const int cnt = max(min(len + 1 - s0, rows_all), 0);
    const bool owns = fs_local >= 0 && fs_local < cnt;
    float m[GT], l[GT], o[GT][4];
#pragma unroll
    for (int h = 0; h < GT; ++h) {
      m[h] = -INFINITY;
      l[h] = o[h][0] = o[h][1] = o[h][2] = o[h][3] = 0.f;
    }
    auto take = [&](int row) {             // the row whose values are in kv: logits, running maxima, sums and outputs
#pragma unroll
      for (int h = 0; h < GT; ++h) {
        if (GT > 1 && h >= G) continue;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fmaf(qv[h][e], kv[0][e], s);      // (zeros from lane HD / 4 on)
#pragma unroll
        for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= scale_log2;
        if (lane == 0) logit_s[h * ld + row] = s;
        const float m_new = fmaxf(m[h], s), f = exp2_fast(m[h] - m_new), p = exp2_fast(s - m_new);
        m[h] = m_new;
        l[h] = fmaf(l[h], f, p);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[h][e] = fmaf(o[h][e], f, p * kv[1][e]);
      }
    };
    if (owns) {
      float nv = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) nv = norm_fold(norm, nv, kv[1][e]);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t par;
        const uint32_t code = q4_row(kv[x], par);
        if (lane < HD / 4 && VATP_INB(s0 + fs_local, cap, dev_status)) {
          unsigned char* row = static_cast<unsigned char*>(x ? c.state.v_cache : c.state.k_cache) + (base + fs_local) * CODES;
          *reinterpret_cast<uint16_t*>(row + q4_byte<HD>(lane >> 3, lane & 7)) = (uint16_t)code;
          if ((lane & 7) == 0) static_cast<uint32_t*>(x ? c.v_params : c.k_params)[(base + fs_local) * NG + (lane >> 3)] = par;
        }
        // the values as stored
#pragma unroll
        for (int e = 0; e < 4; ++e) kv[x][e] = fmaf((float)(code >> (4 * e) & 15u), q4_scale(par), q4_low(par));
      }
      take(fs_local);
#pragma unroll
      for (int x = 16; x; x >>= 1) nv = norm_merge(norm, nv, __shfl_xor_sync(0xffffffffu, nv, x));
      nv = norm_finish(norm, nv);
      if (lane == 0) {
        new_norm_s = nv;
        c.state.vnorm[base + fs_local] = nv;
      }
    }
    for (int row = rows_alloc; row < cnt; ++row) {
      if (row == fs_local) continue;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t code = 0, par = 0;
        if (lane < HD / 4) {
          const int b = q4_byte<HD>(lane >> 3, lane & 7);
          code = load_fresh(reinterpret_cast<const uint32_t*>((x ? vc : kc) + (int64_t)row * CODES + (b & ~3))) >> (8 * (b & 2));
          par = load_fresh(reinterpret_cast<const uint32_t*>((x ? vp : kp) + (int64_t)row * PARAMS) + (lane >> 3));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) kv[x][e] = fmaf((float)(code >> (4 * e) & 15u), q4_scale(par), q4_low(par));
      }
      take(row);
    }
    if (lane == 0) {
#pragma unroll
      for (int h = 0; h < GT; ++h)
        if (GT == 1 || h < G) part_m[WARPS][h] = m[h];
      bar_arrive(s32(&k_done));
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (!bar_wait(s32(&k_done), 0)) bad = true;
#pragma unroll
    for (int h = 0; h < GT; ++h) {
      if (GT > 1 && h >= G) continue;
      float top = m[h];
#pragma unroll
      for (int k = 0; k < WARPS; ++k) top = fmaxf(top, part_m[k][h]);
      const float f = m[h] > -INFINITY ? exp2_fast(m[h] - top) : 0.f;
      if (lane == 0) part_l[WARPS][h] = l[h] * f;
      if (lane < HD / 4) *reinterpret_cast<float4*>(new_o + h * HD + 4 * lane) = make_float4(o[h][0] * f, o[h][1] * f, o[h][2] * f, o[h][3] * f);
    }
  }

  const int len = min(max(len_m, 0), cap - 1), fs = min(max(fs_m, 0), cap - 1);
  const int hi = len + 1;                // slots [0, hi) are live once the new token is in
  const int cnt = max(min(hi - s0, rows_all), 0), cnt_t = min(cnt, rows_alloc);      // live slots, and those in tiles
  const int fs_local = fs - s0, ls_local = ls - s0;
  constexpr int SB = 2;                  // slots of a thread whose state is in registers at a time
  float old_r[SB], norm_r[SB];
  int pos_r[SB];
  long long fx_r[WINDOWED ? SB : 1];
  const float* old_g = WINDOWED ? c.state.ring + ((int64_t)u * w + (t % w)) * cap + s0 : c.state.acc + base;
  auto fetch = [&](int i0) {
#pragma unroll
    for (int k = 0; k < SB; ++k) {
      const int i = i0 + k * WORKERS;
      old_r[k] = norm_r[k] = 0.f;
      pos_r[k] = 0;
      if (WINDOWED) fx_r[k] = 0;
      if (i < cnt) {
        old_r[k] = old_g[i];
        norm_r[k] = c.state.vnorm[base + i];
        pos_r[k] = c.state.pos[base + i];
        if (WINDOWED) fx_r[k] = c.state.acc_fixed[base + i];
      }
    }
  };

  if (wid < WARPS) {
    // ---- the row that the launch ahead appended, if one of this warp's early items of K holds it
    const int n = items_in(cnt_t);
    int ls_item = -1;                         // that item
    uint32_t ls_word = 0u;                    // that row (lanes below CODES / 4: codes, then parameters)
    if (n == n_alloc && ls >= 0 && ls != fs && ls_local >= 0 && ls_local < cnt_t && ls_local / Q4_ROWS % WARPS == wid) {
      ls_item = ls_local / (Q4_ROWS * WARPS);
      if (lane < CODES / 4) ls_word = load_fresh(reinterpret_cast<const uint32_t*>(kc + (int64_t)ls_local * CODES) + lane);
      else if (lane < CODES / 4 + NG) ls_word = load_fresh(reinterpret_cast<const uint32_t*>(kp + (int64_t)ls_local * PARAMS) + (lane - CODES / 4));
    }

    // ---- B operand of K q^T
    uint32_t qb[NG][INT ? 2 : 4], qr[GT > 1 && Q_REST ? NG : 1][4];
    // what a sum is to be multiplied by (INT: of the lane's two digits); sums of q over groups, * scale
    float q_back[2], qsum[INT ? NG / 2 : NG][2];
    {
      float q[QG][8], most = 0.f, gs[QG];
#pragma unroll
      for (int g = 0; g < QG; ++g) q_raw[g].get(q[g]);
#pragma unroll
      for (int g = 0; g < QG; ++g) {
        gs[g] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          most = fmaxf(most, fabsf(q[g][e]));
          gs[g] += q[g][e];
        }
        gs[g] += __shfl_xor_sync(0xffffffffu, gs[g], 1);
        gs[g] += __shfl_xor_sync(0xffffffffu, gs[g], 2);
        gs[g] *= scale_log2;
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1)
        if (!INT) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      if (INT) most = max_of(most);
      const int ex = min(max((int)(__float_as_uint(most) >> 23) - 126, -90), 100);      // 2^ex is above the largest magnitude
      if constexpr (INT) {
        // Q = q 2^(25 - ex) as an integer; byte lo + 16 hi of a row by 16 Q_lo, its upper half 16 hi by Q_hi - 16 Q_lo
        const float up = __uint_as_float((uint32_t)(25 - ex + 127) << 23);
        const uint32_t sel = (uint32_t)(r8 & 3) | (uint32_t)((r8 & 3) + 4) << 4;      // this column's digit of two words
#pragma unroll
        for (int g = 0; g < NG; ++g) qb[g][0] = qb[g][1] = 0u;
#pragma unroll
        for (int g = 0; g < QG; ++g) {
          uint32_t w[2][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int lo = __float2int_rn(q[g][2 * i] * up), hi = __float2int_rn(q[g][2 * i + 1] * up);
            w[0][i] = (uint32_t)(16 * lo) + 0x80808080u;          // (signed digits: a byte each, 128 too large)
            w[1][i] = (uint32_t)(hi - 16 * lo) + 0x80808080u;
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t b = __byte_perm(__byte_perm(w[x][0], w[x][1], sel), __byte_perm(w[x][2], w[x][3], sel), 0x5410u) ^ 0x80808080u;
            if (r8 < 4) qb[2 * g][x] = b;
            else qb[2 * g + 1][x] = b;
          }
          qsum[g][0] = __shfl_sync(0xffffffffu, gs[g], 16 * (t4 >> 1));      // of group 2 g + t4 / 2, in the even lanes
          if (t4 & 1) qsum[g][0] = 0.f;
          qsum[g][1] = 0.f;
        }
        // (integers do not hold what is not finite: the logits become NaN)
        const float back = most < INFINITY ? __uint_as_float((uint32_t)(ex - 29 + 127) << 23) * scale_log2 : __uint_as_float(0x7fff0000u);
        q_back[0] = t4 & 1 ? back * 65536.f : back;
        q_back[1] = q_back[0] * 256.f;
      } else {
        // q to [2^13, 2^14) by a power of two, as a high half and a remainder
        const float up = __uint_as_float((uint32_t)(14 - ex + 127) << 23), back = __uint_as_float((uint32_t)(ex + CODE_EXP - 14 + 127) << 23) * scale_log2;
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float p0 = q[g][x] * up, p1 = q[g][x + 4] * up;
            const __half2 h = __floats2half2_rn(p0, p1);
            qb[g][x] = *reinterpret_cast<const uint32_t*>(&h);
            if constexpr (Q_REST) qr[g][x] = half2_of(p0 - __low2float(h), p1 - __high2float(h));
          }
        // (an accumulator's columns are heads 2 t4 and 2 t4 + 1; their sums are with the lanes of those columns)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          q_back[x] = __shfl_sync(0xffffffffu, back, 4 * (2 * t4 + x));
#pragma unroll
          for (int g = 0; g < NG; ++g) qsum[g][x] = __shfl_sync(0xffffffffu, gs[g], 4 * (2 * t4 + x));
        }
      }
    }

    // ---- the ring: the next item's slot, place and the parity of its barrier; the next item to request
    int slot = 0, next = ahead;
    uint32_t par = 0;
    const unsigned char* item = ring;
    auto arrived = [&]() {
      if (!bar_try(full_a + 8 * slot, par) && !bad && !bar_wait(full_a + 8 * slot, par)) bad = true;
    };
    auto release = [&]() {                    // every lane has read the item: its slot takes the next one
      __syncwarp();
      // (with one head per cache the elected lane's code takes registers that it does not have: 128 x 1025 slots 10.2 -> 11.0 us; with four
      // heads 8 x 13108 18.0 -> 17.5)
      if (next < 2 * n && (GT == 1 ? lane == 0 : elected())) request(next, n, slot);
      ++next;
      item += ITEM;
      if (++slot == depth) { slot = 0; item = ring; par ^= 1; }
    };
    if (n != n_alloc) {                       // fewer tokens than there is room for: what was requested early is dropped
      next = 2 * n;
      for (int j = 0; j < ahead; ++j) { arrived(); release(); }
      next = min(depth, 2 * n);
      if (lane == 0 && !bad)
        for (int j = 0; j < next; ++j) request(j, n, (slot + j) % depth);
      __syncwarp();
    }
    auto patch = [&](int j, uint32_t word) {  // item j of the ring
      if (j < early) {
        unsigned char* to = ring + slot * ITEM;
        const int r = ls_local % Q4_ROWS;
        if (lane < CODES / 4) reinterpret_cast<uint32_t*>(to + r * CODES)[lane] = word;
        else if (lane < CODES / 4 + NG) reinterpret_cast<uint32_t*>(to + Q4_ROWS * CODES + r * PARAMS)[lane - CODES / 4] = word;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (before the next bulk copy into the slot)
        __syncwarp();
      }
    };

    // ---- logits of this warp's tiles and their maximum
    constexpr int MX = GT > 1 ? 2 : 1;
    float m_run[MX];
#pragma unroll
    for (int x = 0; x < MX; ++x) m_run[x] = -INFINITY;
    // rows r0 + r8 + 8 k, k < 2 N, from tile `a0` of the item on
    auto k_rows = [&](int r0, int a0) {
      uint32_t kw[2 * N][KW], pr[2 * N][KP];
      const unsigned char* codes = item + (a0 * Q4_TILE + r8) * CODES + t4 * (HD / 8);
      const unsigned char* params = item + Q4_ROWS * CODES + (a0 * Q4_TILE + r8) * PARAMS;
#pragma unroll
      for (int k = 0; k < 2 * N; ++k) {
        words_of(codes + 8 * k * CODES, kw[k]);
        if constexpr (INT) {
#pragma unroll
          for (int f = 0; f < KP; ++f)       // of groups t4 / 2 and t4 / 2 + 2
            pr[k][f] = *reinterpret_cast<const uint32_t*>(params + 8 * k * PARAMS + 4 * (t4 >> 1) + 8 * f);
        } else {
          words_of(params + 8 * k * PARAMS, pr[k]);
        }
      }
      if (a0 + N == 2) release();
      if constexpr (INT) {
        int d[N][KP][4];                     // groups 2 f (columns 0 - 3) and 2 f + 1 (columns 4 - 7)
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int a = 0; a < N; ++a) {
            // words of chunks 2 t4 (first half of the lane's words) and 2 t4 + 1; a half word is a group
            const uint32_t sel = g & 1 ? 0x7632u : 0x5410u;
            const uint32_t xa = __byte_perm(kw[2 * a][g >> 1], kw[2 * a][KW / 2 + (g >> 1)], sel), xb = __byte_perm(kw[2 * a + 1][g >> 1], kw[2 * a + 1][KW / 2 + (g >> 1)], sel);
            // (sums start at the float 1.5 * 2^23 as an integer: below 2^20, they are that float's low bits)
            if (g & 1) mma_s8(d[a][g >> 1], xa, xb, xa & 0xf0f0f0f0u, xb & 0xf0f0f0f0u, qb[g][0], qb[g][1]);
            else mma_s8(d[a][g >> 1], xa, xb, xa & 0xf0f0f0f0u, xb & 0xf0f0f0f0u, qb[g][0], qb[g][1], 0x4b400000);
          }
        float s[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          s[k] = 0.f;
#pragma unroll
          for (int f = 0; f < KP; ++f) {
            const float d0 = __int_as_float(d[k >> 1][f][2 * (k & 1)]) - 12582912.f, d1 = __int_as_float(d[k >> 1][f][2 * (k & 1) + 1]) - 12582912.f;
            s[k] = fmaf(q4_scale(pr[k][f]), fmaf(d1, q_back[1], d0 * q_back[0]), s[k]);
            s[k] = fmaf(q4_low(pr[k][f]), qsum[f][0], s[k]);
          }
        }
        // the four lanes of a row hold parts of its sum; lane t4 ends up with row r8 + 8 t4
        const bool odd = t4 & 1, up = t4 & 2;
        float a = odd ? s[1] : s[0], b = odd ? s[3] : s[2];
        a += __shfl_xor_sync(0xffffffffu, odd ? s[0] : s[1], 1);
        b += __shfl_xor_sync(0xffffffffu, odd ? s[2] : s[3], 1);
        float x = (up ? b : a) + __shfl_xor_sync(0xffffffffu, up ? a : b, 2);
        const int row = r0 + r8 + 8 * t4;
        if (row >= cnt_t || row == fs_local) x = -INFINITY;      // (the incoming token's slot is the last warp's)
        if (row < cnt_t && row != fs_local) logit_s[row] = x;
        m_run[0] = fmaxf(m_run[0], x);
      } else {
        float acc[N][NG][4];
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int a = 0; a < N; ++a) {
            const uint32_t sel = g & 1 ? 0x7632u : 0x5410u;
            const uint32_t xa = __byte_perm(kw[2 * a][g >> 1], kw[2 * a][KW / 2 + (g >> 1)], sel), xb = __byte_perm(kw[2 * a + 1][g >> 1], kw[2 * a + 1][KW / 2 + (g >> 1)], sel);
            float(&d)[4] = acc[a][g];
            d[0] = d[1] = d[2] = d[3] = 0.f;
            mma_f16(d, codes0(xa), codes0(xb), codes1(xa), codes1(xb), qb[g][0], qb[g][1]);
            mma_f16(d, codes2(xa), codes2(xb), codes3(xa), codes3(xb), qb[g][2], qb[g][3]);
            if constexpr (Q_REST) {
              mma_f16(d, codes0(xa), codes0(xb), codes1(xa), codes1(xb), qr[g][0], qr[g][1]);
              mma_f16(d, codes2(xa), codes2(xb), codes3(xa), codes3(xb), qr[g][2], qr[g][3]);
            }
          }
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) {
          const int row = r0 + r8 + 8 * k;
          const bool live = row < cnt_t && row != fs_local;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float d = 0.f, l = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              d = fmaf(q4_scale(pr[k][g]), acc[k >> 1][g][2 * (k & 1) + x], d);
              l = fmaf(q4_low(pr[k][g]), qsum[g][x], l);
            }
            const float s = live ? fmaf(d, q_back[x], l) : -INFINITY;
            const int h = 2 * t4 + x;
            if (h < G && live) logit_s[h * ld + row] = s;
            m_run[x] = fmaxf(m_run[x], s);
          }
        }
      }
    };
    for (int j = 0; j < n; ++j) {
      arrived();
      if (j == ls_item) patch(j, ls_word);
      const int r0 = item_row(j);
#pragma unroll 1
      for (int a = 0; a < 2; a += N) k_rows(r0 + a * Q4_TILE, a);
    }
    // (after the wait: at most one unfinished predecessor exists while a successor sets up)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
#pragma unroll
    for (int x = 0; x < MX; ++x) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1)
        if (!INT) m_run[x] = fmaxf(m_run[x], __shfl_xor_sync(0xffffffffu, m_run[x], o));
      if (INT) m_run[x] = max_of(m_run[x]);
      const int h = GT > 1 ? 2 * t4 + x : 0;
      if (r8 == 0 && (GT > 1 ? h < G : t4 == 0)) part_m[wid][h] = m_run[x];
    }
    __syncwarp();
    if (lane == 0) bar_arrive(s32(&k_done));

    // ---- O^T += V^T (p sc): A = codes (16 channels x 16 or 32 slots), B = p sc by slot and head, scaled by a power of two to fit fp16
    // (2^(13 - J)) or 32-bit integers (2^(29 - J)).  J follows the largest log2 of p sc (rounded up; p relative to the warp's maximum) with
    // a slack of 2^2; when it moves, what has been summed up is rescaled (a power of two).
    constexpr int X_TOP = INT ? 29 : 13;
    float o_acc[NG][2][4];                   // INT: [group][0]: channels 4 r8 .. + 3 of the group, of this lane's digits
    int o_int[INT ? NG : 1][2][4];           // sums over codes lo + 16 hi of a byte, and over 16 hi
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        o_acc[g][i][0] = o_acc[g][i][1] = o_acc[g][i][2] = o_acc[g][i][3] = 0.f;
        if (INT) o_int[g][i][0] = o_int[g][i][1] = o_int[g][i][2] = o_int[g][i][3] = 0;
      }
    // this warp's maxima, rounded up to integers (0 without a live slot): p is taken relative to them, and what it is scaled by is a power of two
    // (in one exponential with s, 2^29 p would have lost eight bits); of this lane's slots (and groups): sum of p, sum of p lo
    float m_own[GT], l_run[GT], lo_run[GT][PG];
    int J[GT];
#pragma unroll
    for (int h = 0; h < GT; ++h) {
      m_own[h] = GT == 1 || h < G ? ceilf(part_m[wid][h]) : 0.f;
      if (m_own[h] == -INFINITY) m_own[h] = 0.f;
      l_run[h] = 0.f;
      J[h] = Q4_NO_J;
#pragma unroll
      for (int i = 0; i < PG; ++i) lo_run[h][i] = 0.f;
    }
    // N tiles of an item from tile a0 on.  Lane: slot `lane` of the item and all of its groups, or (N == 1) slot lane / 2 of the tile and
    // half of the groups.
    const int my_slot_in = N == 2 ? lane : lane >> 1, my_group = N == 2 ? 0 : (lane & 1) * VW;
    const int x_at = (N == 2 ? (lane >> 4) * (INT ? Q4_TILE : NG * XC * Q4_TILE) : 0) + 4 * (my_slot_in & 3) + (my_slot_in >> 2 & 3);
    bool last = n == 0;                      // (INT: one round more, which only takes the integer sums over)
    const float digits = t4 & 1 ? 65536.f : 1.f;
    auto v_rows = [&](int j, int a0) {
      const int row = item_row(j) + a0 * Q4_TILE + my_slot_in;
      const bool live = row < cnt_t && row != fs_local && !last;
      float s[GT];
      uint32_t pr[PG];
      bool moved = last || (INT && j % (Q4_FLUSH / Q4_ROWS) == Q4_FLUSH / Q4_ROWS - 1);
      float f[GT];
      if (!last) {
#pragma unroll
        for (int h = 0; h < GT; ++h) s[h] = GT == 1 || h < G ? logit_s[h * ld + row] : -INFINITY;
        words_of(item + Q4_ROWS * CODES + (a0 * Q4_TILE + my_slot_in) * PARAMS + 4 * my_group, pr);
      }
      if (!live) {                           // (its logit is another's, or nobody's; its parameters may be anything)
#pragma unroll
        for (int h = 0; h < GT; ++h) s[h] = -INFINITY;
#pragma unroll
        for (int i = 0; i < PG; ++i) pr[i] = 0u;
      }
      // 126 + exponent of the largest scale, rounded up (scales below 2^-94 count as that: with J 2 less, 2^(J - 29) is then still a normal number)
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < PG; ++i) most = fmaxf(most, q4_scale(pr[i]));
      const int ev = max((int)(__float_as_uint(most) >> 23), 32);
#pragma unroll
      for (int h = 0; h < GT; ++h) {
        f[h] = 1.f;
        if (GT == 1 || h < G) {
          s[h] -= m_own[h];                  // log2 p: not above 0, -inf for a slot that is not live
          const int top = __reduce_max_sync(0xffffffffu, __float2int_ru(s[h]) + ev);      // (-inf: the least integer)
          if (top > J[h] + 2) {
            f[h] = exp2_fast((float)(J[h] - top));
            J[h] = top;
            moved = true;
          }
        }
      }
      if (moved && (!INT || j > 0)) {        // (INT, j = 0: nothing has been summed up)
        if constexpr (INT) {
          // The integer sums go into the float ones: a lane's two digits make one number, below 2^31 for up to Q4_FLUSH slots of a warp.
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int h0 = o_int[g][1][2 * i], h1 = o_int[g][1][2 * i + 1];
              o_acc[g][0][2 * i] = f[0] * fmaf((float)((o_int[g][0][2 * i] - h0) + 256 * (o_int[g][0][2 * i + 1] - h1)), digits, o_acc[g][0][2 * i]);
              o_acc[g][0][2 * i + 1] = f[0] * fmaf((float)((h0 >> 4) + 16 * h1), digits, o_acc[g][0][2 * i + 1]);
              o_int[g][0][2 * i] = o_int[g][0][2 * i + 1] = o_int[g][1][2 * i] = o_int[g][1][2 * i + 1] = 0;
            }
        } else {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float fx = f[0];                 // of column 2 t4 + x
#pragma unroll
            for (int h = 1; h < GT; ++h) fx = (GT > 4 ? 2 * t4 + x : t4) == h ? f[h] : fx;
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
              for (int i = 0; i < 2; ++i) { o_acc[g][i][x] *= fx; o_acc[g][i][2 + x] *= fx; }
          }
        }
      }
      if (last) return;
      uint32_t vw[N][4][VW];
#pragma unroll
      for (int a = 0; a < N; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i) words_of(item + ((a0 + a) * Q4_TILE + 4 * i + t4) * CODES + r8 * (HD / 16), vw[a][i]);
#pragma unroll
      for (int h = 0; h < GT; ++h)
        if (GT == 1 || h < G) {
          // (a NaN stays one, and the sums with it)
          const float p = exp2_fast(s[h]), y = p * pow2(126 + X_TOP - J[h]);
          l_run[h] += p;
#pragma unroll
          for (int i = 0; i < PG; ++i) {
            lo_run[h][i] = fmaf(p, q4_low(pr[i]), lo_run[h][i]);
            if constexpr (INT) {             // a column for each byte
              const uint32_t X = __float2uint_rn(y * q4_scale(pr[i]));
              unsigned char* to = xs[wid] + (my_group + i) * 4 * 2 * Q4_TILE + x_at;
#pragma unroll
              for (int d = 0; d < 4; ++d) to[d * 2 * Q4_TILE] = (unsigned char)(X >> (8 * d));
            } else if ((i & 1) == 0) {
              const int i1 = PG > 1 ? i + 1 : i;
              const float x0 = y * q4_scale(pr[i]), x1 = y * q4_scale(pr[i1]);
              const __half2 hh = __floats2half2_rn(x0, x1);
              uint16_t* to = reinterpret_cast<uint16_t*>(xs[wid]) + ((my_group + i) * XC + x_col(h, 0)) * Q4_TILE + x_at;
              to[0] = __half_as_ushort(__low2half(hh));
              if (PG > 1) to[XC * Q4_TILE] = __half_as_ushort(__high2half(hh));
              const __half2 hl = __floats2half2_rn(x0 - __low2float(hh), x1 - __high2float(hh));
              to += (x_col(h, 1) - x_col(h, 0)) * Q4_TILE;
              to[0] = __half_as_ushort(__low2half(hl));
              if (PG > 1) to[XC * Q4_TILE] = __half_as_ushort(__high2half(hl));
            }
          }
        }
      if (a0 + N == 2) release();            // (with a barrier of the warp)
      else __syncwarp();
      if constexpr (INT) {
        // bytes of four slots side by side: a lane's words of slots t4, t4 + 4, t4 + 8, t4 + 12, transposed
        uint32_t tr[N][VW][4];
#pragma unroll
        for (int a = 0; a < N; ++a)
#pragma unroll
          for (int x = 0; x < VW; ++x) {
            const uint32_t p0 = __byte_perm(vw[a][0][x], vw[a][1][x], 0x5140u), p1 = __byte_perm(vw[a][2][x], vw[a][3][x], 0x5140u);
            const uint32_t p2 = __byte_perm(vw[a][0][x], vw[a][1][x], 0x7362u), p3 = __byte_perm(vw[a][2][x], vw[a][3][x], 0x7362u);
            tr[a][x][0] = __byte_perm(p0, p1, 0x5410u);
            tr[a][x][1] = __byte_perm(p0, p1, 0x7632u);
            tr[a][x][2] = __byte_perm(p2, p3, 0x5410u);
            tr[a][x][3] = __byte_perm(p2, p3, 0x7632u);
          }
        const uint32_t* xw = reinterpret_cast<const uint32_t*>(xs[wid]) + (r8 & 3) * 2 * Q4_TILE / 4 + t4;      // (columns from 4 on are not used)
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          // rows 0 - 7: the group's first byte (channels 4 r8, + 1), rows 8 - 15: its second
          const uint32_t b0 = xw[g * 2 * Q4_TILE], b1 = xw[g * 2 * Q4_TILE + Q4_TILE / 4];
          const uint32_t a0 = tr[0][g >> 1][2 * (g & 1)], a1 = tr[0][g >> 1][2 * (g & 1) + 1], a2 = tr[1][g >> 1][2 * (g & 1)], a3 = tr[1][g >> 1][2 * (g & 1) + 1];
          mma_u8(o_int[g][0], a0, a1, a2, a3, b0, b1);
          mma_u8(o_int[g][1], a0 & 0xf0f0f0f0u, a1 & 0xf0f0f0f0u, a2 & 0xf0f0f0f0u, a3 & 0xf0f0f0f0u, b0, b1);
        }
      } else {
#pragma unroll
        for (int a = 0; a < N; ++a)
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const uint16_t* xh = reinterpret_cast<const uint16_t*>(xs[wid]) + ((a * NG + g) * XC + r8) * Q4_TILE + 4 * t4;
            const uint2 b = *reinterpret_cast<const uint2*>(xh);
            const uint32_t sel = g & 1 ? 0x7632u : 0x5410u;
            const uint32_t xa = __byte_perm(vw[a][0][g >> 1], vw[a][1][g >> 1], sel), xb = __byte_perm(vw[a][2][g >> 1], vw[a][3][g >> 1], sel);
            mma_f16(o_acc[g][0], codes0(xa), codes1(xa), codes0(xb), codes1(xb), b.x, b.y);
            mma_f16(o_acc[g][1], codes2(xa), codes3(xa), codes2(xb), codes3(xb), b.x, b.y);
            if constexpr (GT > 4) {
              const uint2 d = *reinterpret_cast<const uint2*>(xh + 8 * Q4_TILE);
              mma_f16(o_acc[g][0], codes0(xa), codes1(xa), codes0(xb), codes1(xb), d.x, d.y);
              mma_f16(o_acc[g][1], codes2(xa), codes3(xa), codes2(xb), codes3(xb), d.x, d.y);
            }
          }
      }
      __syncwarp();
    };
    for (int j = 0; !last; ++j) {
      if (j < n) {
        arrived();
      }
      last = j == n;
      if (last && !INT) break;
#pragma unroll 1
      for (int a = 0; a < 2; a += N) v_rows(j, a);
    }
    fetch(tid);
    // ---- the warp's partial, relative to the CTA's maximum: sums of p (even lanes) and of p lo, and O^T with its constant factor,
    // into the ring
    if (!bad && !bar_wait(s32(&k_done), 0)) bad = true;
    __syncwarp();
    constexpr int COLS = GT > 4 ? 2 : 1;     // heads of this lane's columns of the accumulators: 2 t4 + x or t4
    float fm[COLS], fo[COLS];                // factors of its sums of p and of its outputs
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      const int hc = GT == 1 ? 0 : COLS * t4 + x;
      float mo = m_own[0], m = part_m[0][hc];
      int j = J[0];
#pragma unroll
      for (int h = 1; h < GT; ++h)
        if (h == hc) { mo = m_own[h]; j = J[h]; }
#pragma unroll
      for (int k = 1; k <= WARPS; ++k) m = fmaxf(m, part_m[k][hc]);
      const bool any = hc < G && part_m[wid][hc] > -INFINITY;
      fm[x] = any ? exp2_fast(mo - m) : 0.f;
      fo[x] = any ? fm[x] * pow2(j - 126 - X_TOP + (INT ? 0 : CODE_EXP)) : 0.f;
    }
    {
      constexpr int LOW = N == 2 ? 1 : 2;    // (neighbouring lanes have halves of a slot's groups with N == 1)
      sum_over<GT, LOW>(l_run, lane);
      float lo_all[GT * PG];
#pragma unroll
      for (int h = 0; h < GT; ++h)
#pragma unroll
        for (int i = 0; i < PG; ++i) lo_all[h * PG + i] = lo_run[h][i];
      sum_over<GT * PG, LOW>(lo_all, lane);
      constexpr int L_LANES = 32 / GT, LO_LANES = 32 / (GT * PG);
      const int hl = lane / L_LANES, ho = lane / LO_LANES / PG, io = lane / LO_LANES % PG;
      float fl = __shfl_sync(0xffffffffu, fm[0], hl / COLS), fi = __shfl_sync(0xffffffffu, fm[0], ho / COLS);
      if (COLS > 1) {
        const float fl1 = __shfl_sync(0xffffffffu, fm[COLS - 1], hl / COLS), fi1 = __shfl_sync(0xffffffffu, fm[COLS - 1], ho / COLS);
        if (hl & 1) fl = fl1;
        if (ho & 1) fi = fi1;
      }
      if (lane % L_LANES == 0) part_l[wid][hl] = l_run[0] * fl;
      if (lane % LO_LANES < LOW) part_lo[wid][ho][my_group + io] = lo_all[0] * fi;
    }
    float* po = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int x = 0; x < (GT > 4 ? 2 : 1); ++x) {
      const int h = GT > 4 ? 2 * t4 + x : t4;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {        // channel 4 r8 + i of the group
          if constexpr (INT) {
            o[i] = o_acc[g][0][i] + __shfl_xor_sync(0xffffffffu, o_acc[g][0][i], 1);      // (the upper digits' columns)
            o[i] *= fo[0];
          } else {                           // the remainder's column beside the head's
            o[i] = GT > 4 ? o_acc[g][i >> 1][2 * (i & 1) + x] : o_acc[g][i >> 1][2 * (i & 1)] + o_acc[g][i >> 1][2 * (i & 1) + 1];
            o[i] *= fo[x];
          }
        }
        if (h < G) *reinterpret_cast<float4*>(po + h * HD + 32 * g + 4 * r8) = make_float4(o[0], o[1], o[2], o[3]);
      }
    }
  }
  __syncthreads();
  if (split > 1) cluster_wait_acquire();

  // ---- to the unit's CTAs: maximum and sum to every one, channel slice r of the partial output to rank r
  if (tid < split * G) {
    const int h = tid / split, dst = tid - h * split;
    float m = part_m[WARPS][h], l = part_l[WARPS][h];
#pragma unroll
    for (int k = 0; k < WARPS; ++k) {
      m = fmaxf(m, part_m[k][h]);
      l += part_l[k][h];
    }
    send2(at_rank(s32(&ex_ml[rank][h]), dst), m, l, at_rank(s32(&ex_bar), dst));
  }
  for (int i = tid; i < G * HD; i += THREADS) {
    const int h = i / HD, ch = i - h * HD;
    float a = new_o[i];
#pragma unroll
    for (int k = 0; k < WARPS; ++k) a += reinterpret_cast<const float*>(dyn + (size_t)k * ring_bytes)[i] + part_lo[k][h][ch >> 5];
    const int dst = ch >> slice_log2;
    send(at_rank(s32(&xo[(rank * G + h) * slice + (ch & (slice - 1))]), dst), a, at_rank(s32(&ex_bar), dst));
  }
  if (!bar_wait(s32(&ex_bar), 0)) bad = true;

  // ---- every CTA: the unit's normaliser (all data is local now) and its slice of the output.  Lane r has CTA r's maximum and sum.
  float m_all = -INFINITY, inv_all = 0.f, fr = 0.f;      // of the one head (all warps), or of head `wid`
  if (GT == 1 || wid < G) {
    const float2 ml = lane < split ? ex_ml[lane][GT == 1 ? 0 : wid] : make_float2(-INFINITY, 0.f);
    m_all = max_of(ml.x);
    fr = ml.x > -INFINITY ? exp2_fast(ml.x - m_all) : 0.f;
    float L = ml.y * fr;
#pragma unroll
    for (int o = Q4_SPLIT / 2; o; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
    inv_all = 1.f / __shfl_sync(0xffffffffu, L, 0);
  }
  if constexpr (GT == 1) {
    if (writes && wid * 32 < slice) {
      float a = 0.f;
      for (int r = 0; r < split; ++r) a = fmaf(xo[r * slice + min(tid, slice - 1)], __shfl_sync(0xffffffffu, fr, r), a);
      if (tid < slice) to_out(out + (int64_t)u * HD + rank * slice + tid, a * inv_all);
    }
  } else {
    if (wid < G) {
      if (lane < split) fr_s[lane][wid] = fr;
      if (lane == 0) { all_m[wid] = m_all; all_inv[wid] = inv_all; }
    }
    __syncthreads();
    for (int i = tid; i < (writes ? G * slice : 0); i += THREADS) {
      const int h = i >> slice_log2, ch = i & (slice - 1);
      float a = 0.f;
      for (int r = 0; r < split; ++r) a = fmaf(xo[(r * G + h) * slice + ch], fr_s[r][h], a);
      to_out(out + ((int64_t)u * G + h) * HD + rank * slice + ch, a * all_inv[h]);
    }
  }

  // ---- indicator update (Eq. 2 / Eq. 3) and importance (Eq. 4) of this CTA's slots, every warp's arg-min to rank 0
  const bool evicting = hi > B;
  if (wid < WARPS) {
    unsigned long long my_key = Q4_NO_KEY;
    int my_slot = -1, my_pos = -1;
    for (int i0 = tid; i0 < cnt;) {
#pragma unroll
      for (int k = 0; k < SB; ++k) {
        const int i = i0 + k * WORKERS;
        if (i >= cnt) continue;
        float p;
        if constexpr (GT == 1) {
          p = exp2_fast(logit_s[i] - m_all) * inv_all;
        } else {                             // the mean of the heads' probabilities
          p = 0.f;
#pragma unroll
          for (int h = 0; h < GT; ++h)
            if (h < G) p = fmaf(exp2_fast(logit_s[h * ld + i] - all_m[h]), all_inv[h], p);
          p /= (float)G;
        }
        const bool is_new = i == fs_local;
        const int64_t o = base + i;
        float S;
        if (WINDOWED) {
          const long long fx = is_new ? prob_to_fixed(p) : fx_r[k] + prob_to_fixed(p) - prob_to_fixed(old_r[k]);
          c.state.ring[((int64_t)u * w + (t % w)) * cap + s0 + i] = p;
          c.state.acc_fixed[o] = fx;
          S = fixed_to_prob(fx);
        } else {
          S = is_new ? p : old_r[k] + p;
        }
        if (VATP_INB(s0 + i, cap, dev_status)) c.state.acc[o] = S;
        const int ps = is_new ? t : pos_r[k];
        if (evicting && ps >= F && ps <= t - R) {
          const unsigned long long key = q4_evict_key(S * (is_new ? new_norm_s : norm_r[k]), ps);
          if (key < my_key) { my_key = key; my_slot = s0 + i; my_pos = ps; }
        }
      }
      i0 += SB * WORKERS;
      if (i0 < cnt) fetch(i0);
    }
    if (WINDOWED) {
      // recycled slot: the other rows of its ring column belong to the previous occupant (shared out over the unit's CTAs)
      for (int r = rank * WORKERS + tid; r < w; r += split * WORKERS)
        if (r != t % w) c.state.ring[((int64_t)u * w + r) * cap + fs] = 0.f;
    }
    if (evicting) {
      // (positions are unique: one lane holds the winning key)
      const unsigned long long win = min_key(my_key);
      if (win == Q4_NO_KEY ? lane == 0 : my_key == win)
        send4(at_rank(s32(&cand[rank * WARPS + wid]), 0), (uint32_t)win, (uint32_t)(win >> 32), (uint32_t)my_slot, (uint32_t)my_pos, at_rank(s32(&cand_bar), 0));
    }
  } else if (rank == 0) {
    int out_slot = hi, left = hi, ev = -1;                         // not evicting: the cache grows
    bool write = lane == 0;
    if (evicting) {
      if (!bar_wait(s32(&cand_bar), 0)) bad = true;
      Q4Candidate best{Q4_NO_KEY, -1, -1};
      for (int i = lane; i < split * WARPS; i += 32)
        if (cand[i].key < best.key) best = cand[i];
      const unsigned long long win = min_key(best.key);
      if (win != Q4_NO_KEY) {
        write = best.key == win;
        out_slot = best.slot;
        ev = best.pos;
        left = hi - 1;
      } else {                             // nothing eligible (cannot happen when F + R <= B): keep the state consistent
        out_slot = min(hi, cap - 1);
      }
    }
    if (write) {
      // (both positions by one thread, in this order: they are the same word where the incoming token goes at once)
      if (fs < hi) c.state.pos[(int64_t)u * cap + fs] = t;
      if (left < hi && VATP_INB(out_slot, cap, dev_status)) c.state.pos[(int64_t)u * cap + out_slot] = -1;
      c.state.len[u] = left;
      c.state.free_slot[u] = out_slot;
      c.state.next_pos[u] = t + 1;
      c.state.last_slot[u] = fs;
      if (evicted) evicted[u] = ev;
    }
  }
  if (bad) {
    // Something never arrived: say so, give copies that may still be in flight time to land, and stay until the unit's other CTAs have
    // sent what they send here (threads that exit count as arrived).
    if (dev_status) atomicExch(dev_status, (int)VATP_ERR_TIMEOUT);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
}

// How many clusters of `split` CTAs with an SM each run at once (they lie within a GPC, which is not a multiple of them); asked for
// once per device and size.  0 where the runtime does not say: a unit then stays on fewer CTAs in this call.
using ClusterCounts = KnownCounts<16, Q4_SPLIT + 1>;
template <typename Kernel>
int clusters_at_once(ClusterCounts& known, Kernel kern, int split, int threads, size_t dyn) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  return known.get(dev, split, [&] {
    int n = 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)split);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = dyn;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = split;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dyn) != cudaSuccess ||
        cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
      cudaGetLastError();
      return -1;
    }
    return n;
  });
}

template <typename T, int HD, int GT>
cudaError_t launch_gt(int units, int G, int B, int F, int R, int window, int norm, float scale, const vatp_cache_q4& c, const void* q,
                      const void* k, const void* v, void* out, int32_t* evicted, int32_t* dev_status, cudaStream_t st) {
  const int cap = cache_capacity(B), sms = device_sm_count();
  constexpr int ITEM = q4_item<HD>;
  // Static arrays and what the system takes, rounded up (of a CTA of sixteen warps, of one of eight).
  constexpr size_t fixed16 = (GT > 4 ? 47 : GT > 1 ? 41 : 18) * 1024, fixed8 = (GT > 4 ? 28 : GT > 1 ? 24 : 11) * 1024;
  const bool win = window > 0;
  auto kern16 = win ? decode_q4_kernel<T, HD, true, GT, 16, true> : decode_q4_kernel<T, HD, false, GT, 16, true>;
  auto kern8 = win ? decode_q4_kernel<T, HD, true, GT, 8, true> : decode_q4_kernel<T, HD, false, GT, 8, true>;
  auto pair8 = win ? decode_q4_kernel<T, HD, true, GT, 8, false> : decode_q4_kernel<T, HD, false, GT, 8, false>;
  const size_t most16 = 226 * 1024 - fixed16, most8 = 226 * 1024 - fixed8;
  static ClusterCounts known[2];         // (of kern16, without and with a history)
  // Units on fewer CTAs than SMs: an SM to a CTA (two of a launch on one SM while others idle: 32 units x 2049 slots, four CTAs each,
  // 8.0 and 7.3 us per step, with the same kernel), a power of two of them per unit that run at once and find some slots, of sixteen warps when there
  // are more than three rounds for eight (74 units x 4097: 15.7 and 14.0 us; 32 x 1025: 6.0 and 6.8, which is why not always).  More units
  // than SMs: one CTA of eight warps each, two on an SM.
  int split = 1;
  while (split < Q4_SPLIT && units * split * 2 <= sms && cap / split >= 4 * Q4_ROWS && clusters_at_once(known[win], kern16, split * 2, 17 * 32, most16) >= units) split *= 2;
  // Then any other number that would save eight warps a round (CTAs that get sixteen below have fewer): clusters lie within a GPC, seven of sixteen CTAs run at once, fifteen of eight, but
  // eleven of ten, 22 of six (16 units x 4002 slots, four heads: four CTAs each 12.8 us per step, six 10.7; 40 x 2049: two 9.1, three 7.7).
  // Of clusters of three and of five, the last two of those said to fit have been seen to wait (of three, 43 units 7.7 us and 45 10.4).
  auto rounds_of = [&](int split) { return (B + 1 - Q4_EXTRA + 8 * Q4_ROWS * split - 1) / (8 * Q4_ROWS * split); };
  for (int more = split + 1; more <= Q4_SPLIT && units * more <= sms; ++more)
    if (rounds_of(more) < rounds_of(split) && clusters_at_once(known[win], kern16, more, 17 * 32, most16) >= units + (more & 1) * 2) split = more;
  const bool alone = units <= sms;
  // a ring takes the warp's partial output in the end
  const int least = (G * HD * 4 + ITEM - 1) / ITEM > 2 ? (G * HD * 4 + ITEM - 1) / ITEM : 2;
  auto chunk_of = [&](int split) { return ((cap + split - 1) / split + Q4_ROWS - 1) / Q4_ROWS * Q4_ROWS; };
  int warps = 8;
  auto bytes = [&](int split, int depth) { return (size_t)warps * depth * ITEM + (size_t)G * HD * 12 + (size_t)G * (chunk_of(split) + 2 * Q4_EXTRA) * 4; };
  const size_t half = 113 * 1024 - fixed8;
  if (alone ? (cap + split - 1) / split > 3 * 8 * Q4_ROWS : bytes(split, least) > half) warps = 16;      // (half: two CTAs on an SM)
  // (rather eight warps than more CTAs than SMs where the logits leave no room for sixteen rings: 32 units x 13001 slots, eight heads: 95 -> 55 us)
  if (alone && warps == 16 && bytes(split, least) > most16) warps = 8;
  const size_t most = warps == 16 ? most16 : most8;
  while (split < Q4_SPLIT && bytes(split, least) > most) split = split * 2 < Q4_SPLIT ? split * 2 : Q4_SPLIT;      // (the logits of a CTA's slots stand in shared memory)
  int chunk = chunk_of(split), ld = chunk;
  // A few slots more than whole rounds of the warps (the incoming token's, where the budget fills them): the last warp of the last
  // CTA takes them.
  const int round = warps * Q4_ROWS * split, rounds = (B + 1) / round, extra = B + 1 - rounds * round;
  if (rounds > 0 && extra > 0 && extra <= Q4_EXTRA && rounds * warps * Q4_ROWS <= chunk) {
    chunk = rounds * warps * Q4_ROWS;
    ld = chunk + 2 * Q4_EXTRA;           // (the capacity is the slots' number rounded up to eight)
  }
  const int per_warp = (chunk / Q4_ROWS + warps - 1) / warps;
  int depth = 2 * per_warp;
  depth = depth < least ? least : depth > Q4_DEPTH ? Q4_DEPTH : depth;
  const size_t limit = !alone && warps == 8 ? half : most;
  while (depth > least && bytes(split, depth) > limit) --depth;
  size_t dyn = bytes(split, depth);
  if (dyn > most || (int64_t)units * split > 0x7fffffffll) return cudaErrorNotSupported;
  if (alone && dyn < 120 * 1024 - fixed8) dyn = 120 * 1024 - fixed8;
  auto kern = warps == 16 ? kern16 : alone ? kern8 : pair8;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
  if (e == cudaSuccess && split > 8) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * split));
  cfg.blockDim = dim3((unsigned)(warps * 32 + 32));
  cfg.dynamicSmemBytes = dyn;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // may start before the previous launch has drained
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, G, split, chunk, ld, depth, B, cap, F, R, window, norm, scale * Q4_LOG2E, c, (const T*)q,
                            (const T*)k, (const T*)v, (T*)out, evicted, dev_status);
}

template <typename T, int HD>
cudaError_t launch_hd(int units, int G, int B, int F, int R, int window, int norm, float scale, const vatp_cache_q4& c, const void* q,
                      const void* k, const void* v, void* out, int32_t* evicted, int32_t* dev_status, cudaStream_t st) {
  auto f = G == 1 ? launch_gt<T, HD, 1> : G <= 4 ? launch_gt<T, HD, 4> : launch_gt<T, HD, 8>;
  return f(units, G, B, F, R, window, norm, scale, c, q, k, v, out, evicted, dev_status, st);
}

}  // namespace

cudaError_t launch_decode_q4(int units, int G, int d, int dtype, int B, int F, int R, int window, int norm, float scale, const vatp_cache_q4& c,
                             const void* q, const void* k, const void* v, void* out, int32_t* evicted, int32_t* dev_status, cudaStream_t st) {
  if (G > Q4_HEADS) return cudaErrorNotSupported;
  auto f = dtype == VATP_F32 ? (d == 64 ? launch_hd<float, 64> : launch_hd<float, 128>)
                             : (d == 64 ? launch_hd<__nv_bfloat16, 64> : launch_hd<__nv_bfloat16, 128>);
  return f(units, G, B, F, R, window, norm, scale, c, q, k, v, out, evicted, dev_status, st);
}

}  // namespace vatp
