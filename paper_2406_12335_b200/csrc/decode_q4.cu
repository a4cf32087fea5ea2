// Decode step on a cache whose rows are held in 4 bits: append (quantised), attend (Eq. 1), indicator update (Eq. 2 / Eq. 3),
// importance (Eq. 4), release of the lowest-importance unprotected slot.
//
// With the values lo_ig + sc_ig code_ic of row i, group g and channel c:
//   s_i = scale * sum_g ( sc_ig * sum_{c in g} q_c code_ic + lo_ig * sum_{c in g} q_c ),   p = softmax(s)
//   o_c = sum_i p_i lo_ig + sum_i (p_i sc_ig) code_ic
// The sums over codes run on the warp-level tensor-core path (mma.sync m16n8k16, fp16 in, fp32 accumulate), the rest in fp32:
//   * a code in the low bits of a 16-bit word IS the fp16 number code * 2^-24 (subnormal), one in bits 4-7 is code * 2^-20: unpacking
//     is one AND per two codes and one shift per eight; the constant factors go into the other operand and the result;
//   * that operand is exact to 2^-22 whatever its magnitude: q is scaled by a power of two per head, p_i sc_ig by one per warp and
//     head that the largest of them determines, and both are taken as a high fp16 half and a remainder (q of bf16 inputs has none);
//   * rows are stored so that the 16 bytes a lane loads hold the channels it needs in an MMA operand, of every group: rows go from
//     global memory into operand registers by plain 8- and 16-byte loads, without shared memory.
// A unit is split over a thread-block cluster; the slots of a CTA over its eight warps, sixteen at a time.  A warp keeps its own
// softmax (its maximum, sum and partial output; no barrier between the two products); the CTA joins them, the cluster joins the
// CTAs' by st.async into the partners' shared memory, and every CTA then updates the indicators of its own slots and sends its
// eviction candidate to rank 0.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "q4.cuh"

namespace cg = cooperative_groups;

namespace vatp {
namespace {

constexpr int Q4_WARPS = 8, Q4_THREADS = Q4_WARPS * 32;
constexpr int Q4_TILE = 16;            // slots of a warp at a time
constexpr int Q4_SPLIT = 8;            // CTAs of a unit at most
constexpr int Q4_HEADS = 8;            // query heads of a unit at most (columns of the MMA tiles)
constexpr int Q4_AHEAD = 2;            // tiles in flight per warp
constexpr float Q4_LOG2E = 1.4426950408889634f;
constexpr unsigned long long Q4_NO_KEY = ~0ull;

__device__ __forceinline__ uint32_t s32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* bar) { asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(s32(bar)) : "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(s32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* bar) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], 0;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(s32(bar)) : "memory");
  return ok != 0;
}
// bounded wait (about a second) for the barrier's first phase: false when what it counts never arrived
__device__ __forceinline__ bool bar_wait(uint64_t* bar) {
  if (bar_try(bar)) return true;
  uint64_t t0, t1;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  while (!bar_try(bar)) {
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
    if (t1 - t0 > 1000000000ull) return false;
  }
  return true;
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
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Rows are read once, past L1: a step may request rows before its predecessor has finished, and what it requests again afterwards
// must come from L2.
__device__ __forceinline__ uint32_t load_row(const uint32_t* p) {
  uint32_t x;
  asm volatile("ld.global.cg.u32 %0, [%1];" : "=r"(x) : "l"(p));
  return x;
}
__device__ __forceinline__ uint2 load_row(const uint2* p) {
  uint2 x;
  asm volatile("ld.global.cg.v2.u32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "l"(p));
  return x;
}
__device__ __forceinline__ uint4 load_row(const uint4* p) {
  uint4 x;
  asm volatile("ld.global.cg.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
  return x;
}
template <int N> __device__ __forceinline__ void load_words(const void* p, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = load_row(static_cast<const uint32_t*>(p));
  } else if constexpr (N == 2) {
    const uint2 x = load_row(static_cast<const uint2*>(p));
    w[0] = x.x; w[1] = x.y;
  } else {
    const uint4 x = load_row(static_cast<const uint4*>(p));
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  }
}
template <int N> __device__ __forceinline__ void copy_words(const unsigned char* p, uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
}

// eight or four consecutive channels of a new row
__device__ __forceinline__ void load_new(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 r = load_behind_wait(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
}
__device__ __forceinline__ void load_new(const float* p, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float4 r = load_behind_wait(reinterpret_cast<const float4*>(p) + k);
    x[4 * k] = r.x; x[4 * k + 1] = r.y; x[4 * k + 2] = r.z; x[4 * k + 3] = r.w;
  }
}
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
// Dynamic shared memory: partial outputs of the warps [8][G][HD] | logits [G][ld].
template <typename T, int HD, bool WINDOWED, int GT>
__global__ void __launch_bounds__(Q4_THREADS, 2)
decode_q4_kernel(int G_arg, int split, int chunk, int ld, int B, int cap, int F, int R, int w, int norm, float scale_log2, vatp_cache_q4 c, const T* q_new,
                 const T* k_new, const T* v_new, T* out, int32_t* evicted, int32_t* dev_status) {
  constexpr int NG = HD / 32, KW = HD / 32, VW = HD / 64;       // groups of a row; 32-bit words of a lane in a K row and a V row
  constexpr int KP = GT == 1 ? 1 : NG;                          // parameter words of a lane per K row
  constexpr bool SPLIT_Q = sizeof(T) == 4;                      // q has a remainder beyond its high half
  const int G = GT == 1 ? 1 : G_arg;
  extern __shared__ float dyn[];
  float* part_o = dyn;
  float* logit_s = dyn + Q4_WARPS * G * HD;
  constexpr int XC = GT > 4 ? 16 : 8, X_LOW = XC / 2;           // columns of the second product's operand; the remainders' first one
  __shared__ __align__(16) uint16_t xs[Q4_WARPS][NG][XC][Q4_TILE];     // [group][column][slot]
  __shared__ __align__(16) unsigned char new_row[2][HD / 2 + 4 * NG];  // the incoming token's K and V row: codes, parameters
  __shared__ float part_m[Q4_WARPS][GT], part_j[Q4_WARPS][GT], part_l[Q4_WARPS][GT], part_lo[Q4_WARPS][GT][NG];
  __shared__ float f_m[Q4_WARPS][GT], f_j[Q4_WARPS][GT];      // the warps' factors towards the CTA's maximum
  __shared__ float xo[GT * HD];                                        // slices of partial outputs received [split][G][HD / split]
  __shared__ float2 ex_ml[Q4_SPLIT][GT];                               // per rank and head: maximum of its logits, sum of exp2(s - m)
  __shared__ float fr_s[Q4_SPLIT][GT], all_m[GT], all_inv[GT], new_norm_s;
  __shared__ Q4Candidate cand[Q4_SPLIT];
  __shared__ unsigned long long warp_key[Q4_WARPS];
  __shared__ __align__(8) uint64_t ex_bar, cand_bar;

  const int rank = split > 1 ? (int)cg::this_cluster().block_rank() : 0;
  const int tid = threadIdx.x, lane = tid & 31, wid = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int r8 = lane >> 2, t4 = lane & 3;
  const int u = blockIdx.x / split;
  const int s0 = min(rank * chunk, cap), rows_alloc = min(chunk, cap - s0);      // this CTA's slots of the unit
  const int64_t base = (int64_t)u * cap + s0;
  if (tid == 0) {
    bar_init(&ex_bar);
    bar_init(&cand_bar);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (split > 1) {
      bar_expect(&ex_bar, (uint32_t)(8 * G * split + 4 * G * HD));
      if (rank == 0) bar_expect(&cand_bar, (uint32_t)(split * sizeof(Q4Candidate)));
    }
  }
  for (int i = lane; i < NG * XC * Q4_TILE / 2; i += 32) reinterpret_cast<uint32_t*>(xs[wid])[i] = 0u;      // (columns without a head stay 0)
  __syncthreads();
  if (split > 1) cluster_arrive_release();

  // ---- a tile's rows: K rows r8 and r8 + 8 with the channels of chunks 2 t4 and 2 t4 + 1, V rows 4 t4 .. + 3 with those of chunk r8
  const unsigned char* kc = static_cast<const unsigned char*>(c.state.k_cache) + base * (HD / 2);
  const unsigned char* vc = static_cast<const unsigned char*>(c.state.v_cache) + base * (HD / 2);
  const uint32_t* kp = static_cast<const uint32_t*>(c.k_params) + base * NG;
  const uint32_t* vp = static_cast<const uint32_t*>(c.v_params) + base * NG;
  struct KTile { uint32_t w[2][KW], p[2][KP], v[2]; };      // v: V's parameters of group t4, for the bound on p sc
  struct VTile { uint32_t w[4][VW], p[VW]; };               // p: parameters of slot lane / 2, groups VW (lane mod 2) ..
  auto load_k = [&](KTile& x, int r0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = min(r0 + r8 + 8 * i, rows_alloc - 1);      // (rows beyond the last are not used)
      load_words(kc + (int64_t)row * (HD / 2) + t4 * (HD / 8), x.w[i]);
      if constexpr (GT == 1) x.p[i][0] = t4 < NG ? load_row(kp + (int64_t)row * NG + t4) : 0u;
      else load_words(kp + (int64_t)row * NG, x.p[i]);
      x.v[i] = t4 < NG ? load_row(vp + (int64_t)row * NG + t4) : 0u;
    }
  };
  auto load_v = [&](VTile& x, int r0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) load_words(vc + (int64_t)min(r0 + 4 * t4 + i, rows_alloc - 1) * (HD / 2) + r8 * (HD / 16), x.w[i]);
    load_words(vp + (int64_t)min(r0 + (lane >> 1), rows_alloc - 1) * NG + (lane & 1) * VW, x.p);
  };
  constexpr int RSTEP = Q4_WARPS * Q4_TILE;
  const int first = wid * Q4_TILE;
  KTile kt[Q4_AHEAD];
#pragma unroll
  for (int a = 0; a < Q4_AHEAD; ++a)
    if (first + a * RSTEP < rows_alloc) load_k(kt[a], first + a * RSTEP);
  // Nothing but K and V rows is read before the previous launch has completed.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int len = min(max(c.state.len[u], 0), cap - 1), fs = min(max(c.state.free_slot[u], 0), cap - 1);
  const int t = c.state.next_pos[u], ls = c.state.last_slot[u];
  const int hi = len + 1;                // slots [0, hi) are live once the new token is in
  const int cnt = max(min(hi - s0, rows_alloc), 0);
  const int fs_local = fs - s0;
  const bool owns_new = fs_local >= 0 && fs_local < cnt;
  const int new_warp = owns_new ? (fs_local / Q4_TILE) % Q4_WARPS : -1;
  // The row that the previous step appended may have been requested before it was stored.
  const int ls_local = ls - s0;
#pragma unroll
  for (int a = 0; a < Q4_AHEAD; ++a) {
    const int r0 = first + a * RSTEP;
    if (ls >= 0 && r0 < rows_alloc && ls_local >= r0 && ls_local < r0 + Q4_TILE) load_k(kt[a], r0);
  }
  VTile vt[Q4_AHEAD];
#pragma unroll
  for (int a = 0; a < Q4_AHEAD; ++a)
    if (first + a * RSTEP < cnt) load_v(vt[a], first + a * RSTEP);

  // ---- B operand of K q^T.  Lane (n = r8, t4): channels 8 t4 .. 8 t4 + 7 of every group of its column's head.
  // GT == 1: column 2 g carries the high half of group g alone, column 2 g + 1 its remainder: every lane of a row's four then
  // holds one group's sum, to be scaled by that group's parameters.  Else: column n is head n.
  uint32_t qb[NG][4], qr[GT > 1 && SPLIT_Q ? NG : 1][4];
  float q_back, qsum[GT > 1 ? NG : 1][2];      // 2^24 / (the head's power of two) * scale; sums of q over groups, * scale
  {
    const T* qp = q_new + ((int64_t)u * G + (GT == 1 ? 0 : min(r8, G - 1))) * HD + 8 * t4;
    float q[NG][8], most = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g)
      load_new(qp + 32 * g, q[g]);
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(q[g][e]));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    // power of two that brings the largest to [2^13, 2^14)
    const int ex = min(max(13 + 127 - (int)(__float_as_uint(most) >> 23), -100), 126);
    const float up = __uint_as_float((uint32_t)(ex + 127) << 23), back = __uint_as_float((uint32_t)(24 - ex + 127) << 23) * scale_log2;
    float gs[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s += q[g][e];
      s += __shfl_xor_sync(0xffffffffu, s, 1);
      s += __shfl_xor_sync(0xffffffffu, s, 2);
      gs[g] = s * scale_log2;
      float a[8], rest[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = q[g][e] * (e & 1 ? up * 0.0625f : up);      // (odd channels' codes stand four bits higher)
        a[e] = __half2float(__float2half_rn(x));
        rest[e] = x - a[e];
      }
      const bool low = GT == 1 && SPLIT_Q && (r8 & 1), mine = GT > 1 || (r8 >> 1) == g;
      if (GT == 1 && !SPLIT_Q && (r8 & 1)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = 0.f;
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        qb[g][x] = mine ? (low ? half2_of(rest[x], rest[x + 4]) : half2_of(a[x], a[x + 4])) : 0u;
        if constexpr (GT > 1 && SPLIT_Q) qr[g][x] = half2_of(rest[x], rest[x + 4]);
      }
    }
    if constexpr (GT == 1) {
      q_back = back;
      float s = gs[0];
#pragma unroll
      for (int g = 1; g < NG; ++g) s = t4 == g ? gs[g] : s;
      qsum[0][0] = t4 < NG ? s : 0.f;
      qsum[0][1] = 0.f;
    } else {
      // (an accumulator's columns are heads 2 t4 and 2 t4 + 1; their sums are with the lanes of those columns)
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int x = 0; x < 2; ++x) qsum[g][x] = __shfl_sync(0xffffffffu, gs[g], 4 * (2 * t4 + x));
      q_back = back;
    }
  }
  float q_back2[2];
  if constexpr (GT > 1) {
#pragma unroll
    for (int x = 0; x < 2; ++x) q_back2[x] = __shfl_sync(0xffffffffu, q_back, 4 * (2 * t4 + x));
  }

  // ---- the incoming token: quantised, stored, and kept for the tiles that hold its slot; its norm (Eq. 4)
  if (wid == new_warp) {
    float norm_v = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float y[4] = {0.f, 0.f, 0.f, 0.f};
      if (lane < HD / 4) load_new((x ? v_new : k_new) + (int64_t)u * HD + 4 * lane, y);
      uint32_t par;
      const uint32_t code = q4_row(y, par);
      if (lane < HD / 4) {
        *reinterpret_cast<uint16_t*>(new_row[x] + q4_byte<HD>(lane >> 3, lane & 7)) = (uint16_t)code;
        if ((lane & 7) == 0) reinterpret_cast<uint32_t*>(new_row[x] + HD / 2)[lane >> 3] = par;
      }
      if (x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) norm_v = norm_fold(norm, norm_v, y[e]);
#pragma unroll
        for (int o = 16; o; o >>= 1) norm_v = norm_merge(norm, norm_v, __shfl_xor_sync(0xffffffffu, norm_v, o));
        norm_v = norm_finish(norm, norm_v);
      }
    }
    __syncwarp();
    constexpr int CW = HD / 8;             // words of a row's codes
    const int x = lane >> 4, i = lane & 15;
    const uint32_t* from = reinterpret_cast<const uint32_t*>(new_row[x]);
    if (i < CW) reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(x ? c.state.v_cache : c.state.k_cache) + (base + fs_local) * (HD / 2))[i] = from[i];
    if (i < NG) static_cast<uint32_t*>(x ? c.v_params : c.k_params)[(base + fs_local) * NG + i] = from[CW + i];
    if (lane == 0) {
      new_norm_s = norm_v;
      c.state.vnorm[base + fs_local] = norm_v;
      c.state.pos[base + fs_local] = t;
    }
  }

  // ---- logits of this warp's tiles, their maximum and that of s + log2 sc_v (J, rounded up: what p sc may amount to)
  constexpr int MX = GT > 1 ? 2 : 1;
  float m_run[MX], j_run[MX];
#pragma unroll
  for (int x = 0; x < MX; ++x) m_run[x] = j_run[x] = -INFINITY;
  for (int r0 = first; r0 < cnt; r0 += Q4_AHEAD * RSTEP) {
#pragma unroll
    for (int a = 0; a < Q4_AHEAD; ++a) {
      const int rt = r0 + a * RSTEP;
      if (rt >= cnt) break;
      KTile& k = kt[a];
      if (wid == new_warp && fs_local >= rt && fs_local < rt + Q4_TILE) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (rt + r8 + 8 * i == fs_local) {
            copy_words(new_row[0] + t4 * (HD / 8), k.w[i]);
            copy_words(new_row[0] + HD / 2 + (GT == 1 ? 4 * min(t4, NG - 1) : 0), k.p[i]);
            if (GT == 1 && t4 >= NG) k.p[i][0] = 0u;
            if (t4 < NG) k.v[i] = reinterpret_cast<const uint32_t*>(new_row[1] + HD / 2)[t4];
          }
      }
      float acc[GT > 1 ? NG : 2][4];
#pragma unroll
      for (int g = 0; g < (GT > 1 ? NG : 2); ++g) acc[g][0] = acc[g][1] = acc[g][2] = acc[g][3] = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        // words of chunks 2 t4 (first half of the lane's words) and 2 t4 + 1; a half word is a group
        const uint32_t sel = g & 1 ? 0x7632u : 0x5410u;
        const uint32_t xa = __byte_perm(k.w[0][g >> 1], k.w[0][KW / 2 + (g >> 1)], sel);
        const uint32_t xb = __byte_perm(k.w[1][g >> 1], k.w[1][KW / 2 + (g >> 1)], sel);
        float(&d0)[4] = acc[GT > 1 ? g : 0];
        float(&d1)[4] = acc[GT > 1 ? g : 1];
        mma_f16(d0, xa & 0x000f000fu, xb & 0x000f000fu, xa & 0x00f000f0u, xb & 0x00f000f0u, qb[g][0], qb[g][1]);
        mma_f16(d1, xa >> 8 & 0x000f000fu, xb >> 8 & 0x000f000fu, xa >> 8 & 0x00f000f0u, xb >> 8 & 0x00f000f0u, qb[g][2], qb[g][3]);
        if constexpr (GT > 1 && SPLIT_Q) {
          mma_f16(d0, xa & 0x000f000fu, xb & 0x000f000fu, xa & 0x00f000f0u, xb & 0x00f000f0u, qr[g][0], qr[g][1]);
          mma_f16(d1, xa >> 8 & 0x000f000fu, xb >> 8 & 0x000f000fu, xa >> 8 & 0x00f000f0u, xb >> 8 & 0x00f000f0u, qr[g][2], qr[g][3]);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = rt + r8 + 8 * i;
        const bool live = row < cnt;
        float s[MX];
        if constexpr (GT == 1) {
          const float d = (acc[0][2 * i] + acc[1][2 * i]) + (acc[0][2 * i + 1] + acc[1][2 * i + 1]);
          s[0] = fmaf(q4_scale(k.p[i][0]) * q_back, d, q4_low(k.p[i][0]) * qsum[0][0]);
          s[0] += __shfl_xor_sync(0xffffffffu, s[0], 1);
          s[0] += __shfl_xor_sync(0xffffffffu, s[0], 2);
        } else {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float d = 0.f, l = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              d = fmaf(q4_scale(k.p[i][g]), acc[g][2 * i + x], d);
              l = fmaf(q4_low(k.p[i][g]), qsum[g][x], l);
            }
            s[x] = fmaf(d, q_back2[x], l);
          }
        }
        // exponent of the largest scale of V's row, rounded up
        int ev = max((int)(k.v[i] >> 7 & 0xffu) - 126, -100);
        ev = max(ev, __shfl_xor_sync(0xffffffffu, ev, 1));
        ev = max(ev, __shfl_xor_sync(0xffffffffu, ev, 2));
#pragma unroll
        for (int x = 0; x < MX; ++x) {
          if (!live) s[x] = -INFINITY;
          const int h = GT > 1 ? 2 * t4 + x : 0;
          if (GT > 1 ? h < G : t4 == 0) logit_s[h * ld + row] = s[x];
          m_run[x] = fmaxf(m_run[x], s[x]);
          j_run[x] = fmaxf(j_run[x], s[x] + (float)ev);
        }
      }
      if (rt + Q4_AHEAD * RSTEP < cnt) load_k(kt[a], rt + Q4_AHEAD * RSTEP);
    }
  }
  // (after the wait: at most one unfinished predecessor exists while a successor sets up)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
#pragma unroll
  for (int x = 0; x < MX; ++x) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      m_run[x] = fmaxf(m_run[x], __shfl_xor_sync(0xffffffffu, m_run[x], o));
      j_run[x] = fmaxf(j_run[x], __shfl_xor_sync(0xffffffffu, j_run[x], o));
    }
    const int h = GT > 1 ? 2 * t4 + x : 0;
    if (r8 == 0 && (GT > 1 ? h < G : t4 == 0)) { part_m[wid][h] = m_run[x]; part_j[wid][h] = j_run[x]; }
  }
  __syncwarp();

  // ---- O^T += V^T (p sc): A = codes (16 channels x 16 slots), B = p sc by slot and head
  float o_acc[NG][2][4];
#pragma unroll
  for (int g = 0; g < NG; ++g)
#pragma unroll
    for (int i = 0; i < 2; ++i) o_acc[g][i][0] = o_acc[g][i][1] = o_acc[g][i][2] = o_acc[g][i][3] = 0.f;
  float l_run[GT], lo_run[GT][VW];        // of this lane's slots (and groups): sum of p, sum of p lo
#pragma unroll
  for (int h = 0; h < GT; ++h) {
    l_run[h] = 0.f;
#pragma unroll
    for (int i = 0; i < VW; ++i) lo_run[h][i] = 0.f;
  }
  for (int r0 = first; r0 < cnt; r0 += Q4_AHEAD * RSTEP) {
#pragma unroll
    for (int a = 0; a < Q4_AHEAD; ++a) {
      const int rt = r0 + a * RSTEP;
      if (rt >= cnt) break;
      VTile& v = vt[a];
      if (wid == new_warp && fs_local >= rt && fs_local < rt + Q4_TILE) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (rt + 4 * t4 + i == fs_local) copy_words(new_row[1] + r8 * (HD / 16), v.w[i]);
        if (rt + (lane >> 1) == fs_local) copy_words(new_row[1] + HD / 2 + (lane & 1) * VW * 4, v.p);
      }
      const int slot = rt + (lane >> 1);
      const bool live = slot < cnt;
#pragma unroll
      for (int h = 0; h < GT; ++h) {
        if (GT > 1 && h >= G) break;
        const float s = logit_s[h * ld + slot];      // (-inf from cnt on)
        const float p = live ? exp2_fast(s - part_m[wid][h]) : 0.f, y = live ? exp2_fast(s - part_j[wid][h] + 14.f) : 0.f;
        l_run[h] += p;
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          const float x = live ? y * q4_scale(v.p[i]) : 0.f;
          if (live) lo_run[h][i] = fmaf(p, q4_low(v.p[i]), lo_run[h][i]);
          const __half hh = __float2half_rn(x), hl = __float2half_rn(x - __half2float(hh));
          const int g = (lane & 1) * VW + i;
          xs[wid][g][h][lane >> 1] = __half_as_ushort(hh);
          xs[wid][g][h + X_LOW][lane >> 1] = __half_as_ushort(hl);
        }
      }
      __syncwarp();
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint2 b = *reinterpret_cast<const uint2*>(&xs[wid][g][r8][4 * t4]);
        const uint32_t sel = g & 1 ? 0x7632u : 0x5410u;
        const uint32_t xa = __byte_perm(v.w[0][g >> 1], v.w[1][g >> 1], sel), xb = __byte_perm(v.w[2][g >> 1], v.w[3][g >> 1], sel);
        mma_f16(o_acc[g][0], xa & 0x000f000fu, xa & 0x00f000f0u, xb & 0x000f000fu, xb & 0x00f000f0u, b.x, b.y);
        mma_f16(o_acc[g][1], xa >> 8 & 0x000f000fu, xa >> 8 & 0x00f000f0u, xb >> 8 & 0x000f000fu, xb >> 8 & 0x00f000f0u, b.x, b.y);
        if constexpr (GT > 4) {
          const uint2 d = *reinterpret_cast<const uint2*>(&xs[wid][g][X_LOW + r8][4 * t4]);
          mma_f16(o_acc[g][0], xa & 0x000f000fu, xa & 0x00f000f0u, xb & 0x000f000fu, xb & 0x00f000f0u, d.x, d.y);
          mma_f16(o_acc[g][1], xa >> 8 & 0x000f000fu, xa >> 8 & 0x00f000f0u, xb >> 8 & 0x000f000fu, xb >> 8 & 0x00f000f0u, d.x, d.y);
        }
      }
      __syncwarp();
      if (rt + Q4_AHEAD * RSTEP < cnt) load_v(vt[a], rt + Q4_AHEAD * RSTEP);
    }
  }
  // ---- the warp's partial: sums of p (even lanes), of p lo, and O^T with its constant factors (codes in odd channels stand four
  // bits higher)
#pragma unroll
  for (int h = 0; h < GT; ++h) {
    if (GT > 1 && h >= G) break;
#pragma unroll
    for (int o = 2; o < 32; o <<= 1) {
      l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], o);
#pragma unroll
      for (int i = 0; i < VW; ++i) lo_run[h][i] += __shfl_xor_sync(0xffffffffu, lo_run[h][i], o);
    }
    if (lane < 2) {
      if (lane == 0) part_l[wid][h] = l_run[h];
#pragma unroll
      for (int i = 0; i < VW; ++i) part_lo[wid][h][lane * VW + i] = lo_run[h][i];
    }
  }
#pragma unroll
  for (int g = 0; g < NG; ++g)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float o = o_acc[g][i][x];
        if (GT <= 4) o += __shfl_xor_sync(0xffffffffu, o, 2);      // (the remainder's column)
        const int h = 2 * t4 + (x & 1);
        if (h < G) part_o[((size_t)wid * G + h) * HD + 32 * g + 4 * r8 + 2 * i + (x >> 1)] = x & 2 ? o * 0.0625f : o;
      }
  // ---- the state of this thread's slots tid, tid + 256, ...: the first ones read while the CTAs exchange
  constexpr int SB = 2;
  float old_r[SB], norm_r[SB];
  int pos_r[SB];
  long long fx_r[WINDOWED ? SB : 1];
  const float* old_g = WINDOWED ? c.state.ring + ((int64_t)u * w + (t % w)) * cap + s0 : c.state.acc + base;
  auto fetch = [&](int i0) {
#pragma unroll
    for (int k = 0; k < SB; ++k) {
      const int i = i0 + k * Q4_THREADS;
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
  fetch(tid);
  __syncthreads();
  if (tid < Q4_WARPS * G) {
    const int k = tid / G, h = tid - k * G;
    float m = part_m[0][h];
#pragma unroll
    for (int i = 1; i < Q4_WARPS; ++i) m = fmaxf(m, part_m[i][h]);
    const bool any = part_m[k][h] > -INFINITY;
    f_m[k][h] = any ? exp2_fast(part_m[k][h] - m) : 0.f;
    f_j[k][h] = any ? exp2_fast(part_j[k][h] + 10.f - m) : 0.f;
  }
  __syncthreads();
  // (another CTA's shared memory may only be written once that CTA runs and its barriers are armed)
  if (split > 1) cluster_wait_acquire();

  // ---- to the unit's CTAs: maximum and sum to every one, channel slice r of the partial output to rank r
  const int slice = HD / split, slice_log2 = 31 - __clz(slice);
  if (tid < split * G) {
    const int h = tid / split, dst = tid - h * split;
    float m = part_m[0][h], l = 0.f;
#pragma unroll
    for (int k = 0; k < Q4_WARPS; ++k) {
      m = fmaxf(m, part_m[k][h]);
      l = fmaf(part_l[k][h], f_m[k][h], l);
    }
    if (split > 1) send2(at_rank(s32(&ex_ml[rank][h]), dst), m, l, at_rank(s32(&ex_bar), dst));
    else ex_ml[0][h] = make_float2(m, l);
  }
  for (int i = tid; i < G * HD; i += Q4_THREADS) {
    const int h = i / HD, ch = i - h * HD;
    float a = 0.f;
#pragma unroll
    for (int k = 0; k < Q4_WARPS; ++k) {
      a = fmaf(part_o[((size_t)k * G + h) * HD + ch], f_j[k][h], a);
      a = fmaf(part_lo[k][h][ch >> 5], f_m[k][h], a);
    }
    const int dst = ch >> slice_log2, off = (rank * G + h) * slice + (ch & (slice - 1));
    if (split > 1) send(at_rank(s32(&xo[off]), dst), a, at_rank(s32(&ex_bar), dst));
    else xo[off] = a;
  }
  bool bad = false;                      // this thread's wait ran out: the results are void
  if (split > 1) bad = !bar_wait(&ex_bar);
  else __syncthreads();

  // ---- every CTA: the unit's normaliser (all data is local now) and its slice of the output
  float m_all = -INFINITY, inv_all = 0.f;      // of the one head
  auto join = [&](int h, float (&fr)[Q4_SPLIT]) {
    float2 ml[Q4_SPLIT];
    float L = 0.f;
    m_all = -INFINITY;
#pragma unroll
    for (int r = 0; r < Q4_SPLIT; ++r) {
      ml[r] = r < split ? ex_ml[r][h] : make_float2(-INFINITY, 0.f);
      m_all = fmaxf(m_all, ml[r].x);
    }
#pragma unroll
    for (int r = 0; r < Q4_SPLIT; ++r) {
      fr[r] = ml[r].x > -INFINITY ? exp2_fast(ml[r].x - m_all) : 0.f;
      L = fmaf(ml[r].y, fr[r], L);
    }
    inv_all = 1.f / L;
  };
  if constexpr (GT == 1) {
    float fr[Q4_SPLIT];
    join(0, fr);
    if (tid < slice) {
      float a = 0.f;
#pragma unroll
      for (int r = 0; r < Q4_SPLIT; ++r)
        if (r < split) a = fmaf(xo[r * slice + tid], fr[r], a);
      to_out(out + (int64_t)u * HD + rank * slice + tid, a * inv_all);
    }
  } else {
    if (tid < G) {
      float fr[Q4_SPLIT];
      join(tid, fr);
#pragma unroll
      for (int r = 0; r < Q4_SPLIT; ++r) fr_s[r][tid] = fr[r];
      all_m[tid] = m_all;
      all_inv[tid] = inv_all;
    }
    __syncthreads();
    for (int i = tid; i < G * slice; i += Q4_THREADS) {
      const int h = i >> slice_log2, ch = i & (slice - 1);
      float a = 0.f;
#pragma unroll
      for (int r = 0; r < Q4_SPLIT; ++r)
        if (r < split) a = fmaf(xo[(r * G + h) * slice + ch], fr_s[r][h], a);
      to_out(out + ((int64_t)u * G + h) * HD + rank * slice + ch, a * all_inv[h]);
    }
  }

  // ---- indicator update (Eq. 2 / Eq. 3) and importance (Eq. 4) of this CTA's slots, its arg-min
  const bool evicting = hi > B;
  unsigned long long my_key = Q4_NO_KEY;
  int my_slot = -1, my_pos = -1;
  for (int i0 = tid; i0 < cnt;) {
#pragma unroll
    for (int k = 0; k < SB; ++k) {
      const int i = i0 + k * Q4_THREADS;
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
      c.state.acc[o] = S;
      const int ps = is_new ? t : pos_r[k];
      if (evicting && ps >= F && ps <= t - R) {
        const unsigned long long key = q4_evict_key(S * (is_new ? new_norm_s : norm_r[k]), ps);
        if (key < my_key) { my_key = key; my_slot = s0 + i; my_pos = ps; }
      }
    }
    i0 += SB * Q4_THREADS;
    if (i0 < cnt) fetch(i0);
  }
  if (WINDOWED) {
    // recycled slot: the other rows of its ring column belong to the previous occupant (shared out over the unit's CTAs)
    for (int r = rank * Q4_THREADS + tid; r < w; r += split * Q4_THREADS)
      if (r != t % w) c.state.ring[((int64_t)u * w + r) * cap + fs] = 0.f;
  }
  if (evicting) {
    // this CTA's candidate (positions are unique: one thread holds the winning key), sent to rank 0
    const unsigned long long wkey = min_key(my_key);
    if (lane == 0) warp_key[wid] = wkey;
    __syncthreads();
    const unsigned long long win = min_key(lane < Q4_WARPS ? warp_key[lane] : Q4_NO_KEY);
    if (win == Q4_NO_KEY ? tid == 0 : my_key == win) {
      if (split > 1)
        send4(at_rank(s32(&cand[rank]), 0), (uint32_t)win, (uint32_t)(win >> 32), (uint32_t)my_slot, (uint32_t)my_pos, at_rank(s32(&cand_bar), 0));
      else
        cand[0] = Q4Candidate{win, my_slot, my_pos};
    }
    if (split == 1) __syncthreads();
  }
  if (rank == 0 && tid == 0) {
    int out_slot = hi, left = hi, ev = -1;                         // not evicting: the cache grows
    if (evicting) {
      if (split > 1 && !bar_wait(&cand_bar)) bad = true;
      Q4Candidate best{Q4_NO_KEY, -1, -1};
      for (int r = 0; r < split; ++r)
        if (cand[r].key < best.key) best = cand[r];
      if (best.key != Q4_NO_KEY) {
        out_slot = best.slot;
        ev = best.pos;
        left = hi - 1;
        c.state.pos[(int64_t)u * cap + out_slot] = -1;
      } else {                             // nothing eligible (cannot happen when F + R <= B): keep the state consistent
        out_slot = min(hi, cap - 1);
      }
    }
    c.state.len[u] = left;
    c.state.free_slot[u] = out_slot;
    c.state.next_pos[u] = t + 1;
    c.state.last_slot[u] = fs;
    if (evicted) evicted[u] = ev;
  }
  if (bad) {
    // Something never arrived: say so, and stay until the unit's other CTAs have sent what they send here (threads that exit count
    // as arrived).
    if (dev_status) atomicExch(dev_status, (int)VATP_ERR_TIMEOUT);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
}

template <typename T, int HD, int GT>
cudaError_t launch_gt(int units, int G, int B, int F, int R, int window, int norm, float scale, const vatp_cache_q4& c, const void* q,
                      const void* k, const void* v, void* out, int32_t* evicted, int32_t* dev_status, cudaStream_t st) {
  const int cap = cache_capacity(B), sms = device_sm_count();
  // The logits of a CTA's slots stand in shared memory beside the warps' partial outputs.
  const size_t most = 200 * 1024, partials = (size_t)Q4_WARPS * G * HD * 4;
  auto chunk_of = [&](int split) { return ((cap + split - 1) / split + Q4_TILE - 1) / Q4_TILE * Q4_TILE; };
  int split = 1;
  while (split < Q4_SPLIT && units * split * 2 <= 2 * sms && cap / (split * 2) >= 4 * Q4_TILE) split *= 2;
  while (split < Q4_SPLIT && partials + (size_t)G * chunk_of(split) * 4 > most) split *= 2;
  const int chunk = chunk_of(split);
  const size_t dyn = partials + (size_t)G * chunk * 4;
  if (dyn > most || (int64_t)units * split > 0x7fffffffll) return cudaErrorNotSupported;
  auto kern = window > 0 ? decode_q4_kernel<T, HD, true, GT> : decode_q4_kernel<T, HD, false, GT>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * split));
  cfg.blockDim = dim3(Q4_THREADS);
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
  return cudaLaunchKernelEx(&cfg, kern, G, split, chunk, chunk, B, cap, F, R, window, norm, scale * Q4_LOG2E, c, (const T*)q, (const T*)k,
                            (const T*)v, (T*)out, evicted, dev_status);
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
