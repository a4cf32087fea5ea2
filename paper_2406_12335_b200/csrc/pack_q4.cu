// Rows of K and V to and from their 4-bit form: compaction of a prompt's kept rows, conversion of a decode state, and back.
//
// Bound by memory where the number of instructions allows: a row of 128 bf16 channels is 256 bytes in one form and 80 in the other.
// 256 units x 1639 slots: rows into 4 bits 45.4 us (6.25 TB/s, 0.96 of a copy's rate), gathered out of prompts of 8192 tokens 54.7 (rows
// of 256 bytes anywhere), back 47.9.
#include "cache_copy.cuh"
#include "q4.cuh"

namespace vatp {
namespace {

constexpr int PK_WARPS = 2, PK_THREADS = PK_WARPS * 32;      // (8 warps a CTA, which end together: 256 units x 1639 slots 48.8 us, so 45.3)
constexpr int UP_THREADS = 256;

// CTA `i` of those that copy a state from a to c; false for i < 0 (a CTA that has rows to do).  The unit's words go with its first CTA.
template <int THREADS>
__device__ __forceinline__ bool copy_state(const CopyPlan& plan, int i, const vatp_cache& a, const vatp_cache& c) {
  if (i < 0) return false;
  const int u = i / plan.ctas, cta = i - u * plan.ctas;
  if (cta == 0 && threadIdx.x == 0) copy_unit_words(a, u, c, u);
  copy_words<THREADS>(plan, cta, u, [&](auto f) { f(u); });
  return true;
}

// A group of a row as it is stored: its least and largest value, and each of them.
template <typename T> struct Group32;
template <> struct Group32<__nv_bfloat16> {
  uint32_t w[16];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 r = load_behind_wait(reinterpret_cast<const uint4*>(p) + i);
      w[4 * i] = r.x; w[4 * i + 1] = r.y; w[4 * i + 2] = r.z; w[4 * i + 3] = r.w;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
  __device__ __forceinline__ void range(float& mn, float& mx) const {      // two values an instruction
    __nv_bfloat162 a = reinterpret_cast<const __nv_bfloat162&>(w[0]), b = a;
#pragma unroll
    for (int i = 1; i < 16; ++i) {
      const __nv_bfloat162 x = reinterpret_cast<const __nv_bfloat162&>(w[i]);
      a = __hmin2_nan(a, x);
      b = __hmax2_nan(b, x);
    }
    mn = min_nan(__low2float(a), __high2float(a));
    mx = max_nan(__low2float(b), __high2float(b));
  }
};
template <> struct Group32<float> {
  float x[32];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float4 r = load_behind_wait(reinterpret_cast<const float4*>(p) + i);
      x[4 * i] = r.x; x[4 * i + 1] = r.y; x[4 * i + 2] = r.z; x[4 * i + 3] = r.w;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = 0.f;
  }
  __device__ __forceinline__ float at(int i) const { return x[i]; }
  __device__ __forceinline__ void range(float& mn, float& mx) const {
    mn = mx = x[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) { mn = min_nan(mn, x[i]); mx = max_nan(mx, x[i]); }
  }
};

// A warp takes 1024 / HD consecutive slots of a unit, a lane one group of a row: its range needs no exchange, the arithmetic of a
// group's parameters is done once.  The codes pass through 512 bytes of shared memory so that they leave as full 16-byte words.
// (What bounds it is the number of instructions: with half a group a lane, 17 a value where this has 9.)
// kept != nullptr (compaction): slot s of unit u takes row kept[u][s] of the prompt, and the decode state is initialised.
// kept == nullptr (conversion): slot s takes slot s of the cache k, v where its state `a` says that it holds a token; further CTAs copy
// that state (STATE: plan; a kernel of its own, since its copies in flight take registers: 256 units x 1639 slots without them 45.4 us, in
// one kernel 50.0; the way back 47.9 and 60.4).
template <typename T, int HD, bool STATE>
__global__ void __launch_bounds__(PK_THREADS)
pack_q4_kernel(const __grid_constant__ CopyPlan plan, Shape sh, int B, int cap, int blocks_per_unit, const T* k, const T* v, const int32_t* kept,
               vatp_cache a, const float* attn_acc, const float* vnorm, vatp_cache_q4 c, int32_t* dev_status) {
  constexpr int NG = HD / 32, ROWS = 32 / NG;                    // lanes a row, rows of a warp
  __shared__ __align__(16) unsigned char stage[PK_WARPS][2][512];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int u = blockIdx.x / blocks_per_unit;
  const int first = ((blockIdx.x - u * blocks_per_unit) * PK_WARPS + wid) * ROWS;      // this warp's first slot
  const int g = lane % NG, s = first + lane / NG;                 // this lane's group and slot
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if constexpr (STATE)
    if (copy_state<PK_THREADS>(plan, blockIdx.x - sh.units * blocks_per_unit, a, c.state)) return;
  if (first >= cap) return;
  const int len = min(sh.T, B);
  const int64_t o = (int64_t)u * cap + s;
  int src = -1;                                                   // row of the prompt, or slot
  int64_t from = 0;
  if (kept) {
    if (s < len) src = kept[(int64_t)u * B + s];
    if (src >= 0 && !VATP_INB(src, sh.T, dev_status)) src = -1;
    from = unit_offset(sh, u) + (int64_t)src * sh.st;
  } else {
    if (s < cap && a.pos[o] >= 0) src = s;
    from = o * HD;
  }
  Group32<T> x[2];
  if (src >= 0) {
    x[0].load(k + from + 32 * g);
    x[1].load(v + from + 32 * g);
  } else {
    x[0].clear();
    x[1].clear();
  }
  if (kept && g == 0 && s < cap) {
    c.state.pos[o] = src;
    c.state.acc[o] = src >= 0 ? attn_acc[(int64_t)u * sh.T + src] : 0.f;
    c.state.vnorm[o] = src >= 0 ? vnorm[(int64_t)u * sh.T + src] : 0.f;
    if (s == 0) {
      c.state.len[u] = len;
      c.state.free_slot[u] = len;
      c.state.next_pos[u] = sh.T;
      c.state.last_slot[u] = -1;
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    float mn, mx;
    x[t].range(mn, mx);
    const Q4Group q = q4_group(mn, mx);
    if (src >= 0) reinterpret_cast<uint32_t*>(t ? c.v_params : c.k_params)[o * NG + g] = q4_params(q);
    unsigned char* row = stage[wid][t] + (lane / NG) * (HD / 2);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *reinterpret_cast<uint16_t*>(row + q4_byte<HD>(g, j)) = (uint16_t)q4_codes(q, x[t].at(4 * j), x[t].at(4 * j + 1), x[t].at(4 * j + 2), x[t].at(4 * j + 3));
  }
  const uint32_t rows = __ballot_sync(0xffffffffu, src >= 0 && g == 0);           // bit NG * r: row r is live
  __syncwarp();                                                   // (a vote orders no memory)
  const int at = lane * 16, r = at / (HD / 2);
  if (rows >> (NG * r) & 1u) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      unsigned char* dst = static_cast<unsigned char*>(t ? c.state.v_cache : c.state.k_cache) + ((int64_t)u * cap + first) * (HD / 2) + at;
      *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(stage[wid][t] + at);
    }
  }
}

__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&x)[4]) {
  __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(reinterpret_cast<uint32_t&>(a), reinterpret_cast<uint32_t&>(b));
}
__device__ __forceinline__ void store4(float* p, const float (&x)[4]) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }

// A lane takes HD / 16 bytes of a row, i.e. four channels of each of its groups; eight lanes a row.  A warp's stores of one group
// cover four rows, 64 or 128 bytes each.
template <typename T, int HD, bool STATE>
__global__ void __launch_bounds__(UP_THREADS)
unpack_q4_kernel(const __grid_constant__ CopyPlan plan, int row_ctas, int64_t slots, vatp_cache_q4 c, vatp_cache to) {
  constexpr int G = HD / 32;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if constexpr (STATE)
    if (copy_state<UP_THREADS>(plan, blockIdx.x - row_ctas, c.state, to)) return;
  T* k = static_cast<T*>(to.k_cache);
  T* v = static_cast<T*>(to.v_cache);
  const int64_t i = (int64_t)blockIdx.x * (UP_THREADS / 8) + threadIdx.x / 8;    // the slot
  const int j = threadIdx.x & 7;
  if (i >= slots || c.state.pos[i] < 0) return;
  uint32_t w[2][G / 2], pr[2][G];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const unsigned char* codes = static_cast<const unsigned char*>(t ? c.state.v_cache : c.state.k_cache) + i * (HD / 2) + j * (HD / 16);
    const uint32_t* params = static_cast<const uint32_t*>(t ? c.v_params : c.k_params) + i * G;
#pragma unroll
    for (int x = 0; x < G / 2; ++x) w[t][x] = load_behind_wait(reinterpret_cast<const uint32_t*>(codes) + x);
#pragma unroll
    for (int x = 0; x < G; ++x) pr[t][x] = load_behind_wait(params + x);
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t code = w[t][g / 2] >> (16 * (g & 1));
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = fmaf((float)(code >> (4 * e) & 15u), q4_scale(pr[t][g]), q4_low(pr[t][g]));
      store4((t ? v : k) + i * HD + 32 * g + 4 * j, x);
    }
}

template <typename T, int HD>
cudaError_t pack_hd(const Shape& s, int B, const void* k, const void* v, const int32_t* kept, const CacheArray* arrays, int n, const vatp_cache& a,
                    const float* attn_acc, const float* vnorm, const vatp_cache_q4& c, int32_t* dev_status, cudaStream_t st) {
  constexpr int SLOTS = PK_WARPS * 1024 / HD;      // of a CTA
  const int cap = cache_capacity(B), per_unit = (cap + SLOTS - 1) / SLOTS;
  CopyPlan plan;
  if (!make_copy_plan(&plan, arrays, n, true, cap, cap, PK_THREADS)) return cudaErrorInvalidValue;
  if (!plan.ctas && unit_words_apart(a, c.state)) plan.ctas = 1;
  const int64_t ctas = (int64_t)s.units * ((int64_t)per_unit + plan.ctas);
  if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  DependentLaunch dl(dim3((unsigned)ctas), dim3(PK_THREADS), 0, st);
  return cudaLaunchKernelEx(&dl.cfg, plan.ctas ? pack_q4_kernel<T, HD, true> : pack_q4_kernel<T, HD, false>, plan, s, B, cap, per_unit, (const T*)k, (const T*)v, kept, a, attn_acc, vnorm, c, dev_status);
}

template <typename T, int HD>
cudaError_t unpack_hd(int units, int B, const vatp_cache_q4& c, const CacheArray* arrays, int n, const vatp_cache& to, cudaStream_t st) {
  const int cap = cache_capacity(B);
  const int64_t slots = (int64_t)units * cap, ctas = (slots + UP_THREADS / 8 - 1) / (UP_THREADS / 8);
  CopyPlan plan;
  if (!make_copy_plan(&plan, arrays, n, true, cap, cap, UP_THREADS)) return cudaErrorInvalidValue;
  if (!plan.ctas && unit_words_apart(c.state, to)) plan.ctas = 1;
  if (ctas + (int64_t)units * plan.ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  DependentLaunch dl(dim3((unsigned)(ctas + (int64_t)units * plan.ctas)), dim3(UP_THREADS), 0, st);
  return cudaLaunchKernelEx(&dl.cfg, plan.ctas ? unpack_q4_kernel<T, HD, true> : unpack_q4_kernel<T, HD, false>, plan, (int)ctas, slots, c, to);
}

}  // namespace

cudaError_t launch_compact_q4(const Shape& s, int dtype, int B, const void* k, const void* v, const int32_t* kept, const float* attn_acc,
                              const float* vnorm, const float* win_rows, const vatp_cache_q4& c, int32_t* dev_status, cudaStream_t st) {
  auto f = dtype == VATP_F32 ? (s.d == 64 ? pack_hd<float, 64> : pack_hd<float, 128>)
                             : (s.d == 64 ? pack_hd<__nv_bfloat16, 64> : pack_hd<__nv_bfloat16, 128>);
  cudaError_t e = f(s, B, k, v, kept, nullptr, 0, c.state, attn_acc, vnorm, c, dev_status, st);
  if (e == cudaSuccess && s.window > 0) e = launch_ring(s, B, win_rows, kept, c.state, dev_status, st);
  return e;
}

cudaError_t launch_pack_q4(int units, int d, int dtype, int B, const vatp_cache& from, const CacheArray* arrays, int n, const vatp_cache_q4& to,
                           int32_t* dev_status, cudaStream_t st) {
  Shape s;
  memset(&s, 0, sizeof(s));
  s.units = units;
  s.heads = 1;
  auto f = dtype == VATP_F32 ? (d == 64 ? pack_hd<float, 64> : pack_hd<float, 128>) : (d == 64 ? pack_hd<__nv_bfloat16, 64> : pack_hd<__nv_bfloat16, 128>);
  return f(s, B, from.k_cache, from.v_cache, nullptr, arrays, n, from, nullptr, nullptr, to, dev_status, st);
}

cudaError_t launch_unpack_q4(int units, int d, int dtype, int B, const vatp_cache_q4& from, const CacheArray* arrays, int n, const vatp_cache& to,
                             cudaStream_t st) {
  auto f = dtype == VATP_F32 ? (d == 64 ? unpack_hd<float, 64> : unpack_hd<float, 128>)
                             : (d == 64 ? unpack_hd<__nv_bfloat16, 64> : unpack_hd<__nv_bfloat16, 128>);
  return f(units, B, from, arrays, n, to, st);
}

}  // namespace vatp
