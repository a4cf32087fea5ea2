// Decode step on a cache whose rows are held in 4 bits: append (quantised), attend (Eq. 1), indicator update (Eq. 2 / Eq. 3),
// importance (Eq. 4), release of the lowest-importance unprotected slot.
//
// With the values lo_ig + sc_ig code_ic of row i, group g and channel c:
//   s_i = scale * sum_g ( sc_ig * sum_{c in g} q_c code_ic + lo_ig * sum_{c in g} q_c ),   p = softmax(s)
//   o_c = sum_i p_i lo_ig + sum_i (p_i sc_ig) code_ic
#include "q4.cuh"

namespace vatp {
namespace {

constexpr int Q4_THREADS = 256, Q4_WARPS = Q4_THREADS / 32;
constexpr float Q4_LOG2E = 1.4426950408889634f;

__device__ __forceinline__ unsigned long long q4_evict_key(float I, int pos) {
  return ((unsigned long long)__float_as_uint(I) << 32) | (unsigned)(0x7fffffff - pos);
}
__device__ __forceinline__ float block_reduce(float x, bool max, float* tmp) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const float y = __shfl_xor_sync(0xffffffffu, x, o);
    x = max ? fmaxf(x, y) : x + y;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) tmp[threadIdx.x >> 5] = x;
  __syncthreads();
  x = tmp[0];
  for (int i = 1; i < Q4_WARPS; ++i) x = max ? fmaxf(x, tmp[i]) : x + tmp[i];
  return x;
}

// One CTA per unit.
template <typename T, int HD, bool WINDOWED>
__global__ void __launch_bounds__(Q4_THREADS)
decode_q4_kernel(int G, int B, int cap, int F, int R, int w, int norm, float scale_log2, vatp_cache_q4 c, const T* q_new, const T* k_new,
                 const T* v_new, T* out, int32_t* evicted, int32_t* dev_status) {
  constexpr int NG = HD / 32;
  extern __shared__ float logit_s[];        // [G][cap]
  __shared__ float q_s[8][HD], qsum_s[8][NG], tmp[Q4_WARPS], inv_l[8], new_norm_s;
  __shared__ unsigned long long keys[Q4_WARPS];
  const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int len = min(max(c.state.len[u], 0), cap - 1), fs = min(max(c.state.free_slot[u], 0), cap - 1), t = c.state.next_pos[u];
  const int hi = len + 1;
  const int64_t base = (int64_t)u * cap;
  for (int i = tid; i < G * HD; i += Q4_THREADS) q_s[i / HD][i % HD] = to_f32(q_new[(int64_t)u * G * HD + i]);
  if (wid < 2) {
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (lane < HD / 4)
      for (int e = 0; e < 4; ++e) x[e] = to_f32((wid ? v_new : k_new)[(int64_t)u * HD + 4 * lane + e]);
    uint32_t params;
    const uint32_t code = q4_row(x, params);
    if (lane < HD / 4) {
      unsigned char* row = static_cast<unsigned char*>(wid ? c.state.v_cache : c.state.k_cache) + (base + fs) * (HD / 2);
      *reinterpret_cast<uint16_t*>(row + q4_byte<HD>(lane / 8, lane % 8)) = (uint16_t)code;
      if (lane % 8 == 0) static_cast<uint32_t*>(wid ? c.v_params : c.k_params)[(base + fs) * NG + lane / 8] = params;
    }
    if (wid == 1) {
      float n = 0.f;
      for (int e = 0; e < 4; ++e) n = norm_fold(norm, n, x[e]);
      for (int o = 16; o; o >>= 1) n = norm_merge(norm, n, __shfl_xor_sync(0xffffffffu, n, o));
      if (lane == 0) {
        new_norm_s = n = norm_finish(norm, n);
        c.state.vnorm[base + fs] = n;
        c.state.pos[base + fs] = t;
      }
    }
  }
  __syncthreads();
  if (tid < G * NG) {
    float a = 0.f;
    for (int i = 0; i < 32; ++i) a += q_s[tid / NG][(tid % NG) * 32 + i];
    qsum_s[tid / NG][tid % NG] = a;
  }
  __syncthreads();
  const unsigned char* kc = static_cast<const unsigned char*>(c.state.k_cache) + base * (HD / 2);
  const unsigned char* vc = static_cast<const unsigned char*>(c.state.v_cache) + base * (HD / 2);
  const uint32_t* kp = static_cast<const uint32_t*>(c.k_params) + base * NG;
  const uint32_t* vp = static_cast<const uint32_t*>(c.v_params) + base * NG;
  for (int i = tid; i < hi; i += Q4_THREADS)
    for (int h = 0; h < G; ++h) {
      float s = 0.f;
      for (int g = 0; g < NG; ++g) {
        float a = 0.f;
        for (int j = 0; j < 8; ++j) {
          const uint32_t code = *reinterpret_cast<const uint16_t*>(kc + (int64_t)i * (HD / 2) + q4_byte<HD>(g, j));
          for (int e = 0; e < 4; ++e) a = fmaf(q_s[h][32 * g + 4 * j + e], (float)(code >> (4 * e) & 15u), a);
        }
        const uint32_t pr = kp[(int64_t)i * NG + g];
        s = fmaf(q4_scale(pr), a, fmaf(q4_low(pr), qsum_s[h][g], s));
      }
      logit_s[h * cap + i] = s * scale_log2;
    }
  __syncthreads();
  for (int h = 0; h < G; ++h) {
    float m = -INFINITY, l = 0.f;
    for (int i = tid; i < hi; i += Q4_THREADS) m = fmaxf(m, logit_s[h * cap + i]);
    m = block_reduce(m, true, tmp);
    for (int i = tid; i < hi; i += Q4_THREADS) l += logit_s[h * cap + i] = exp2f(logit_s[h * cap + i] - m);
    l = block_reduce(l, false, tmp);
    if (tid == 0) inv_l[h] = 1.f / l;
  }
  __syncthreads();
  for (int x = tid; x < G * HD; x += Q4_THREADS) {
    const int h = x / HD, ch = x % HD, g = ch / 32, j = ch % 32 / 4, e = ch % 4;
    float a = 0.f;
    for (int i = 0; i < hi; ++i) {
      const uint32_t code = *reinterpret_cast<const uint16_t*>(vc + (int64_t)i * (HD / 2) + q4_byte<HD>(g, j)) >> (4 * e) & 15u;
      const uint32_t pr = vp[(int64_t)i * NG + g];
      a = fmaf(logit_s[h * cap + i], fmaf((float)code, q4_scale(pr), q4_low(pr)), a);
    }
    a *= inv_l[h];
    if constexpr (sizeof(T) == 2) out[((int64_t)u * G + h) * HD + ch] = __float2bfloat16(a);
    else out[((int64_t)u * G + h) * HD + ch] = a;
  }
  const bool evicting = hi > B;
  unsigned long long key = ~0ull;
  int key_slot = -1;
  for (int i = tid; i < hi; i += Q4_THREADS) {
    float p = 0.f;
    for (int h = 0; h < G; ++h) p = fmaf(logit_s[h * cap + i], inv_l[h], p);
    p /= (float)G;
    const bool is_new = i == fs;
    float S;
    if (WINDOWED) {
      float* ring = c.state.ring + ((int64_t)u * w + (t % w)) * cap + i;
      const long long fx = is_new ? prob_to_fixed(p) : c.state.acc_fixed[base + i] + prob_to_fixed(p) - prob_to_fixed(*ring);
      *ring = p;
      c.state.acc_fixed[base + i] = fx;
      S = fixed_to_prob(fx);
    } else {
      S = is_new ? p : c.state.acc[base + i] + p;
    }
    c.state.acc[base + i] = S;
    const int ps = is_new ? t : c.state.pos[base + i];
    if (evicting && ps >= F && ps <= t - R) {
      const unsigned long long x = q4_evict_key(S * (is_new ? new_norm_s : c.state.vnorm[base + i]), ps);
      if (x < key) { key = x; key_slot = i; }
    }
  }
  if (WINDOWED)
    for (int r = tid; r < w; r += Q4_THREADS)
      if (r != t % w) c.state.ring[((int64_t)u * w + r) * cap + fs] = 0.f;
  unsigned long long best = key;
  for (int o = 16; o; o >>= 1) { const unsigned long long y = __shfl_xor_sync(0xffffffffu, best, o); best = y < best ? y : best; }
  if (lane == 0) keys[wid] = best;
  __syncthreads();
  for (int i = 0; i < Q4_WARPS; ++i) best = keys[i] < best ? keys[i] : best;
  if (best == ~0ull ? tid == 0 : key == best) {          // (positions are unique: one thread holds the winning key)
    int out_slot = hi, left = hi, ev = -1;
    if (evicting) {
      out_slot = best == ~0ull ? min(hi, cap - 1) : key_slot;
      if (best != ~0ull) {
        left = hi - 1;
        ev = 0x7fffffff - (int)(unsigned)best;
        c.state.pos[base + out_slot] = -1;
      }
    }
    c.state.len[u] = left;
    c.state.free_slot[u] = out_slot;
    c.state.next_pos[u] = t + 1;
    c.state.last_slot[u] = fs;
    if (evicted) evicted[u] = ev;
  }
}

template <typename T, int HD>
cudaError_t launch_hd(int units, int G, int B, int F, int R, int window, int norm, float scale, const vatp_cache_q4& c, const void* q,
                      const void* k, const void* v, void* out, int32_t* evicted, int32_t* dev_status, cudaStream_t st) {
  const int cap = cache_capacity(B);
  const size_t dyn = (size_t)G * cap * 4;
  if (G > 8 || dyn > 200 * 1024) return cudaErrorNotSupported;
  auto kern = window > 0 ? decode_q4_kernel<T, HD, true> : decode_q4_kernel<T, HD, false>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  if (e != cudaSuccess) return e;
  DependentLaunch dl(dim3(units), dim3(Q4_THREADS), dyn, st);
  return cudaLaunchKernelEx(&dl.cfg, kern, G, B, cap, F, R, window, norm, scale * Q4_LOG2E, c, (const T*)q, (const T*)k, (const T*)v, (T*)out,
                            evicted, dev_status);
}

}  // namespace

cudaError_t launch_decode_q4(int units, int G, int d, int dtype, int B, int F, int R, int window, int norm, float scale, const vatp_cache_q4& c,
                             const void* q, const void* k, const void* v, void* out, int32_t* evicted, int32_t* dev_status, cudaStream_t st) {
  auto f = dtype == VATP_F32 ? (d == 64 ? launch_hd<float, 64> : launch_hd<float, 128>)
                             : (d == 64 ? launch_hd<__nv_bfloat16, 64> : launch_hd<__nv_bfloat16, 128>);
  return f(units, G, B, F, R, window, norm, scale, c, q, k, v, out, evicted, dev_status, st);
}

}  // namespace vatp
