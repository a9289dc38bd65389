// Attention of the response span over a cache in 4 bits and the response's own rows.
//
// A workgroup per query row: 256 keys at a time, a logit a thread, the running maximum and sum of the softmax, then the
// values, an element of the head dimension a thread.
#include "mx.hpp"

namespace maskkv {

namespace {

constexpr int kThreads = 256;

struct AttendMxParams {
  View Q, K2, V2, O;
  MxCache cache;
  const int32_t* cu;
  int64_t capacity;
  int H, q_per_kv, n_resp, n_q;
  float c;  // scale * log2(e)
  float* lse;
};

template <typename T>
__device__ __forceinline__ float element(const char* p, int i) {
  if (sizeof(T) == 2) return as_f32((uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << 16);
  return reinterpret_cast<const float*>(p)[i];
}

template <bool MAX>
__device__ __forceinline__ float over_all(float v, float* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float w = __shfl_xor(v, o, 64);
    v = MAX ? fmaxf(v, w) : v + w;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return MAX ? fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])) : (part[0] + part[1]) + (part[2] + part[3]);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void attend_mx_kernel(const AttendMxParams prm) {
  __shared__ float q[D], p[kThreads], part[4], half[2][D];
  const int bh = blockIdx.y, i = blockIdx.x, t = threadIdx.x;
  const int b = bh / prm.H, h = bh % prm.H;
  const int64_t c0 = min((int64_t)prm.cu[bh], prm.capacity), c1 = min((int64_t)prm.cu[bh + 1], prm.capacity);
  const int cached = max((int)(c1 - c0), 0), n = cached + prm.n_resp;
  const char* qrow = prm.Q.group_row(b, h, prm.q_per_kv, prm.n_resp, i);
  if (t < D) q[t] = element<T>(qrow, t);
  float m = kNegBig, l = 0.f, o = 0.f;
  for (int base = 0; base < n; base += kThreads) {
    __syncthreads();
    const int j = base + t;
    float s = 0.f;
    if (j < cached) {
      for (int e = 0; e < D / 8; ++e) {
        float x[8];
        mx_decode_f32(reinterpret_cast<const uint32_t*>(prm.cache.k_codes + (c0 + j) * (D / 2))[e],
                      mx_unit(reinterpret_cast<const uint8_t*>(prm.cache.k_scales)[(c0 + j) * (D / 32) + e / 4]), x);
        for (int u = 0; u < 8; ++u) s = fmaf(q[8 * e + u], x[u], s);
      }
    } else if (j < n) {
      const char* k = prm.K2.row(b, h, j - cached);
      for (int e = 0; e < D; ++e) s = fmaf(q[e], element<T>(k, e), s);
    }
    s *= prm.c;
    const float m_new = fmaxf(m, over_all<true>(j < n ? s : kNegBig, part));
    const float x = j < n ? fast_exp2(s - m_new) : 0.f, alpha = fast_exp2(m - m_new);
    l = l * alpha + over_all<false>(x, part);
    o *= alpha;
    m = m_new;
    p[t] = x;
    __syncthreads();
    const int e = t % D, g = t / D;
    const int many = min(n - base, kThreads);
    for (int u = g; u < many; u += kThreads / D) {
      const int r = base + u;
      float v;
      if (r < cached) {
        float x8[8];
        mx_decode_f32(reinterpret_cast<const uint32_t*>(prm.cache.v_codes + (c0 + r) * (D / 2))[e / 8],
                      mx_unit(reinterpret_cast<const uint8_t*>(prm.cache.v_scales)[(c0 + r) * (D / 32) + e / 32]), x8);
        v = x8[0];
        for (int w = 1; w < 8; ++w) v = e % 8 == w ? x8[w] : v;
      } else {
        v = element<T>(prm.V2.row(b, h, r - cached), e);
      }
      o = fmaf(p[u], v, o);
    }
  }
  __syncthreads();
  if (kThreads / D == 4) {
    if (t >= 2 * D) half[t / D - 2][t % D] = o;
    __syncthreads();
    if (t < 2 * D) o += half[t / D][t % D];
    __syncthreads();
  }
  if (t >= D && t < 2 * D) half[0][t - D] = o;
  __syncthreads();
  if (t < D) {
    o = (o + half[0][t]) / l;
    char* to = prm.O.group_row(b, h, prm.q_per_kv, prm.n_resp, i);
    if (sizeof(T) == 2)
      reinterpret_cast<uint16_t*>(to)[t] = (uint16_t)pack_bf16x2(o, o);
    else
      reinterpret_cast<float*>(to)[t] = o;
  }
  if (t == 0 && prm.lse) prm.lse[(int64_t)bh * prm.n_q + i] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

size_t attend_mx_workspace_bytes(const maskkv_desc*, int64_t) { return 0; }

int launch_attend_mx(const maskkv_desc* d, const View& Q, const MxCache& cache, const int32_t* cu_budget, int64_t capacity, const View& K2,
                     const View& V2, float scale, const View& O, float* lse, void*, hipStream_t stream) {
  AttendMxParams prm;
  prm.Q = Q;
  prm.K2 = K2;
  prm.V2 = V2;
  prm.O = O;
  prm.cache = cache;
  prm.cu = cu_budget;
  prm.capacity = capacity;
  prm.H = d->H;
  prm.q_per_kv = query_heads_per_kv(d);
  prm.n_resp = d->n_resp;
  prm.n_q = prm.q_per_kv * d->n_resp;
  prm.c = scale * kLog2e;
  prm.lse = lse;
  const dim3 grid((unsigned)prm.n_q, (unsigned)(d->B * d->H));
  if (d->dtype == MASKKV_BF16) {
    if (d->d == 128)
      hipLaunchKernelGGL((attend_mx_kernel<bf16_t, 128>), grid, dim3(kThreads), 0, stream, prm);
    else
      hipLaunchKernelGGL((attend_mx_kernel<bf16_t, 64>), grid, dim3(kThreads), 0, stream, prm);
  } else {
    if (d->d == 128)
      hipLaunchKernelGGL((attend_mx_kernel<float, 128>), grid, dim3(kThreads), 0, stream, prm);
    else
      hipLaunchKernelGGL((attend_mx_kernel<float, 64>), grid, dim3(kThreads), 0, stream, prm);
  }
  return check_launch("attend_mx");
}

}  // namespace maskkv
