// The attention that each cached row gets, added up over the denoising steps: for a cached row k of a head
//   out = decay * in + sum_i exp(q_i . k * scale - lse_i)    over the query rows i of the head's group.
//
// A thread per cached row, the query rows in order.
#include "mx.hpp"

namespace maskkv {

namespace {

struct AccumulateParams {
  View Q;
  const char* Kc;
  MxCache cache;
  const int32_t* cu;
  int64_t capacity;
  int H, BH, q_per_kv, n_resp, n_q;
  float c;  // scale * log2(e)
  float decay;
  const float *lse, *in;
  float* out;
};

template <typename T>
__device__ __forceinline__ float element(const char* p, int i) {
  if (sizeof(T) == 2) return as_f32((uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << 16);
  return reinterpret_cast<const float*>(p)[i];
}

template <typename T, int D, bool MX>
__global__ __launch_bounds__(256) void accumulate_kernel(const AccumulateParams prm) {
  const int64_t total = min((int64_t)prm.cu[prm.BH], prm.capacity);
  const int64_t first = (int64_t)blockIdx.x * 256 + (threadIdx.x & ~63);
  if (first >= total) return;
  const int64_t row = min(first + (threadIdx.x & 63), total - 1);
  int bh = head_of_row(prm.cu, prm.BH, (int)first);
  while (bh + 1 < prm.BH && prm.cu[bh + 1] <= row) ++bh;
  float k[D];
  if (MX) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      float x[8];
      mx_decode_f32(reinterpret_cast<const uint32_t*>(prm.cache.k_codes + row * (D / 2))[i],
                    mx_unit(reinterpret_cast<const uint8_t*>(prm.cache.k_scales)[row * (D / 32) + i / 4]), x);
#pragma unroll
      for (int j = 0; j < 8; ++j) k[8 * i + j] = x[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < D; ++i) k[i] = element<T>(prm.Kc + row * (D * (int)sizeof(T)), i);
  }
  float sum = 0.f;
  for (int i = 0; i < prm.n_q; ++i) {
    const char* q = prm.Q.group_row(bh / prm.H, bh % prm.H, prm.q_per_kv, prm.n_resp, i);
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < D; ++j) s = fmaf(element<T>(q, j), k[j], s);
    sum += fast_exp2(fmaf(s, prm.c, -prm.lse[(int64_t)bh * prm.n_q + i] * kLog2e));
  }
  if (first + (threadIdx.x & 63) < total) prm.out[row] = prm.decay > 0.f ? fmaf(prm.decay, prm.in[row], sum) : sum;
}

template <typename T, int D>
void launch_one(const AccumulateParams& prm, hipStream_t stream) {
  const dim3 grid((unsigned)((prm.capacity + 255) / 256));
  if (prm.Kc)
    hipLaunchKernelGGL((accumulate_kernel<T, D, false>), grid, dim3(256), 0, stream, prm);
  else
    hipLaunchKernelGGL((accumulate_kernel<T, D, true>), grid, dim3(256), 0, stream, prm);
}

}  // namespace

int launch_accumulate(const maskkv_desc* d, const View& Q, const void* Kc, const MxCache& cache, const int32_t* cu_budget, int64_t capacity,
                      float scale, const float* row_lse, float decay, const float* weights_in, float* weights_out, hipStream_t stream) {
  if (capacity == 0) return MASKKV_OK;
  AccumulateParams prm;
  prm.Q = Q;
  prm.Kc = reinterpret_cast<const char*>(Kc);
  prm.cache = cache;
  prm.cu = cu_budget;
  prm.capacity = capacity;
  prm.H = d->H;
  prm.BH = d->B * d->H;
  prm.q_per_kv = query_heads_per_kv(d);
  prm.n_resp = d->n_resp;
  prm.n_q = prm.q_per_kv * d->n_resp;
  prm.c = scale * kLog2e;
  prm.decay = decay;
  prm.lse = row_lse;
  prm.in = weights_in;
  prm.out = weights_out;
  if (d->dtype == MASKKV_BF16)
    d->d == 128 ? launch_one<bf16_t, 128>(prm, stream) : launch_one<bf16_t, 64>(prm, stream);
  else
    d->d == 128 ? launch_one<float, 128>(prm, stream) : launch_one<float, 64>(prm, stream);
  return check_launch("accumulate");
}

}  // namespace maskkv
