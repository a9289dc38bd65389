// Further eviction from a packed cache: of each head the rows of largest weight stay.
//
// Two launches.  The first, a workgroup per head, finds the smallest weight that stays by a search over the bits of the
// weights' order, and lists the rows that stay, ascending.  The second moves them: a packed row's number is all it needs, so
// no search for heads comes before its loads.
#include "kernels.hpp"

namespace maskkv {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

struct EvictParams {
  const float* weights;
  const int32_t *cu, *budgets, *idx;
  int64_t capacity, capacity_out;
  int BH;
  int32_t *rows, *idx_out, *cu_out;
  float* weights_out;
  MovedRows moved;
};

// Weights in the order of unsigned numbers: NaN, -infinity ... -0 = 0 ... infinity.
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = as_u32(w);
  if (w != w) return 0u;
  if (u << 1 == 0) return 0x80000000u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int length_of(const EvictParams& prm, int bh, int& first) {
  const int capacity = (int)prm.capacity;
  first = min(prm.cu[bh], capacity);
  return max(min(prm.cu[bh + 1], capacity) - first, 0);
}
__device__ __forceinline__ int stay_of(const EvictParams& prm, int bh) {
  int first;
  const int n = length_of(prm, bh, first);
  return min(max(prm.budgets[bh], 0), n);
}

// The sum of a value over the workgroup.
__device__ __forceinline__ int sum_all(int v, int* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += part[w];
  return s;
}

__global__ __launch_bounds__(kThreads) void evict_rows_kernel(const EvictParams prm) {
  __shared__ int part[kWaves], ties_of[kWaves];
  const int bh = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int before = 0;
  for (int i = t; i < bh; i += kThreads) before += stay_of(prm, i);
  before = sum_all(before, part);
  int first;
  const int n = length_of(prm, bh, first), k = stay_of(prm, bh);
  if (t == 0) {
    prm.cu_out[bh] = before;
    if (bh == prm.BH - 1) prm.cu_out[prm.BH] = before + k;
  }
  if (k == 0) return;
  const float* w = prm.weights + first;
  uint32_t least = 0;  // the largest order that k rows have at least
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
    int c = 0;
    for (int i = t; i < n; i += kThreads) c += order_of(w[i]) >= (least | bit);
    if (sum_all(c, part) >= k) least |= bit;
  }
  int above = 0;
  for (int i = t; i < n; i += kThreads) above += order_of(w[i]) > least;
  int ties = k - sum_all(above, part);  // so many of the rows at `least` stay, the first ones
  int at = before;
  for (int base = 0; base < n; base += kThreads) {
    const int i = base + t;
    const uint32_t o = i < n ? order_of(w[i]) : 0u;
    const uint64_t over = __ballot(i < n && o > least), same = __ballot(i < n && o == least);
    __syncthreads();
    if (lane == 0) {
      part[wave] = __popcll(over);
      ties_of[wave] = __popcll(same);
    }
    __syncthreads();
    int overs = 0, sames = 0, all_overs = 0, all_sames = 0;  // before this wave, and of all waves
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      overs += v < wave ? part[v] : 0;
      sames += v < wave ? ties_of[v] : 0;
      all_overs += part[v];
      all_sames += ties_of[v];
    }
    const uint64_t below = (1ull << lane) - 1;
    overs += __popcll(over & below);
    sames += __popcll(same & below);
    const bool stays = (over >> lane & 1) || ((same >> lane & 1) && sames < ties);
    const int to = at + overs + min(sames, ties);
    if (stays && to < prm.capacity_out) prm.rows[to] = first + i;
    at += all_overs + min(all_sames, ties);
    ties -= min(all_sames, ties);
  }
}

// A wave moves one row's bytes of every array, 2 a lane and step.
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams prm) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= min((int64_t)prm.cu_out[prm.BH], prm.capacity_out)) return;
  const int64_t from = prm.rows[row];
#pragma unroll
  for (int m = 0; m < kMoved; ++m)
    for (int i = lane * 2; i < prm.moved.bytes[m]; i += 128)
      *reinterpret_cast<uint16_t*>(prm.moved.to[m] + row * prm.moved.bytes[m] + i) =
          *reinterpret_cast<const uint16_t*>(prm.moved.from[m] + from * prm.moved.bytes[m] + i);
  if (lane == 0 && prm.idx) prm.idx_out[row] = prm.idx[from];
  if (lane == 0 && prm.weights_out) prm.weights_out[row] = prm.weights[from];
}

}  // namespace

int launch_evict(const maskkv_desc* d, const float* weights, const int32_t* cu_budget, int64_t capacity, const int32_t* budgets,
                 const MovedRows& moved, const int32_t* idx, int32_t* idx_out, int32_t* rows, float* weights_out, int32_t* cu_out,
                 int64_t capacity_out, hipStream_t stream) {
  EvictParams prm;
  prm.weights = weights;
  prm.cu = cu_budget;
  prm.budgets = budgets;
  prm.idx = idx;
  prm.capacity = capacity;
  prm.capacity_out = capacity_out;
  prm.BH = d->B * d->H;
  prm.rows = rows;
  prm.idx_out = idx_out;
  prm.cu_out = cu_out;
  prm.weights_out = weights_out;
  prm.moved = moved;
  hipLaunchKernelGGL(evict_rows_kernel, dim3(prm.BH), dim3(kThreads), 0, stream, prm);
  if (int e = check_launch("evict (rows)")) return e;
  const int64_t most = capacity_out < capacity ? capacity_out : capacity;  // (no more rows stay than there are)
  if (most == 0) return MASKKV_OK;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)((most + 3) / 4)), dim3(256), 0, stream, prm);
  return check_launch("evict (move)");
}

}  // namespace maskkv
