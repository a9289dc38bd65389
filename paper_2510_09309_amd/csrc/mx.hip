// The cache in 4 bits: eviction that stores the kept rows so, and the values that such rows stand for.
//
// Both are streams: 2 d eb bytes of K and V in and 2 (d/2 + d/32) out for a row that is stored, the reverse for one that is expanded.
// A lane takes 16 bytes of a row of K and the same of V, so that loads are whole rows and the lanes of a group of 32 elements are
// four (bf16) or eight (fp32) neighbours, which find the group's largest magnitude by exchanges inside a row of lanes, without the LDS.
//
// The scale is a power of two, so the only rounding is the one to 4 bits: dividing by it and multiplying with it again are exact.
//
// Bound by HBM where there are many rows, by the latency of arguments, positions and rows where there are few.  256 heads x 64 ... 1024 bf16
// rows of 128 (89 k in all): stored in 15.0 us (45 MB by rows of 256 bytes in, 12 MB out; from the memory-side cache 12.9, 12.4 without the conversion),
// expanded in 10.2 (5 TB/s).  32 heads x 250 rows: 4.4 and 3.0 on the device, as long as the host takes to launch them.
#include "mx.hpp"

namespace maskkv {

namespace {

constexpr int kThreads = 256;

struct CompactMxParams {
  View K, V;
  Lens lens;
  int H, BH;
  int d;
  const int32_t* idx;
  const int32_t* cu;
  int64_t capacity;
  MxCache out;
};

// The largest magnitude of a group, as the bits of an fp32, in all of its lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false));
}
template <typename T>
__device__ __forceinline__ uint32_t group_most(const u32x4& x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = x[i];
    if (sizeof(T) == 2)
      m = max(m, max(w << 16 & 0x7FFF0000u, w & 0x7FFF0000u));
    else
      m = max(m, w & 0x7FFFFFFFu);
  }
  m = max_with<0xB1>(m);                       // neighbours
  m = max_with<0x4E>(m);                       // pairs
  if (sizeof(T) == 4) m = max_with<0x141>(m);  // the other four of eight
  return m;
}

template <typename T>
__device__ __forceinline__ void store_group(const u32x4& x, char* codes, char* scales, int piece) {
  const uint32_t scale = mx_scale(group_most<T>(x));
  const uint32_t c = mx_encode<T>(x, scale);
  if (sizeof(T) == 2)
    reinterpret_cast<uint32_t*>(codes)[piece] = c;
  else
    reinterpret_cast<uint16_t*>(codes)[piece] = (uint16_t)c;
  constexpr int kLanes = kMxGroup * sizeof(T) / 16;
  if (piece % kLanes == 0) scales[piece / kLanes] = (char)scale;
}

// A wave stores kRounds times as many rows as it has room for in its lanes, side by side, and asks for all of them before it uses the first
// (the 89 k rows above from the memory-side cache: one round 14.5 us, two 12.9, three 13.0, four 13.4).
// Positions and the heads' ends are asked for at once, so that three waits in turn come before the first row is stored:
// arguments, these, and the rows.
constexpr int kRounds = 2;
constexpr int kEnds = 256;  // heads up to which a wave holds the ends of all of them in its lanes; more are searched, a latency for each halving

template <typename T, bool ONCE>
__global__ __launch_bounds__(kThreads) void compact_mx_kernel(const CompactMxParams prm) {
  typedef CompactMxParams A;
  fetch_arguments({MASKKV_VIEW_ARGUMENTS(A, K), MASKKV_VIEW_ARGUMENTS(A, V), MASKKV_ARGUMENT(A, lens), MASKKV_ARGUMENT(A, H),
                   MASKKV_ARGUMENT(A, out)});
  const int pieces = prm.d * (int)sizeof(T) / 16;  // of a row: 8, 16 or 32
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine = 64 / pieces, piece = lane % pieces;
  const int capacity = (int)prm.capacity;
  const int64_t first64 = ((int64_t)group_number() * (kThreads / 64) + wave) * (mine * kRounds);  // of this wave
  if (first64 >= capacity) return;
  const int first = (int)first64;
  int position[kRounds];
#pragma unroll
  for (int u = 0; u < kRounds; ++u) position[u] = prm.idx[min(first + u * mine + lane / pieces, capacity - 1)];
  int total, bh, end;  // the head of the first row, and where its rows end
  if (prm.BH <= kEnds) {
    int ends[kEnds / 64];
#pragma unroll
    for (int i = 0; i < kEnds / 64; ++i) ends[i] = prm.cu[min(i * 64 + lane + 1, prm.BH)];
    static_assert(kEnds == 256 && kRounds == 2, "what is waited for at once");
    asm volatile("" : "+v"(ends[0]), "+v"(ends[1]), "+v"(ends[2]), "+v"(ends[3]), "+v"(position[0]), "+v"(position[1]));
    total = min(__builtin_amdgcn_readlane(ends[kEnds / 64 - 1], 63), capacity);
    if (first >= total) return;
    bh = 0;
#pragma unroll
    for (int i = 0; i < kEnds / 64; ++i) bh += __popcll(__ballot(ends[i] <= first));  // (heads behind the last count as it does)
    end = 0;
#pragma unroll
    for (int i = 0; i < kEnds / 64; ++i)
      if (i == bh / 64) end = __builtin_amdgcn_readlane(ends[i], bh % 64);
  } else {
    total = min(prm.cu[prm.BH], capacity);
    if (first >= total) return;
    bh = head_of_row(prm.cu, prm.BH, first);
    end = prm.cu[bh + 1];
  }
  u32x4 k[kRounds], v[kRounds];
  auto load = [&](int u, int h, int b) {
    // a position outside the prompt is clamped rather than read out of bounds
    const int src = min(max(position[u], 0), max(prm.lens.P[b] - 1, 0));
    k[u] = read_piece<ONCE>(prm.K.row(b, h, src) + piece * 16);
    v[u] = read_piece<ONCE>(prm.V.row(b, h, src) + piece * 16);
  };
  if (min(first + kRounds * mine, total) <= end) {  // all rows are of one head
    const int b = bh / prm.H, h = bh % prm.H;
#pragma unroll
    for (int u = 0; u < kRounds; ++u) load(u, h, b);
  } else {
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
      const int row = min(first + u * mine + lane / pieces, total - 1);  // (lanes behind the last row do it again, and store nothing)
      int own = bh;
      while (own + 1 < prm.BH && prm.cu[own + 1] <= row) ++own;
      load(u, own % prm.H, own / prm.H);
    }
  }
#pragma unroll
  for (int u = 0; u < kRounds; ++u) {
    const int64_t row = first + u * mine + lane / pieces;
    if (row >= total) return;  // (all lanes of a row at once: the exchanges below stay inside a row)
    store_group<T>(k[u], prm.out.k_codes + row * (prm.d / 2), prm.out.k_scales + row * (prm.d / kMxGroup), piece);
    store_group<T>(v[u], prm.out.v_codes + row * (prm.d / 2), prm.out.v_scales + row * (prm.d / kMxGroup), piece);
  }
}

struct ExpandParams {
  MxCache in;
  const int32_t* total;  // cu[BH]
  int64_t capacity;
  int d;
  char *Kc, *Vc;
};

// Eight elements a thread, of K and of V.
template <typename T>
__global__ __launch_bounds__(kThreads) void expand_mx_kernel(const ExpandParams prm) {
  const int pieces = prm.d / 8;
  const int64_t i = (int64_t)group_number() * kThreads + threadIdx.x;
  if (i >= min((int64_t)prm.total[0], prm.capacity) * pieces) return;
  const uint32_t codes[2] = {reinterpret_cast<const uint32_t*>(prm.in.k_codes)[i], reinterpret_cast<const uint32_t*>(prm.in.v_codes)[i]};
  const uint32_t scales[2] = {reinterpret_cast<const uint8_t*>(prm.in.k_scales)[i / 4], reinterpret_cast<const uint8_t*>(prm.in.v_scales)[i / 4]};
  char* const to[2] = {prm.Kc, prm.Vc};
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const uint32_t c = codes[n];
    const float unit = mx_unit(scales[n]);
    if (sizeof(T) == 2) {
      reinterpret_cast<u32x4*>(to[n])[i] = mx_decode_bf16(c, unit);
    } else {
      float x[8];
      mx_decode_f32(c, unit, x);
      reinterpret_cast<float4*>(to[n])[2 * i] = make_float4(x[0], x[1], x[2], x[3]);
      reinterpret_cast<float4*>(to[n])[2 * i + 1] = make_float4(x[4], x[5], x[6], x[7]);
    }
  }
}

}  // namespace

int launch_compact_mx(const maskkv_desc* d, const Lens& lens, const View& K, const View& V, const int32_t* idx, const int32_t* cu_budget,
                      int64_t capacity, const MxCache& cache, hipStream_t stream) {
  if (capacity == 0) return MASKKV_OK;
  CompactMxParams prm;
  prm.K = K;
  prm.V = V;
  prm.lens = lens;
  prm.H = d->H;
  prm.BH = d->B * d->H;
  prm.d = d->d;
  prm.idx = idx;
  prm.cu = cu_budget;
  prm.capacity = capacity;
  prm.out = cache;
  const int rows = kRounds * kThreads / (d->d * (d->dtype == MASKKV_BF16 ? 2 : 4) / 16);  // of a workgroup
  const dim3 grid = grid_of((capacity + rows - 1) / rows);
  // (89 k rows of 2.1 GB of prompt: 15.0 us past the cache, 16.8 through it, and 12.9 through it where just these rows were there)
  const bool bf16 = d->dtype == MASKKV_BF16, once = 2ll * prm.BH * d->P_max * d->d * (bf16 ? 2 : 4) > kSideCache;
  const auto kernel = bf16 ? once ? compact_mx_kernel<bf16_t, true> : compact_mx_kernel<bf16_t, false>
                           : once ? compact_mx_kernel<float, true> : compact_mx_kernel<float, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, prm);
  return check_launch("compact_mx");
}

int launch_expand_mx(const maskkv_desc* d, const MxCache& cache, const int32_t* cu_budget, int64_t capacity, void* Kc, void* Vc,
                     hipStream_t stream) {
  if (capacity == 0) return MASKKV_OK;
  ExpandParams prm;
  prm.in = cache;
  prm.total = cu_budget + (int64_t)d->B * d->H;
  prm.capacity = capacity;
  prm.d = d->d;
  prm.Kc = reinterpret_cast<char*>(Kc);
  prm.Vc = reinterpret_cast<char*>(Vc);
  const dim3 grid = grid_of((capacity * (d->d / 8) + kThreads - 1) / kThreads);
  if (d->dtype == MASKKV_BF16)
    hipLaunchKernelGGL(expand_mx_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, prm);
  else
    hipLaunchKernelGGL(expand_mx_kernel<float>, grid, dim3(kThreads), 0, stream, prm);
  return check_launch("expand_mx");
}

}  // namespace maskkv
