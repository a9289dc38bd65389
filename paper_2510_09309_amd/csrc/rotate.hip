// Rotary positions: pairs of a row's elements turned by position * frequency.
//
// A workgroup takes 8 to 32 tokens and some of their heads.  The sines and cosines of its tokens are formed once, by all threads together, and
// kept in LDS; a thread then has one place of a token's rows - as many pairs as two pieces of 16 bytes hold - and turns them in one head after the other.
// The angle is reduced in 64 bits: in whole turns, position * (frequency / 2 pi), of which the fraction is exact; what is left is
// rounded to 32 bits, by 2^-26 turns at most.  2 pi, the frequency in turns and the product have 64 bits: off by less than 2^-51 of the turns together, which at one
// radian a position is 2^-26 turns up to position 2^28 and 2^-23 at 2^31.
//
// Bound by the memory: 32768 tokens of 32 + 32 heads (1.07 GB) 196 us, 5.5 TB/s, as fast as a copy; 8192 tokens of 32 + 8 heads, a token's heads together,
// 29; 256 tokens of 32 + 32 heads 5.1, one token 4.7, of which the launch is most.
#include <type_traits>

#include "kernels.hpp"

namespace maskkv {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 32;  // of a workgroup, at most
constexpr int kAtOnce = 4;   // heads whose rows a thread asks for before it turns the first

struct RotateParams {
  View q, k, q_out, k_out;
  double turns[64];   // of pair i for one position
  int32_t len[MASKKV_MAX_BATCH];
  const int32_t* positions;
  int n_tokens;
  int hq, heads;      // of the queries; of both
  int per;            // heads of a workgroup
  int width, half;
  int items_log2;     // places of a row: d / (2 * V)
  int tokens_log2;    // tokens of a workgroup
  float amplitude;
};

// V elements of a row as floats.
template <typename T, int V>
struct Piece {
  static constexpr int kBytes = V * (int)sizeof(T);
  typedef uint32_t Words __attribute__((ext_vector_type(kBytes < 4 ? 1 : kBytes / 4)));
  Words w;
  template <bool PAST>
  __device__ __forceinline__ void load(const char* from) {
    if constexpr (kBytes == 2)
      w[0] = *reinterpret_cast<const uint16_t*>(from);
    else if constexpr (PAST)
      w = __builtin_nontemporal_load(reinterpret_cast<const Words*>(from));
    else
      w = *reinterpret_cast<const Words*>(from);
  }
  template <bool PAST>
  __device__ __forceinline__ void store(char* to) const {
    if constexpr (kBytes == 2)
      *reinterpret_cast<uint16_t*>(to) = (uint16_t)w[0];
    else if constexpr (PAST)
      __builtin_nontemporal_store(w, reinterpret_cast<Words*>(to));
    else
      *reinterpret_cast<Words*>(to) = w;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return as_f32(w[i]);
    const uint32_t u = w[i / 2];
    return as_f32(i % 2 ? u & 0xFFFF0000u : u << 16);
  }
  __device__ __forceinline__ void set(const float (&x)[V]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = as_u32(x[i]);
    } else if constexpr (V == 1) {
      w[0] = pack_bf16x2(x[0], 0.f);
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2) w[i / 2] = pack_bf16x2(x[i], x[i + 1]);
    }
  }
};

// PAST: rows are written (1), or read and written (2), past the memory-side cache.
template <typename T, int V, bool PAIRS, int PAST>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateParams prm) {
  __shared__ float2 turned[kTokens * 64];  // [token][pair]
  typedef RotateParams A;
  fetch_arguments({MASKKV_VIEW_ARGUMENTS(A, q), MASKKV_VIEW_ARGUMENTS(A, k), MASKKV_VIEW_ARGUMENTS(A, q_out), MASKKV_VIEW_ARGUMENTS(A, k_out),
                   MASKKV_ARGUMENT(A, turns), MASKKV_ARGUMENT(A, len), MASKKV_ARGUMENT(A, positions), MASKKV_ARGUMENT(A, amplitude)});
  const int b = blockIdx.z, tokens = 1 << prm.tokens_log2, t0 = blockIdx.x << prm.tokens_log2;
  const int len = prm.len[b];
  if (t0 >= len) return;
  const int item = threadIdx.x & ((1 << prm.items_log2) - 1), slot = threadIdx.x >> prm.items_log2;
  const int tt = slot & (tokens - 1), step = kThreads >> prm.items_log2 >> prm.tokens_log2;
  const int t = min(t0 + tt, len - 1), end = min((int)(blockIdx.y + 1) * prm.per, prm.heads);
  const bool mine = t0 + tt < len, turns = item < prm.half / V;
  // the two pieces, as bytes of a row
  const int rest = prm.width + (item - prm.half / V) * 2 * V;
  const int first = (turns ? item * (PAIRS ? 2 * V : V) : rest) * (int)sizeof(T);
  const int second = (turns ? (PAIRS ? (2 * item + 1) * V : prm.half + item * V) : rest + V) * (int)sizeof(T);

  Piece<T, V> x[kAtOnce], y[kAtOnce];
  auto fetch = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int h = h0 + u * step;
      if (h >= end || !mine) continue;
      const char* row = h < prm.hq ? prm.q.row(b, h, t) : prm.k.row(b, h - prm.hq, t);
      x[u].template load<PAST == 2>(row + first);
      y[u].template load<PAST == 2>(row + second);
    }
  };
  int h0 = blockIdx.y * prm.per + (slot >> prm.tokens_log2);
  fetch(h0);  // (under way beside the angles)
  for (int i = threadIdx.x; i < prm.half << prm.tokens_log2; i += kThreads) {
    const int token = i / prm.half, pair = i - token * prm.half;
    const double a = (double)prm.positions[(int64_t)b * prm.n_tokens + min(t0 + token, len - 1)] * prm.turns[pair];
    const float left = (float)(a - rint(a));
    float s, c;
    sincospif(2.f * left, &s, &c);
    turned[token * 64 + pair] = make_float2(c * prm.amplitude, s * prm.amplitude);
  }
  __syncthreads();
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float2 v = turned[tt * 64 + (turns ? item * V + i : 0)];
    c[i] = v.x;
    s[i] = v.y;
  }
  for (; h0 < end; h0 += kAtOnce * step) {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int h = h0 + u * step;
      if (h >= end || !mine) continue;
      char* row = h < prm.hq ? prm.q_out.row(b, h, t) : prm.k_out.row(b, h - prm.hq, t);
      if (turns) {
        float p[V], q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float a, e;
          if constexpr (PAIRS) {  // elements 2i and 2i + 1 of both pieces in a row
            a = 2 * i < V ? x[u].get(2 * i % V) : y[u].get(2 * i % V);
            e = 2 * i + 1 < V ? x[u].get((2 * i + 1) % V) : y[u].get((2 * i + 1) % V);
          } else {
            a = x[u].get(i);
            e = y[u].get(i);
          }
          const float to_a = fmaf(a, c[i], -(e * s[i])), to_e = fmaf(e, c[i], a * s[i]);
          if constexpr (PAIRS) {
            (2 * i < V ? p[2 * i % V] : q[2 * i % V]) = to_a;
            (2 * i + 1 < V ? p[(2 * i + 1) % V] : q[(2 * i + 1) % V]) = to_e;
          } else {
            p[i] = to_a;
            q[i] = to_e;
          }
        }
        x[u].set(p);
        y[u].set(q);
      }
      x[u].template store<PAST != 0>(row + first);
      y[u].template store<PAST != 0>(row + second);
    }
    fetch(h0 + kAtOnce * step);
  }
}

template <typename T, int V, int PAST>
void launch_pieces(const RotateParams& prm, bool pairs, dim3 grid, hipStream_t stream) {
  if (pairs)
    hipLaunchKernelGGL((rotate_kernel<T, V, true, PAST>), grid, dim3(kThreads), 0, stream, prm);
  else
    hipLaunchKernelGGL((rotate_kernel<T, V, false, PAST>), grid, dim3(kThreads), 0, stream, prm);
}

// What is read and written, in bytes, from which on it goes past the memory-side cache, which holds 256 MB (out of it, a step finds what the one before has
// left): stores from 128 MB on, 8192 tokens of 32 + 8 heads (168 MB) 38.9 us with stores that stay and 29.1 past it, 2 x 3000
// tokens of 12 + 12 heads in fp32 (74 MB) 14.9 and 21.0; loads too from 512 MB on, a 32k prompt 202 with stores alone, 196.
constexpr int64_t kStoresPast = (int64_t)128 << 20, kAllPast = (int64_t)512 << 20;

}  // namespace

int launch_rotate(const maskkv_desc* d, const maskkv_rotary* rotary, const int32_t* positions, int n_tokens, const int32_t* lens,
                  const View* Q, const View* Q_out, const View* K, const View* K_out, hipStream_t stream) {
  RotateParams prm{};
  if (Q) prm.q = *Q, prm.q_out = *Q_out;
  if (K) prm.k = *K, prm.k_out = *K_out;
  prm.width = rotary->width;
  prm.half = rotary->width / 2;
  for (int i = 0; i < prm.half; ++i) prm.turns[i] = rotary->freq[i] / 6.283185307179586476925;
  int longest = 0;
  for (int b = 0; b < d->B; ++b) {
    prm.len[b] = lens ? lens[b] : n_tokens;
    longest = prm.len[b] > longest ? prm.len[b] : longest;
  }
  if (longest == 0) return MASKKV_OK;
  prm.positions = positions;
  prm.n_tokens = n_tokens;
  prm.hq = Q ? d->H * query_heads_per_kv(d) : 0;
  prm.heads = prm.hq + (K ? d->H : 0);
  prm.amplitude = (float)rotary->amplitude;
  // pieces of 16 bytes, or as much less as halves that are no multiple of them ask for
  const bool bf16 = d->dtype == MASKKV_BF16;
  int V = bf16 ? 8 : 4;
  while (prm.half % V) V /= 2;
  while (1 << prm.items_log2 < d->d / (2 * V)) ++prm.items_log2;
  // as many tokens as still leave a workgroup or two for each compute unit: a head's rows of 32 tokens lie in one stretch of memory, of 8 in four
  // (32k prompt, 64 heads: 8 tokens 246 us, 16 232, 32 202; 256 tokens of 64 heads 5.1, 8.1, 12.7)
  const int slots = kThreads >> prm.items_log2;
  int most_tokens = 8;
  while (most_tokens < kTokens && (int64_t)d->B * longest / (2 * most_tokens) >= 448) most_tokens *= 2;
  while (1 << prm.tokens_log2 < most_tokens && 1 << prm.tokens_log2 < longest && 1 << prm.tokens_log2 < slots) ++prm.tokens_log2;
  const int tokens = 1 << prm.tokens_log2, step = slots >> prm.tokens_log2;
  const int tiles = (longest + tokens - 1) / tokens;
  // heads to several workgroups as long as these do not fill the chip
  const int64_t groups = (int64_t)tiles * d->B, most = (prm.heads + step - 1) / step;
  int64_t parts = (1024 + groups - 1) / groups;
  parts = parts < most ? parts : most;
  prm.per = (int)((most + parts - 1) / parts) * step;
  const dim3 grid((unsigned)tiles, (unsigned)((prm.heads + prm.per - 1) / prm.per), (unsigned)d->B);
  const int64_t bytes = 2 * (int64_t)d->B * longest * prm.heads * d->d * (bf16 ? 2 : 4);
  const bool pairs = rotary->layout == MASKKV_ROTARY_PAIRS;
  auto whole = [&](auto past) {  // (halves of whole pieces)
    constexpr int kPast = decltype(past)::value;
    if (bf16)
      launch_pieces<bf16_t, 8, kPast>(prm, pairs, grid, stream);
    else
      launch_pieces<float, 4, kPast>(prm, pairs, grid, stream);
  };
  if (V == (bf16 ? 8 : 4)) {
    if (bytes >= kAllPast)
      whole(std::integral_constant<int, 2>());
    else if (bytes >= kStoresPast)
      whole(std::integral_constant<int, 1>());
    else
      whole(std::integral_constant<int, 0>());
  } else if (bf16) {
    if (V == 4) launch_pieces<bf16_t, 4, 0>(prm, pairs, grid, stream);
    if (V == 2) launch_pieces<bf16_t, 2, 0>(prm, pairs, grid, stream);
    if (V == 1) launch_pieces<bf16_t, 1, 0>(prm, pairs, grid, stream);
  } else {
    if (V == 2) launch_pieces<float, 2, 0>(prm, pairs, grid, stream);
    if (V == 1) launch_pieces<float, 1, 0>(prm, pairs, grid, stream);
  }
  return check_launch("rotate");
}

}  // namespace maskkv
