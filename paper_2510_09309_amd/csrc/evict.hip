// Further eviction from a packed cache: of each head the rows of largest weight stay.
//
// One launch.  A workgroup moves up to `per` rows of the smaller cache that belong to one head.  It finds that head from the
// budgets, and which of the head's rows they are by itself, from all of the head's weights: several workgroups of a head do
// the same search, which costs the latency of one, where a list made by one of them would cost a launch between the two.
//
// The search is for the smallest weight that stays, and ends when a candidate has as many rows as stay.  Up to 512 rows every wave
// holds all of them and goes through the bits of the weights' order by itself, by ballots: no barrier and no LDS.  Beyond that it goes
// by histograms of eight bits in LDS.  The rows of a thread stay in registers, up to 32 of them; a longer head's are read again every round.
#include "mx.hpp"

namespace maskkv {

namespace {

struct EvictParams {
  const float* weights;
  const int32_t *cu, *budgets, *idx;
  int64_t capacity, capacity_out;
  int BH;
  int per;        // rows of a workgroup at most
  int row_shift;  // 16-byte pieces of a row, both large arrays together: 1 << row_shift
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

struct HeadRows {
  int first, n, stay;
};
__device__ __forceinline__ HeadRows rows_of(const EvictParams& prm, int bh, int capacity) {
  const int budget = prm.budgets[bh], a = min(prm.cu[bh], capacity), z = min(prm.cu[bh + 1], capacity);
  HeadRows x;
  x.first = a;
  x.n = max(z - a, 0);
  x.stay = min(max(budget, 0), x.n);
  return x;
}

// How many rows stay of the heads before each, by one wave.
__device__ __forceinline__ void write_prefix(const EvictParams& prm) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < prm.BH; base += 64) {
    const int bh = base + lane;
    const int stay = bh < prm.BH ? rows_of(prm, bh, (int)prm.capacity).stay : 0;
    const int upto = wave_prefix(stay);
    if (bh < prm.BH) prm.cu_out[bh] = before + upto - stay;
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  if (lane == 0) prm.cu_out[prm.BH] = before;
}

// The numbers of the rows that stay with ranks lo .. hi-1 among the head's, into `list`; every wave by itself, up to 64 * VALUES rows.
// (All waves come to the same ranks; each writes those of its share of the rows.)
template <int THREADS, int VALUES>
__device__ __forceinline__ void list_rows_alone(const float* w, int n, int k, int lo, int hi, int32_t* list) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t held[VALUES];
#pragma unroll
  for (int v = 0; v < VALUES; ++v) {
    const float x = w[min(v * 64 + lane, n - 1)];
    held[v] = v * 64 + lane < n ? order_of(x) : 0u;
  }
  uint32_t least = 0;   // a row at or above it stays, or may
  bool exact = k == n;  // just those stay
  for (uint32_t bit = 0x80000000u; bit && !exact; bit >>= 1) {
    int c = 0;
#pragma unroll
    for (int v = 0; v < VALUES; ++v) c += __popcll(__ballot(held[v] >= (least | bit)));
    if (c >= k) least |= bit;
    exact = c == k;
  }
  int ties = k;  // so many of the rows at `least` stay, the first ones
  if (!exact) {
#pragma unroll
    for (int v = 0; v < VALUES; ++v) ties -= __popcll(__ballot(held[v] > least));
  }
  int overs = 0, sames = 0;
#pragma unroll
  for (int v = 0; v < VALUES; ++v) {
    const bool live = v * 64 + lane < n;
    const uint64_t a = __ballot(live && (exact ? held[v] >= least : held[v] > least)), b = __ballot(live && !exact && held[v] == least);
    if (v % (THREADS / 64) == wave) {
      const uint64_t below = (1ull << lane) - 1;
      const int before = sames + __popcll(b & below), rank = overs + __popcll(a & below) + min(before, ties);
      const bool stays = (a >> lane & 1) || ((b >> lane & 1) && before < ties);
      if (stays && rank >= lo && rank < hi) list[rank - lo] = v * 64 + lane;
    }
    overs += __popcll(a);
    sames += __popcll(b);
  }
}

// The same by the whole workgroup.  VALUES: rows of a thread, in registers, or 0.
template <int THREADS, int VALUES>
__device__ __forceinline__ void list_rows(const float* w, int n, int k, int lo, int hi, int32_t* list, int* bins, int (*counts)[4]) {
  constexpr int kWaves = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int each = VALUES ? VALUES : (n + THREADS - 1) / THREADS;
  const int row0 = wave * each * 64 + lane;  // a wave's rows lie side by side, 64 a step
  uint32_t held[VALUES ? VALUES : 1];
  auto read = [&](int v) {
    const int row = row0 + v * 64;
    const float x = w[min(row, n - 1)];
    return row < n ? order_of(x) : 0u;
  };
  if constexpr (VALUES > 0) {
#pragma unroll
    for (int v = 0; v < VALUES; ++v) held[v] = read(v);
  }
  auto over_rows = [&](auto f) {
    if constexpr (VALUES > 0) {
#pragma unroll
      for (int v = 0; v < VALUES; ++v) f(held[v], v);
    } else {
#pragma unroll 8
      for (int v = 0; v < each; ++v) f(read(v), v);
    }
  };

  // Eight bits of `least` a round: how many of the rows that agree with it so far have which next eight bits; then the highest
  // of these with at least as many rows at or above it as are still to be found.
  uint32_t least = 0;   // a row at or above it stays, or may
  bool exact = k == n;  // just those stay
  int wanted = k;       // of the rows that agree with `least` in the bits so far
  for (int shift = 24; shift >= 0 && !exact; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += THREADS) bins[i] = 0;
    __syncthreads();
    over_rows([&](uint32_t o, int v) {
      if (row0 + v * 64 < n && (shift == 24 || (o ^ least) >> (shift + 8) == 0)) atomicAdd(&bins[o >> shift & 255], 1);
    });
    __syncthreads();
    // every wave by itself: a lane holds four bins from the top, 255 - 4 lane ..
    const int4 four = *reinterpret_cast<const int4*>(bins + 252 - 4 * lane);
    const int own = four.x + four.y + four.z + four.w;
    const int upto = wave_prefix(own);
    const int at = __builtin_ctzll(__ballot(upto >= wanted));  // (there is one: all the rows that agree are `wanted` or more)
    int above = __builtin_amdgcn_readlane(upto - own, at);     // rows above the bin in question
    const int in[4] = {__builtin_amdgcn_readlane(four.w, at), __builtin_amdgcn_readlane(four.z, at), __builtin_amdgcn_readlane(four.y, at),
                       __builtin_amdgcn_readlane(four.x, at)};
    int j = 0;
    while (j < 3 && above + in[j] < wanted) above += in[j++];
    least |= (uint32_t)(255 - 4 * at - j) << shift;
    exact = above + in[j] == wanted;
    wanted -= above;
    __syncthreads();
  }
  const auto over = [&](uint32_t o, int v) { return __ballot(row0 + v * 64 < n && (exact ? o >= least : o > least)); };
  const auto same = [&](uint32_t o, int v) { return __ballot(row0 + v * 64 < n && !exact && o == least); };
  int overs = 0, sames = 0;
  over_rows([&](uint32_t o, int v) {
    overs += __popcll(over(o, v));
    sames += __popcll(same(o, v));
  });
  if constexpr (VALUES > 0) {  // (the ballots are formed again below: kept from here to there they would take all registers)
#pragma unroll
    for (int v = 0; v < VALUES; ++v) asm volatile("" : "+v"(held[v]));
  }
  if (lane == 0) {
    counts[wave][0] = overs;
    counts[wave][1] = sames;
  }
  __syncthreads();
  int ties = k;  // so many of the rows at `least` stay, the first ones
  overs = sames = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const int a = counts[i][0], b = counts[i][1];
    ties -= a;
    overs += i < wave ? a : 0;
    sames += i < wave ? b : 0;
  }
  ties = __builtin_amdgcn_readfirstlane(ties);
  overs = __builtin_amdgcn_readfirstlane(overs);
  sames = __builtin_amdgcn_readfirstlane(sames);
  const uint64_t below = (1ull << lane) - 1;
  over_rows([&](uint32_t o, int v) {
    const uint64_t a = over(o, v), b = same(o, v);
    const int before = sames + __popcll(b & below);
    const int rank = overs + __popcll(a & below) + min(before, ties);
    const bool stays = (a >> lane & 1) || ((b >> lane & 1) && before < ties);
    if (stays && rank >= lo && rank < hi) list[rank - lo] = row0 + v * 64;
    overs += __popcll(a);
    sames += __popcll(b);
  });
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_kernel(const EvictParams prm) {
  extern __shared__ int32_t list[];  // [per]
  __shared__ __attribute__((aligned(16))) int bins[256];
  __shared__ int counts[THREADS / 64][4];
  typedef EvictParams A;
  fetch_arguments({MASKKV_ARGUMENT(A, weights), MASKKV_ARGUMENT(A, rows), MASKKV_ARGUMENT(A, moved), (uint32_t)(offsetof(A, moved) + 64)});
  const int lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && threadIdx.x < 64) write_prefix(prm);

  // ---- the head of this workgroup's rows, how many rows stay of the heads before it, and which of its own these are
  constexpr int kSets = 4;
  const int unit = blockIdx.x, capacity = (int)prm.capacity;
  int before = 0, units_before = 0, bh = -1, part = 0;
  HeadRows x = {0, 0, 0};
  for (int base = 0; base < prm.BH && bh < 0; base += 64 * kSets) {
    HeadRows some[kSets];
#pragma unroll
    for (int i = 0; i < kSets; ++i) some[i] = rows_of(prm, min(base + i * 64 + lane, prm.BH - 1), capacity);
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      if (base + i * 64 >= prm.BH || bh >= 0) break;
      const int stay = base + i * 64 + lane < prm.BH ? some[i].stay : 0;
      const int units = (int)(((uint32_t)stay + prm.per - 1) / prm.per);
      const int rows_upto = wave_prefix(stay), upto = wave_prefix(units);
      const uint64_t found = __ballot(units_before + upto > unit);
      if (found) {
        const int at = __builtin_ctzll(found);
        bh = base + i * 64 + at;
        x = {__builtin_amdgcn_readlane(some[i].first, at), __builtin_amdgcn_readlane(some[i].n, at), __builtin_amdgcn_readlane(stay, at)};
        part = unit - units_before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(units, at));
        before += __builtin_amdgcn_readlane(rows_upto, at) - x.stay;
      } else {
        units_before += __builtin_amdgcn_readlane(upto, 63);
        before += __builtin_amdgcn_readlane(rows_upto, 63);
      }
    }
  }
  if (bh < 0) return;
  const int lo = part * prm.per;
  const int64_t to = (int64_t)before + lo;
  const int rows = (int)min((int64_t)min(x.stay - lo, prm.per), prm.capacity_out - to);
  if (rows <= 0) return;

  const float* w = prm.weights + x.first;
  if (x.n <= 64)
    list_rows_alone<THREADS, 1>(w, x.n, x.stay, lo, lo + rows, list);
  else if (x.n <= 256)
    list_rows_alone<THREADS, 4>(w, x.n, x.stay, lo, lo + rows, list);
  else if (x.n <= 512)
    list_rows_alone<THREADS, 8>(w, x.n, x.stay, lo, lo + rows, list);
  else if (x.n <= THREADS * 4)
    list_rows<THREADS, 4>(w, x.n, x.stay, lo, lo + rows, list, bins, counts);
  else if (x.n <= THREADS * 16)
    list_rows<THREADS, 16>(w, x.n, x.stay, lo, lo + rows, list, bins, counts);
  else if (x.n <= THREADS * 32)
    list_rows<THREADS, 32>(w, x.n, x.stay, lo, lo + rows, list, bins, counts);
  else
    list_rows<THREADS, 0>(w, x.n, x.stay, lo, lo + rows, list, bins, counts);
  __syncthreads();

  // ---- the rows, 16 bytes a thread and step
  const int pieces = 1 << prm.row_shift, half = pieces / 2;
  constexpr int kAtOnce = 4;
  for (int i0 = threadIdx.x; i0 < rows << prm.row_shift; i0 += kAtOnce * THREADS) {
    u32x4 x4[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = min(i0 + u * THREADS, (rows << prm.row_shift) - 1), piece = i & (pieces - 1), m = piece >= half;
      const int64_t from = x.first + list[i >> prm.row_shift];
      x4[u] = *reinterpret_cast<const u32x4*>(prm.moved.from[m] + (from * half + (piece - m * half)) * 16);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = i0 + u * THREADS, piece = i & (pieces - 1), m = piece >= half;
      if (i < rows << prm.row_shift)
        *reinterpret_cast<u32x4*>(prm.moved.to[m] + ((to + (i >> prm.row_shift)) * half + (piece - m * half)) * 16) = x4[u];
    }
  }
  for (int i = threadIdx.x; i < rows; i += THREADS) {
    const int64_t from = x.first + list[i];
    prm.rows[to + i] = (int32_t)from;
    if (prm.idx) prm.idx_out[to + i] = prm.idx[from];
    if (prm.weights_out) prm.weights_out[to + i] = prm.weights[from];
    if (prm.moved.bytes[2] == 4) {
      reinterpret_cast<uint32_t*>(prm.moved.to[2])[to + i] = reinterpret_cast<const uint32_t*>(prm.moved.from[2])[from];
      reinterpret_cast<uint32_t*>(prm.moved.to[3])[to + i] = reinterpret_cast<const uint32_t*>(prm.moved.from[3])[from];
    } else if (prm.moved.bytes[2] == 2) {
      reinterpret_cast<uint16_t*>(prm.moved.to[2])[to + i] = reinterpret_cast<const uint16_t*>(prm.moved.from[2])[from];
      reinterpret_cast<uint16_t*>(prm.moved.to[3])[to + i] = reinterpret_cast<const uint16_t*>(prm.moved.from[3])[from];
    }
  }
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
  prm.row_shift = 0;
  while (16 << prm.row_shift < 2 * moved.bytes[0]) ++prm.row_shift;
  // Workgroups for two of every compute unit, of 16 rows at least and of no more than the list has room for.
  const int64_t most = capacity_out < capacity ? capacity_out : capacity;  // (no more rows stay than there are)
  int64_t per = (most + 511) / 512;
  per = per < 16 ? 16 : per > 8192 ? 8192 : per;
  prm.per = (int)per;
  const int64_t groups = most / per + prm.BH;  // (each head's last one may have fewer)
  if (capacity / prm.BH <= 2048)
    hipLaunchKernelGGL(evict_kernel<256>, dim3((unsigned)groups), dim3(256), per * 4, stream, prm);
  else
    hipLaunchKernelGGL(evict_kernel<1024>, dim3((unsigned)groups), dim3(1024), per * 4, stream, prm);
  return check_launch("evict");
}

}  // namespace maskkv
