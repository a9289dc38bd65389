// Further eviction from a packed cache: of each head the rows of largest weight stay.
//
// One launch.  A workgroup moves up to `per` rows of the smaller cache that belong to one head.  It finds that head from the
// budgets, and which of the head's rows they are by itself, from all of the head's weights: several workgroups of a head do
// the same search, which costs the latency of one, where a list made by one of them would cost a launch between the two.
//
// The search is for the smallest weight that stays, two bits of the weights' order a round: every wave counts its rows at or above
// three candidates by ballots and the waves' counts meet in LDS, one barrier a round; it ends when a candidate has as many rows as
// stay.  The rows of a thread stay in registers, up to 32 of them; a longer head's are read again every round.
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
__device__ __forceinline__ HeadRows rows_of(const EvictParams& prm, int bh) {
  const int capacity = (int)prm.capacity;
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
    const int stay = bh < prm.BH ? rows_of(prm, bh).stay : 0;
    const int upto = wave_prefix(stay);
    if (bh < prm.BH) prm.cu_out[bh] = before + upto - stay;
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  if (lane == 0) prm.cu_out[prm.BH] = before;
}

// The numbers of the rows that stay with ranks lo .. hi-1 among the head's, into `list`.  VALUES: rows of a thread, in registers, or 0.
template <int THREADS, int VALUES>
__device__ __forceinline__ void list_rows(const float* w, int n, int k, int lo, int hi, int32_t* list, int (*counts)[THREADS / 64][4]) {
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

  uint32_t least = 0;     // a row at or above it stays, or may
  bool exact = k == n;    // just those stay
  for (int shift = 30, round = 0; shift >= 0 && !exact; shift -= 2, ++round) {
    int c[3] = {0, 0, 0};
    over_rows([&](uint32_t o, int) {
#pragma unroll
      for (int j = 0; j < 3; ++j) c[j] += __popcll(__ballot(o >= (least | (uint32_t)(j + 1) << shift)));
    });
    int* mine = counts[round & 1][wave];
    if (lane == 0) {
      mine[0] = c[0];
      mine[1] = c[1];
      mine[2] = c[2];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      int s;
      if (kWaves == 4) {
        s = counts[round & 1][0][j] + counts[round & 1][1][j] + counts[round & 1][2][j] + counts[round & 1][3][j];
      } else {
        s = counts[round & 1][lane % kWaves][j];  // (16 waves: the sum over a row of 16 lanes)
        s = plus_dpp<0x121, 0xf>(s);
        s = plus_dpp<0x122, 0xf>(s);
        s = plus_dpp<0x124, 0xf>(s);
        s = plus_dpp<0x128, 0xf>(s);
      }
      c[j] = __builtin_amdgcn_readfirstlane(s);
    }
    uint32_t digit = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (c[j] >= k) {
        digit = j + 1;
        exact = c[j] == k;
      }
    least |= digit << shift;
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
  __syncthreads();
  if (lane == 0) {
    counts[0][wave][0] = overs;
    counts[0][wave][1] = sames;
  }
  __syncthreads();
  int ties = k;  // so many of the rows at `least` stay, the first ones
  overs = sames = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const int a = counts[0][i][0], b = counts[0][i][1];
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
  __shared__ int counts[2][THREADS / 64][4];
  const int lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && threadIdx.x < 64) write_prefix(prm);

  // ---- the head of this workgroup's rows, how many rows stay of the heads before it, and which of its own these are
  const int unit = blockIdx.x;
  int before = 0, units_before = 0, bh = -1, part = 0;
  for (int base = 0; base < prm.BH && bh < 0; base += 64) {
    const int stay = base + lane < prm.BH ? rows_of(prm, base + lane).stay : 0;
    const int units = (int)(((uint32_t)stay + prm.per - 1) / prm.per);
    const int rows_upto = wave_prefix(stay), upto = wave_prefix(units);
    const uint64_t found = __ballot(units_before + upto > unit);
    if (found) {
      const int at = __builtin_ctzll(found);
      bh = base + at;
      part = unit - units_before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(units, at));
      before += __builtin_amdgcn_readlane(rows_upto, at) - __builtin_amdgcn_readlane(stay, at);
    } else {
      units_before += __builtin_amdgcn_readlane(upto, 63);
      before += __builtin_amdgcn_readlane(rows_upto, 63);
    }
  }
  if (bh < 0) return;
  const HeadRows x = rows_of(prm, bh);
  const int lo = part * prm.per;
  const int64_t to = (int64_t)before + lo;
  const int rows = (int)min((int64_t)min(x.stay - lo, prm.per), prm.capacity_out - to);
  if (rows <= 0) return;

  const float* w = prm.weights + x.first;
  if (x.n <= THREADS)
    list_rows<THREADS, 1>(w, x.n, x.stay, lo, lo + rows, list, counts);
  else if (x.n <= THREADS * 4)
    list_rows<THREADS, 4>(w, x.n, x.stay, lo, lo + rows, list, counts);
  else if (x.n <= THREADS * 16)
    list_rows<THREADS, 16>(w, x.n, x.stay, lo, lo + rows, list, counts);
  else if (x.n <= THREADS * 32)
    list_rows<THREADS, 32>(w, x.n, x.stay, lo, lo + rows, list, counts);
  else
    list_rows<THREADS, 0>(w, x.n, x.stay, lo, lo + rows, list, counts);
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
