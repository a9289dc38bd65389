// Further eviction from a packed cache: of each head the rows of largest weight stay.
//
// Short heads take one launch.  A workgroup moves up to `per` rows of the smaller cache that belong to one head; it finds that head from
// the budgets, and which of the head's rows they are by itself, from all of the head's weights: several workgroups of a head do
// the same search, which costs the latency of one, where a list made by one of them would cost a launch between the two.  Long
// heads take that launch: a workgroup of 1024 per head lists the rows that stay, and a second kernel moves them.
//
// The search is for the smallest weight that stays, and ends when a candidate has as many rows as stay.  Up to 512 rows every wave
// holds all of them and goes through the bits of the weights' order by itself, by ballots: no barrier and no LDS.  Beyond that the workgroup
// goes by histograms of eight bits in LDS.  The rows of a thread stay in registers, up to 32 of them; a longer head's are read again
// every round.
//
// Nothing is computed but comparisons and counts: latency, and where there are many rows the copying.  32 heads x 250 bf16 rows, half of them moved: 6.5 us
// a call; 256 heads x 64 ... 1024 rows in 4 bits (89 k, half of them moved: 6 MB in, 7 out) 11.0 us, 60 % of its waves' time spent waiting.
#include "mx.hpp"

namespace maskkv {

namespace {

// Rows of a head up to which the rows that stay are not listed by a launch of their own: on average, or all of the longest one's.  One and two
// launches: 32 heads x 250 rows 8.3 and 11.7 us, x 900 10.8 and 13.9, x 1800 14.6 and 16.4, x 4000 21.5 and 21.1; 4 x 1800 9.4 and 11.8, x 4000 12.8 and 12.9; 256 heads x
// 600 19.2 and 22.7, x 1200 36.1 and 36.9; heads of 1000 ... 8000 rows, 32 of them, 34.0 and 21.3, 4 x 8000 30.0 and 15.4: beyond 4096 a workgroup of 256 reads its
// head again and again.  (With the expansion of what is left, 0.5 ... 5 us.)
constexpr int kShortHead = 1024, kLongestHead = 4096;
constexpr int kMostRows = 4096;   // of a workgroup's list

struct EvictParams {
  const float* weights;
  const int32_t *cu, *budgets, *idx;
  int64_t capacity, capacity_out;
  int BH;
  int per;        // rows of a workgroup at most
  int once;       // the old cache goes past the memory-side cache
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

// Of rows row, row + 64 ... of a head's n.  (All are asked for before the first is used: as the compiler has it, under a condition each, one after the other.)
template <int VALUES>
__device__ __forceinline__ void read_orders(const float* w, int row, int n, uint32_t (&held)[VALUES]) {
  float x[VALUES];
#pragma unroll
  for (int v = 0; v < VALUES; ++v) x[v] = w[min(row + v * 64, n - 1)];
#pragma unroll
  for (int v = 0; v < VALUES; ++v) asm volatile("" : "+v"(x[v]));
#pragma unroll
  for (int v = 0; v < VALUES; ++v) held[v] = row + v * 64 < n ? order_of(x[v]) : 0u;
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

// The numbers (from `base` on) of the rows that stay with ranks lo .. hi-1 among the head's, into `list`; every wave by itself, up to 64 * VALUES rows.
// (All waves come to the same ranks; each writes those of its share of the rows.)
template <int THREADS, int VALUES>
__device__ __forceinline__ void list_rows_alone(const float* w, int n, int k, int lo, int hi, int base, int32_t* list) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t held[VALUES];
  read_orders<VALUES>(w, lane, n, held);
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
      if (stays && rank >= lo && rank < hi) list[rank - lo] = v * 64 + lane + base;
    }
    overs += __popcll(a);
    sames += __popcll(b);
  }
}

// Of each count of a histogram: as many as keep a workgroup's additions apart.
template <int THREADS>
struct Bins {
  static constexpr int kCopies = THREADS == 256 ? 2 : 8;
  static constexpr int kCopy = 256 + 8;  // from one copy to the next: those of a count lie in banks of their own
  static constexpr int kRound = kCopy * kCopies;
};

// The same by the whole workgroup.  VALUES: rows of a thread, in registers, or 0.
template <int THREADS, int VALUES>
__device__ __forceinline__ void list_rows(const float* w, int n, int k, int lo, int hi, int base, int32_t* list, int* all_bins, int (*counts)[4]) {
  constexpr int kWaves = THREADS / 64, kCopies = Bins<THREADS>::kCopies, kBins = Bins<THREADS>::kRound;
  constexpr bool kOneScans = kWaves == 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int each = VALUES ? VALUES : (n + THREADS - 1) / THREADS;
  const int row0 = wave * each * 64 + lane;  // a wave's rows lie side by side, 64 a step
  uint32_t held[VALUES ? VALUES : 1];
  if constexpr (VALUES > 0) read_orders<VALUES>(w, row0, n, held);
  auto over_rows = [&](auto f) {
    if constexpr (VALUES > 0) {
#pragma unroll
      for (int v = 0; v < VALUES; ++v) f(held[v], v);
    } else {
      for (int v0 = 0; v0 < each; v0 += 8) {
        uint32_t some[8];
        read_orders<8>(w, row0 + v0 * 64, n, some);
#pragma unroll
        for (int v = 0; v < 8; ++v)
          if (v0 + v < each) f(some[v], v0 + v);  // (behind these come the next wave's rows)
      }
    }
  };

  // (Weights have a few exponents between them: several counts of each, side by side in LDS, keep a wave's additions apart.)
  // Eight bits of `least` a round: how many of the rows that agree with it so far have which next eight bits; then the highest
  // of these with at least as many rows at or above it as are still to be found.
  uint32_t least = 0;   // a row at or above it stays, or may
  bool exact = k == n;  // just those stay
  int wanted = k;       // of the rows that agree with `least` in the bits so far
  for (int i = threadIdx.x; i < 4 * kBins / 4; i += THREADS) reinterpret_cast<int4*>(all_bins)[i] = make_int4(0, 0, 0, 0);
  __syncthreads();
  for (int shift = 24; shift >= 0 && !exact; shift -= 8) {
    int* const bins = all_bins + shift / 8 * kBins;  // (a round has its own: one barrier each)
    over_rows([&](uint32_t o, int v) {
      if (row0 + v * 64 < n && (shift == 24 || (o ^ least) >> (shift + 8) == 0)) atomicAdd(&bins[lane % kCopies * Bins<THREADS>::kCopy + (o >> shift & 255)], 1);
    });
    __syncthreads();
    // A lane holds four bins from the top, 255 - 4 lane ..: every wave by itself, or, of sixteen, one for all.
    if (!kOneScans || wave == 0) {
      int in[4] = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < kCopies; ++c) {
        const int4 some = *reinterpret_cast<const int4*>(bins + c * Bins<THREADS>::kCopy + 252 - 4 * lane);
        in[0] += some.w, in[1] += some.z, in[2] += some.y, in[3] += some.x;
      }
      const int own = (in[0] + in[1]) + (in[2] + in[3]);
      const int upto = wave_prefix(own);
      const int at = __builtin_ctzll(__ballot(upto >= wanted));  // (there is one: all the rows that agree are `wanted` or more)
      int above = __builtin_amdgcn_readlane(upto - own, at);     // rows above the bin in question
      int digit = 255 - 4 * at, upto_it = above;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int n_j = __builtin_amdgcn_readlane(in[j], at);
        if (upto_it < wanted) {
          digit = 255 - 4 * at - j;
          above = upto_it;
          upto_it += n_j;
        }
      }
      least |= (uint32_t)digit << shift;
      exact = upto_it == wanted;
      wanted -= above;
    }
    if constexpr (kOneScans) {
      if (threadIdx.x == 0) counts[0][2] = (int)least, counts[0][3] = exact ? 0 : wanted;
      __syncthreads();
      least = (uint32_t)__builtin_amdgcn_readfirstlane(counts[0][2]);
      wanted = __builtin_amdgcn_readfirstlane(counts[0][3]);
      exact = wanted == 0;
    }
  }
  // Where `exact`, those at or above `least` stay, else those above it and the first ones of those at it.
  const uint32_t surely = exact ? least : least + 1;  // (`least` is not the largest of all numbers: that would be a NaN's)
  const auto over = [&](uint32_t o, int v) { return __ballot(row0 + v * 64 < n && o >= surely); };
  const auto same = [&](uint32_t o, int v) { return __ballot(row0 + v * 64 < n && o == least); };
  auto fresh = [&] {  // (the ballots are formed again further on: kept from here to there they would take all registers)
    if constexpr (VALUES > 0) {
#pragma unroll
      for (int v = 0; v < VALUES; ++v) asm volatile("" : "+v"(held[v]));
    }
  };
  int overs = 0, sames = 0;
  over_rows([&](uint32_t o, int v) { overs += __popcll(over(o, v)); });
  if (!exact) over_rows([&](uint32_t o, int v) { sames += __popcll(same(o, v)); });
  fresh();
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
  auto before_me = [](uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u)); };
  if (exact) {
    over_rows([&](uint32_t o, int v) {
      const uint64_t a = over(o, v);
      const int rank = overs + before_me(a);
      if (row0 + v * 64 < n && o >= surely && rank >= lo && rank < hi) list[rank - lo] = row0 + v * 64 + base;
      overs += __popcll(a);
    });
  } else {
    over_rows([&](uint32_t o, int v) {
      const uint64_t a = over(o, v), b = same(o, v);
      const int before = sames + before_me(b), rank = overs + before_me(a) + min(before, ties);
      const bool stays = row0 + v * 64 < n && (o >= surely || (o == least && before < ties));
      if (stays && rank >= lo && rank < hi) list[rank - lo] = row0 + v * 64 + base;
      overs += __popcll(a);
      sames += __popcll(b);
    });
  }
}

// `rows` rows from `list` (packed rows) to row `to` of the smaller cache on.
template <int THREADS, bool ONCE>
__device__ __forceinline__ void copy_rows(const EvictParams& prm, const int32_t* list, int64_t to, int rows) {
  const int pieces = 1 << prm.row_shift, half = pieces / 2;
  constexpr int kAtOnce = 4;
  for (int i0 = threadIdx.x; i0 < rows << prm.row_shift; i0 += kAtOnce * THREADS) {  // 16 bytes a thread and step
    u32x4 x4[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = min(i0 + u * THREADS, (rows << prm.row_shift) - 1), piece = i & (pieces - 1), m = piece >= half;
      const int64_t from = list[i >> prm.row_shift];
      x4[u] = read_piece<ONCE>(prm.moved.from[m] + (from * half + (piece - m * half)) * 16);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = i0 + u * THREADS, piece = i & (pieces - 1), m = piece >= half;
      if (i < rows << prm.row_shift)
        *reinterpret_cast<u32x4*>(prm.moved.to[m] + ((to + (i >> prm.row_shift)) * half + (piece - m * half)) * 16) = x4[u];
    }
  }
}
template <int THREADS>
__device__ __forceinline__ void move_rows(const EvictParams& prm, const int32_t* list, int64_t to, int rows) {
  if (prm.once)
    copy_rows<THREADS, true>(prm, list, to, rows);
  else
    copy_rows<THREADS, false>(prm, list, to, rows);
  for (int i = threadIdx.x; i < rows; i += THREADS) {  // (what is small, all of it asked for before the first is stored)
    const int64_t from = list[i];
    int32_t position = 0;
    float weight = 0.f;
    uint32_t scale[2] = {0, 0};
    if (prm.idx) position = prm.idx[from];
    if (prm.weights_out) weight = prm.weights[from];
    if (prm.moved.bytes[2] == 4) {
      scale[0] = reinterpret_cast<const uint32_t*>(prm.moved.from[2])[from];
      scale[1] = reinterpret_cast<const uint32_t*>(prm.moved.from[3])[from];
    } else if (prm.moved.bytes[2] == 2) {
      scale[0] = reinterpret_cast<const uint16_t*>(prm.moved.from[2])[from];
      scale[1] = reinterpret_cast<const uint16_t*>(prm.moved.from[3])[from];
    }
    if (prm.idx) prm.idx_out[to + i] = position;
    if (prm.weights_out) prm.weights_out[to + i] = weight;
    if (prm.moved.bytes[2] == 4) {
      reinterpret_cast<uint32_t*>(prm.moved.to[2])[to + i] = scale[0];
      reinterpret_cast<uint32_t*>(prm.moved.to[3])[to + i] = scale[1];
    } else if (prm.moved.bytes[2] == 2) {
      reinterpret_cast<uint16_t*>(prm.moved.to[2])[to + i] = (uint16_t)scale[0];
      reinterpret_cast<uint16_t*>(prm.moved.to[3])[to + i] = (uint16_t)scale[1];
    }
  }
}

// The head of a unit of `per` rows that stay (bh -1: behind the last), which of its own units it is, and the rows that stay before it.
struct UnitRows {
  int bh, part, before;
  HeadRows head;
};
__device__ __forceinline__ UnitRows rows_of_unit(const EvictParams& prm, int unit, int per) {
  constexpr int kSets = 4;
  const int lane = threadIdx.x & 63, capacity = (int)prm.capacity;
  UnitRows x = {-1, 0, 0, {0, 0, 0}};
  int units_before = 0;
  for (int base = 0; base < prm.BH; base += 64 * kSets) {
    HeadRows some[kSets];
#pragma unroll
    for (int i = 0; i < kSets; ++i) some[i] = rows_of(prm, min(base + i * 64 + lane, prm.BH - 1), capacity);
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      if (base + i * 64 >= prm.BH) break;
      const int stay = base + i * 64 + lane < prm.BH ? some[i].stay : 0;
      const int units = (int)(((uint32_t)stay + per - 1) / per);
      const int rows_upto = wave_prefix(stay), upto = wave_prefix(units);
      const uint64_t found = __ballot(units_before + upto > unit);
      if (found) {
        const int at = __builtin_ctzll(found);
        x.bh = base + i * 64 + at;
        x.head = {__builtin_amdgcn_readlane(some[i].first, at), __builtin_amdgcn_readlane(some[i].n, at), __builtin_amdgcn_readlane(stay, at)};
        x.part = unit - units_before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(units, at));
        x.before += __builtin_amdgcn_readlane(rows_upto, at) - x.head.stay;
        return x;
      }
      units_before += __builtin_amdgcn_readlane(upto, 63);
      x.before += __builtin_amdgcn_readlane(rows_upto, 63);
    }
  }
  return x;
}

__device__ __forceinline__ void fetch_evict_arguments() {
  typedef EvictParams A;
  fetch_arguments({MASKKV_ARGUMENT(A, weights), MASKKV_ARGUMENT(A, rows), MASKKV_ARGUMENT(A, moved), (uint32_t)(offsetof(A, moved) + 64)});
}

// Short heads.
__global__ __launch_bounds__(256) void evict_kernel(const EvictParams prm) {
  extern __shared__ int32_t list[];  // [per]
  __shared__ __attribute__((aligned(16))) int bins[4 * Bins<256>::kRound];
  __shared__ int counts[4][4];
  fetch_evict_arguments();
  if (blockIdx.x == 0 && threadIdx.x < 64) write_prefix(prm);
  const UnitRows x = rows_of_unit(prm, blockIdx.x, prm.per);
  if (x.bh < 0) return;
  const int lo = x.part * prm.per, n = x.head.n, k = x.head.stay, first = x.head.first;
  const int64_t to = (int64_t)x.before + lo;
  const int rows = (int)min((int64_t)min(k - lo, prm.per), prm.capacity_out - to);
  if (rows <= 0) return;
  const float* w = prm.weights + first;
  if (n <= 64)
    list_rows_alone<256, 1>(w, n, k, lo, lo + rows, first, list);
  else if (n <= 256)
    list_rows_alone<256, 4>(w, n, k, lo, lo + rows, first, list);
  else if (n <= 512)
    list_rows_alone<256, 8>(w, n, k, lo, lo + rows, first, list);
  else if (n <= 256 * 4)
    list_rows<256, 4>(w, n, k, lo, lo + rows, first, list, bins, counts);
  else if (n <= 256 * 8)
    list_rows<256, 8>(w, n, k, lo, lo + rows, first, list, bins, counts);
  else if (n <= 256 * 16)
    list_rows<256, 16>(w, n, k, lo, lo + rows, first, list, bins, counts);
  else
    list_rows<256, 0>(w, n, k, lo, lo + rows, first, list, bins, counts);
  __syncthreads();
  for (int i = threadIdx.x; i < rows; i += 256) prm.rows[to + i] = list[i];
  move_rows<256>(prm, list, to, rows);
}

// Long heads: the rows that stay of a head, ...
__global__ __launch_bounds__(1024) void evict_rows_kernel(const EvictParams prm) {
  __shared__ __attribute__((aligned(16))) int bins[4 * Bins<1024>::kRound];
  __shared__ int counts[16][4];
  fetch_evict_arguments();
  if (blockIdx.x == 0 && threadIdx.x < 64) write_prefix(prm);
  const UnitRows x = rows_of_unit(prm, blockIdx.x, 0x7FFFFFFF);  // (a head of which rows stay is one unit)
  if (x.bh < 0) return;
  const int n = x.head.n, k = x.head.stay, first = x.head.first, rows = (int)min((int64_t)k, prm.capacity_out - x.before);
  if (rows <= 0) return;
  const float* w = prm.weights + first;
  int32_t* list = prm.rows + x.before;
  if (n <= 1024 * 2)
    list_rows<1024, 2>(w, n, k, 0, rows, first, list, bins, counts);
  else if (n <= 1024 * 4)
    list_rows<1024, 4>(w, n, k, 0, rows, first, list, bins, counts);
  else if (n <= 1024 * 8)
    list_rows<1024, 8>(w, n, k, 0, rows, first, list, bins, counts);
  else if (n <= 1024 * 16)
    list_rows<1024, 16>(w, n, k, 0, rows, first, list, bins, counts);
  else if (n <= 1024 * 32)
    list_rows<1024, 32>(w, n, k, 0, rows, first, list, bins, counts);
  else
    list_rows<1024, 0>(w, n, k, 0, rows, first, list, bins, counts);
}

// ... and their moving, `per` a workgroup.
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams prm) {
  extern __shared__ int32_t list[];  // [per]
  fetch_evict_arguments();
  const int64_t to = (int64_t)blockIdx.x * prm.per;
  const int rows = (int)min((int64_t)prm.per, min((int64_t)prm.cu_out[prm.BH], prm.capacity_out) - to);
  if (rows <= 0) return;
  for (int i = threadIdx.x; i < rows; i += 256) list[i] = prm.rows[to + i];
  __syncthreads();
  move_rows<256>(prm, list, to, rows);
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
  // (A third of the memory-side cache: the new cache and others are beside it.  Past it and through it, 256 heads of bf16 rows, half of them moved: 66 MB
  // 21.3 and 18.5 us, 79 MB 22.3 and 22.4, 92 MB 24.9 and 25.8, 131 MB 32.0 and 37.9; 139 MB in 4 bits, with their expansion, 117 and 128.)
  prm.once = 2 * capacity * moved.bytes[0] > kSideCache / 3;
  prm.row_shift = 0;
  while (16 << prm.row_shift < 2 * moved.bytes[0]) ++prm.row_shift;
  // Workgroups for two of every compute unit, of 16 rows at least and of no more than the list has room for.
  const int64_t most = capacity_out < capacity ? capacity_out : capacity;  // (no more rows stay than there are)
  int64_t per = (most + 511) / 512;
  per = per < 16 ? 16 : per > kMostRows ? kMostRows : per;
  prm.per = (int)per;
  if (capacity <= (int64_t)kShortHead * prm.BH || d->P_max <= kLongestHead || capacity <= kLongestHead) {
    const int64_t groups = most / per + prm.BH;  // (each head's last one may have fewer)
    hipLaunchKernelGGL(evict_kernel, dim3((unsigned)groups), dim3(256), per * 4, stream, prm);
    return check_launch("evict");
  }
  hipLaunchKernelGGL(evict_rows_kernel, dim3((unsigned)prm.BH), dim3(1024), 0, stream, prm);
  if (int e = check_launch("evict (rows)")) return e;
  if (most == 0) return MASKKV_OK;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)((most + per - 1) / per)), dim3(256), per * 4, stream, prm);
  return check_launch("evict (move)");
}

}  // namespace maskkv
