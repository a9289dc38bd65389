// The attention that each cached row gets, added up over the denoising steps: for a cached row k of a head
//   out = decay * in + sum_i exp(q_i . k * scale - lse_i)    over the query rows i of the head's group.
//
// A wave holds 32 rows of the cache as the A operand of its matrix instructions for as long as it takes all query rows past
// them, 32 at a step: a lane then owns one query, whose normaliser is one number, and adds up what that query gives to 16 of the
// rows; the lanes' sums meet once, at the end.  The queries come through LDS, moved as whole rows.
//
// Where there are many cached rows the four waves of a workgroup hold 32 each and share the queries (SHARE), which come by direct
// transfers into a ring of four steps, three ahead, one barrier a step; where there are few, all waves hold the same 32 and take the steps
// in turn.  Sums have a fixed order either way.
//
// Probabilities stay in fp32: nothing is rounded but the inputs.  A lane's sums of 16 rows run over its queries, so a row's sum has a chain of
// n / 32 additions and five more, in fp32.
//
// Bound by vector instructions where there is much to do: an exponential, a multiply-add and an addition for every (query, row), 24 cycles of the
// vector pipe for 64 of them beside 16 of the matrix pipe at head_dim 128.  512 queries of 256 heads x 64 ... 1024 rows (89 k): 21.9 ... 23.3 us, the vector
// pipe busy half and the matrix pipe a third of the time; the busiest compute units have four workgroups, the average 3.25.  256 queries x 32
// heads x 250 rows: 5.8, the latency of arguments, heads' ends, rows and queries in turn.
// Units dealt to the XCDs in runs of eight, an eighth each, and one at a time: 21.9, 22.5 and 27.1 us for those, 9.2, 11.6 and 10.8 for 64 queries of 256 heads
// x 128 ... 1024 rows, 25.8, 32.2 and 25.8 for 64 of 2048 heads x 16 ... 128 rows, 17.2, 17.2 and 18.0 for 128 of 64 heads of a group of four.
#include <type_traits>

#include "lds.hpp"
#include "mx.hpp"

namespace maskkv {

namespace {

constexpr int kUnits = 256;  // compute units
constexpr int kTile = 32;    // cached rows of a wave, query rows of a step

struct AccumulateParams {
  View Q;
  const char* Kc;
  MxCache cache;
  const int32_t* cu;
  int64_t capacity;
  int H, BH, q_per_kv, n_resp, n_q;
  int groups;  // workgroups, a multiple of 8
  float c;  // scale * log2(e)
  float decay;
  const float *lse, *in;
  float* out;
};

template <typename T, int D, int WAVES, bool SHARE>
struct AccCfg {
  static constexpr int kRowB = D * (int)sizeof(T);
  static constexpr int kPPR = kRowB / 16;             // pieces of 16 bytes in a row
  static constexpr int kMovers = SHARE ? WAVES : 1;   // waves that move a step's queries
  static constexpr int kRPL = kMovers * 64 / kPPR;    // rows of a load of theirs
  static constexpr int kLoads = kTile / kRPL;
  static constexpr int kStepB = kTile * kRowB;
  static constexpr int kRing = 4;                                // steps
  static constexpr int kMoves = kStepB / 1024 / WAVES;           // direct transfers of a wave and step, of 1 KiB
  static constexpr int kNormB = 256;                             // of a wave and step: the queries' normalisers (twice)
  static constexpr int kNormAt = kRing * kStepB;
  static constexpr int kLds = SHARE ? kNormAt + kRing * WAVES * kNormB : WAVES * kStepB;
  __device__ static uint32_t swz(uint32_t row) { return sizeof(T) == 2 && D == 64 ? (row >> 1) & 7 : row & 15; }
};

template <typename T, int D, bool MX, int WAVES, bool SHARE>
__global__ __launch_bounds__(WAVES * 64) void accumulate_kernel(const AccumulateParams prm) {
  using C = AccCfg<T, D, WAVES, SHARE>;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int kRows = SHARE ? WAVES * kTile : kTile;  // cached rows of a workgroup
  extern __shared__ __attribute__((aligned(16))) char acc_lds[];
  __shared__ float part[WAVES][kTile];
  typedef AccumulateParams A;
  fetch_arguments({MASKKV_VIEW_ARGUMENTS(A, Q), MASKKV_ARGUMENT(A, Kc), MASKKV_ARGUMENT(A, BH), MASKKV_ARGUMENT(A, out)});
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, g = lane >> 5;
  // Each XCD (workgroups whose numbers are congruent modulo 8) takes runs of eight units: most of a head's queries stay in one L2, and the units
  // that there may be, but are not, are on all XCDs alike.
  const int group = group_number();
  if (group >= prm.groups) return;
  const int unit = group / 64 * 64 + 64 <= prm.groups ? group / 64 * 64 + group % 8 * 8 + group / 8 % 8 : group;
  const int capacity = (int)prm.capacity;
  const UnitHead head = head_of_unit(prm.cu, prm.BH, capacity, unit, [](int n) { return (int)(((uint32_t)n + kRows - 1) / kRows); });
  const int bh = head.bh;
  if (bh < 0) return;
  const int b = bh / prm.H, h = bh % prm.H;
  const int last = head.first + head.rows - 1;
  const int row0 = head.first + (unit - head.first_unit) * kRows + (SHARE ? wave * kTile : 0);  // of this wave
  const int64_t row = min(row0 + r, last);  // (row0 may lie behind the head's end: nothing of such a wave is stored)

  const int steps = (prm.n_q + kTile - 1) / kTile;
  constexpr int kEvery = SHARE ? 1 : WAVES;  // a wave's steps: every so many
  const int mover = SHARE ? threadIdx.x : lane;
  u32x4 moved[C::kLoads];
  float lse = 0.f;
  auto load_step = [&](int s) {
#pragma unroll
    for (int j = 0; j < C::kLoads; ++j) {
      const int i = min(s * kTile + j * C::kRPL + mover / C::kPPR, prm.n_q - 1);
      moved[j] = *reinterpret_cast<const u32x4*>(prm.Q.group_row(b, h, prm.q_per_kv, prm.n_resp, i) + mover % C::kPPR * 16);
    }
    lse = s * kTile + r < prm.n_q ? prm.lse[(int64_t)bh * prm.n_q + s * kTile + r] : INFINITY;
  };
  auto store_step = [&](char* to) {
#pragma unroll
    for (int j = 0; j < C::kLoads; ++j) {
      const uint32_t i = j * C::kRPL + mover / C::kPPR, p = mover % C::kPPR;
      *reinterpret_cast<u32x4*>(to + i * C::kRowB + ((p ^ C::swz(i)) << 4)) = moved[j];
    }
  };
  // SHARE: a wave moves a quarter of a step's queries, and its own copy of their normalisers.  Rows behind the last one are the last one.
  // (A whole step of a head without a group has a base that all lanes share and offsets that they keep; else every row's head is
  // found by a division.)
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)acc_lds;
  const uint32_t norm_at = lds0 + C::kNormAt + wave * C::kNormB;
  const char* const queries = prm.Q.row(b, h * prm.q_per_kv, 0);
  uint32_t offset[SHARE ? C::kMoves : 1];
  auto row_of = [&](int j) { return (wave * C::kMoves + j) * (1024 / C::kRowB) + lane / C::kPPR; };
  auto piece_of = [&](int j) { return ((uint32_t)lane % C::kPPR ^ C::swz(row_of(j))) * 16; };
  if constexpr (SHARE) {
#pragma unroll
    for (int j = 0; j < C::kMoves; ++j) offset[j] = row_of(j) * (uint32_t)prm.Q.stride_t + piece_of(j);
  }
  auto move_step = [&](int s) {
    const uint32_t to = lds0 + s % C::kRing * C::kStepB + wave * C::kMoves * 1024;
    const int from = s * kTile;
    if (prm.q_per_kv == 1 && from + kTile <= prm.n_q) {
      const char* base = queries + (int64_t)from * prm.Q.stride_t;
#pragma unroll
      for (int j = 0; j < C::kMoves; ++j) dma16(base, offset[j], to + j * 1024);
    } else {
#pragma unroll
      for (int j = 0; j < C::kMoves; ++j)
        dma16_from(prm.Q.group_row(b, h, prm.q_per_kv, prm.n_resp, min(from + row_of(j), prm.n_q - 1)) + piece_of(j), to + j * 1024);
    }
    dma4(reinterpret_cast<const char*>(prm.lse + (int64_t)bh * prm.n_q), (uint32_t)min(from + r, prm.n_q - 1) * 4,
         norm_at + s % C::kRing * (WAVES * C::kNormB));
  };
  if constexpr (SHARE) {
    for (int s = 0; s < C::kRing - 1; ++s)
      if (s < steps) move_step(s);
  }
  const int s0 = wave;
  if (!SHARE && s0 < steps) load_step(s0);

  // ---- this lane's half of a cached row
  u32x4 kf[C::kPPR / 2];
  if constexpr (MX) {
    const char* codes = prm.cache.k_codes + row * (D / 2) + g * (D / 4);
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(prm.cache.k_scales) + row * (D / 32) + g * (D / 64);
    u32x4 c[D / 64];
    float unit_of[D / 64];
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      c[j] = reinterpret_cast<const u32x4*>(codes)[j];
      unit_of[j] = mx_unit(scales[j]);
    }
#pragma unroll
    for (int w = 0; w < D / 16; ++w) {
      const uint32_t word = c[w / 4][w % 4];
      if constexpr (F32) {
        float x[8];
        mx_decode_f32(word, unit_of[w / 4], x);
        kf[2 * w] = u32x4{as_u32(x[0]), as_u32(x[1]), as_u32(x[2]), as_u32(x[3])};
        kf[2 * w + 1] = u32x4{as_u32(x[4]), as_u32(x[5]), as_u32(x[6]), as_u32(x[7])};
      } else {
        kf[w] = mx_decode_bf16(word, unit_of[w / 4]);
      }
    }
  } else {
    const u32x4* k = reinterpret_cast<const u32x4*>(prm.Kc + row * C::kRowB + g * (C::kRowB / 2));
#pragma unroll
    for (int i = 0; i < C::kPPR / 2; ++i) kf[i] = k[i];
  }

  float sum[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i] = 0.f;
  uint32_t fragment[C::kPPR / 2];  // where this lane's half of its query's row lies in a step
#pragma unroll
  for (int i = 0; i < C::kPPR / 2; ++i) fragment[i] = r * C::kRowB + (((g * (C::kPPR / 2) + i) ^ C::swz(r)) << 4);
  auto take = [&](uint32_t base, int imm, float lse_now) __attribute__((always_inline)) {
    f32x16 x = {};
#pragma unroll
    for (int i = 0; i < C::kPPR / 2; ++i) {
      const u32x4 q = *in_lds<const u32x4>(base + fragment[i], imm);
      mfma_step<T>(kf[i], q, x);
    }
    const float by = -lse_now * kLog2e;
    const bool none = lse_now == INFINITY;  // (adds nothing, whatever the query holds)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = fast_exp2(fmaf(x[i], prm.c, by));
    if (__any(none)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = none ? 0.f : x[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] += x[i];
  };
  if constexpr (SHARE) {
#pragma unroll
    for (int i = 0; i < C::kPPR / 2; ++i) fragment[i] += lds0;
    auto step = [&](int s, auto place) __attribute__((always_inline)) {
      constexpr int kPlace = decltype(place)::value;  // s % kRing
      // This wave's part of step s is there when only those of the two steps behind it are under way; behind the barrier so are the other
      // waves', and all of them have read step s - 1, whose place step s + 3 takes.
      __builtin_amdgcn_sched_barrier(0);
      if (s + 2 < steps)
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"(2 * (C::kMoves + 1)) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      if (s + 3 < steps) move_step(s + 3);
      const float norm = *in_lds<const float>(norm_at + r * 4, kPlace * (WAVES * C::kNormB));
      take(0, kPlace * C::kStepB, s * kTile + r < prm.n_q ? norm : INFINITY);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (read before the barrier)
    };
    for (int s = 0; s < steps; s += C::kRing) {
      step(s, std::integral_constant<int, 0>());
      if (s + 1 < steps) step(s + 1, std::integral_constant<int, 1>());
      if (s + 2 < steps) step(s + 2, std::integral_constant<int, 2>());
      if (s + 3 < steps) step(s + 3, std::integral_constant<int, 3>());
    }
  } else {
    char* own = acc_lds + wave * C::kStepB;
    for (int s = s0; s < steps; s += kEvery) {
      store_step(own);
      const float lse_now = lse;
      if (s + kEvery < steps) load_step(s + kEvery);
      asm volatile("" ::: "memory");
      take(lds0 + wave * C::kStepB, 0, lse_now);
      asm volatile("" ::: "memory");
    }
  }

  // ---- a row's sum over the 32 lanes of its half: each exchange leaves a lane half of the rows
#pragma unroll
  for (int half = 8; half > 0; half >>= 1) {
    const bool upper = lane & 2 * half;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const float keep = upper ? sum[half + i] : sum[i], give = upper ? sum[i] : sum[half + i];
      sum[i] = keep + __shfl_xor(give, 2 * half, 64);
    }
  }
  float total = sum[0] + __shfl_xor(sum[0], 1, 64);
  const int i = (lane >> 1) & 15, at = 8 * (i / 4) + 4 * g + i % 4;
  const bool mine = !(lane & 1);
  if constexpr (!SHARE) {
    if (mine) part[wave][at] = total;
    __syncthreads();
    if (wave > 0) return;
    total = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += part[w][at];
  }
  if (mine && row0 + at <= last) prm.out[row0 + at] = prm.decay > 0.f ? fmaf(prm.decay, prm.in[row0 + at], total) : total;
}

template <typename T, int D, bool MX, int WAVES, bool SHARE>
int launch_form(AccumulateParams prm, hipStream_t stream) {
  using C = AccCfg<T, D, WAVES, SHARE>;
  static_assert(C::kLds + WAVES * kTile * 4 <= 160 * 1024, "a workgroup's LDS");
  const int rows = SHARE ? WAVES * kTile : kTile;
  prm.groups = (int)((prm.capacity / rows + prm.BH + 7) / 8 * 8);  // (each head's last ones may be short)
  const auto kernel = accumulate_kernel<T, D, MX, WAVES, SHARE>;
  if (C::kLds > 48 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, C::kLds);
    if (e != hipSuccess) {
      set_error("accumulate: cannot raise dynamic LDS limit: %s", hipGetErrorString(e));
      (void)hipGetLastError();
      return MASKKV_EHIP;
    }
  }
  hipLaunchKernelGGL(kernel, grid_of(prm.groups), dim3(WAVES * 64), C::kLds, stream, prm);
  return check_launch("accumulate");
}

// Few: tiles of cached rows for less than two workgroups a compute unit, and more than one step of queries to deal to waves instead.  In turn and
// shared, 32 heads of one length, 512 queries: 288 tiles 7.2 and 10.6 us, 448 9.7 and 10.6, 512 9.8 and 10.6, 576 11.9 and 11.3, 832 16.2 and 11.6; 128
// queries: 288 tiles 4.4 and 5.2, 448 5.4 and 5.3, 576 6.5 and 5.3; 40 queries 4.1 and 4.7, 4.5 and 4.8, 4.9 and 4.8; fp32, 128 queries, 312 tiles 10.5 and 12.9.
template <typename T, int D, bool MX>
int launch_rows(const AccumulateParams& prm, hipStream_t stream) {
  const int64_t tiles = prm.capacity / kTile + prm.BH;
  const int steps = (prm.n_q + kTile - 1) / kTile;
  if (steps > 1 && tiles < 2 * kUnits) return launch_form<T, D, MX, 4, false>(prm, stream);
  return launch_form<T, D, MX, 4, true>(prm, stream);
}

template <typename T, int D>
int launch_one(const AccumulateParams& prm, hipStream_t stream) {
  return prm.Kc ? launch_rows<T, D, false>(prm, stream) : launch_rows<T, D, true>(prm, stream);
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
    return d->d == 128 ? launch_one<bf16_t, 128>(prm, stream) : launch_one<bf16_t, 64>(prm, stream);
  return d->d == 128 ? launch_one<float, 128>(prm, stream) : launch_one<float, 64>(prm, stream);
}

}  // namespace maskkv
