// Attention of the response span over a cache in 4 bits and the response's own rows: one pass over the keys with the running maximum and
// sum of a softmax.  Three kernels: up to 16 query rows a head (bf16), 32 a workgroup, and 128 a workgroup (bf16); which of them a launch
// takes, and whether a head's keys go to several workgroups, is chosen by what it is expected to take (`deal_of`).
//
// 32 query rows: four waves serve 32 query rows of a head.  Logits are formed transposed (keys on the matrix instruction's row
// axis), so that a lane owns one query and its probabilities are the B operand of O^T = V^T P^T as they stand.  The waves take
// tiles of 32 keys in turn, each through registers and LDS of its own, without a barrier, and are merged at the end.  A
// row's two halves along the head dimension belong to the two halves of a wave: a lane's codes of a key are 16 (8) whole words
// in a row, its scales two bytes (one), and the conversion of a word is an operand of a matrix instruction.  Values are converted on
// their way into LDS, from where a transposing read brings them as V^T.  The response's tiles come first: what is read of the
// cache for the first of its tiles is under way meanwhile.  Rows of the response are moved whole and pass through LDS: as the product wants them, half
// a row a lane, a load would touch 64 lines of memory (32 heads x 512 queries x 250 rows 19.8 us that way and 18.3 this, x 256 queries the same 10.1).
//
// The values of 4 bits are exact in bf16, so the logits are those of the stored values; sums, maxima and outputs are fp32 throughout.
// Probabilities are rounded to bf16, by at most 2^-8 of each, as the operand of the second product: fp32 operands have a sixteenth of its rate.
// The sum that divides them is of the unrounded ones.  Partial results are fp32.
//
// Where the keys are dealt out, or only those of long heads, a second kernel joins the partial results: in the same launch it would take a counter that is zero
// when the call begins, and a workspace need not be.
//
// Bound by latency where there is little to do: 32 heads x 256 queries x 250 + 256 rows, head_dim 128, 10.1 us, of which 6.5 are the launch, the
// first loads and the merging of the waves; one query row of 7 heads over 4 x 30k rows 7.6 + 3.0 us (16 MB, 3.2 at a large copy's rate).
// By the two phases of a tile where there is much: 256 heads x 512 queries x 64 ... 1024 rows 77 ... 82 us by the board, 700 ... 745 TFLOP/s, the matrix pipe busy
// 38 % and the vector pipe 44 % of the time, at a clock that the board's power lowers to 1.85 GHz; the same from a cache in bf16 takes 75.5.
// By the memory where few queries meet a cache that is larger than the memory-side one: a token of 64 heads of four x 16384 rows (143 MB) 33 us, 4.4 TB/s, 128 heads of
// eight x 32768 (570 MB) 108, 5.3; the former over rows of bf16, 537 MB, takes 171 in maskkv_attend.
#include <cmath>
#include <type_traits>

#include "attend.hpp"
#include "mx.hpp"

namespace maskkv {

namespace {

constexpr int kUnits = 256;  // compute units
constexpr int kTile = 32;    // keys of a tile, and query rows of a workgroup
constexpr int kWaves = 4;

struct AttendMxParams {
  View Q, K2, V2, O;
  MxCache cache;
  const int32_t* cu;
  int64_t capacity;
  int H, BH, q_per_kv, n_resp, n_q, qtiles;
  int units;      // at most
  int chunk;      // tiles of a workgroup, or 0: all of its head
  int extras;     // (see Work) or 0
  int tile_rows;  // query rows of a workgroup
  int part_rows;  // of a partial result
  float c;        // scale * log2(e)
  float* lse;
  float* part_o;    // [places * qtiles][part_rows][D], a place a unit (with extras: see Work)
  float2* part_ml;  // [places * qtiles][part_rows]
  int2* parts;      // [BH] a head's first unit, and how many it has (with extras: not used)
};

__device__ __forceinline__ void fetch_attend_mx_arguments() {
  typedef AttendMxParams A;
  fetch_arguments({MASKKV_VIEW_ARGUMENTS(A, Q), MASKKV_VIEW_ARGUMENTS(A, K2), MASKKV_VIEW_ARGUMENTS(A, V2), MASKKV_VIEW_ARGUMENTS(A, O),
                   MASKKV_ARGUMENT(A, cache), MASKKV_ARGUMENT(A, H), (uint32_t)(offsetof(A, parts) + 4)});
}

template <typename T, int D>
struct MxCfg {
  static constexpr int kRowB = D * (int)sizeof(T);
  static constexpr int kPPR = kRowB / 16;        // pieces of 16 bytes in a row
  static constexpr int kLoads = kPPR / 2;        // of 16 bytes a lane, of a tile's V
  static constexpr int kRPL = 64 / kPPR;         // rows of such a load
  static constexpr int kWords = D / 16;          // code words of a lane's half row
  static constexpr int kDB = D / 32;
  static constexpr int kTileB = kTile * kRowB;     // K, then V of a wave
  static constexpr int kSumP = D / 2 + 4;          // floats from one query's sums to the next while the waves are merged, half a row at a time
  static constexpr int kSumB = kTile * kSumP * 4;
  static constexpr int kMlAt = kWaves * (kTileB > kSumB ? kTileB : kSumB);
  static constexpr int kLds = kMlAt + kWaves * kTile * 8;
  // Rows that are read by halves, 16 bytes a lane: neighbouring rows on different banks.
  __device__ static uint32_t slot(uint32_t row, uint32_t p) { return p ^ (kPPR == 8 ? (row >> 1) & 7 : row & 15); }
  // V: bf16 see v_swizzle; fp32: blocks of 32 columns, exchanged in every other four rows.
  __device__ static uint32_t v_slot(uint32_t row, uint32_t p) {
    return sizeof(T) == 2 ? (p ^ v_swizzle<D>(row) << 1) : p ^ ((row >> 2) & 1) << 3;
  }
};

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) == 2 ? 2 : 1) void attend_mx_kernel(const AttendMxParams prm) {
  using C = MxCfg<T, D>;
  constexpr bool F32 = sizeof(T) == 4;
  extern __shared__ __attribute__((aligned(1024))) char mx_lds[];
  fetch_attend_mx_arguments();
  const Place place = place_of(blockIdx.x, prm.units, prm.qtiles);
  const int unit = place.unit, qtile = place.qtile;
  const int resp_tiles = (prm.n_resp + kTile - 1) / kTile;
  auto tiles_of = [&](int rows) { return (int)(((uint32_t)rows + kTile - 1) / kTile) + resp_tiles; };  // those of the response first
  const int capacity = (int)prm.capacity;
  UnitHead head;
  if (prm.chunk) {
    head = head_of_unit(prm.cu, prm.BH, capacity, unit, [&](int rows) { return (tiles_of(rows) + prm.chunk - 1) / prm.chunk; });
    if (head.bh < 0) return;
  } else {
    const int first = min(prm.cu[unit], capacity);
    head = {unit, unit, 1, first, max(min(prm.cu[unit + 1], capacity) - first, 0)};
  }
  const int bh = head.bh, units = head.units, cached = head.rows, tiles = tiles_of(cached);
  const int b = bh / prm.H, h = bh % prm.H;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, g = lane >> 5;
  if (prm.chunk && unit == head.first_unit && qtile == 0 && threadIdx.x == 0) prm.parts[bh] = make_int2(head.first_unit, units);
  const int t0 = prm.chunk ? (unit - head.first_unit) * prm.chunk : 0;
  const int t1 = prm.chunk ? min(tiles, t0 + prm.chunk) : tiles;

  char* const v_lds = mx_lds + wave * C::kTileB;
  const uint32_t v_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)v_lds;

  // ---- what is under way: two tiles of the cache, and one of the response
  struct Cached {
    u32x4 k[D / 64], v[D / 64];
    uint32_t ks, vs;
  } one, two;
  struct Resp {
    u32x4 k[C::kLoads], v[C::kLoads];  // whole rows
  } ahead;
  auto load_resp = [&](int t, Resp& x) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < C::kLoads; ++j) {
      const int row = min(t * kTile + j * C::kRPL + lane / C::kPPR, prm.n_resp - 1);
      x.k[j] = *reinterpret_cast<const u32x4*>(prm.K2.row(b, h, row) + lane % C::kPPR * 16);
      x.v[j] = *reinterpret_cast<const u32x4*>(prm.V2.row(b, h, row) + lane % C::kPPR * 16);
    }
  };
  // (A tile's first row is the same in all lanes: their offsets from it are all that is formed for each.)
  auto load_cached = [&](int t, Cached& x) __attribute__((always_inline)) {
    const int64_t base = (int64_t)head.first + t * kTile;
    const uint32_t row = min(r, cached - t * kTile - 1);  // (rows behind the last one are the last one)
    const uint32_t at = row * (D / 2) + g * (D / 4), scale = row * (D / 32) + g * (D / 64);
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      x.k[j] = *reinterpret_cast<const u32x4*>(prm.cache.k_codes + base * (D / 2) + at + 16 * j);
      x.v[j] = *reinterpret_cast<const u32x4*>(prm.cache.v_codes + base * (D / 2) + at + 16 * j);
    }
    const char *ks = prm.cache.k_scales + base * (D / 32) + scale, *vs = prm.cache.v_scales + base * (D / 32) + scale;
    x.ks = D == 128 ? *reinterpret_cast<const uint16_t*>(ks) : *reinterpret_cast<const uint8_t*>(ks);
    x.vs = D == 128 ? *reinterpret_cast<const uint16_t*>(vs) : *reinterpret_cast<const uint8_t*>(vs);
  };
  // This wave's tiles: t0 + wave, and every fourth from there; those of the response are the first `resp` of them.
  const int mine = max(t1 - t0 - wave + kWaves - 1, 0) / kWaves;
  const int resp = min(max(min(resp_tiles, t1) - t0 - wave + kWaves - 1, 0) / kWaves, mine);
  auto tile_of = [&](int i) { return t0 + wave + i * kWaves; };
  if (resp > 0) load_resp(tile_of(0), ahead);
  if (mine > resp) load_cached(tile_of(resp) - resp_tiles, one);
  if (mine > resp + 1) load_cached(tile_of(resp + 1) - resp_tiles, two);

  // ---- this lane's query: half of its row, as the B operand of the first product
  u32x4 qf[C::kPPR / 2];
  {
    const char* q = prm.Q.group_row(b, h, prm.q_per_kv, prm.n_resp, min(qtile * kTile + r, prm.n_q - 1)) + g * (C::kRowB / 2);
#pragma unroll
    for (int i = 0; i < C::kPPR / 2; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + 16 * i);
  }

  f32x16 o[C::kDB], s;
#pragma unroll
  for (int db = 0; db < C::kDB; ++db) o[db] = f32x16{};
  float m = kNegBig, l = 0.f;

  auto logits_step = [&](int i, const u32x4& x) __attribute__((always_inline)) {  // bf16: word i of the lane's half row
    mfma_step<bf16_t>(x, qf[i], s);
  };
  auto logits_step_f32 = [&](int i, const float (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t q = qf[2 * i + e / 4][e % 4];
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], as_f32(q), s, 0, 0, 0);
    }
  };

  // ---- softmax of a tile with `left` rows, and the output update.  Lanes l and l ^ 32 have the same query.
  auto update = [&](int left) __attribute__((always_inline)) {
    if (left < kTile) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i / 4) + i % 4 >= left - 4 * g) s[i] = -INFINITY;
    }
    float bm = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) bm = fmaxf(bm, s[i]);
    const float cand = max_halves(bm) * prm.c;
    const bool bump = cand > m + kLazyBump;  // (see attend.hip)
    if (__any(bump)) {
      const float m_new = bump ? cand : m;
      const float alpha = fast_exp2(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < C::kDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = fast_exp2(fmaf(s[i], prm.c, -m));
      s[i] = p;
      l += p;
    }
    if constexpr (!F32) {
      uint32_t from = v_at + v_read_offset<D>(lane, 0);
      asm volatile("" : "+v"(from));  // (an address for each block would be kept in a register of its own)
#pragma unroll
      for (int tp = 0; tp < 2; ++tp) {
        u32x4 pf;
#pragma unroll
        for (int w = 0; w < 4; ++w) pf[w] = pack_bf16x2(s[8 * tp + 2 * w], s[8 * tp + 2 * w + 1]);
#pragma unroll
        for (int db = 0; db < C::kDB; ++db) {
          const u32x2 lo = read_transposed(from ^ db << 6, 16 * tp * C::kRowB), hi = read_transposed(from ^ db << 6, (16 * tp + 8) * C::kRowB);
          mfma_step<bf16_t>(u32x4{lo[0], lo[1], hi[0], hi[1]}, pf, o[db]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = 8 * (i / 4) + 4 * g + i % 4;
#pragma unroll
        for (int db = 0; db < C::kDB; ++db) {
          const float v = *reinterpret_cast<const float*>(v_lds + row * C::kRowB + ((db ^ ((row >> 2) & 1)) * 32 + r) * 4);
          o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[i], o[db], 0, 0, 0);
        }
      }
    }
  };

  for (int i = 0; i < resp; ++i) {
    const int t = tile_of(i);
    auto rows_to_lds = [&](const u32x4 (&x)[C::kLoads], auto slot) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < C::kLoads; ++j) {
        const uint32_t row = j * C::kRPL + lane / C::kPPR, p = lane % C::kPPR;
        *reinterpret_cast<u32x4*>(v_lds + row * C::kRowB + (slot(row, p) << 4)) = x[j];
      }
    };
    rows_to_lds(ahead.k, [](uint32_t row, uint32_t p) { return C::slot(row, p); });
    asm volatile("" ::: "memory");
    s = f32x16{};
#pragma unroll
    for (int w = 0; w < C::kPPR / 2; ++w)
      mfma_step<T>(*reinterpret_cast<const u32x4*>(v_lds + r * C::kRowB + (C::slot(r, g * (C::kPPR / 2) + w) << 4)), qf[w], s);
    asm volatile("" ::: "memory");
    rows_to_lds(ahead.v, [](uint32_t row, uint32_t p) { return C::v_slot(row, p); });
    if (i + 1 < resp) load_resp(tile_of(i + 1), ahead);
    asm volatile("" ::: "memory");
    update(prm.n_resp - t * kTile);
    asm volatile("" ::: "memory");
  }
  auto take = [&](int i, Cached& x) __attribute__((always_inline)) {
    const int t = tile_of(i) - resp_tiles;
    // V on its way into LDS, K into the first product
    uint32_t to = v_at + r * C::kRowB + (C::v_slot(r, g * (C::kPPR / 2)) << 4);
    asm volatile("" : "+v"(to));
#pragma unroll
    for (int w = 0; w < C::kWords; ++w) {
      const uint32_t word = x.v[w / 4][w % 4];
      const float unit = mx_unit(x.vs >> (8 * (w / 4)) & 255);
      if constexpr (F32) {
        float y[8];
        mx_decode_f32(word, unit, y);
        *in_lds<u32x4>(to ^ 2 * w << 4) = u32x4{as_u32(y[0]), as_u32(y[1]), as_u32(y[2]), as_u32(y[3])};
        *in_lds<u32x4>(to ^ (2 * w + 1) << 4) = u32x4{as_u32(y[4]), as_u32(y[5]), as_u32(y[6]), as_u32(y[7])};
      } else {
        *in_lds<u32x4>(to ^ w << 4) = mx_decode_bf16(word, unit);
      }
    }
    asm volatile("" ::: "memory");
    s = f32x16{};
#pragma unroll
    for (int w = 0; w < C::kWords; ++w) {
      const uint32_t word = x.k[w / 4][w % 4];
      const float unit = mx_unit(x.ks >> (8 * (w / 4)) & 255);
      if constexpr (F32) {
        float y[8];
        mx_decode_f32(word, unit, y);
        logits_step_f32(w, y);
      } else {
        logits_step(w, mx_decode_bf16(word, unit));
      }
    }
    if (i + 2 < mine) load_cached(t + 2 * kWaves, x);
    update(cached - t * kTile);
    asm volatile("" ::: "memory");
  };
  for (int i = resp; i < mine; i += 2) {
    take(i, one);
    if (i + 1 < mine) take(i + 1, two);
  }

  // ---- the waves' results become one: sums of each wave, in units of the largest reference, through LDS
  l = sum_halves(l);
  float2* const ml = reinterpret_cast<float2*>(mx_lds + C::kMlAt);
  if (g == 0) ml[wave * kTile + r] = make_float2(m, l);
  __syncthreads();
  float top = kNegBig;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w * kTile + r].x);
  const float mine_by = fast_exp2(m - top);
  float* const sums = reinterpret_cast<float*>(mx_lds);
  constexpr int kEach = 8;                // elements of a row that a thread writes
  constexpr int kPerRow = D / 2 / kEach;  // threads of half a row
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half) __syncthreads();
    if (qtile * kTile + r < prm.n_q)
#pragma unroll
      for (int n = 0; n < C::kDB / 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x16& from = o[half * (C::kDB / 2) + n];
          *reinterpret_cast<float4*>(sums + (wave * kTile + r) * C::kSumP + 32 * n + 8 * i + 4 * g) =
              make_float4(from[4 * i] * mine_by, from[4 * i + 1] * mine_by, from[4 * i + 2] * mine_by, from[4 * i + 3] * mine_by);
        }
    __syncthreads();
    const int row = threadIdx.x / kPerRow, q = qtile * kTile + row, at = threadIdx.x % kPerRow * kEach;  // (256 threads: 32 rows or more)
    if (row >= kTile || q >= prm.n_q) continue;
    float mq = kNegBig, lq = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mq = fmaxf(mq, ml[w * kTile + row].x);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) lq += ml[w * kTile + row].y * fast_exp2(ml[w * kTile + row].x - mq);
    float x[kEach];
#pragma unroll
    for (int e = 0; e < kEach; e += 4) {
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float4 z = *reinterpret_cast<const float4*>(sums + (w * kTile + row) * C::kSumP + at + e);
        y.x += z.x, y.y += z.y, y.z += z.z, y.w += z.w;
      }
      x[e] = y.x, x[e + 1] = y.y, x[e + 2] = y.z, x[e + 3] = y.w;
    }
    const int to_at = half * (D / 2) + at;
    if (units > 1) {
      const int64_t part = ((int64_t)unit * prm.qtiles + qtile) * prm.part_rows + row;
      float4* to = reinterpret_cast<float4*>(prm.part_o + part * D + to_at);
      to[0] = make_float4(x[0], x[1], x[2], x[3]);
      to[1] = make_float4(x[4], x[5], x[6], x[7]);
      if (to_at == 0) prm.part_ml[part] = make_float2(mq, lq);
      continue;
    }
    const float by = 1.f / lq;
    char* to = prm.O.group_row(b, h, prm.q_per_kv, prm.n_resp, q) + to_at * (int)sizeof(T);
    if constexpr (F32) {
      reinterpret_cast<float4*>(to)[0] = make_float4(x[0] * by, x[1] * by, x[2] * by, x[3] * by);
      reinterpret_cast<float4*>(to)[1] = make_float4(x[4] * by, x[5] * by, x[6] * by, x[7] * by);
    } else {
      *reinterpret_cast<u32x4*>(to) = u32x4{pack_bf16x2(x[0] * by, x[1] * by), pack_bf16x2(x[2] * by, x[3] * by),
                                            pack_bf16x2(x[4] * by, x[5] * by), pack_bf16x2(x[6] * by, x[7] * by)};
    }
    if (to_at == 0 && prm.lse) prm.lse[(int64_t)bh * prm.n_q + q] = (mq + __builtin_amdgcn_logf(lq)) * kLn2;
  }
}

// ---- up to 16 query rows of bf16 (single tokens, a few of a grouped head): eight waves on the 16-row form of the matrix instructions.
//
// The layout is that of the kernel above with quarters of a wave for halves: a lane's share of a key is a quarter of its row, at head_dim
// 128 one group with one scale, and a lane has 8 instead of 16 probabilities of a tile.  What a call of few queries takes is the reading
// of the cache and the time of one tile from its first load to its last product; half the registers leave room for twice the
// waves, so that most waves have one tile or two.  Against 32 query rows a workgroup: one token of 7 heads over 4 x 30k rows 11.4 and 12.5 us, of 32 heads
// x 1000 rows 8.2 and 10.5, 16 tokens 8.8 and 11.0; 16 heads x 5 queries x 60 rows 6.6 and 6.4.
template <int D>
struct FewCfg {
  static constexpr int kWaves = 8;
  static constexpr int kQueries = 16;
  static constexpr int kRowB = 2 * D;
  static constexpr int kPPR = kRowB / 16;
  static constexpr int kWords = D / 32;                // code words of a lane's quarter row
  static constexpr int kBlocks = D / 16;               // of 16 output rows
  static constexpr int kLoads = kTile * kPPR / 64;     // of 16 bytes a lane, of a tile's V
  static constexpr int kWaveB = kTile * kRowB;         // V
  static constexpr int kSumP = D + 4;
  static constexpr int kSumB = kQueries * kSumP * 4;
  static constexpr int kLds = kWaves * (kWaveB > kSumB ? kWaveB : kSumB) + kWaves * kQueries * 8;
};

typedef __attribute__((ext_vector_type(4))) float f32x4;
__device__ __forceinline__ void mfma16(const u32x4& a, const u32x4& b, f32x4& acc) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
// Over the quarters of a wave.
__device__ __forceinline__ float max_quarters(float v) {
  const auto x = __builtin_amdgcn_permlane16_swap(as_u32(v), as_u32(v), false, false);
  const uint32_t a = x[0], b = x[1];
  return max_halves(fmaxf(as_f32(a), as_f32(b)));
}
__device__ __forceinline__ float sum_quarters(float v) {
  const auto x = __builtin_amdgcn_permlane16_swap(as_u32(v), as_u32(v), false, false);
  const uint32_t a = x[0], b = x[1];
  return sum_halves(as_f32(a) + as_f32(b));
}

template <int D>
__global__ __launch_bounds__(512, 4) void attend_mx_few_kernel(const AttendMxParams prm) {
  using C = FewCfg<D>;
  constexpr int kWaves = C::kWaves;
  extern __shared__ __attribute__((aligned(1024))) char mx_lds[];
  fetch_attend_mx_arguments();
  const int unit = blockIdx.x;
  const int resp_tiles = (prm.n_resp + kTile - 1) / kTile;
  auto tiles_of = [&](int rows) { return (int)(((uint32_t)rows + kTile - 1) / kTile) + resp_tiles; };  // those of the response first
  const int capacity = (int)prm.capacity;
  UnitHead head;
  if (prm.chunk) {
    head = head_of_unit(prm.cu, prm.BH, capacity, unit, [&](int rows) { return (tiles_of(rows) + prm.chunk - 1) / prm.chunk; });
    if (head.bh < 0) return;
  } else {
    const int first = min(prm.cu[unit], capacity);
    head = {unit, unit, 1, first, max(min(prm.cu[unit + 1], capacity) - first, 0)};
  }
  const int bh = head.bh, units = head.units, cached = head.rows, tiles = tiles_of(cached);
  const int b = bh / prm.H, h = bh % prm.H;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  if (prm.chunk && unit == head.first_unit && threadIdx.x == 0) prm.parts[bh] = make_int2(head.first_unit, units);
  const int t0 = prm.chunk ? (unit - head.first_unit) * prm.chunk : 0;
  const int t1 = prm.chunk ? min(tiles, t0 + prm.chunk) : tiles;
  char* const v_lds = mx_lds + wave * C::kWaveB;
  const uint32_t v_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)v_lds;

  typedef __attribute__((ext_vector_type(C::kWords))) uint32_t Codes;
  struct Cached {  // of keys r and 16 + r of a tile
    Codes k[2], v[2];
    uint32_t ks[2], vs[2];
  } ahead;
  // (A tile's first row is the same in all lanes: their offsets from it are all that is formed for each.)
  auto load_cached = [&](int t, Cached& x) __attribute__((always_inline)) {
    const int64_t base = (int64_t)head.first + t * kTile;
    const int last = cached - t * kTile - 1;  // (rows behind the last one are the last one)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t row = min(16 * u + r, last);
      const uint32_t at = row * (D / 2) + g * (D / 8), scale = row * (D / 32) + g * (D / 32) / 4;
      x.k[u] = *reinterpret_cast<const Codes*>(prm.cache.k_codes + base * (D / 2) + at);
      x.v[u] = *reinterpret_cast<const Codes*>(prm.cache.v_codes + base * (D / 2) + at);
      x.ks[u] = *reinterpret_cast<const uint8_t*>(prm.cache.k_scales + base * (D / 32) + scale);
      x.vs[u] = *reinterpret_cast<const uint8_t*>(prm.cache.v_scales + base * (D / 32) + scale);
    }
  };
  // This wave's tiles: t0 + wave, and every eighth from there; those of the response are the first `resp` of them.
  const int mine = max(t1 - t0 - wave + kWaves - 1, 0) / kWaves;
  const int resp = min(max(min(resp_tiles, t1) - t0 - wave + kWaves - 1, 0) / kWaves, mine);
  auto tile_of = [&](int i) { return t0 + wave + i * kWaves; };
  u32x4 qf[C::kWords];
  {
    const char* q = prm.Q.group_row(b, h, prm.q_per_kv, prm.n_resp, min(r, prm.n_q - 1)) + g * (C::kRowB / 4);
#pragma unroll
    for (int i = 0; i < C::kWords; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + 16 * i);
  }
  f32x4 o[C::kBlocks], s[2];
#pragma unroll
  for (int i = 0; i < C::kBlocks; ++i) o[i] = f32x4{};
  float m = kNegBig, l = 0.f;

  // Rows 4g .. 4g+3 and 16 on of V: lane i of 16 points at 8 bytes of row i / 4 of them and receives column i of a block.
  const uint32_t read_row = 4 * g + (r >> 2);
  const uint32_t read_at = v_at + read_row * C::kRowB + (v_swizzle<D>(read_row) << 5) + (r & 3) * 8;
  const uint32_t write_at = v_at + r * C::kRowB + ((g * C::kWords ^ v_swizzle<D>(r) << 1) << 4);

  // Softmax of a tile with `left` rows, and the output update.  Lanes with the same r have the same query.
  auto update = [&](int left) __attribute__((always_inline)) {
    if (left < kTile) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * u + i >= left - 4 * g) s[u][i] = -INFINITY;
    }
    float bm = s[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) bm = fmaxf(bm, s[i / 4][i % 4]);
    const float cand = max_quarters(bm) * prm.c;
    const bool bump = cand > m + kLazyBump;  // (see attend.hip)
    if (__any(bump)) {
      const float m_new = bump ? cand : m;
      const float alpha = fast_exp2(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int n = 0; n < C::kBlocks; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] *= alpha;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = fast_exp2(fmaf(s[i / 4][i % 4], prm.c, -m));
      l += p[i];
    }
    const u32x4 pf = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
    uint32_t from = read_at;
    asm volatile("" : "+v"(from));  // (an address for each block would be kept in a register of its own)
#pragma unroll
    for (int n = 0; n < C::kBlocks; ++n) {
      const u32x2 lo = read_transposed(from ^ n << 5, 0), hi = read_transposed(from ^ n << 5, 16 * C::kRowB);
      mfma16(u32x4{lo[0], lo[1], hi[0], hi[1]}, pf, o[n]);
    }
  };

  for (int i = 0; i < resp; ++i) {
    const int t = tile_of(i);
    u32x4 v[C::kLoads];
#pragma unroll
    for (int j = 0; j < C::kLoads; ++j) {
      const int row = j * (64 / C::kPPR) + lane / C::kPPR;
      v[j] = *reinterpret_cast<const u32x4*>(prm.V2.row(b, h, min(t * kTile + row, prm.n_resp - 1)) + lane % C::kPPR * 16);
    }
#pragma unroll
    for (int j = 0; j < C::kLoads; ++j) {
      const uint32_t row = j * (64 / C::kPPR) + lane / C::kPPR, p = lane % C::kPPR;
      *reinterpret_cast<u32x4*>(v_lds + row * C::kRowB + ((p ^ v_swizzle<D>(row) << 1) << 4)) = v[j];
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const char* k = prm.K2.row(b, h, min(t * kTile + 16 * u + r, prm.n_resp - 1)) + g * (C::kRowB / 4);
      s[u] = f32x4{};
#pragma unroll
      for (int w = 0; w < C::kWords; ++w) mfma16(*reinterpret_cast<const u32x4*>(k + 16 * w), qf[w], s[u]);
    }
    asm volatile("" ::: "memory");
    update(prm.n_resp - t * kTile);
    asm volatile("" ::: "memory");
  }
  auto take = [&](int i, Cached& x) __attribute__((always_inline)) {
    const int t = tile_of(i) - resp_tiles;
    uint32_t to = write_at;
    asm volatile("" : "+v"(to));
#pragma unroll
    for (int w = 0; w < C::kWords; ++w)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        *in_lds<u32x4>(to ^ w << 4, 16 * u * C::kRowB) = mx_decode_bf16(x.v[u][w], mx_unit(x.vs[u]));
    s[0] = s[1] = f32x4{};
#pragma unroll
    for (int w = 0; w < C::kWords; ++w) {
#pragma unroll
      for (int u = 0; u < 2; ++u) mfma16(mx_decode_bf16(x.k[u][w], mx_unit(x.ks[u])), qf[w], s[u]);
      if (w % 2) __builtin_amdgcn_sched_barrier(0);  // (all words converted before the first product: 35 registers more than there are)
    }
    if (i + 1 < mine) load_cached(t + kWaves, x);
    asm volatile("" ::: "memory");
    update(cached - t * kTile);
    asm volatile("" ::: "memory");
  };
  // (The response is one tile of one wave of a head: what is asked for ahead of it would take the registers of all.)
  if (mine > resp) load_cached(tile_of(resp) - resp_tiles, ahead);
  for (int i = resp; i < mine; ++i) take(i, ahead);

  // ---- the waves' results become one
  l = sum_quarters(l);
  float2* const ml = reinterpret_cast<float2*>(mx_lds + C::kLds - kWaves * C::kQueries * 8);
  if (g == 0) ml[wave * C::kQueries + r] = make_float2(m, l);
  __syncthreads();
  float top = kNegBig;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w * C::kQueries + r].x);
  const float mine_by = fast_exp2(m - top);
  float* const sums = reinterpret_cast<float*>(mx_lds);
  if (r < prm.n_q)
#pragma unroll
    for (int n = 0; n < C::kBlocks; ++n)
      *reinterpret_cast<float4*>(sums + (wave * C::kQueries + r) * C::kSumP + 16 * n + 4 * g) =
          make_float4(o[n][0] * mine_by, o[n][1] * mine_by, o[n][2] * mine_by, o[n][3] * mine_by);
  __syncthreads();
  constexpr int kPerRow = D / 4;
  const int q = threadIdx.x / kPerRow, at = threadIdx.x % kPerRow * 4;  // (512 threads: 16 rows at head_dim 128)
  if (q >= prm.n_q) return;
  float mq = kNegBig, lq = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) mq = fmaxf(mq, ml[w * C::kQueries + q].x);
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    lq += ml[w * C::kQueries + q].y * fast_exp2(ml[w * C::kQueries + q].x - mq);
    const float4 z = *reinterpret_cast<const float4*>(sums + (w * C::kQueries + q) * C::kSumP + at);
    x = make_float4(x.x + z.x, x.y + z.y, x.z + z.z, x.w + z.w);
  }
  if (units > 1) {
    const int64_t part = (int64_t)unit * prm.part_rows + q;
    *reinterpret_cast<float4*>(prm.part_o + part * D + at) = x;
    if (at == 0) prm.part_ml[part] = make_float2(mq, lq);
    return;
  }
  const float by = 1.f / lq;
  *reinterpret_cast<u32x2*>(prm.O.group_row(b, h, prm.q_per_kv, prm.n_resp, q) + at * 2) =
      u32x2{pack_bf16x2(x.x * by, x.y * by), pack_bf16x2(x.z * by, x.w * by)};
  if (at == 0 && prm.lse) prm.lse[(int64_t)bh * prm.n_q + q] = (mq + __builtin_amdgcn_logf(lq)) * kLn2;
}

// ---- many query rows of bf16: a workgroup of four waves serves 128 of a head, 32 a wave, over tiles of 64 keys that all of them read
// from LDS as bf16.  Two workgroups share a compute unit, so that one's softmax runs beside the other's products, and within a
// wave the logits of the next tile are formed beside the softmax of this one.
//
// Iteration t reads K(t+1) and V(t), and brings K(t+2) and V(t+1) into the other two of four buffers, which iteration t-1 has
// read: one barrier an iteration.  Tiles of the cache come through registers, read an iteration ahead and converted on their way
// into LDS; those of the response by direct transfers.
constexpr int kWideTile = 64;
constexpr int kWideQueries = 128;

template <int D>
struct WideCfg {
  static constexpr int kRowB = 2 * D;
  static constexpr int kPPR = kRowB / 16;
  static constexpr int kSteps = D / 16;
  static constexpr int kDB = D / 32;
  static constexpr int kTileB = kWideTile * kRowB;
  static constexpr int kLds = 4 * kTileB;                  // K(t), K(t+1), V(t), V(t+1)
  static constexpr int kMoves = kWideTile * kRowB / 4096;  // direct transfers of 1 KiB a wave and tile
  static constexpr int kMoveRows = 1024 / kRowB;
  static constexpr int kWords = D / 32;                    // code words of a thread: a quarter of a row
  __device__ static uint32_t swz_k(uint32_t row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
};

// The head of a given rank by descending number of tiles, equal ones by ascending number: the lanes of a wave hold all heads'
// ends, which are asked for at once; a bit of the wanted count of tiles takes a ballot per 64 heads.
constexpr int kRanked = 256;  // heads up to which their order is found so
template <typename F>
__device__ __forceinline__ UnitHead head_of_rank(const int32_t* cu, int BH, int capacity, int rank, F tiles_of) {
  constexpr int N = kRanked / 64;
  const int lane = threadIdx.x & 63;
  int from[N], to[N], tiles[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int bh = min(i * 64 + lane, BH - 1);
    from[i] = cu[bh];
    to[i] = cu[bh + 1];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(from[i]), "+v"(to[i]));
#pragma unroll
  for (int i = 0; i < N; ++i) {
    from[i] = min(from[i], capacity);
    to[i] = max(min(to[i], capacity) - from[i], 0);  // (rows)
    tiles[i] = i * 64 + lane < BH ? min(tiles_of(to[i]), 0xFFFF) : 0;
  }
  int found = 0, above = 0;  // the count, and how many heads have more tiles
  for (int bit = 1 << 15; bit > 0; bit >>= 1) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __popcll(__ballot(tiles[i] >= (found | bit)));
    if (n > rank)
      found |= bit;
    else
      above = n;
  }
  int left = rank - above;
  UnitHead x = {0, rank, 1, 0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint64_t same = __ballot(tiles[i] == found);
    const int n = __popcll(same);
    if (left >= 0 && left < n) {
      const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
      const int at = __builtin_ctzll(__ballot(tiles[i] == found && before == left));
      x.bh = i * 64 + at;
      x.first = __builtin_amdgcn_readlane(from[i], at);
      x.rows = __builtin_amdgcn_readlane(to[i], at);
    }
    left -= n;
  }
  x.bh = __builtin_amdgcn_readfirstlane(x.bh);
  x.first = __builtin_amdgcn_readfirstlane(x.first);
  x.rows = __builtin_amdgcn_readfirstlane(x.rows);
  return x;
}

// What a unit is: tiles t0 .. t1 - 1 of a head, and the place of its partial result where the head has several units.  Three ways:
//   no chunk         a unit is a head, by rank up to kRanked of them;
//   chunk            units of so many tiles, head after head, a place each;
//   chunk, extras    (up to kRanked heads) units of what is left of the heads behind their first `chunk` tiles, which take longest, head after
//                    head, as many as there are; then each head's first tiles, which is all of most, by rank.  Places: `extras` for the
//                    former, then one for the first tiles of each head that is cut.  (The units that there may be, but are not, come last: in front
//                    of 1024 workgroups 124 of them cost 5 us, as the heads' order then is not that of the compute units.)
// False: a unit behind the last one.
struct Work {
  UnitHead head;
  int t0, t1, place;
};
__device__ __forceinline__ int units_of_tiles(int tiles, int chunk) { return (tiles + chunk - 1) / chunk; }
template <typename F>
__device__ __forceinline__ bool work_of(const AttendMxParams& prm, int unit, int qtile, F tiles_of, Work& w) {
  const int capacity = (int)prm.capacity;
  int part = 0;
  w.place = unit;
  if (prm.chunk && !prm.extras) {
    w.head = head_of_unit(prm.cu, prm.BH, capacity, unit, [&](int rows) { return units_of_tiles(tiles_of(rows), prm.chunk); });
    if (w.head.bh < 0) return false;
    part = unit - w.head.first_unit;
    if (part == 0 && qtile == 0 && threadIdx.x == 0) prm.parts[w.head.bh] = make_int2(unit, w.head.units);
  } else {
    int others = 0;  // units of what is left
    if (prm.extras) {
      w.head = head_of_unit(prm.cu, prm.BH, capacity, unit, [&](int rows) { return units_of_tiles(tiles_of(rows), prm.chunk) - 1; });
      others = w.head.first_unit;
      part = unit - others + 1;
      w.head.units += 1;
    }
    if (!prm.extras || w.head.bh < 0) {
      part = 0;
      const int i = unit - others;
      if (i >= prm.BH) return false;
      if (prm.BH <= kRanked) {
        w.head = head_of_rank(prm.cu, prm.BH, capacity, i, tiles_of);
      } else {
        const int first = min(prm.cu[i], capacity);
        w.head = {i, i, 1, first, max(min(prm.cu[i + 1], capacity) - first, 0)};
      }
      if (prm.extras && tiles_of(w.head.rows) > prm.chunk) {
        w.head.units = units_of_tiles(tiles_of(w.head.rows), prm.chunk);
        w.place = prm.extras + sum_before(prm.cu, w.head.bh, capacity, [&](int rows) { return tiles_of(rows) > prm.chunk ? 1 : 0; });
      }
    }
  }
  const int tiles = tiles_of(w.head.rows);
  w.t0 = part * prm.chunk;
  w.t1 = prm.chunk ? min(tiles, w.t0 + prm.chunk) : tiles;
  return true;
}

template <int D>
__global__ __launch_bounds__(256, 2) void attend_mx_wide_kernel(const AttendMxParams prm) {
  using C = WideCfg<D>;
  extern __shared__ __attribute__((aligned(1024))) char mx_lds[];
  fetch_attend_mx_arguments();
  const Place place = place_of(blockIdx.x, prm.units, prm.qtiles);
  const int unit = place.unit, qtile = place.qtile;
  const int resp_tiles = (prm.n_resp + kWideTile - 1) / kWideTile;
  auto tiles_of = [&](int rows) { return (int)(((uint32_t)rows + kWideTile - 1) / kWideTile) + resp_tiles; };  // those of the response first
  Work work;
  if (!work_of(prm, unit, qtile, tiles_of, work)) return;
  const UnitHead& head = work.head;
  const int bh = head.bh, first = head.first, cached = head.rows, t0 = work.t0, tiles = work.t1;  // this workgroup's: t0 .. tiles - 1
  const int b = bh / prm.H, h = bh % prm.H;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, g = lane >> 5;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mx_lds;

  // ---- tiles on their way.  Of the cache a thread takes a quarter of a row; of the response a wave takes a quarter of the rows.
  const int my_row = threadIdx.x >> 2, quarter = threadIdx.x & 3;
  const char* const codes_k = prm.cache.k_codes + (int64_t)first * (D / 2);
  const char* const codes_v = prm.cache.v_codes + (int64_t)first * (D / 2);
  const char* const scales_k = prm.cache.k_scales + (int64_t)first * (D / 32);
  const char* const scales_v = prm.cache.v_scales + (int64_t)first * (D / 32);
  uint32_t kc[C::kWords], vc[C::kWords], ks = 0, vs = 0;
  // (An LDS write of 16 bytes a lane takes eight lanes at a time, here two rows: the words of a thread are read, and written, in another order
  // in every other row, or half of a row, so that the eight fall on different banks.)
  const uint32_t turn_k = D == 128 ? quarter & 2 : my_row & 1, turn_v = (D == 128 ? quarter & 2 : 0) ^ (my_row & 1);
  auto read = [&](int t, const char* codes, const char* scales, uint32_t turn, uint32_t (&c)[C::kWords], uint32_t& s) {
    const int base = (t - resp_tiles) * kWideTile;
    if (base < 0 || base >= cached) return;
    const uint32_t row = min(my_row, cached - base - 1);
    const char* from = codes + (int64_t)base * (D / 2);
#pragma unroll
    for (int w = 0; w < C::kWords; ++w) c[w] = *reinterpret_cast<const uint32_t*>(from + (row * (D / 2) + quarter * (D / 8) + 4 * (w ^ turn)));
    s = *reinterpret_cast<const uint8_t*>(scales + (int64_t)base * (D / 32) + (row * (D / 32) + quarter * (D / 32) / 4));
  };
  const char* const resp_k = prm.K2.row(b, h, 0);
  const char* const resp_v = prm.V2.row(b, h, 0);
  const uint32_t moved = wave * (kWideTile / 4) + (uint32_t)lane / C::kPPR;  // this lane's row of the wave's first transfer
  const uint32_t piece_k = ((uint32_t)lane % C::kPPR ^ C::swz_k(moved)) << 4, piece_v = ((uint32_t)lane % C::kPPR ^ v_swizzle<D>(moved) << 1) << 4;
  auto transfer = [&](int t, const char* from, int64_t stride, uint32_t piece, uint32_t step, uint32_t to) {
    const int left = prm.n_resp - t * kWideTile;
    from += (int64_t)t * kWideTile * stride;
#pragma unroll
    for (int j = 0; j < C::kMoves; ++j) {  // (a row's permutation changes from a transfer to the next by an exclusive-or of its own)
      const uint32_t row = min((int)moved + j * C::kMoveRows, left - 1);
      dma16(from, row * (uint32_t)stride + (piece ^ (j * step & (C::kRowB - 1))), to + (wave * C::kMoves + j) * 1024);
    }
  };
  // where this thread's quarter of a row goes, as the byte to which a word's number is added by an exclusive-or
  const uint32_t to_k = my_row * C::kRowB + ((quarter * C::kWords ^ C::swz_k(my_row) ^ turn_k) << 4);
  const uint32_t to_v = my_row * C::kRowB + ((quarter * C::kWords ^ v_swizzle<D>(my_row) << 1 ^ turn_v) << 4);
  auto convert = [&](const uint32_t (&c)[C::kWords], uint32_t s, uint32_t to) {
    const float unit = mx_unit(s);
#pragma unroll
    for (int w = 0; w < C::kWords; ++w) *in_lds<u32x4>(lds0 + (to ^ w << 4)) = mx_decode_bf16(c[w], unit);
  };
  // K(t), V(t) into the buffer of an even or odd tile (counted from the first one of this workgroup)
  auto bring_k = [&](int t, uint32_t odd) {
    if (t >= tiles) return;
    if (t < resp_tiles)
      transfer(t, resp_k, prm.K2.stride_t, piece_k, C::swz_k(C::kMoveRows) << 4, lds0 + odd * C::kTileB);
    else
      convert(kc, ks, to_k + odd * C::kTileB);
  };
  auto bring_v = [&](int t, uint32_t odd) {
    if (t >= tiles) return;
    if (t < resp_tiles)
      transfer(t, resp_v, prm.V2.stride_t, piece_v, 0, lds0 + (2 + odd) * C::kTileB);
    else
      convert(vc, vs, to_v + (2 + odd) * C::kTileB);
  };
  auto read_k = [&](int t) { read(t, codes_k, scales_k, turn_k, kc, ks); };
  auto read_v = [&](int t) { read(t, codes_v, scales_v, turn_v, vc, vs); };
  auto arrive = [] {  // what this wave has moved and written is there, and so is everyone's behind the barrier
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  read_k(t0);
  read_v(t0);
  const int q0 = qtile * kWideQueries + wave * 32;
  u32x4 qf[C::kSteps];
  {
    const char* q = prm.Q.group_row(b, h, prm.q_per_kv, prm.n_resp, min(q0 + r, prm.n_q - 1)) + g * D;
#pragma unroll
    for (int i = 0; i < C::kSteps; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + 16 * i);
  }
  bring_k(t0, 0);
  read_k(t0 + 1);
  bring_v(t0, 0);
  read_v(t0 + 1);
  bring_k(t0 + 1, 1);
  read_k(t0 + 2);
  arrive();

  f32x16 o[C::kDB], even[2], odd[2];
#pragma unroll
  for (int db = 0; db < C::kDB; ++db) o[db] = f32x16{};
  float m = kNegBig, l = 0.f, top = 0.f;  // top: the largest logit of the tile whose turn comes next
  const float c = prm.c;
  uint32_t k_at[C::kSteps], v_at[C::kDB];
#pragma unroll
  for (int i = 0; i < C::kSteps; ++i) k_at[i] = lds0 + r * C::kRowB + (((C::kPPR / 2 * g + i) ^ C::swz_k(r)) << 4);
#pragma unroll
  for (int db = 0; db < C::kDB; ++db) v_at[db] = lds0 + 2 * C::kTileB + v_read_offset<D>(lane, db);
  // Fragment n of a tile: 0 .. kQK-1 of its keys (two chains of products, one for 32 keys each), from kQK on of the values of the tile before.
  constexpr int kQK = 2 * C::kSteps, kPV = 4 * C::kDB, kAhead = 2;
  u32x4 fr[kAhead + 1];
  auto fetch = [&](int n, uint32_t odd_k) {
    u32x4& f = fr[n % (kAhead + 1)];
    if (n < kQK) {
      f = *in_lds<const u32x4>(k_at[n / 2], odd_k * C::kTileB + n % 2 * 32 * C::kRowB);
    } else {
      const int i = n - kQK, imm = (1 - odd_k) * C::kTileB + i / C::kDB * 16 * C::kRowB;
      const u32x2 lo = read_transposed(v_at[i % C::kDB], imm), hi = read_transposed(v_at[i % C::kDB], imm + 8 * C::kRowB);
      f = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  };
  auto mask = [&](int t, f32x16 (&s)[2]) {  // keys behind the last one of the response, or of the cache
    const int left = t < resp_tiles ? prm.n_resp - t * kWideTile : cached - (t - resp_tiles) * kWideTile;
    if (left >= kWideTile) return;
    const int mine = left - 4 * g;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (kb * 32 + 8 * (i / 4) + i % 4 >= mine) s[kb][i] = -INFINITY;
  };
#pragma unroll
  for (int n = 0; n < kQK; ++n) {
    fetch(n, 0);
    if (n < 2) even[n] = f32x16{};
    mfma_step<bf16_t>(fr[n % (kAhead + 1)], qf[n / 2], even[n % 2]);
  }
  mask(t0, even);
  top = even[0][0];
#pragma unroll
  for (int i = 0; i < 32; ++i) top = fmaxf(top, even[i / 16][i % 16]);
  arrive();  // (K(2) takes the place of K(0))

  // Tile t (odd or not) with its logits in `s`; with MORE those of the next into `next`.  The next tile's logits are formed beside
  // this one's exponentials, this one's part of the output beside the search for the next one's largest logit.
  auto step = [&](int t, auto odd_tile, auto more, f32x16 (&s)[2], f32x16 (&next)[2]) {
    constexpr uint32_t kOdd = decltype(odd_tile)::value;
    constexpr bool kMore = decltype(more)::value;
    constexpr int kFrom = kMore ? 0 : kQK;
    if constexpr (kMore) {
      bring_k(t + 2, kOdd);
      bring_v(t + 1, 1 - kOdd);
      read_k(t + 3);
      read_v(t + 2);
    }
    const float cand = max_halves(top) * c;
    const bool bump = cand > m + kLazyBump;  // (see attend.hip)
    if (__any(bump)) {
      const float m_new = bump ? cand : m;
      const float alpha = fast_exp2(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < C::kDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    }
    u32x4 pf[4];
    auto probabilities = [&](int i) {  // values i and i + 1 of the 32
      const float p0 = fast_exp2(fmaf(s[i / 16][i % 16], c, -m)), p1 = fast_exp2(fmaf(s[i / 16][i % 16 + 1], c, -m));
      l += p0 + p1;
      uint32_t both = pack_bf16x2(p0, p1);
      asm volatile("" : "+v"(both), "+v"(l));  // (formed here, beside the products, and not where it is first needed)
      pf[i / 8][i % 8 / 2] = both;
    };
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < kAhead; ++n) fetch(kFrom + n, 1 - kOdd);
    if constexpr (kMore) {
#pragma unroll
      for (int n = 0; n < kQK; ++n) {
        fetch(n + kAhead, 1 - kOdd);
        if (n < 2) next[n] = f32x16{};
        mfma_step<bf16_t>(fr[n % (kAhead + 1)], qf[n / 2], next[n % 2]);
#pragma unroll
        for (int i = n * 32 / kQK; i < (n + 1) * 32 / kQK; i += 2) probabilities(i);
        __builtin_amdgcn_sched_barrier(0);
      }
      mask(t + 1, next);
    } else {
#pragma unroll
      for (int i = 0; i < 32; i += 2) probabilities(i);
    }
    float high = -INFINITY;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = kQK; n < kQK + kPV; ++n) {
      if (n + kAhead < kQK + kPV) fetch(n + kAhead, 1 - kOdd);
      mfma_step<bf16_t>(fr[n % (kAhead + 1)], pf[(n - kQK) / C::kDB], o[(n - kQK) % C::kDB]);
      if constexpr (kMore) {
#pragma unroll
        for (int i = (n - kQK) * 32 / kPV; i < (n + 1 - kQK) * 32 / kPV; ++i) high = fmaxf(high, next[i / 16][i % 16]);
        asm volatile("" : "+v"(high));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    top = high;
    arrive();
  };
  using Yes = std::true_type;
  using No = std::false_type;
  int t = t0;
  for (; t + 2 < tiles; t += 2) {
    step(t, No(), Yes(), even, odd);
    step(t + 1, Yes(), Yes(), odd, even);
  }
  if (t + 1 < tiles) {
    step(t, No(), Yes(), even, odd);
    step(t + 1, Yes(), No(), odd, even);
  } else {
    step(t, No(), No(), even, odd);
  }

  // ---- out, by way of LDS: whole rows
  l = sum_halves(l);
  if (head.units > 1) {
    if (q0 + r >= prm.n_q) return;
    const int64_t part = ((int64_t)work.place * prm.qtiles + qtile) * prm.part_rows + wave * 32 + r;
#pragma unroll
    for (int db = 0; db < C::kDB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(prm.part_o + part * D + 32 * db + 8 * i + 4 * g) =
            make_float4(o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]);
    if (g == 0) prm.part_ml[part] = make_float2(m, l);
    return;
  }
  const float by = 1.f / l;
  char* own = mx_lds + wave * 32 * (C::kRowB + 16);
#pragma unroll
  for (int db = 0; db < C::kDB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(own + r * (C::kRowB + 16) + (32 * db + 8 * i + 4 * g) * 2) =
          u32x2{pack_bf16x2(o[db][4 * i] * by, o[db][4 * i + 1] * by), pack_bf16x2(o[db][4 * i + 2] * by, o[db][4 * i + 3] * by)};
  asm volatile("" ::: "memory");
#pragma unroll
  for (int j = 0; j < 32 * C::kPPR / 64; ++j) {
    const int row = (j * 64 + lane) / C::kPPR, p = lane % C::kPPR;
    if (q0 + row < prm.n_q)
      *reinterpret_cast<u32x4*>(prm.O.group_row(b, h, prm.q_per_kv, prm.n_resp, q0 + row) + p * 16) =
          *reinterpret_cast<const u32x4*>(own + row * (C::kRowB + 16) + p * 16);
  }
  if (prm.lse && g == 0 && q0 + r < prm.n_q) prm.lse[(int64_t)bh * prm.n_q + q0 + r] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// The partial results of the heads that have several units: sums in units of the largest reference.  D/4 threads take a query row and
// ask for kAtOnce of its partial results before they use the first; where a head has many, the eight groups of a workgroup share one
// row (SHARED) and meet in LDS, else each has a row of its own.
constexpr int kJoinGroups = 8;
template <typename T, int D, bool SHARED>
__global__ __launch_bounds__(kJoinGroups * D / 4) void attend_mx_join_kernel(const AttendMxParams prm) {
  constexpr int kPer = D / 4, kAtOnce = 8, kStep = SHARED ? kJoinGroups : 1;
  __shared__ float4 sums[kJoinGroups][kPer];
  __shared__ float2 tops[kJoinGroups];
  fetch_attend_mx_arguments();
  const int grp = threadIdx.x / kPer, at = threadIdx.x % kPer;
  const int64_t step = (int64_t)prm.qtiles * prm.part_rows;
  const int q = SHARED ? blockIdx.x : blockIdx.x * kJoinGroups + grp;
  int bh = blockIdx.y, units, first, first_place;  // places of a head's units: first_place, first + 1, first + 2, ...
  if (SHARED || !prm.extras) {
    first_place = first = prm.parts[bh].x;
    units = prm.parts[bh].y;
  } else {  // the head of that number among the ones that are cut
    const int capacity = (int)prm.capacity, resp_tiles = (prm.n_resp + kWideTile - 1) / kWideTile;
    auto units_of = [&](int rows) { return units_of_tiles((int)(((uint32_t)rows + kWideTile - 1) / kWideTile) + resp_tiles, prm.chunk); };
    const UnitHead head = head_of_unit(prm.cu, prm.BH, capacity, bh, [&](int rows) { return units_of(rows) > 1 ? 1 : 0; });
    if (head.bh < 0) return;
    first_place = prm.extras + bh;
    bh = head.bh;
    units = units_of(head.rows);
    first = sum_before(prm.cu, bh, capacity, [&](int rows) { return units_of(rows) - 1; }) - 1;
  }
  if (units <= 1 || q >= prm.n_q) return;
  const int64_t in_unit = (int64_t)(q / prm.tile_rows) * prm.part_rows + q % prm.tile_rows;
  float m = kNegBig, l = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int u0 = SHARED ? grp : 0; u0 < units; u0 += kAtOnce * kStep) {
    float2 ml[kAtOnce];
    float4 y[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      ml[i] = make_float2(kNegBig, 0.f);
      y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (u0 + i * kStep < units) {
        const int u = u0 + i * kStep;
        const int64_t part = (u ? first + u : first_place) * step + in_unit;
        ml[i] = prm.part_ml[part];
        y[i] = *reinterpret_cast<const float4*>(prm.part_o + part * D + at * 4);
      }
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, ml[i].x);
    const float old = fast_exp2(m - top);
    m = top;
    l *= old;
    x = make_float4(x.x * old, x.y * old, x.z * old, x.w * old);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float by = fast_exp2(ml[i].x - m);
      l = fmaf(ml[i].y, by, l);
      x = make_float4(fmaf(y[i].x, by, x.x), fmaf(y[i].y, by, x.y), fmaf(y[i].z, by, x.z), fmaf(y[i].w, by, x.w));
    }
  }
  if constexpr (SHARED) {
    sums[grp][at] = x;
    if (at == 0) tops[grp] = make_float2(m, l);
    __syncthreads();
    if (grp > 0) return;
    m = kNegBig;
#pragma unroll
    for (int i = 0; i < kJoinGroups; ++i) m = fmaxf(m, tops[i].x);
    l = 0.f;
    x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kJoinGroups; ++i) {
      const float by = fast_exp2(tops[i].x - m);
      const float4 y = sums[i][at];
      l = fmaf(tops[i].y, by, l);
      x = make_float4(fmaf(y.x, by, x.x), fmaf(y.y, by, x.y), fmaf(y.z, by, x.z), fmaf(y.w, by, x.w));
    }
  }
  const float by = 1.f / l;
  char* to = prm.O.group_row(bh / prm.H, bh % prm.H, prm.q_per_kv, prm.n_resp, q) + at * 4 * (int)sizeof(T);
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<float4*>(to) = make_float4(x.x * by, x.y * by, x.z * by, x.w * by);
  else
    *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(x.x * by, x.y * by), pack_bf16x2(x.z * by, x.w * by)};
  if (at == 0 && prm.lse) prm.lse[(int64_t)bh * prm.n_q + q] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// How the tiles are dealt out.
struct Deal {
  bool few;       // up to 16 query rows
  bool wide;      // 128 query rows a workgroup
  int tile_rows, qtiles, part_rows;
  int chunk;      // tiles of a unit, or 0: a unit per head
  int extras;     // (see Work) or 0
  int cut;        // heads of more than `chunk` tiles, at most, where there are extras
  int64_t units;  // at most
  int64_t places() const { return extras ? extras + cut : units; }  // of partial results
};
// Units of a head on average above which a query row's partial results are read by a whole workgroup instead of an eighth of one: 59 units 11.4 and
// 16.1 us a call, 32 11.4 and 12.6; 8 units 15.0 and 14.1.
constexpr int kSharedUnits = 16;

// What a launch of each kernel takes, in us: fitted to 170 launches of bf16 and 50 of fp32 over 4 ... 256 heads, 4 ... 3700 query rows and
// 3 ... 8500 cached rows a head (longest to shortest up to 8), each timed with whole heads and with units for 128 ... 1024 workgroups, in every
// form that takes it; off by 12 % (root of the mean square). Over 400 other launches the form and units that it chooses took 1.03 times
// as long as the best that were timed (bf16 1.024, fp32 1.030, up to 16 query rows 1.015), 1.11 times with fixed limits on the numbers of heads
// and tiles. The worst, 1.3 ... 1.7 (fp32 2.0), are heads of very different lengths left whole: the host does not know their lengths.
// Both sides: 64 heads x 354 queries x 250 rows 22.8 whole and wide, 25.1 narrow, 28.1 ... 35.9 dealt out; 32 x 512 x 250 19.8 narrow, 24.2 wide; 8 x 400 x
// 5582 38.8 whole, 31.0 dealt out; 28 heads x 27 queries x 1106 rows 16.6 whole, 12.6 dealt out; 28 heads (head_dim 64) of 455 ... 6037 rows, 115
// queries: 27 whole, 14 dealt out.
struct Form {
  int tile_rows, keys;  // query rows of a workgroup, keys of a tile
  int tiles;            // that its waves take in one step
  int least;            // tiles of a unit
  int at_once;          // workgroups of a compute unit
  float start, round;   // the launch, the first loads and the last stores; the same of each round of workgroups
  float fixed, per_d;   // a step: fixed + per_d * d / 128
  float beside;         // ... of a workgroup that shares its compute unit: so many times that, for each
  float part;           // a million bytes of partial results, written and read
  float uneven;         // kUneven where no compute unit has a second workgroup that would fill the wait for the longest head
};
constexpr Form kFew = {16, kTile, 8, 16, 2, 4.5f, 1.3f, 0.f, 1.2f, 1.f, 0.8f, 1.15f};
constexpr Form kNarrow = {kTile, kTile, kWaves, 8, 2, 5.2f, 1.3f, 0.f, 0.75f, 1.13f, 0.8f, 1.5f};
constexpr Form kWide = {kWideQueries, kWideTile, 1, 2, 2, 7.f, 0.f, 0.4f, 0.9f, 0.8f, 0.5f, 1.15f};
constexpr Form kNarrowF32 = {kTile, kTile, kWaves, 4, 1, 2.f, 3.f, 0.f, 5.5f, 1.f, 0.8f, 1.15f};
constexpr float kJoin = 4.3f;      // the second kernel
constexpr float kUneven = 1.15f;   // a launch of whole heads waits for the longest ones: by so much on average (1 ... 1.3 choose about as well)
// Whole heads: what one may take that has all the rows of the longest prompt.  Beyond, the keys are dealt out, though most heads may be short; in the kernel of 128
// rows only heads are cut that take longer than the launch is expected to.  Both sides, 8 x 32 heads x 512 queries: 64 ... 1024 rows of each, whole
// 77.5 us, to be cut 82.2 (a second launch, which finds nothing to join), dealt out 96.9; with 18000 rows in one of them 367, 110 and 109 ... 114.
constexpr float kLongest = 400.f;

// Capacities are planned for in steps of a sixteenth of the power of two below (up to 6 % more rows than there are; the units past the last
// head end at once): so few different plans can be looked over for the workspace of all smaller capacities.
int64_t planned(int64_t capacity) {
  int64_t step = 1;
  while (step * 32 <= capacity) step *= 2;
  return (capacity + step - 1) / step * step;
}

Deal deal_of(const maskkv_desc* d, int64_t room) {
  const int64_t capacity = planned(room);
  const int n_q = query_heads_per_kv(d) * d->n_resp;
  const int64_t BH = (int64_t)d->B * d->H;
  const bool bf16 = d->dtype == MASKKV_BF16;
  // What the host knows of the heads' lengths: no head has more rows than the longest prompt, and all of them as many as there is room for.
  const int64_t most = (d->P_max < capacity ? d->P_max : capacity) + d->n_resp;
  Deal best;
  float best_cost = -1.f;
  auto consider = [&](const Form& f) {
    const int qtiles = (n_q + f.tile_rows - 1) / f.tile_rows;
    const int64_t resp = (d->n_resp + f.keys - 1) / f.keys;
    const float tiles = (float)(BH * resp + capacity / f.keys) + 0.5f * BH, mean = tiles / BH;  // (half a tile of a head is empty, on average)
    const float step = f.fixed + f.per_d * (float)d->d / 128.f;
    auto cost = [&](float units, float steps) {
      const float rounds = units * qtiles / kUnits;
      const float a_step = rounds <= 1.f ? step : step * (f.at_once == 1 ? (rounds < 3.f ? ceilf(rounds) : rounds) : f.beside * fmaxf(rounds, 2.f));
      return f.start + f.round * fmaxf(rounds, 1.f) + ceilf(steps) * a_step;
    };
    auto take = [&](float cost, int chunk, int extras = 0, int cut = 0) {
      if (best_cost >= 0.f && cost >= best_cost) return;
      best_cost = cost;
      best.few = &f == &kFew;
      best.wide = &f == &kWide;
      best.tile_rows = f.tile_rows;
      best.qtiles = qtiles;
      best.part_rows = n_q < f.tile_rows ? n_q : f.tile_rows;
      best.chunk = chunk;
      best.extras = extras;
      best.cut = cut;
      best.units = extras ? extras + BH : chunk ? (capacity / f.keys + BH * (resp + 1)) / chunk + BH : BH;
    };
    const float whole = cost((float)BH, mean * (BH * qtiles <= kUnits ? f.uneven : kUneven) / f.tiles);
    const bool fits = step * ((float)most / (f.keys * f.tiles)) <= kLongest;
    if (fits) take(whole, 0);
    // (The other kernels, and more heads than are ordered, are better off with all heads dealt out: 512 heads x 16 queries x 100 ... 1000 rows and one of 40000
    // 23.5 and 21.6 us, 130 x 64 x 100 ... 2000 33.9 and 23.4, 400 x 300 x 50 ... 400 85.3 and 79.5; where none is long -4 ... 15 us.)
    if (const int64_t chunk = (int64_t)ceilf(whole / step) * f.tiles; !fits && &f == &kWide && BH <= kRanked && chunk >= 2 * mean) {  // (else most are cut)
      // A head that is cut has more than chunk - resp tiles of the cache, and a unit for every `chunk` tiles, or part of them, behind its first.
      const int64_t cached = capacity / f.keys + BH, most_cut = cached / (chunk + 1 - resp), cut = most_cut < BH ? most_cut : BH;
      if (cut == 0)
        take(whole, 0);  // (there is no room for a head that long)
      else
        take(whole + kJoin, (int)chunk, (int)((cached + cut * (resp - 1)) / chunk), (int)cut);
    }
    auto dealt = [&](float wanted) {
      int64_t chunk = (int64_t)fmaxf(ceilf(wanted), (float)f.least);
      chunk = (chunk + f.tiles - 1) / f.tiles * f.tiles;
      if (fits && chunk * f.keys >= most + 2 * f.keys) return;  // (a head's last tiles of both kinds may be short)
      const float units = fmaxf(tiles / chunk + 0.5f * BH, BH * ceilf(mean / chunk));
      take(cost(units, fminf((float)chunk, mean) / f.tiles) + kJoin + f.part * units * n_q * d->d * 4e-6f, (int)chunk);
    };
    for (int k = 1; k <= f.at_once; ++k) {  // a unit for every compute unit, or for every place in them:
      const float places = (float)(k * kUnits) / qtiles;
      dealt(tiles / fmaxf(places - 0.5f * BH, 0.5f * BH));  // for heads of any length, of which half a unit is empty,
      dealt(mean / fmaxf(floorf(places / BH), 1.f));        // and for heads of one length
    }
  };
  if (!bf16) {
    consider(kNarrowF32);
  } else if (n_q <= kFew.tile_rows) {
    consider(kFew);
  } else {
    consider(kNarrow);
    if (n_q > kWideQueries / 2) consider(kWide);
  }
  return best;
}

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T, int D>
int launch_one(const AttendMxParams& prm, const Deal& deal, hipStream_t stream) {
  using C = MxCfg<T, D>;
  static_assert(C::kLds <= 160 * 1024, "a workgroup's LDS");
  auto kernel = &attend_mx_kernel<T, D>;
  int threads = kWaves * 64, lds = C::kLds;
  const int64_t groups = deal.units * deal.qtiles;
  if constexpr (sizeof(T) == 2) {
    if (deal.wide) {
      kernel = &attend_mx_wide_kernel<D>;
      lds = WideCfg<D>::kLds;
    }
    if (deal.few) {
      kernel = &attend_mx_few_kernel<D>;
      threads = FewCfg<D>::kWaves * 64;
      lds = FewCfg<D>::kLds;
    }
  }
  if (groups * threads > 0xFFFFFFFF) {  // (threads of a launch along a dimension)
    set_error("attend_mx: %lld workgroups are more than a launch can have", (long long)groups);
    return MASKKV_ESHAPE;
  }
  if (lds > 48 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) {
      set_error("attend_mx: hipFuncSetAttribute: %s", hipGetErrorString(e));
      (void)hipGetLastError();
      return MASKKV_EHIP;
    }
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), lds, stream, prm);
  if (int e = check_launch("attend_mx")) return e;
  if (!deal.chunk) return MASKKV_OK;
  if (deal.extras)
    hipLaunchKernelGGL((attend_mx_join_kernel<T, D, false>), dim3((unsigned)(prm.n_q + kJoinGroups - 1) / kJoinGroups, (unsigned)deal.cut),
                       dim3(kJoinGroups * D / 4), 0, stream, prm);
  else if (deal.units > (int64_t)kSharedUnits * prm.BH)
    hipLaunchKernelGGL((attend_mx_join_kernel<T, D, true>), dim3((unsigned)prm.n_q, (unsigned)prm.BH), dim3(kJoinGroups * D / 4), 0, stream, prm);
  else
    hipLaunchKernelGGL((attend_mx_join_kernel<T, D, false>), dim3((unsigned)(prm.n_q + kJoinGroups - 1) / kJoinGroups, (unsigned)prm.BH),
                       dim3(kJoinGroups * D / 4), 0, stream, prm);
  return check_launch("attend_mx (join)");
}

}  // namespace

AttendMxPlan attend_mx_plan(const maskkv_desc* d, int64_t capacity) {
  const Deal x = deal_of(d, capacity);
  const int64_t BH = (int64_t)d->B * d->H;
  return {x.tile_rows, x.qtiles, x.chunk, x.units, x.wide && (!x.chunk || x.extras) && BH <= kRanked, x.chunk && !x.extras && x.units > kSharedUnits * BH,
          x.extras, x.cut};
}

size_t attend_mx_needs(const maskkv_desc* d, int64_t capacity) {
  const Deal x = deal_of(d, capacity);
  if (!x.chunk) return 0;
  const size_t rows = (size_t)x.places() * x.qtiles * x.part_rows;
  return pad256(rows * d->d * 4) + pad256(rows * 8) + (x.extras ? 0 : pad256((size_t)d->B * d->H * 8));
}

// The most that any capacity up to this one needs: fewer rows may be dealt out finer.  (A cache that shrinks keeps its workspace.)
size_t attend_mx_workspace_bytes(const maskkv_desc* d, int64_t capacity) {
  size_t most = 0;
  for (int64_t rows = planned(capacity);;) {
    const size_t bytes = attend_mx_needs(d, rows);
    most = bytes > most ? bytes : most;
    if (rows == 0) return most;
    int64_t step = 1;
    while (step * 32 < rows) step *= 2;
    rows -= step;
  }
}

int launch_attend_mx(const maskkv_desc* d, const View& Q, const MxCache& cache, const int32_t* cu_budget, int64_t capacity, const View& K2,
                     const View& V2, float scale, const View& O, float* lse, void* workspace, hipStream_t stream) {
  const Deal deal = deal_of(d, capacity);
  AttendMxParams prm;
  prm.Q = Q;
  prm.K2 = K2;
  prm.V2 = V2;
  prm.O = O;
  prm.cache = cache;
  prm.cu = cu_budget;
  prm.capacity = capacity;
  prm.H = d->H;
  prm.BH = d->B * d->H;
  prm.q_per_kv = query_heads_per_kv(d);
  prm.n_resp = d->n_resp;
  prm.n_q = prm.q_per_kv * d->n_resp;
  prm.qtiles = deal.qtiles;
  prm.units = (int)deal.units;
  prm.chunk = deal.chunk;
  prm.extras = deal.extras;
  prm.tile_rows = deal.tile_rows;
  prm.part_rows = deal.part_rows;
  prm.c = scale * kLog2e;
  prm.lse = lse;
  const size_t rows = (size_t)deal.places() * deal.qtiles * deal.part_rows;
  char* ws = reinterpret_cast<char*>(workspace);
  prm.part_o = reinterpret_cast<float*>(ws);
  prm.part_ml = reinterpret_cast<float2*>(ws + pad256(rows * d->d * 4));
  prm.parts = reinterpret_cast<int2*>(ws + pad256(rows * d->d * 4) + pad256(rows * 8));
  if (d->dtype == MASKKV_BF16)
    return d->d == 128 ? launch_one<bf16_t, 128>(prm, deal, stream) : launch_one<bf16_t, 64>(prm, deal, stream);
  return d->d == 128 ? launch_one<float, 128>(prm, deal, stream) : launch_one<float, 64>(prm, deal, stream);
}

}  // namespace maskkv
