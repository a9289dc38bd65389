// Attention of response rows that do not all see each other - trees of drafted tokens, blocks in order - over a packed cache and the
// response's own rows: one pass over the keys with the running maximum and sum of a softmax, a bit per query and response row.
//
// A workgroup has eight waves (fp32 at head_dim 128: four) and serves 32 query rows of a head.  Logits are formed transposed (keys on the matrix instruction's row axis), so that a
// lane owns one query, its word of the mask covers a tile of 32 response rows, and its probabilities are the B operand of
// O^T = V^T P^T as they stand.  The waves take tiles of 32 keys in turn, each through LDS of its own and without a barrier: K and V come by direct
// transfers, K of the next tile while this one's softmax runs, V of the next behind this one's product.  (The compiler waits for the query's fragments in front of the
// first product of every turn, not of the first one only, and so for all transfers: the logits of a tile wait for its V too.)  The waves are merged at the end.
//
// The keys of a head go to several workgroups where the launch would not fill the chip (`deal_of`), and a second kernel joins the partial results.
//
// What a row does not see must not reach it, be it infinite or NaN: a product of the matrix pipe would turn a probability of 0 times such
// a value into NaN.  Tiles of the response are looked through for them, and one that has any takes the product key by key (`add_seen`).  Cached rows
// are seen by all queries of their head; a tile's places behind the last row hold that row again, as a key that is masked, and zeros as a value.
//
// Sums, maxima and outputs are fp32; probabilities are rounded to bf16, by at most 2^-8 of each, as the operand of the second product: fp32 operands have a
// sixteenth of its rate.  The sum that divides them is of the unrounded ones.
//
// By latency (of that wait, too) and memory where few rows meet a long cache: 64 rows of 32 heads x 4096 (69 MB) 17.3 us, 4.0 TB/s, waves waiting 42 % of their
// cycles, and 3.9 to 4.7 for the joining launch; 8 rows over 32 x 8192 (134 MB) 31 together.  By latency where there is little: 256 heads x 32 rows x 64 ... 1024
// 14.8 (54 MB), four heads of 8 fp32 rows 6.8.  With many rows (the second kernel) by matrix and softmax phases: 4 heads of 336 rows x 30011 33.8 us, 700 TFLOP/s
// with the padding to 384 rows, both pipes busy 40 % of the time; joining 7.4.
// Eight waves a workgroup and one of these a compute unit, not two of four waves (both sides in their own best number of units): ragged batch 18.7 and 15.1 us, single token
// of 7 heads x 30k rows 17.8 and 17.2, 64 rows over 4096 21.0 and 20.9.
#include <cmath>
#include <type_traits>

#include "attend.hpp"
#include "mx.hpp"

namespace maskkv {

namespace {

constexpr int kUnits = 256;  // compute units
constexpr int kTile = 32;    // keys of a tile, and query rows of a workgroup

struct TreeParams {
  View Q, K2, V2, O;
  const char* Kc;
  const char* Vc;
  const int32_t* cu;
  const uint32_t* mask;
  int64_t capacity;
  int H, BH, q_per_kv, n_resp, n_q, qtiles, words;
  int units;      // at most
  int chunk;      // tiles of a workgroup, or 0: all of its head
  int tile_rows;  // query rows of a workgroup
  int part_rows;  // of a partial result
  float c;        // scale * log2(e)
  float* lse;
  float* part_o;    // [units * qtiles][part_rows][D]
  float2* part_ml;  // [units * qtiles][part_rows]
  int2* parts;      // [BH] a head's first unit, and how many it has
};

__device__ __forceinline__ void fetch_tree_arguments() {
  typedef TreeParams A;
  fetch_arguments({MASKKV_VIEW_ARGUMENTS(A, Q), MASKKV_VIEW_ARGUMENTS(A, K2), MASKKV_VIEW_ARGUMENTS(A, V2), MASKKV_VIEW_ARGUMENTS(A, O),
                   MASKKV_ARGUMENT(A, Kc), MASKKV_ARGUMENT(A, H), (uint32_t)(offsetof(A, parts) + 4)});
}

template <typename T, int D>
struct TreeCfg {
  static constexpr int kWaves = D * (int)sizeof(T) == 512 ? 4 : 8;  // as many as LDS has room for, up to two a SIMD
  static constexpr int kThreads = kWaves * 64;
  static constexpr int kRowB = D * (int)sizeof(T);
  static constexpr int kPPR = kRowB / 16;           // pieces of 16 bytes in a row
  static constexpr int kDB = D / 32;
  static constexpr int kTileB = kTile * kRowB;      // K, then V of a wave
  static constexpr int kMoves = kTileB / 1024;      // direct transfers of a tile
  static constexpr int kMoveRows = 64 / kPPR;       // rows of one
  static constexpr int kSumP = D / 2 + 4;           // floats from one query's sums to the next while the waves are merged, half a row at a time
  static constexpr int kMlAt = kWaves * 2 * kTileB;
  static constexpr int kLds = kMlAt + kWaves * kTile * 8;
  static_assert(kTile * kSumP * 4 <= 2 * kTileB && kTile * kTile * 4 <= kTileB, "LDS of a wave");
  // Rows that are read by halves, 16 bytes a lane: neighbouring rows on different banks.
  __device__ static uint32_t k_slot(uint32_t row, uint32_t p) { return p ^ (kPPR == 8 ? (row >> 1) & 7 : row & 15); }
  // V: bf16 see v_swizzle; fp32: blocks of 32 columns, exchanged in every other four rows.
  __device__ static uint32_t v_slot(uint32_t row, uint32_t p) {
    return sizeof(T) == 2 ? p ^ v_swizzle<D>(row) << 1 : p ^ ((row >> 2) & 1) << 3;
  }
};

// The larger of each of two numbers of 16 bits.
__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

template <int N>
__device__ __forceinline__ void wait_moves() {  // all but the last N transfers have arrived
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void lds_is_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

template <typename T, int D>
__global__ __launch_bounds__((TreeCfg<T, D>::kThreads), (TreeCfg<T, D>::kWaves / 4)) void attend_tree_kernel(const TreeParams prm) {
  using C = TreeCfg<T, D>;
  constexpr int kWaves = C::kWaves;
  constexpr bool F32 = sizeof(T) == 4;
  extern __shared__ __attribute__((aligned(1024))) char tree_lds[];
  fetch_tree_arguments();
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

  char* const k_lds = tree_lds + wave * 2 * C::kTileB;
  char* const v_lds = k_lds + C::kTileB;
  const uint32_t k_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)k_lds, v_at = k_at + C::kTileB;

  // This wave's tiles: t0 + wave, and every one as many on as there are waves.
  const int mine = max(t1 - t0 - wave + kWaves - 1, 0) / kWaves;
  auto tile_of = [&](int i) { return t0 + wave + i * kWaves; };
  // A transfer brings the pieces that belong to consecutive places of LDS.  (Rows behind the last one are the last one.)
  auto move = [&](const char* from, int64_t stride, int left, uint32_t to, auto slot) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < C::kMoves; ++j) {
      const uint32_t row = j * C::kMoveRows + lane / C::kPPR;
      dma16(from, (uint32_t)min((int)row, left - 1) * (uint32_t)stride + (slot(row, lane % C::kPPR) << 4), to + j * 1024);
    }
  };
  auto move_k = [&](int t) __attribute__((always_inline)) {
    auto slot = [](uint32_t row, uint32_t p) { return C::k_slot(row, p); };
    if (t < resp_tiles)
      move(prm.K2.row(b, h, t * kTile), prm.K2.stride_t, prm.n_resp - t * kTile, k_at, slot);
    else
      move(prm.Kc + ((int64_t)head.first + (t - resp_tiles) * kTile) * C::kRowB, C::kRowB, cached - (t - resp_tiles) * kTile, k_at, slot);
  };
  auto move_v = [&](int t) __attribute__((always_inline)) {
    auto slot = [](uint32_t row, uint32_t p) { return C::v_slot(row, p); };
    if (t < resp_tiles)
      move(prm.V2.row(b, h, t * kTile), prm.V2.stride_t, prm.n_resp - t * kTile, v_at, slot);
    else
      move(prm.Vc + ((int64_t)head.first + (t - resp_tiles) * kTile) * C::kRowB, C::kRowB, cached - (t - resp_tiles) * kTile, v_at, slot);
  };

  // ---- this lane's query: half of its row, as the B operand of the first product
  const int query = min(qtile * kTile + r, prm.n_q - 1);
  u32x4 qf[C::kPPR / 2];
  {
    const char* q = prm.Q.group_row(b, h, prm.q_per_kv, prm.n_resp, query) + g * (C::kRowB / 2);
#pragma unroll
    for (int i = 0; i < C::kPPR / 2; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + 16 * i);
  }
  const uint32_t* const my_mask = prm.mask + ((int64_t)b * prm.n_resp + query % prm.n_resp) * prm.words;
  if (mine > 0) {
    move_k(tile_of(0));
    move_v(tile_of(0));
  }

  f32x16 o[C::kDB], s;
#pragma unroll
  for (int db = 0; db < C::kDB; ++db) o[db] = f32x16{};
  float m = kNegBig, l = 0.f;

  // The product for a tile of the response that holds an infinity or NaN: key by key, of those that the lane's query sees.
  auto add_seen = [&](uint32_t word) __attribute__((always_inline)) {
    float* const p_lds = reinterpret_cast<float*>(k_lds);  // [key][query] (K has been read)
#pragma unroll
    for (int i = 0; i < 16; ++i) p_lds[(8 * (i / 4) + 4 * g + i % 4) * kTile + r] = s[i];
    lds_is_read();
#pragma unroll 1
    for (int j = 0; j < kTile; ++j) {
      const float p = p_lds[j * kTile + r];
      const bool sees = word >> j & 1;
#pragma unroll
      for (int db = 0; db < C::kDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // four elements of the row
          const uint32_t e = 32 * db + 8 * q + 4 * g;
          float v[4];
          if constexpr (F32) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(v_lds + j * C::kRowB + (C::v_slot(j, e / 4) << 4));
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint32_t bits = w[x];
              v[x] = as_f32(bits);
            }
          } else {
            const u32x2 w = *reinterpret_cast<const u32x2*>(v_lds + j * C::kRowB + (C::v_slot(j, e / 8) << 4) + e % 8 * 2);
            const uint32_t w0 = w[0], w1 = w[1];
            v[0] = as_f32(w0 << 16), v[1] = as_f32(w0 & 0xFFFF0000u), v[2] = as_f32(w1 << 16), v[3] = as_f32(w1 & 0xFFFF0000u);
          }
#pragma unroll
          for (int x = 0; x < 4; ++x) o[db][4 * q + x] = sees ? fmaf(p, v[x], o[db][4 * q + x]) : o[db][4 * q + x];
        }
    }
    lds_is_read();
  };
  auto holds_infinite = [&]() __attribute__((always_inline)) {
    u32x4 most = {};  // of the values, without signs (bf16: as pairs)
#pragma unroll
    for (int j = 0; j < C::kMoves; ++j) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(v_lds + j * 1024 + lane * 16);
#pragma unroll
      for (int x = 0; x < 4; ++x) most[x] = F32 ? max(most[x], w[x] & 0x7FFFFFFFu) : max_pairs(most[x], w[x] & 0x7FFF7FFFu);
    }
    bool any = false;
#pragma unroll
    for (int x = 0; x < 4; ++x) any |= most[x] >= 0x7F800000u || (!F32 && (most[x] & 0xFFFFu) >= 0x7F80u);
    return __any(any);
  };

  // ---- a tile: logits, softmax, output.  Lanes l and l ^ 32 have the same query.
  auto take = [&](int i, auto of_response) __attribute__((always_inline)) {
    constexpr bool kResp = decltype(of_response)::value;
    const int t = tile_of(i), left = kResp ? prm.n_resp - t * kTile : cached - (t - resp_tiles) * kTile;
    const bool more = i + 1 < mine;
    uint32_t word = 0;
    if constexpr (kResp) {
      word = my_mask[t];
      if (left < kTile) word &= (1u << left) - 1;
      wait_moves<0>();
    } else {
      wait_moves<C::kMoves>();
    }
    s = f32x16{};
#pragma unroll
    for (int w = 0; w < C::kPPR / 2; ++w)
      mfma_step<T>(*reinterpret_cast<const u32x4*>(k_lds + r * C::kRowB + (C::k_slot(r, g * (C::kPPR / 2) + w) << 4)), qf[w], s);
    lds_is_read();
    if (!kResp && more) move_k(tile_of(i + 1));
    if constexpr (kResp) {
      const uint32_t own = word >> (4 * g);
#pragma unroll
      for (int x = 0; x < 16; ++x) s[x] = own >> (8 * (x / 4) + x % 4) & 1 ? s[x] : -INFINITY;
    } else if (left < kTile) {
#pragma unroll
      for (int x = 0; x < 16; ++x)
        if (8 * (x / 4) + x % 4 >= left - 4 * g) s[x] = -INFINITY;
    }
    float bm = s[0];
#pragma unroll
    for (int x = 1; x < 16; ++x) bm = fmaxf(bm, s[x]);
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
        for (int x = 0; x < 16; ++x) o[db][x] *= alpha;
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const float p = fast_exp2(fmaf(s[x], prm.c, -m));
      s[x] = p;
      l += p;
    }
    bool plain = true;
    if constexpr (kResp) {
      if (holds_infinite()) {
        add_seen(word);
        plain = false;
      }
      if (more) move_k(tile_of(i + 1));
    } else if (more) {
      wait_moves<C::kMoves>();
    } else {
      wait_moves<0>();
    }
    if (!kResp && left < kTile) {  // (places behind the last row: 0 times an infinite value would be NaN)
      for (int at = left * C::kRowB + lane * 16; at < C::kTileB; at += 1024) *reinterpret_cast<u32x4*>(v_lds + at) = u32x4{};
      lds_is_read();
    }
    if (plain) {
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
        for (int x = 0; x < 16; ++x) {
          const int row = 8 * (x / 4) + 4 * g + x % 4;
#pragma unroll
          for (int db = 0; db < C::kDB; ++db) {
            const float v = *reinterpret_cast<const float*>(v_lds + row * C::kRowB + ((db ^ ((row >> 2) & 1)) * 32 + r) * 4);
            o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[x], o[db], 0, 0, 0);
          }
        }
      }
    }
    lds_is_read();
    if (more) move_v(tile_of(i + 1));
  };
  {
    const int resp = min(max(min(resp_tiles, t1) - t0 - wave + kWaves - 1, 0) / kWaves, mine);
    int i = 0;
    for (; i < resp; ++i) take(i, std::true_type());
    for (; i < mine; ++i) take(i, std::false_type());
  }

  // ---- the waves' results become one: sums of each wave, in units of the largest reference, through LDS
  l = sum_halves(l);
  float2* const ml = reinterpret_cast<float2*>(tree_lds + C::kMlAt);
  if (g == 0) ml[wave * kTile + r] = make_float2(m, l);
  __syncthreads();
  float top = kNegBig;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w * kTile + r].x);
  const float mine_by = fast_exp2(m - top);
  float* const sums = reinterpret_cast<float*>(tree_lds);
  constexpr int kEach = kTile * D / 2 / C::kThreads < 4 ? 4 : kTile * D / 2 / C::kThreads;  // elements of a row that a thread writes
  constexpr int kPerRow = D / 2 / kEach;                                                    // threads of half a row
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
    const int row = threadIdx.x / kPerRow, q = qtile * kTile + row, at = threadIdx.x % kPerRow * kEach;  // (32 rows or more)
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
#pragma unroll
      for (int e = 0; e < kEach; e += 4) to[e / 4] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      if (to_at == 0) prm.part_ml[part] = make_float2(mq, lq);
      continue;
    }
    const float by = lq == 0.f ? 0.f : 1.f / lq;  // (a row that sees nothing)
    char* to = prm.O.group_row(b, h, prm.q_per_kv, prm.n_resp, q) + to_at * (int)sizeof(T);
#pragma unroll
    for (int e = 0; e < kEach; e += 4) {
      if constexpr (F32)
        reinterpret_cast<float4*>(to)[e / 4] = make_float4(x[e] * by, x[e + 1] * by, x[e + 2] * by, x[e + 3] * by);
      else
        reinterpret_cast<u32x2*>(to)[e / 4] = u32x2{pack_bf16x2(x[e] * by, x[e + 1] * by), pack_bf16x2(x[e + 2] * by, x[e + 3] * by)};
    }
    if (to_at == 0 && prm.lse) prm.lse[(int64_t)bh * prm.n_q + q] = (mq + __builtin_amdgcn_logf(lq)) * kLn2;
  }
}

// ---- many query rows of bf16: a workgroup of four waves serves 128 of a head, 32 a wave, over tiles of 64 keys that all of them read from LDS.  Two
// workgroups share a compute unit, so that one's softmax runs beside the other's products, and within a wave the logits of the next
// tile are formed beside the softmax of this one.
//
// Iteration t reads K(t+1) and V(t), and brings K(t+2) and V(t+1) into the other two of four buffers, which iteration t-1 has read: one barrier an
// iteration.  Tiles of the response are taken first, each by itself: they are few, have a mask, and may hold what must not be multiplied.
constexpr int kWideTile = 64;
constexpr int kWideQueries = 128;

template <int D>
struct WideCfg {
  static constexpr int kRowB = 2 * D;
  static constexpr int kPPR = kRowB / 16;
  static constexpr int kSteps = D / 16;
  static constexpr int kDB = D / 32;
  static constexpr int kTileB = kWideTile * kRowB;
  static constexpr int kMoves = kWideTile * kRowB / 4096;  // direct transfers of 1 KiB a wave and tile
  static constexpr int kMoveRows = 1024 / kRowB;
  static constexpr int kProbs = 4 * kTileB;                // then: probabilities of a wave for 32 keys, fp32 (see add_seen)
  static constexpr int kLds = kProbs + 4 * kTile * kTile * 4;
  __device__ static uint32_t swz_k(uint32_t row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
};

template <int D>
__global__ __launch_bounds__(256, 2) void attend_tree_wide_kernel(const TreeParams prm) {
  using C = WideCfg<D>;
  extern __shared__ __attribute__((aligned(1024))) char tree_lds[];
  fetch_tree_arguments();
  const Place place = place_of(blockIdx.x, prm.units, prm.qtiles);
  const int unit = place.unit, qtile = place.qtile;
  const int resp_tiles = (prm.n_resp + kWideTile - 1) / kWideTile;
  auto tiles_of = [&](int rows) { return (int)(((uint32_t)rows + kWideTile - 1) / kWideTile) + resp_tiles; };  // those of the response first
  const int capacity = (int)prm.capacity;
  UnitHead head;
  if (prm.chunk) {
    head = head_of_unit(prm.cu, prm.BH, capacity, unit, [&](int rows) { return (tiles_of(rows) + prm.chunk - 1) / prm.chunk; });
    if (head.bh < 0) return;
  } else {
    const int first = min(prm.cu[unit], capacity);
    head = {unit, unit, 1, first, max(min(prm.cu[unit + 1], capacity) - first, 0)};
  }
  const int bh = head.bh, cached = head.rows, all_tiles = tiles_of(cached);
  const int b = bh / prm.H, h = bh % prm.H;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, g = lane >> 5;
  if (prm.chunk && unit == head.first_unit && qtile == 0 && threadIdx.x == 0) prm.parts[bh] = make_int2(head.first_unit, head.units);
  const int t0 = prm.chunk ? (unit - head.first_unit) * prm.chunk : 0;
  const int t1 = prm.chunk ? min(all_tiles, t0 + prm.chunk) : all_tiles;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)tree_lds;

  // ---- tiles on their way: a wave takes a quarter of the rows
  const uint32_t moved = wave * (kWideTile / 4) + (uint32_t)lane / C::kPPR;  // this lane's row of the wave's first transfer
  const uint32_t piece_k = ((uint32_t)lane % C::kPPR ^ C::swz_k(moved)) << 4, piece_v = ((uint32_t)lane % C::kPPR ^ v_swizzle<D>(moved) << 1) << 4;
  auto transfer = [&](const char* from, int64_t stride, int left, uint32_t piece, uint32_t step, uint32_t to) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < C::kMoves; ++j) {  // (a row's permutation changes from a transfer to the next by an exclusive-or of its own)
      const uint32_t row = min((int)moved + j * C::kMoveRows, left - 1);
      dma16(from, row * (uint32_t)stride + (piece ^ (j * step & (C::kRowB - 1))), to + (wave * C::kMoves + j) * 1024);
    }
  };
  const char* const kc = prm.Kc + (int64_t)head.first * C::kRowB;
  const char* const vc = prm.Vc + (int64_t)head.first * C::kRowB;
  // K and V of a tile of the cache (t: counted from its first one) into the buffer of even or odd tiles
  auto bring_k = [&](int t, uint32_t odd) __attribute__((always_inline)) {
    transfer(kc + (int64_t)t * C::kTileB, C::kRowB, cached - t * kWideTile, piece_k, C::swz_k(C::kMoveRows) << 4, lds0 + odd * C::kTileB);
  };
  auto bring_v = [&](int t, uint32_t odd) __attribute__((always_inline)) {
    transfer(vc + (int64_t)t * C::kTileB, C::kRowB, cached - t * kWideTile, piece_v, 0, lds0 + (2 + odd) * C::kTileB);
  };
  auto arrive = [] {  // what this wave has moved is there, and so is everyone's behind the barrier
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  const int q0 = qtile * kWideQueries + wave * 32, query = min(q0 + r, prm.n_q - 1);
  u32x4 qf[C::kSteps];
  {
    const char* q = prm.Q.group_row(b, h, prm.q_per_kv, prm.n_resp, query) + g * D;
#pragma unroll
    for (int i = 0; i < C::kSteps; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + 16 * i);
  }

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

  auto raise = [&]() __attribute__((always_inline)) {  // the reference, where the tile's largest logit asks for it
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
  };

  // Fragment n of a tile: 0 .. kQK-1 of its keys (two chains of products, one for 32 keys each), from kQK on of values; in which buffers.
  constexpr int kQK = 2 * C::kSteps, kPV = 4 * C::kDB, kAhead = 2;
  u32x4 fr[kAhead + 1];
  auto fetch = [&](int n, uint32_t odd_k, uint32_t odd_v) __attribute__((always_inline)) {
    u32x4& f = fr[n % (kAhead + 1)];
    if (n < kQK) {
      f = *in_lds<const u32x4>(k_at[n / 2] + odd_k * C::kTileB, n % 2 * 32 * C::kRowB);
    } else {
      const int i = n - kQK, imm = i / C::kDB * 16 * C::kRowB;
      const uint32_t at = v_at[i % C::kDB] + odd_v * C::kTileB;
      const u32x2 lo = read_transposed(at, imm), hi = read_transposed(at, imm + 8 * C::kRowB);
      f = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  };

  // ---- tiles of the response, in the buffers of even and odd tiles in turn: the next one, and its words, are under way meanwhile
  const uint32_t* const my_mask = prm.mask + ((int64_t)b * prm.n_resp + query % prm.n_resp) * prm.words;
  const int resp_end = min(t1, resp_tiles), begin = max(t0 - resp_tiles, 0), tiles = t1 - resp_tiles;  // those of the cache: counted from its first one
  auto bring_resp = [&](int t, uint32_t odd) __attribute__((always_inline)) {
    const int left = prm.n_resp - t * kWideTile;
    transfer(prm.K2.row(b, h, t * kWideTile), prm.K2.stride_t, left, piece_k, C::swz_k(C::kMoveRows) << 4, lds0 + odd * C::kTileB);
    transfer(prm.V2.row(b, h, t * kWideTile), prm.V2.stride_t, left, piece_v, 0, lds0 + (2 + odd) * C::kTileB);
  };
  uint32_t ahead[2] = {0, 0};
  auto words_of = [&](int t) __attribute__((always_inline)) {
    const int left = prm.n_resp - t * kWideTile;
    ahead[0] = my_mask[2 * t];
    ahead[1] = 2 * t + 1 < prm.words ? my_mask[2 * t + 1] : 0;
    if (left < 32) ahead[0] &= (1u << left) - 1;
    if (left > 32 && left < 64) ahead[1] &= (1u << (left - 32)) - 1;
  };
  if (t0 < resp_end) {
    words_of(t0);
    bring_resp(t0, 0);
  }
  for (int t = t0; t < resp_end; ++t) {
    const uint32_t odd_tile = (t - t0) & 1, k_off = odd_tile * C::kTileB, v0 = lds0 + (2 + odd_tile) * C::kTileB;
    const uint32_t word[2] = {ahead[0], ahead[1]};
    arrive();  // (and the tile before has been read)
    if (t + 1 < resp_end) {
      words_of(t + 1);
      bring_resp(t + 1, 1 - odd_tile);
    }
    if (!__any((word[0] | word[1]) != 0)) continue;  // (none of the wave's queries sees any of it)
#pragma unroll
    for (int n = 0; n < kAhead; ++n) fetch(n, odd_tile, odd_tile);
#pragma unroll
    for (int n = 0; n < kQK; ++n) {
      if (n + kAhead < kQK) fetch(n + kAhead, odd_tile, odd_tile);
      if (n < 2) even[n] = f32x16{};
      mfma_step<bf16_t>(fr[n % (kAhead + 1)], qf[n / 2], even[n % 2]);
    }
    u32x4 most = {};  // of the values, without signs, as pairs of 16 bits
#pragma unroll
    for (int j = 0; j < C::kTileB / 1024; ++j) {
      const u32x4 w = *in_lds<const u32x4>(v0 + j * 1024 + lane * 16);
#pragma unroll
      for (int x = 0; x < 4; ++x) most[x] = max_pairs(most[x], w[x] & 0x7FFF7FFFu);
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const uint32_t own = word[kb] >> (4 * g);
#pragma unroll
      for (int i = 0; i < 16; ++i) even[kb][i] = own >> (8 * (i / 4) + i % 4) & 1 ? even[kb][i] : -INFINITY;
    }
    top = even[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, even[i / 16][i % 16]);
    raise();
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float p = fast_exp2(fmaf(even[i / 16][i % 16], c, -m));
      even[i / 16][i % 16] = p;
      l += p;
    }
    const uint32_t m01 = max_pairs(most[0], most[1]), m23 = max_pairs(most[2], most[3]), all = max_pairs(m01, m23);
    const bool any = all >= 0x7F800000u || (all & 0xFFFFu) >= 0x7F80u;
    if (__any(any)) {  // (see attend_tree_kernel: key by key, of those that the lane's query sees)
      const uint32_t own = lds0 + C::kProbs + wave * kTile * kTile * 4;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        lds_is_read();
#pragma unroll
        for (int i = 0; i < 16; ++i) *in_lds<float>(own + ((8 * (i / 4) + 4 * g + i % 4) * kTile + r) * 4) = even[kb][i];
        lds_is_read();
#pragma unroll 1
        for (int j = 0; j < kTile; ++j) {
          const float p = *in_lds<const float>(own + (j * kTile + r) * 4);
          const bool sees = word[kb] >> j & 1;
          const uint32_t row = kb * kTile + j;
#pragma unroll
          for (int db = 0; db < C::kDB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint32_t e = 32 * db + 8 * q + 4 * g;
              const u32x2 w = *in_lds<const u32x2>(v0 + row * C::kRowB + ((e / 8 ^ v_swizzle<D>(row) << 1) << 4) + e % 8 * 2);
              const uint32_t w0 = w[0], w1 = w[1];
              const float v[4] = {as_f32(w0 << 16), as_f32(w0 & 0xFFFF0000u), as_f32(w1 << 16), as_f32(w1 & 0xFFFF0000u)};
#pragma unroll
              for (int x = 0; x < 4; ++x) o[db][4 * q + x] = sees ? fmaf(p, v[x], o[db][4 * q + x]) : o[db][4 * q + x];
            }
        }
      }
    } else {
      u32x4 pf[4];
#pragma unroll
      for (int i = 0; i < 32; i += 2) pf[i / 8][i % 8 / 2] = pack_bf16x2(even[i / 16][i % 16], even[i / 16][i % 16 + 1]);
#pragma unroll
      for (int n = kQK; n < kQK + kAhead; ++n) fetch(n, odd_tile, odd_tile);
#pragma unroll
      for (int n = kQK; n < kQK + kPV; ++n) {
        if (n + kAhead < kQK + kPV) fetch(n + kAhead, odd_tile, odd_tile);
        mfma_step<bf16_t>(fr[n % (kAhead + 1)], pf[(n - kQK) / C::kDB], o[(n - kQK) % C::kDB]);
      }
    }
  }

  // ---- tiles of the cache
  if (begin < tiles) {
    if (t0 < resp_tiles) arrive();  // (the response's last tile has been read)
    bring_k(begin, 0);
    bring_v(begin, 0);
    if (begin + 1 < tiles) bring_k(begin + 1, 1);
    arrive();
    auto mask = [&](int t, f32x16 (&s)[2]) __attribute__((always_inline)) {  // keys behind the last one
      const int left = cached - t * kWideTile;
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
      fetch(n, 0, 0);
      if (n < 2) even[n] = f32x16{};
      mfma_step<bf16_t>(fr[n % (kAhead + 1)], qf[n / 2], even[n % 2]);
    }
    mask(begin, even);
    top = even[0][0];
#pragma unroll
    for (int i = 0; i < 32; ++i) top = fmaxf(top, even[i / 16][i % 16]);
    arrive();  // (K(2) takes the place of K(0))

    // Tile t (odd or not) with its logits in `s`; with MORE those of the next into `next`.  The next tile's logits are formed beside this one's
    // exponentials, this one's part of the output beside the search for the next one's largest logit.
    auto step = [&](int t, auto odd_tile, auto more, f32x16 (&s)[2], f32x16 (&next)[2]) __attribute__((always_inline)) {
      constexpr uint32_t kOdd = decltype(odd_tile)::value;
      constexpr bool kMore = decltype(more)::value;
      constexpr int kFrom = kMore ? 0 : kQK;
      if constexpr (kMore) {
        if (t + 2 < tiles) bring_k(t + 2, kOdd);
        bring_v(t + 1, 1 - kOdd);
      } else if (const int left = cached - t * kWideTile; left < kWideTile) {  // (places behind the last row: 0 times an infinite value would be NaN)
        for (int at = left * C::kRowB + threadIdx.x * 16; at < C::kTileB; at += 256 * 16) *in_lds<u32x4>(lds0 + (2 + kOdd) * C::kTileB + at) = u32x4{};
        arrive();
      }
      raise();
      u32x4 pf[4];
      auto probabilities = [&](int i) __attribute__((always_inline)) {  // values i and i + 1 of the 32
        const float p0 = fast_exp2(fmaf(s[i / 16][i % 16], c, -m)), p1 = fast_exp2(fmaf(s[i / 16][i % 16 + 1], c, -m));
        l += p0 + p1;
        uint32_t both = pack_bf16x2(p0, p1);
        asm volatile("" : "+v"(both), "+v"(l));  // (formed here, beside the products, and not where it is first needed)
        pf[i / 8][i % 8 / 2] = both;
      };
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < kAhead; ++n) fetch(kFrom + n, 1 - kOdd, kOdd);
      if constexpr (kMore) {
#pragma unroll
        for (int n = 0; n < kQK; ++n) {
          fetch(n + kAhead, 1 - kOdd, kOdd);
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
        if (n + kAhead < kQK + kPV) fetch(n + kAhead, 1 - kOdd, kOdd);
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
    int t = begin;
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
  } else {
    arrive();  // (what follows writes where the response's last tile was read)
  }

  // ---- out, by way of LDS: whole rows
  l = sum_halves(l);
  if (head.units > 1) {
    if (q0 + r >= prm.n_q) return;
    const int64_t part = ((int64_t)unit * prm.qtiles + qtile) * prm.part_rows + wave * 32 + r;
#pragma unroll
    for (int db = 0; db < C::kDB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(prm.part_o + part * D + 32 * db + 8 * i + 4 * g) =
            make_float4(o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]);
    if (g == 0) prm.part_ml[part] = make_float2(m, l);
    return;
  }
  const float by = l == 0.f ? 0.f : 1.f / l;  // (a row that sees nothing)
  char* own = tree_lds + wave * 32 * (C::kRowB + 16);
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

// The partial results of the heads that have several units: sums in units of the largest reference.  D/4 threads take a query row and ask for
// kAtOnce of its partial results before they use the first; where a head has many, the eight groups of a workgroup share one row
// (SHARED) and meet in LDS, else each has a row of its own.
constexpr int kJoinGroups = 8;
template <typename T, int D, bool SHARED>
__global__ __launch_bounds__(kJoinGroups * D / 4) void attend_tree_join_kernel(const TreeParams prm) {
  constexpr int kPer = D / 4, kAtOnce = 8, kStep = SHARED ? kJoinGroups : 1;
  __shared__ float4 sums[kJoinGroups][kPer];
  __shared__ float2 tops[kJoinGroups];
  fetch_tree_arguments();
  const int grp = threadIdx.x / kPer, at = threadIdx.x % kPer, bh = blockIdx.y;
  const int q = SHARED ? blockIdx.x : blockIdx.x * kJoinGroups + grp;
  const int first = prm.parts[bh].x, units = prm.parts[bh].y;
  if (units <= 1 || q >= prm.n_q) return;
  const int64_t step = (int64_t)prm.qtiles * prm.part_rows;
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
        const int64_t part = (first + u0 + i * kStep) * step + in_unit;
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
  const float by = l == 0.f ? 0.f : 1.f / l;
  char* to = prm.O.group_row(bh / prm.H, bh % prm.H, prm.q_per_kv, prm.n_resp, q) + at * 4 * (int)sizeof(T);
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<float4*>(to) = make_float4(x.x * by, x.y * by, x.z * by, x.w * by);
  else
    *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(x.x * by, x.y * by), pack_bf16x2(x.z * by, x.w * by)};
  if (at == 0 && prm.lse) prm.lse[(int64_t)bh * prm.n_q + q] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- who sees whom in drafted trees: a thread a row, which walks up from it.  The rows above have ever smaller numbers, so the words are
// finished one after the other, the last one first.  Trees of up to kTreeRows rows lie in LDS, parents and words, so that a step of the walk waits for LDS
// and the words leave in order (64 trees of 512: 9.3 us with both in memory, 7.9 in LDS).
constexpr int kTreeRows = 1024;
constexpr int kMaskThreads = 256;
template <bool LDS>
__global__ __launch_bounds__(kMaskThreads) void tree_mask_kernel(const int32_t* parents, int n, int words, uint32_t* mask) {
  __shared__ int32_t own_parents[LDS ? kTreeRows : 1];
  __shared__ uint32_t own_words[LDS ? kMaskThreads * (kTreeRows / 32 + 1) : 1];
  const int b = blockIdx.y, first = blockIdx.x * kMaskThreads, i = first + threadIdx.x;
  const int32_t* up = parents + (int64_t)b * n;
  if constexpr (LDS) {
    for (int j = threadIdx.x; j < min(n, first + kMaskThreads); j += kMaskThreads) own_parents[j] = up[j];
    __syncthreads();
    up = own_parents;
  }
  if (i < n) {
    const int pitch = words | 1;  // (neighbouring rows on different banks)
    uint32_t* const to = LDS ? own_words + threadIdx.x * pitch : mask + ((int64_t)b * n + i) * words;
    int p = up[i], at = words - 1, node = i;
    uint32_t bits = 0;
    auto put = [&](int j) {
      for (; at > j / 32; --at) {
        to[at] = bits;
        bits = 0;
      }
      bits |= 1u << (j % 32);
    };
    if (p >= -1) {
      put(i);
      while (p >= 0 && p < node) {
        const int above = up[p];
        if (above < -1) break;  // (there is no such row)
        put(p);
        node = p;
        p = above;
      }
    }
    for (; at >= 0; --at) {
      to[at] = bits;
      bits = 0;
    }
  }
  if constexpr (LDS) {
    __syncthreads();
    uint32_t* const to = mask + ((int64_t)b * n + first) * words;
    const int count = min(n - first, kMaskThreads) * words, pitch = words | 1;
    for (int j = threadIdx.x; j < count; j += kMaskThreads) to[j] = own_words[j / words * pitch + j % words];
  }
}

// How the tiles are dealt out.
struct Deal {
  bool wide;      // 128 query rows a workgroup
  int tile_rows, qtiles, part_rows;
  int chunk;      // tiles of a unit, or 0: a unit per head
  int64_t units;  // at most
};
constexpr int kSharedUnits = 16;  // units of a head on average above which a query row's partial results are read by a whole workgroup

// What a launch of each kernel takes, in us: start + round * rounds + steps * step, from launches of 2 ... 64 heads, 48 ... 1792 query rows and 200 ... 32000
// rows a head.  Both sides: 32 heads x 160 rows x 1000, whole 17, dealt out 27; 4 heads x 256 rows x 4000 16.6 by 32 rows a
// workgroup, 26 by 128; 4 heads of seven x 64 rows x 32000 84 and 49; 64 heads of seven x 256 x 200 128 and 49.
struct Form {
  int tile_rows, keys;  // query rows of a workgroup, keys of a tile
  int tiles;            // that its waves take in one step
  int least;            // tiles of a unit
  int at_once;          // workgroups of a compute unit
  float start, round;   // the launch; the first loads, the merging and the last stores of each round of workgroups
  float step;           // of a workgroup alone on its compute unit
  float beside;         // ... of one that shares it: so many times that, for each
};
constexpr float kJoin = 4.f, kPart = 0.15f;  // the second kernel, and a million bytes of partial results, written and read

Form form_of(const maskkv_desc* d, bool wide) {
  const bool small = d->d == 64;
  if (wide) return {kWideQueries, kWideTile, 1, 4, 2, 8.f, 0.f, small ? 0.85f : 1.3f, 0.8f};
  if (d->dtype == MASKKV_BF16) return {kTile, kTile, 8, 8, small ? 2 : 1, 3.f, 6.f, small ? 0.9f : 1.45f, 0.8f};
  return {kTile, kTile, small ? 8 : 4, small ? 8 : 4, 1, 2.f, 4.f, small ? 4.f : 5.5f, 1.f};
}
// Units that a launch is dealt out into, at most: of any capacity.
int64_t most_units(const Form& f, int qtiles, int64_t BH) {
  const int64_t wanted = f.at_once * kUnits / qtiles + 1;
  return (wanted > BH ? wanted : BH) + BH;
}
// Tiles that a head has, at most.
int64_t longest_of(const maskkv_desc* d, const Form& f, int64_t capacity) {
  return (d->P_max < capacity ? d->P_max : capacity) / f.keys + 1 + (d->n_resp + f.keys - 1) / f.keys;
}

Deal deal_of(const maskkv_desc* d, int64_t capacity) {
  const int n_q = query_heads_per_kv(d) * d->n_resp;
  const int64_t BH = (int64_t)d->B * d->H;
  Deal best;
  float best_cost = -1.f;
  for (int wide = 0; wide < (d->dtype == MASKKV_BF16 && n_q > kWideQueries / 2 ? 2 : 1); ++wide) {
    const Form f = form_of(d, wide);
    const int qtiles = (n_q + f.tile_rows - 1) / f.tile_rows;
    const int64_t resp = (d->n_resp + f.keys - 1) / f.keys, longest = longest_of(d, f, capacity);
    const float tiles = (float)(BH * resp + capacity / f.keys) + 0.5f * BH, mean = tiles / BH;  // (half a tile of a head is empty, on average)
    auto cost = [&](float units, float steps) {
      const float wgs = units * qtiles, rounds = ceilf(wgs / (f.at_once * kUnits));
      const float step = wgs <= kUnits ? f.step : f.step * f.beside * f.at_once;
      return f.start + rounds * (f.round + ceilf(steps) * step);
    };
    auto take = [&](float us, int64_t chunk) {
      if (best_cost >= 0.f && us >= best_cost) return;
      best_cost = us;
      best = {wide != 0, f.tile_rows, qtiles, n_q < f.tile_rows ? n_q : f.tile_rows, (int)chunk, BH};
      if (chunk) best.units = (capacity / f.keys + BH * (resp + 1)) / chunk + BH;
    };
    // A whole head: the host does not know their lengths, but that none is longer than the longest prompt.
    const float whole = fminf((float)longest, fmaxf(1.25f * mean, 0.25f * longest));
    take(cost((float)BH, whole / f.tiles), 0);
    auto dealt = [&](float wanted) {
      int64_t chunk = (int64_t)fmaxf(ceilf(wanted), (float)f.least);
      chunk = (chunk + f.tiles - 1) / f.tiles * f.tiles;
      if (chunk >= longest || (capacity / f.keys + BH * (resp + 1)) / chunk + BH > most_units(f, qtiles, BH)) return;
      const float units = fmaxf(tiles / chunk + 0.5f * BH, BH * ceilf(mean / chunk));
      take(cost(units, fminf((float)chunk, mean) / f.tiles) + kJoin + kPart * units * n_q * d->d * 4e-6f, chunk);
    };
    for (int k = 1; k <= f.at_once; ++k) {  // a unit for every compute unit, or for every place in them:
      const float places = (float)(k * kUnits) / qtiles;
      dealt(tiles / fmaxf(places - 0.5f * BH, 0.5f * BH));  // for heads of any length, of which half a unit is empty,
      dealt(mean / fmaxf(floorf(places / BH), 1.f));        // and for heads of one length
    }
  }
  return best;
}

bool shared_rows(const Deal& x, int64_t BH) { return x.chunk && x.units > kSharedUnits * BH; }

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

size_t bytes_of(const maskkv_desc* d, int64_t units, int qtiles, int part_rows) {
  const size_t rows = (size_t)units * qtiles * part_rows;
  return pad256(rows * d->d * 4) + pad256(rows * 8) + pad256((size_t)d->B * d->H * 8);
}

template <typename T, int D>
int launch_one(const TreeParams& prm, const Deal& deal, hipStream_t stream) {
  static_assert(TreeCfg<T, D>::kLds <= 160 * 1024, "a workgroup's LDS");
  auto kernel = &attend_tree_kernel<T, D>;
  int lds = TreeCfg<T, D>::kLds, threads = TreeCfg<T, D>::kThreads;
  if constexpr (sizeof(T) == 2) {
    if (deal.wide) {
      kernel = &attend_tree_wide_kernel<D>;
      lds = WideCfg<D>::kLds;
      threads = 256;
    }
  }
  const int64_t groups = deal.units * deal.qtiles;
  if (groups * threads > 0xFFFFFFFF) {  // (threads of a launch along a dimension)
    set_error("attend_tree: %lld workgroups are more than a launch can have", (long long)groups);
    return MASKKV_ESHAPE;
  }
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) {
    set_error("attend_tree: hipFuncSetAttribute: %s", hipGetErrorString(e));
    (void)hipGetLastError();
    return MASKKV_EHIP;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), lds, stream, prm);
  if (int e = check_launch("attend_tree")) return e;
  if (!deal.chunk) return MASKKV_OK;
  if (shared_rows(deal, prm.BH))
    hipLaunchKernelGGL((attend_tree_join_kernel<T, D, true>), dim3((unsigned)prm.n_q, (unsigned)prm.BH), dim3(kJoinGroups * D / 4), 0, stream, prm);
  else
    hipLaunchKernelGGL((attend_tree_join_kernel<T, D, false>), dim3((unsigned)(prm.n_q + kJoinGroups - 1) / kJoinGroups, (unsigned)prm.BH),
                       dim3(kJoinGroups * D / 4), 0, stream, prm);
  return check_launch("attend_tree (join)");
}

}  // namespace

size_t attend_tree_needs(const maskkv_desc* d, int64_t capacity) {
  const Deal x = deal_of(d, capacity);
  return x.chunk ? bytes_of(d, x.units, x.qtiles, x.part_rows) : 0;
}

AttendTreePlan attend_tree_plan(const maskkv_desc* d, int64_t capacity) {
  const Deal x = deal_of(d, capacity);
  return {x.tile_rows, x.qtiles, x.chunk, x.units, shared_rows(x, (int64_t)d->B * d->H), attend_tree_needs(d, capacity)};
}

// (No unit is dealt out where no head has more tiles than the least of a unit.)
size_t attend_tree_workspace_bytes(const maskkv_desc* d, int64_t capacity) {
  const int n_q = query_heads_per_kv(d) * d->n_resp;
  size_t most = 0;
  for (int wide = 0; wide < (d->dtype == MASKKV_BF16 && n_q > kWideQueries / 2 ? 2 : 1); ++wide) {
    const Form f = form_of(d, wide);
    const int qtiles = (n_q + f.tile_rows - 1) / f.tile_rows;
    if (longest_of(d, f, capacity) <= f.least) continue;
    const size_t bytes = bytes_of(d, most_units(f, qtiles, (int64_t)d->B * d->H), qtiles, n_q < f.tile_rows ? n_q : f.tile_rows);
    most = bytes > most ? bytes : most;
  }
  return most;
}

int launch_attend_tree(const maskkv_desc* d, const View& Q, const void* Kc, const void* Vc, const int32_t* cu_budget, int64_t capacity,
                       const View& K2, const View& V2, const uint32_t* mask, float scale, const View& O, float* lse, void* workspace,
                       hipStream_t stream) {
  const Deal deal = deal_of(d, capacity);
  TreeParams prm;
  prm.Q = Q;
  prm.K2 = K2;
  prm.V2 = V2;
  prm.O = O;
  prm.Kc = reinterpret_cast<const char*>(Kc);
  prm.Vc = reinterpret_cast<const char*>(Vc);
  prm.cu = cu_budget;
  prm.mask = mask;
  prm.capacity = capacity;
  prm.H = d->H;
  prm.BH = d->B * d->H;
  prm.q_per_kv = query_heads_per_kv(d);
  prm.n_resp = d->n_resp;
  prm.n_q = prm.q_per_kv * d->n_resp;
  prm.words = (d->n_resp + 31) / 32;
  prm.qtiles = deal.qtiles;
  prm.units = (int)deal.units;
  prm.chunk = deal.chunk;
  prm.tile_rows = deal.tile_rows;
  prm.part_rows = deal.part_rows;
  prm.c = scale * kLog2e;
  prm.lse = lse;
  const size_t rows = (size_t)deal.units * deal.qtiles * deal.part_rows;
  char* ws = reinterpret_cast<char*>(workspace);
  prm.part_o = reinterpret_cast<float*>(ws);
  prm.part_ml = reinterpret_cast<float2*>(ws + pad256(rows * d->d * 4));
  prm.parts = reinterpret_cast<int2*>(ws + pad256(rows * d->d * 4) + pad256(rows * 8));
  if (d->dtype == MASKKV_BF16)
    return d->d == 128 ? launch_one<bf16_t, 128>(prm, deal, stream) : launch_one<bf16_t, 64>(prm, deal, stream);
  return d->d == 128 ? launch_one<float, 128>(prm, deal, stream) : launch_one<float, 64>(prm, deal, stream);
}

int launch_tree_mask(const int32_t* parents, int B, int n, uint32_t* mask, hipStream_t stream) {
  const auto kernel = n <= kTreeRows ? &tree_mask_kernel<true> : &tree_mask_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((n + kMaskThreads - 1) / kMaskThreads), (unsigned)B), dim3(kMaskThreads), 0, stream, parents, n,
                     (n + 31) / 32, mask);
  return check_launch("tree_mask");
}

}  // namespace maskkv
