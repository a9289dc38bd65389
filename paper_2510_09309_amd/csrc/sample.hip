// Tokens from logits, with given random numbers: temperature, top-k, top-p, min-p.
//
// Two kernels.  The first reads every row once: a wave takes a part of a row (4 KB) and leaves its largest logit, its mass relative to that
// at the row's temperature and at temperature 1, and, where the row has limits, the largest logit of each group of 128 bytes.  The second
// has a workgroup a row: it adds up the parts and, without limits, reads the one part again in which the wanted mass is reached.  With limits,
// the groups' largest logits say how small a token that stays can be (`floor_of`): few groups reach that, and the tokens of these that do are ranked in
// LDS (`draw_few`).  Where too many do, a top-p's last token is looked for between two bounds of the row's masses (`draw_between`); what is left - a top-k of
// thousands, thousands of equal logits - takes histograms over all bits of the logits' order (`border_of`), and the row is read part by part again.
//
// Which token is drawn must not depend on roundings: in a flat row of 10^5 tokens an error of 10^-7 of the mass is a hundredth of a token.
// Masses are therefore 64 bits wide from the exponential on: 2^f on [-1/2, 1/2] as 1 + f q(f), q the polynomial of degree 8 through
// (2^f - 1)/f at nine Chebyshev points, off by 4e-14, on a vector unit that does 64-bit operations at the rate of 32-bit ones.
// Histograms add up whole numbers, so that the order in which threads come to them has no part in the result.
//
// The one exception is the confidence of bf16 rows, whose terms are fp32 exponentials added up in 64 bits: nothing is drawn by them.
//
// Bound by the vector pipe where all masses are needed: 256 rows of 126464 (65 MB, 12.7 us at a copy's rate) 36.0 + 5.7 us, the pipe busy all of the
// first kernel's time with 34 instructions a logit: 17 for its mass (16 of them in 64 bits), the others for its term of the confidence, the largest logits and
// what a logit is read with.  By latency where masses are not needed: one row of 32001 with top-k and top-p 4.5 + 10.4 us.
// By one compute unit in a nearly flat row with a top-p: 64 rows of 152064 with mixed limits 33 us a call where no row is, 96 to 117 where one is; and in a row
// that is searched whole, 64 of 152064 with a top-k of 50000 and a top-p 340.
// (Such rows dealt to the whole chip by three launches more: 64 rows with mixed limits 129 -> 94 us and 64 rows with a top-p at temperature 1.4 120 -> 115, but
// sharp ones 27.5 -> 32.5, 256 of 126464 48.8 -> 55.3, 100 of 50000 with a top-k 16.7 -> 22.5.)
#include <type_traits>

#include "kernels.hpp"

namespace maskkv {

namespace {

constexpr int kPartBlocks = 256;  // blocks of 16 bytes of a row's part
constexpr int kLoads = kPartBlocks / 64;
constexpr int kGroupBlocks = 8;   // ... of a group
constexpr int kGroups = kPartBlocks / kGroupBlocks;

struct Part {
  double mass;   // sum of exp((l - top) / temperature)
  double plain;  // sum of exp(l - top)
  union {
    float top;   // largest logit
    int first;   // once that is known: where its tokens lie in a list,
  };
  int many;      // and how many
  __device__ Part() {}
  __device__ Part(double a, double b, float c) : mass(a), plain(b), top(c), many(0) {}
  __device__ Part(double a, double b, int c, int n) : mass(a), plain(b), first(c), many(n) {}
};

struct SampleParams {
  const char* logits;
  int64_t row_bytes;
  int rows, V, parts;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniform;
  int32_t* token;
  float* prob;
  float* logprob;
  Part* part;    // [rows][parts]
  float* group;  // [rows][parts * kGroups]
};

// What a row is drawn with.
struct Limits {
  float T;
  int k;        // 0: none
  float p, m;   // 1, 0: none
  bool greedy, some, masses;  // masses: those of all tokens are needed
  __device__ __forceinline__ Limits(const SampleParams& prm, int r) {
    T = prm.temperature ? prm.temperature[r] : 1.f;
    k = prm.top_k ? prm.top_k[r] : 0;
    p = prm.top_p ? prm.top_p[r] : 1.f;
    m = prm.min_p ? prm.min_p[r] : 0.f;
    if (k <= 0 || k >= prm.V) k = 0;
    if (!(p < 1.f)) p = 1.f;
    if (!(m > 0.f)) m = 0.f;
    if (m > 1.f) m = 1.f;
    greedy = !(T > 0.f);
    some = !greedy && (k || p < 1.f || m > 0.f);
    masses = !greedy && !k && (p < 1.f || !(m > 0.f));
  }
  // (at an infinite temperature all finite logits have one mass, and -infinity none)
  __device__ __forceinline__ double c() const { return fmax(1.4426950408889634074 / (double)T, 1e-290); }
};

// 2^t for t = d * c, t <= 0, d >= -1000 / c: what is below 2^-1000, or NaN, is 2^-1000, which is nothing beside the largest one's 1; 2^0 is 1 exactly.
// A sum with 1.5 * 2^52 rounds t to a whole number, which is the low word of the sum; it is added to the exponent as it is.
struct Power {
  double c, least, first;  // first: of the polynomial's coefficients
  __device__ __forceinline__ explicit Power(double by) : c(by), least(-1000.0 / by), first(1.0203121070622722e-07) {
    asm("" : "+v"(first));  // (two constants are more than an instruction takes: this one in registers, once)
  }
  __device__ __forceinline__ double operator()(double d) const {
    constexpr double kRound = 0x1.8p52;
    d = fmax(d, least);
    const double n = fma(d, c, kRound), f = fma(d, c, kRound - n);
    double q = first;
    q = fma(q, f, 1.325522487501112e-06);
    q = fma(q, f, 1.5252686846270554e-05);
    q = fma(q, f, 0.00015403455852469646);
    q = fma(q, f, 0.0013333558179043094);
    q = fma(q, f, 0.00961812915940254);
    q = fma(q, f, 0.055504108664760424);
    q = fma(q, f, 0.2402265069581299);
    q = fma(q, f, 0.6931471805599453);
    const double m = fma(q, f, 1.0);
    return __hiloint2double(__double2hiint(m) + (__double2loint(n) << 20), __double2loint(m));
  }
  // The mass of a logit relative to the largest one.
  __device__ __forceinline__ double of(float l, float top) const { return (*this)((double)l - (double)top); }
};
constexpr double kLog2e64 = 1.4426950408889634074;

// A row in blocks of 16 bytes that begin at multiples of 16 bytes: its first and last one may be another row's in part.
template <typename T>
struct Row {
  static constexpr int E = 16 / (int)sizeof(T);
  const char* first;  // block 0
  int lead, V, blocks;
  __device__ __forceinline__ Row(const SampleParams& prm, int r) {
    const char* p = prm.logits + (int64_t)r * prm.row_bytes;
    lead = (int)((uintptr_t)p & 15) / (int)sizeof(T);
    first = p - lead * (int)sizeof(T);
    V = prm.V;
    blocks = (V + lead + E - 1) / E;
  }
  __device__ __forceinline__ int number(int block) const { return block * E - lead; }  // of a block's first element
  __device__ __forceinline__ bool whole(int block) const { return number(block) >= 0 && number(block) + E <= V; }
  __device__ __forceinline__ u32x4 load(int block) const { return *reinterpret_cast<const u32x4*>(first + (int64_t)block * 16); }
  __device__ __forceinline__ static void spread(const u32x4& w, float (&x)[E]) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const uint32_t u = sizeof(T) == 4 ? w[i] : w[i / 2];
      // (-0 counts as 0, NaN as -infinity)
      x[i] = fmaxf(as_f32(sizeof(T) == 4 ? u : i % 2 ? u & 0xFFFF0000u : u << 16) + 0.f, -INFINITY);
    }
  }
  // Elements of a block that is not wholly this row's: -infinity for the others.
  __device__ __forceinline__ void edge(int block, float (&x)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int at = number(block) + i;
      float v = -INFINITY;
      if (at >= 0 && at < V) {
        const char* p = first + ((int64_t)block * 16 + i * (int)sizeof(T));
        v = sizeof(T) == 4 ? *reinterpret_cast<const float*>(p) : as_f32((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
      }
      x[i] = fmaxf(v + 0.f, -INFINITY);
    }
  }
  __device__ __forceinline__ void read(int block, float (&x)[E]) const {
    if (whole(block))
      spread(load(block), x);
    else
      edge(block, x);
  }
};
// Where a row's largest logit is +infinity, its infinite logits count as 0 and the others as -infinity.
__device__ __forceinline__ float finite_top(float l) { return l == INFINITY ? 0.f : -INFINITY; }

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return as_f32((uint32_t)__builtin_amdgcn_update_dpp(0, (int)as_u32(v), CTRL, 0xf, 0xf, false));
}
// The largest of eight, of all lanes.
__device__ __forceinline__ float max_eight(float v) {
  v = fmaxf(v, dpp<0xB1>(v));   // neighbours
  v = fmaxf(v, dpp<0x4E>(v));   // pairs
  return fmaxf(v, dpp<0x141>(v));  // halves of eight
}
__device__ __forceinline__ float max_wave(float v) {
  v = max_eight(v);
  v = fmaxf(v, dpp<0x140>(v));  // halves of sixteen
  const auto x = __builtin_amdgcn_permlane16_swap(as_u32(v), as_u32(v), false, false);
  const uint32_t a = x[0], b = x[1];
  return max_halves(fmaxf(as_f32(a), as_f32(b)));
}
__device__ __forceinline__ double sum_wave(double v) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) v += __shfl_xor(v, i);
  return v;
}

// ---- every part of every row
template <typename T>
__global__ __launch_bounds__(256) void sample_parts_kernel(const SampleParams prm) {
  constexpr int E = Row<T>::E;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t task = (int64_t)blockIdx.x * 4 + wave;
  const int r = (int)(task / prm.parts), i = (int)(task - (int64_t)r * prm.parts);
  if (r >= prm.rows) return;
  const Row<T> row(prm, r);
  float x[kLoads][E];
  {
    u32x4 w[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int block = i * kPartBlocks + j * 64 + lane;
      if (block < row.blocks && row.whole(block)) w[j] = row.load(block);
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int block = i * kPartBlocks + j * 64 + lane;
      if (block >= row.blocks) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[j][e] = -INFINITY;
      } else if (row.whole(block)) {
        row.spread(w[j], x[j]);
      } else {
        row.edge(block, x[j]);
      }
    }
  }
  const Limits lim(prm, r);
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    float most = x[j][0];
#pragma unroll
    for (int e = 1; e < E; ++e) most = fmaxf(most, x[j][e]);
    if (lim.some) {
      const float of_group = max_eight(most);
      if (lane % kGroupBlocks == 0)
        prm.group[((int64_t)r * prm.parts + i) * kGroups + j * (64 / kGroupBlocks) + lane / kGroupBlocks] = of_group;
    }
    top = fmaxf(top, most);
  }
  top = max_wave(top);
  float ref = top;
  if (top == INFINITY) {
    ref = 0.f;
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
      for (int e = 0; e < E; ++e) x[j][e] = finite_top(x[j][e]);
  }
  double mass = 0.0, plain = 0.0;
  if (ref > -INFINITY) {
    if (prm.logprob) {
      const Power plainly(kLog2e64);
      // (of bf16 the differences are exact but for logits below 2^-12 or so; of fp32 they are not)
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e)
          plain += sizeof(T) == 2 ? (double)fast_exp2((x[j][e] - ref) * kLog2e) : plainly.of(x[j][e], ref);
    }
    if (lim.masses) {
      const Power power(lim.c());
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) mass += power.of(x[j][e], ref);
    }
  }
  if (prm.logprob) plain = sum_wave(plain);
  if (lim.masses) mass = sum_wave(mass);
  if (lane == 0) prm.part[(int64_t)r * prm.parts + i] = Part(mass, plain, top);
}

// ---- a token for every row
constexpr int kBins = 1024;      // of the groups' largest logits
constexpr int kWide = 2048;      // bins of a row's logits
constexpr int kFewGroups = 4096; // that are looked into, at most
constexpr int kRounds = 4;       // groups of a thread that are asked for at once
constexpr int kFew = 2048;       // tokens that are ranked, at most
constexpr int kList = 4096;      // tokens among which the last one that stays is looked for, at most
constexpr int kDigits = 2048;    // values of eleven bits

template <int N>
struct AskShared {
  double sums[2][N / 64];
  int ints[2][N / 64];
  float floats[2][2][N / 64];
  int found;
  int count;
  double value;
};
// (rows without limits need no more)
template <int N>
struct DrawShared : AskShared<N> {
  union {
    struct {
      uint32_t count[kBins];
      unsigned long long mass[kBins];
    } bins;
    unsigned long long wide[kWide];  // how many there are (from kCountAt on), and the sum of how far they lie in the bin, in 2^-15
    struct {
      uint32_t count[kDigits];
      unsigned long long mass[kDigits];
    } digits;
    double ranked[kFew];  // in the order of their ranks: the mass before each
  };
  float logit[kList];
  int number[kList];
  uint32_t groups[kFewGroups];
  int rounds[2][kRounds][N / 64];
  int taken;
  unsigned long long whole;
  uint32_t key;
};

// What is added up over the lanes up to this one: inside rows of sixteen by shifts, then the ends of rows into the rows behind.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned long long shifted(unsigned long long v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  return (unsigned long long)hi << 32 | lo;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted(double v) {
  return __builtin_bit_cast(double, shifted<CTRL, ROWS>(__builtin_bit_cast(unsigned long long, v)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int shifted(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
template <typename V>
__device__ __forceinline__ V upto_lane(V v) {
  v += shifted<0x111, 0xf>(v);
  v += shifted<0x112, 0xf>(v);
  v += shifted<0x114, 0xf>(v);
  v += shifted<0x118, 0xf>(v);
  v += shifted<0x142, 0xa>(v);
  v += shifted<0x143, 0xc>(v);
  return v;
}

// What all N threads of a workgroup ask each other.  `turn` alternates between two places, so that one barrier a question is enough.
template <int N>
struct Ask {
  static constexpr int kWaves = N / 64;
  AskShared<N>& s;
  int turn = 0;
  __device__ __forceinline__ explicit Ask(AskShared<N>& shared) : s(shared) {}
  __device__ __forceinline__ int wave() const { return threadIdx.x >> 6; }
  __device__ __forceinline__ int lane() const { return threadIdx.x & 63; }
  // The sum before this thread; of all in `total`.
  template <typename V>
  __device__ __forceinline__ V before_in(V* places, V v, V& total) {
    const V upto = upto_lane(v);
    if (lane() == 63) places[wave()] = upto;
    __syncthreads();
    V base = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave()) base = total;
      total += places[w];
    }
    // (of masses not `upto - v`, which would round once more: the lane before has it)
    return base + shifted<0x138, 0xf>(upto);
  }
  __device__ __forceinline__ double before(double v, double& total) {
    turn ^= 1;
    return before_in(s.sums[turn], v, total);
  }
  __device__ __forceinline__ unsigned long long before(unsigned long long v, unsigned long long& total) {
    turn ^= 1;
    return before_in(reinterpret_cast<unsigned long long*>(s.sums[turn]), v, total);
  }
  __device__ __forceinline__ int before(int v, int& total) {
    turn ^= 1;
    return before_in(s.ints[turn], v, total);
  }
  // The first (last) thread for which it is so, or -1.
  __device__ __forceinline__ int first(bool so) {
    const uint64_t b = __ballot(so);
    turn ^= 1;
    if (lane() == 0) s.ints[turn][wave()] = b ? (wave() << 6) + __builtin_ctzll(b) : -1;
    __syncthreads();
    int v = -1;
#pragma unroll
    for (int w = kWaves - 1; w >= 0; --w) v = s.ints[turn][w] >= 0 ? s.ints[turn][w] : v;
    return v;
  }
  __device__ __forceinline__ int last(bool so) {
    const uint64_t b = __ballot(so);
    turn ^= 1;
    if (lane() == 0) s.ints[turn][wave()] = b ? (wave() << 6) + 63 - __builtin_clzll(b) : -1;
    __syncthreads();
    int v = -1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v = s.ints[turn][w] >= 0 ? s.ints[turn][w] : v;
    return v;
  }
  __device__ __forceinline__ void most(float& a, float& b) {
    a = max_wave(a);
    b = max_wave(b);
    turn ^= 1;
    if (lane() == 0) {
      s.floats[turn][0][wave()] = a;
      s.floats[turn][1][wave()] = b;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      a = fmaxf(a, s.floats[turn][0][w]);
      b = fmaxf(b, s.floats[turn][1][w]);
    }
  }
};

// A logit's place in the order of all, as a whole number (of bf16 16 bits are enough).
template <typename T>
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t u = as_u32(l), key = u & 0x80000000u ? ~u : u | 0x80000000u;
  return sizeof(T) == 2 ? key >> 16 : key;
}
template <typename T>
__device__ __forceinline__ float logit_of(uint32_t key) {
  const uint32_t k = sizeof(T) == 4 ? key : key & 0x8000u ? key << 16 : key << 16 | 0xFFFFu;
  return as_f32(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// kDraw threads draw the token of a row.
template <typename T, int kDraw, typename Shared>
struct Drawer {
  static constexpr int E = Row<T>::E, kWaves = kDraw / 64;
  static constexpr int kCounted = kDraw / 2;  // tokens that are ranked by comparing each with each
  static_assert(kDraw >= kPartBlocks, "a part is drawn from by a thread a block");
  const SampleParams& prm;
  Shared& s;
  Ask<kDraw> ask;
  const Row<T> row;
  const Limits lim;
  const int r;
  Part* const part;
  const float* const group;
  const int groups, groups_each, parts_each;  // of the row; of a thread
  float4 first_groups;                        // the first of a thread
  float top = 0.f, ref = 0.f;                 // the largest logit, and what masses are relative to
  float least = 0.f;                          // the smallest of the groups' largest
  const Power power;           // with the temperature
  double u = 0.0;
  double masses = 0.0, plain = 0.0;  // of all tokens
  double mine = 0.0;                 // of this thread's parts, and before them
  double before = 0.0;
  int number = -1;  // the token,
  double prob = 0.0;

  __device__ __forceinline__ Drawer(const SampleParams& p, Shared& shared, int number)
      : prm(p), s(shared), ask(shared), row(p, number), lim(p, number), r(number), part(p.part + (int64_t)number * p.parts),
        group(p.group + (int64_t)number * p.parts * kGroups), groups((row.blocks + kGroupBlocks - 1) / kGroupBlocks),
        groups_each((groups + 4 * kDraw - 1) / (4 * kDraw) * 4), parts_each((p.parts + kDraw - 1) / kDraw), power(lim.greedy ? 1.0 : lim.c()) {}

  __device__ __forceinline__ float seen(float l) const { return top == INFINITY ? finite_top(l) : l; }
  __device__ __forceinline__ void read(int block, float (&x)[E]) const {
    row.read(block, x);
    if (top == INFINITY) {
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = finite_top(x[e]);
    }
  }
  // (What is about 2^-1000 is nothing: a part of which no token has a mass is none that is drawn from.)
  static __device__ __forceinline__ double or_nothing(double m, double least) { return m > least ? m : 0.0; }
  __device__ __forceinline__ double mass(float l) const { return or_nothing(power.of(l, ref), 0x1p-999); }
  __device__ __forceinline__ double part_unit(float part_top, const Power& by) const {
    return part_top == top ? 1.0 : top == INFINITY ? 0.0 : or_nothing(by.of(part_top, ref), 0x1p-990);
  }
  // This thread's parts, and its groups' largest logits in their order (f(logit, group)).
  __device__ __forceinline__ int from_part() const { return min((int)threadIdx.x * parts_each, prm.parts); }
  __device__ __forceinline__ int to_part() const { return min((int)(threadIdx.x + 1) * parts_each, prm.parts); }
  template <typename F>
  __device__ __forceinline__ void each_group(F f) {
    const int from = threadIdx.x * groups_each;
    for (int i = 0; i < groups_each && from + i < groups; i += 4) {
      const float4 v = i ? *reinterpret_cast<const float4*>(group + from + i) : first_groups;
      if (from + i < groups) f(v.x, from + i);
      if (from + i + 1 < groups) f(v.y, from + i + 1);
      if (from + i + 2 < groups) f(v.z, from + i + 2);
      if (from + i + 3 < groups) f(v.w, from + i + 3);
    }
  }

  __device__ __forceinline__ void answer() {
    if (threadIdx.x) return;
    prm.token[r] = number;
    if (prm.prob) prm.prob[r] = (float)prob;
    if (prm.logprob) {
      float l = -INFINITY;
      if (number >= 0) {
        const char* p = prm.logits + (int64_t)r * prm.row_bytes + (int64_t)number * (int)sizeof(T);
        l = sizeof(T) == 4 ? *reinterpret_cast<const float*>(p) : as_f32((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
        l = (float)((double)seen(l) - (double)ref - log(plain));
      }
      prm.logprob[r] = l;
    }
  }

  // The parts together.
  __device__ __forceinline__ void sum_up() {
    const int from = from_part(), to = to_part();
    Part one;
    one.top = -INFINITY;
    if (from < to) one = part[from];
    if (lim.some && (int)threadIdx.x * groups_each < groups) first_groups = *reinterpret_cast<const float4*>(group + threadIdx.x * groups_each);
    float most = -INFINITY, low = -INFINITY;
    for (int i = from; i < to; ++i) most = fmaxf(most, i == from ? one.top : part[i].top);
    if (lim.some) each_group([&](float l, int) { low = l > -INFINITY ? fmaxf(low, -l) : low; });
    ask.most(most, low);
    top = most;
    ref = top == INFINITY ? 0.f : top;
    least = top == INFINITY ? 0.f : -low;
    double own = 0.0;
    const Power plainly(kLog2e64);
    for (int i = from; i < to; ++i) {
      const Part x = i == from ? one : part[i];
      if (lim.masses) mine += x.mass * part_unit(x.top, power);
      if (prm.logprob) own += x.plain * part_unit(x.top, plainly);
    }
    if (prm.logprob) ask.before(own, plain);
    if (lim.masses) before = ask.before(mine, masses);
  }

  __device__ __forceinline__ void greedy() {
    const int from = from_part(), to = to_part();
    int own = -1;
    for (int i = to - 1; i >= from; --i)
      if (part[i].top == top) own = i;
    const int who = ask.first(own >= 0);
    if ((int)threadIdx.x == who) s.found = own;
    __syncthreads();
    const int block = s.found * kPartBlocks + threadIdx.x;
    int at = -1;
    if (threadIdx.x < kPartBlocks && block < row.blocks) {
      float x[E];
      row.read(block, x);
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (x[e] == top) at = row.number(block) + e;
    }
    const int has = ask.first(at >= 0);
    if ((int)threadIdx.x == has) s.count = at;
    __syncthreads();
    number = s.count;
    prob = 1.0;
  }

  // The thread in whose masses (`own`, behind `base`) `target` is exceeded, or the last one with any.
  __device__ __forceinline__ int thread_with(double target, double own, double base) {
    const int who = ask.first(own > 0.0 && base + own > target);
    return who >= 0 ? who : ask.last(own > 0.0);  // (roundings)
  }

  // Of the parts' masses (own: of a thread's, behind `base`) the part in which `target` is exceeded, or the last one with any.
  template <typename F>
  __device__ __forceinline__ int part_with(double target, double own, double base, F mass_in, double& base_of_part) {
    const int who = thread_with(target, own, base);
    if ((int)threadIdx.x == who) {
      int at = from_part();
      double sum = base, before_it = base;
      for (int i = from_part(); i < to_part(); ++i) {
        const double m = mass_in(i);
        if (m > 0.0) {
          at = i;
          before_it = sum;
        }
        sum += m;
        if (m > 0.0 && sum > target) break;
      }
      s.found = at;
      s.value = before_it;
    }
    __syncthreads();
    base_of_part = s.value;
    return s.found;
  }

  // Where the token is: in part i, before which the tokens that stay have the mass `base` and `equal` tokens are as large as `last`: those above
  // `last` stay, and of its equals the first `left`.
  struct Where {
    int i;
    double base, target, total;
    float last;
    int equal, left;
  };
  __device__ __forceinline__ void draw_in(const Where& w) {
    const int block = w.i * kPartBlocks + threadIdx.x;
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = -INFINITY;
    if (threadIdx.x < kPartBlocks && block < row.blocks) read(block, x);
    int nth = 0;
    if (w.last > -INFINITY) {
      int same = 0, all;
#pragma unroll
      for (int e = 0; e < E; ++e) same += x[e] == w.last;
      nth = w.equal + ask.before(same, all);
    }
    double m[E], own = 0.0, unused;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool stays = x[e] > w.last || (x[e] == w.last && nth < w.left);
      nth += x[e] == w.last;
      const double y = mass(x[e]);
      m[e] = stays && x[e] > -INFINITY && y >= (double)lim.m ? y : 0.0;
      own += m[e];
    }
    const double from = w.base + ask.before(own, unused);
    const int who = thread_with(w.target, own, from);
    if ((int)threadIdx.x == who) {
      double sum = from;
      int at = 0;
      bool done = false;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (m[e] > 0.0 && !done) {
          at = e;
          sum += m[e];
          done = sum > w.target;
          s.value = m[e];
        }
      }
      s.found = row.number(block) + at;
    }
    __syncthreads();
    number = s.found;
    prob = s.value / w.total;
  }

  __device__ __forceinline__ Where draw_all() {
    double base;
    const double target = u * masses;
    const int i = part_with(target, mine, before, [&](int j) { return part[j].mass * part_unit(part[j].top, power); }, base);
    return {i, base, target, masses, -INFINITY, 0, 0};
  }

  // ---- few tokens stay
  float slope = 0.f;
  int mass_floor = 0;  // what top-p alone asks for
  __device__ __forceinline__ int bin_of(float l) const { return (int)fminf((ref - l) * slope, kBins - 1.f); }

  // The lowest of the bins of logits in which a token that stays can be (from the largest logit down to the smallest of the groups' largest in
  // equal steps).  With a top-k as many groups' largest logits lie above; with a top-p, so much of their mass.
  __device__ __forceinline__ int floor_of() {
    const bool by_mass = lim.masses && lim.p < 1.f;
    for (int i = threadIdx.x; i < kBins; i += kDraw) {
      s.bins.count[i] = 0;
      s.bins.mass[i] = 0;
    }
    slope = least < ref ? (kBins - 1) / (ref - least) : 0.f;
    __syncthreads();
    each_group([&](float l, int) {
      l = seen(l);
      if (l == -INFINITY) return;
      if (lim.k) atomicAdd(&s.bins.count[bin_of(l)], 1u);
      if (by_mass) atomicAdd(&s.bins.mass[bin_of(l)], (unsigned long long)(mass(l) * 0x1p40));
    });
    __syncthreads();
    int floor = kBins - 1;
    constexpr int kOwn = kBins / kDraw;
    auto lower = [&](auto sum_in, auto reached) __attribute__((always_inline)) {  // the first bin up to which the sum has been reached
      decltype(sum_in(0)) own[kOwn], sum = 0, all;
#pragma unroll
      for (int q = 0; q < kOwn; ++q) sum += own[q] = sum_in(threadIdx.x * kOwn + q);
      auto upto = ask.before(sum, all);
      int at = -1;
#pragma unroll
      for (int q = 0; q < kOwn; ++q) {
        upto += own[q];
        if (at < 0 && reached(upto)) at = threadIdx.x * kOwn + q;
      }
      const int who = ask.first(at >= 0);
      if (who == (int)threadIdx.x) s.found = at;
      __syncthreads();
      if (who >= 0) floor = min(floor, s.found);
    };
    if (lim.k) lower([&](int i) { return (int)s.bins.count[i]; }, [&](int n) { return n >= lim.k; });
    if (by_mass) {
      const double goal = masses * (double)lim.p * (1.0 + 1e-9);
      lower([&](int i) { return s.bins.mass[i]; }, [&](unsigned long long m) { return (double)m * 0x1p-40 >= goal; });
    }
    mass_floor = floor;
    // a little below the smallest logit that min_p lets stay (a top-p of what top-k leaves asks for the mass of all of that)
    if (lim.m > 0.f && !(lim.k && lim.p < 1.f)) {
      const float depth = -__builtin_amdgcn_logf(lim.m) * kLn2 * lim.T;
      const float low = ref - (depth * 1.0001f + 1e-4f * (fabsf(ref) + lim.T));
      if (low < ref) floor = min(floor, bin_of(low));
    }
    return floor;
  }

  // The tokens down to a bin into s.logit and s.number, in their order; how many, or -1: too many.
  __device__ __forceinline__ int list_down_to(int floor) {
    int own = 0, chosen;
    each_group([&](float l, int) {
      l = seen(l);
      own += l > -INFINITY && bin_of(l) <= floor;
    });
    int at = ask.before(own, chosen);
    if (chosen > kFewGroups) return -1;
    each_group([&](float l, int i) {
      l = seen(l);
      if (l > -INFINITY && bin_of(l) <= floor) s.groups[at++] = i;
    });
    __syncthreads();
    int n = 0;
    for (int base = 0; base < chosen; base += kRounds * (kDraw / kGroupBlocks)) {
      float x[kRounds][E];
      int block[kRounds], many[kRounds], upto[kRounds];
      ask.turn ^= 1;
#pragma unroll
      for (int q = 0; q < kRounds; ++q) {
        const int g = base + q * (kDraw / kGroupBlocks) + threadIdx.x / kGroupBlocks;
        block[q] = row.blocks;
        if (g < chosen) block[q] = s.groups[g] * kGroupBlocks + threadIdx.x % kGroupBlocks;
#pragma unroll
        for (int e = 0; e < E; ++e) x[q][e] = -INFINITY;
        if (block[q] < row.blocks) read(block[q], x[q]);
      }
#pragma unroll
      for (int q = 0; q < kRounds; ++q) {
        many[q] = upto[q] = 0;
        if (base + q * (kDraw / kGroupBlocks) < chosen) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (bin_of(x[q][e]) > floor) x[q][e] = -INFINITY;
            many[q] += x[q][e] > -INFINITY;
          }
          upto[q] = upto_lane(many[q]);
        }
        if (ask.lane() == 63) s.rounds[ask.turn][q][ask.wave()] = upto[q];
      }
      __syncthreads();
      int sum = n;
#pragma unroll
      for (int q = 0; q < kRounds; ++q)
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          if (w == ask.wave()) upto[q] += sum - many[q];
          sum += s.rounds[ask.turn][q][w];
        }
      n = sum;
      if (n > kFew) return -1;
#pragma unroll
      for (int q = 0; q < kRounds; ++q)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (x[q][e] > -INFINITY) {
            s.logit[upto[q]] = x[q][e];
            s.number[upto[q]] = row.number(block[q]) + e;
            ++upto[q];
          }
    }
    __syncthreads();
    return n;
  }

  // The n tokens of the list and which of them stay (a thread has the tokens kOwn * t on).
  template <int kOwn>
  __device__ __forceinline__ void draw_of(int n, const double (&stay)[kOwn]) {
    double own = 0.0, total;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) own += stay[q];
    const double from = ask.before(own, total), target = u * total;
    const int who = thread_with(target, own, from);
    if ((int)threadIdx.x == who) {
      double upto = from;
      bool done = false;
#pragma unroll
      for (int q = 0; q < kOwn; ++q)
        if (stay[q] > 0.0 && !done) {
          upto += stay[q];
          done = upto > target;
          s.found = s.number[threadIdx.x * kOwn + q];
          s.value = stay[q];
        }
    }
    __syncthreads();
    number = s.found;
    prob = s.value / total;
  }

  // Up to kCounted tokens: each is compared with each, by two threads.
  __device__ __forceinline__ bool draw_counted(int n, bool all_there) {
    const int i = threadIdx.x / 2, half = threadIdx.x & 1;
    const bool in = i < n;
    const float l = in ? s.logit[i] : -INFINITY;
    int rank = 0;
    if (in) {
#pragma unroll 4
      for (int j = half; j < n; j += 2) {
        const float o = s.logit[j];
        rank += o > l || (o == l && j < i);
      }
    }
    rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, false);  // (the neighbour's half)
    const double m = in ? mass(l) : 0.0;
    const bool first_k = !lim.k || rank < lim.k;
    bool stays = in && first_k && m >= (double)lim.m;
    if (lim.p < 1.f) {
      if (in && half == 0) s.ranked[rank] = first_k ? m : 0.0;
      __syncthreads();
      double ranked;
      const double own = threadIdx.x < n ? s.ranked[threadIdx.x] : 0.0;
      const double upto = ask.before(own, ranked);
      if ((int)threadIdx.x < n) s.ranked[threadIdx.x] = upto;
      __syncthreads();
      const double limit = (double)lim.p * (lim.k ? ranked : masses);
      // (roundings: the last one that stays may not be among these)
      if (!lim.k && !all_there && !(ranked >= limit)) return false;
      stays = stays && (rank == 0 || s.ranked[rank] < limit);
    }
    const double stay[1] = {stays && half == 0 ? m : 0.0};
    // (two threads a token: the list is looked up by the pair)
    double total;
    const double from = ask.before(stay[0], total), target = u * total;
    const int who = thread_with(target, stay[0], from);
    if ((int)threadIdx.x == who) {
      s.found = s.number[i];
      s.value = m;
    }
    __syncthreads();
    number = s.found;
    prob = s.value / total;
    return true;
  }

  // The tokens of a list, or all of the row where n is negative.
  template <typename F>
  __device__ __forceinline__ void each_of(int n, F f) const {
    if (n < 0) return each_logit(f);
    for (int i = threadIdx.x; i < n; i += kDraw) f(s.logit[i]);
  }

  // The last token in rank that stays when the first `goal` tokens do (by_mass: those before which less than `goal_mass` lies), found up to eleven bits at a time
  // of how far its logit's place is behind the first one's: that logit, and how many tokens and (by_mass) how much mass lie above it, and how many are
  // its equals.  Of the n tokens of the list, or of all of the row where n is negative, down to the logit `low`; `above` and `mass_above` lie above all of these.
  // Masses are added up as whole numbers, in units of at most 2^-61 of `held`, which is the mass of all that are looked at: each is off by half a unit,
  // 2^24 of them by 2^-38 of `held`.
  struct Last {
    float logit;
    int above, equal;
    double mass_above;
  };
  struct Span {  // the first one's place, and in how many bits the others' distances from it fit
    uint32_t first;
    int bits;
  };
  __device__ __forceinline__ Span span_of(int n) {
    if (n < 0) return {key_of<T>(ref), 8 * (int)sizeof(T)};
    float high = -INFINITY, low = -INFINITY;
    for (int i = threadIdx.x; i < n; i += kDraw) {
      high = fmaxf(high, s.logit[i]);
      low = fmaxf(low, -s.logit[i]);
    }
    ask.most(high, low);
    const uint32_t first = key_of<T>(high + 0.f), far = first - key_of<T>(-low + 0.f);
    return {first, 32 - __builtin_clz(far | 1)};
  }
  __device__ __forceinline__ Last last_of(int n, const Span& span, float low, double held, bool by_mass, int goal, double goal_mass, int above, double mass_above) {
    const double unit = ldexp(1.0, 61 - ilogb(held));
    unsigned long long whole_above = by_mass ? (unsigned long long)rint(mass_above * unit) : 0;
    const unsigned long long whole_goal = by_mass ? (unsigned long long)fmin(fmax(ceil(goal_mass * unit), 0.0), 0x1p62) : 0;
    uint32_t far = 0;  // as much as is known of the distance
    int equal = 0;
#pragma unroll 1
    for (int left = span.bits; left > 0;) {
      const int bits = min(left, 11), shift = left - bits;
      __syncthreads();
      for (int i = threadIdx.x; i < kDigits; i += kDraw) {
        s.digits.count[i] = 0;
        s.digits.mass[i] = 0;
      }
      __syncthreads();
      auto take = [&](float l) {
        if (l == -INFINITY || l < low) return;
        const uint32_t z = span.first - key_of<T>(l);
        if (left < 32 && z >> left != far >> left) return;
        const int digit = z >> shift & ((1 << bits) - 1);
        atomicAdd(&s.digits.count[digit], 1u);
        if (by_mass) atomicAdd(&s.digits.mass[digit], (unsigned long long)rint(mass(l) * unit));
      };
      each_of(n, take);
      __syncthreads();
      // some digits a thread
      constexpr int kOwn = kDigits / kDraw;
      int many[kOwn], sum = 0, all;
      unsigned long long whole[kOwn], whole_sum = 0, whole_upto = 0, whole_all;
#pragma unroll
      for (int q = 0; q < kOwn; ++q) {
        const int digit = threadIdx.x * kOwn + q;
        sum += many[q] = s.digits.count[digit];
        whole_sum += whole[q] = s.digits.mass[digit];
      }
      int upto = above + ask.before(sum, all);
      if (by_mass) whole_upto = whole_above + ask.before(whole_sum, whole_all);
      // the first one with which the goal is reached; or the last one there is
      int at = -1, last = -1, at_above = 0, last_above = 0, at_many = 0, last_many = 0;
      unsigned long long at_whole = 0, last_whole = 0;
#pragma unroll
      for (int q = 0; q < kOwn; ++q) {
        if (!many[q]) continue;
        last = threadIdx.x * kOwn + q;
        last_above = upto, last_many = many[q], last_whole = whole_upto;
        upto += many[q];
        whole_upto += whole[q];
        if (at < 0 && (by_mass ? whole_upto >= whole_goal : upto >= goal)) {
          at = last;
          at_above = last_above, at_many = last_many, at_whole = last_whole;
        }
      }
      int who = ask.first(at >= 0);
      if (who < 0) {
        who = ask.last(last >= 0);
        at = last, at_above = last_above, at_many = last_many, at_whole = last_whole;
      }
      if (who == (int)threadIdx.x) {
        s.key = far | (uint32_t)at << shift;
        s.found = at_above;
        s.count = at_many;
        s.whole = at_whole;
      }
      __syncthreads();
      far = s.key;
      above = s.found;
      equal = s.count;
      whole_above = s.whole;
      left = shift;
    }
    return {logit_of<T>(span.first - far), above, equal, (double)whole_above / unit};
  }

  // Which tokens stay: those above `last`, and the first `left` of its equals.
  struct Border {
    float last;
    int left;
  };
  __device__ __forceinline__ Border border_of(int n, int above, double mass_above) {
    Border x = {-INFINITY, 0};
    double all = masses, held = masses;  // of what top-k leaves; of that and of all equals of its last one
    const Span span = span_of(n);
#pragma unroll 1
    for (int by_mass = lim.k ? 0 : 1; by_mass < (lim.p < 1.f ? 2 : 1); ++by_mass) {
      const double goal = (double)lim.p * all;
      const Last y = last_of(n, span, x.last, by_mass ? held : 1.0, by_mass, lim.k, goal, above, mass_above);
      if (!by_mass) {
        x = {y.logit, min(lim.k - y.above, y.equal)};
        if (!(lim.p < 1.f)) break;
        // (`held` is at most 1 + equals / k times `all`, for the least of k masses is at most a k-th of them: in `all` the limit is
        // known to (k + equals) 2^-62, 2^-37 at most)
        double own = 0.0;
        each_of(n, [&](float l) { own += l > x.last ? mass(l) : 0.0; });
        ask.before(own, held);
        all = held + x.left * mass(x.last);
        held += y.equal * mass(x.last);
        continue;
      }
      const double room = ceil((goal - y.mass_above) / mass(y.logit));
      int many = room < y.equal ? (int)fmax(room, 0.0) : y.equal;
      if (y.above == 0 && many < 1) many = 1;
      if (lim.k && y.logit == x.last) many = min(many, x.left);
      if (!lim.k || y.logit >= x.last) x = {y.logit, many};
    }
    return x;
  }

  // More than kCounted tokens of the list.
  __device__ __forceinline__ bool draw_listed(int n, bool all_there) {
    constexpr int kOwn = kFew / kDraw;
    float l[kOwn];
    double m[kOwn], sum = 0.0;
    int same = 0;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
      const int i = threadIdx.x * kOwn + q;
      l[q] = i < n ? s.logit[i] : -INFINITY;
      m[q] = i < n ? mass(l[q]) : 0.0;
      sum += m[q];
    }
    if (lim.p < 1.f && !lim.k && !all_there) {
      double listed;
      ask.before(sum, listed);
      if (!(listed >= (double)lim.p * masses)) return false;
    }
    Border x = {-INFINITY, 0};
    if (lim.k || lim.p < 1.f) x = border_of(n, 0, 0.0);
#pragma unroll
    for (int q = 0; q < kOwn; ++q) same += l[q] == x.last;
    int all;
    int nth = ask.before(same, all);
    double stay[kOwn];
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
      const bool in = l[q] > x.last || (l[q] == x.last && nth < x.left);
      nth += l[q] == x.last;
      stay[q] = in && m[q] >= (double)lim.m ? m[q] : 0.0;
    }
    draw_of(n, stay);
    return true;
  }

  // ---- any number of them stays
  // kLoads blocks of a thread, at, at + step, ..., all asked for at once and then taken one by one: f(block, its logits).
  struct Blocks {
    u32x4 w0, w1, w2, w3;
  };
  __device__ __forceinline__ void ask_for(int at, int step, Blocks& b) const {
    static_assert(kLoads == 4, "blocks in flight");
    if (row.whole(at)) b.w0 = row.load(at);
    if (row.whole(at + step)) b.w1 = row.load(at + step);
    if (row.whole(at + 2 * step)) b.w2 = row.load(at + 2 * step);
    if (row.whole(at + 3 * step)) b.w3 = row.load(at + 3 * step);
  }
  template <typename F>
  __device__ __forceinline__ void take(int at, int step, Blocks b, F f) const {
#pragma unroll 1
    for (int j = 0; j < kLoads; ++j) {
      float x[E];
      row.spread(b.w0, x);
      if (!row.whole(at)) row.edge(at, x);
      if (top == INFINITY) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = finite_top(x[e]);
      }
      f(at, x);
      at += step;
      b.w0 = b.w1, b.w1 = b.w2, b.w2 = b.w3;
    }
  }
  // All logits of the row.
  template <typename F>
  __device__ __forceinline__ void each_logit(F f) const {
    Blocks now = {}, next = {};
    ask_for(threadIdx.x, kDraw, now);
    for (int base = threadIdx.x; base < row.blocks; base += kLoads * kDraw) {
      ask_for(base + kLoads * kDraw, kDraw, next);
      take(base, kDraw, now, [&](int, const float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) f(x[e]);
      });
      now = next;
    }
  }
  // The parts, a wave each: f(part, take_part), and take_part(g) calls g(block, its logits) for its blocks.
  template <typename F>
  __device__ __forceinline__ void each_part(F f) const {
    Blocks now = {}, next = {};
    auto at = [&](int i) { return i * kPartBlocks + ask.lane(); };
    ask_for(at(ask.wave()), 64, now);
    for (int i = ask.wave(); i < prm.parts; i += kWaves) {
      ask_for(at(i + kWaves), 64, next);
      f(i, [&](auto g) { take(at(i), 64, now, g); });
      now = next;
    }
  }

  // Where the token is, once each part's mass above the last token that stays is known, and how many of its tokens are that one's equals.
  __device__ __forceinline__ Where where_of(const Border& x) {
    const int from = from_part(), to = to_part();
    int same = 0, unused;
    for (int i = from; i < to; ++i) same += part[i].many;
    const int same_before = ask.before(same, unused);
    double each = x.last > -INFINITY ? mass(x.last) : 0.0;
    if (!(each >= (double)lim.m)) each = 0.0;
    int nth = same_before;
    auto mass_in = [&](int j) {
      const Part y = part[j];
      const int stay = min(max(x.left - nth, 0), y.many);
      nth += y.many;
      return y.mass + stay * each;
    };
    double own = 0.0, total;
    for (int i = from; i < to; ++i) own += mass_in(i);
    const double base = ask.before(own, total), target = u * total;
    nth = same_before;
    double base_of_part;
    const int i = part_with(target, own, base, mass_in, base_of_part);
    int equal = 0, equal_all;  // in the parts before
    for (int j = threadIdx.x; j < i; j += kDraw) equal += part[j].many;
    ask.before(equal, equal_all);
    return {i, base_of_part, target, total, x.last, equal_all, x.left};
  }

  // With a top-p and no top-k: the last token that stays is looked for among those of a few bins.  A token of less than the share (1 - p) / V of all mass never
  // stays (all of them together have less than 1 - p); from there to the largest logit the row's logits are counted in kWide bins, and how far they lie in their bin
  // is added up.  The masses of a bin are at least those of as many tokens at the mean place, and at most what the bin's ends would have if
  // that were the mean place of tokens at them (the exponential is convex): that is within 10^-4 of each other, so the limit lies in one bin or two.  Those above these
  // stay for sure: their mass is added up part by part.  False: too many are in those bins.
  static constexpr int kCountAt = 39;
  __device__ __forceinline__ bool draw_between(Border& border) {
    const float depth = -(float)log((1.0 - (double)lim.p) * masses / prm.V) * lim.T;  // (of the smallest that can stay)
    const float range = depth * 1.0001f + 1e-4f * (fabsf(ref) + lim.T);
    if (!(range > 0.f) || !(range < 1e30f)) return false;
    const float to_bin = kWide / range;
    __syncthreads();
    for (int i = threadIdx.x; i < kWide; i += kDraw) s.wide[i] = 0;
    if (threadIdx.x == 0) s.taken = 0;
    __syncthreads();
    each_logit([&](float l) {
      const float at = (ref - l) * to_bin;
      if (at < (float)kWide) atomicAdd(&s.wide[(int)at], (1ull << kCountAt) + (uint32_t)((at - (float)(int)at) * 0x1p15f));
    });
    __syncthreads();
    constexpr int kOwn = kWide / kDraw;
    const double step = -(double)range / kWide, goal = (double)lim.p * masses;
    const double ratio = power(step);  // of the masses at a bin's ends
    double least[kOwn], most[kOwn], least_sum = 0.0, most_sum = 0.0, all;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
      const int bin = threadIdx.x * kOwn + q;
      const unsigned long long w = s.wide[bin];
      // (places are known in 32 bits, to 2^-10 of a bin, and are cut to 2^-15)
      const double n = (double)(w >> kCountAt), mean = n > 0.0 ? (double)(w & ((1ull << kCountAt) - 1)) * 0x1p-15 / n : 0.0;
      const double begin = power(fmin((bin - 0.002) * step, 0.0));
      most_sum += most[q] = n * begin * (1.0 + (ratio - 1.0) * fmax(mean - 0.002, 0.0));
      least_sum += least[q] = n * power((bin + mean + 0.002) * step);
    }
    double most_upto = ask.before(most_sum, all), least_upto = ask.before(least_sum, all);
    int begin = kWide, end = kWide;  // the limit lies in no bin before `begin`, and no token behind `end` stays
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
      most_upto += most[q];
      least_upto += least[q];
      if (begin == kWide && most_upto >= goal * (1.0 - 1e-9)) begin = threadIdx.x * kOwn + q;
      if (end == kWide && least_upto >= goal * (1.0 + 1e-9)) end = threadIdx.x * kOwn + q;
    }
    {
      const int who = ask.first(begin < kWide);
      if (who < 0) return false;
      if (who == (int)threadIdx.x) s.found = begin;
      const int then = ask.first(end < kWide);
      if (then == (int)threadIdx.x) s.count = end;
      __syncthreads();
      begin = s.found;
      end = then < 0 ? kWide - 1 : s.count;
    }
    // the parts' sure masses, and the tokens between: a stretch of the list for each part
    double sure = 0.0;
    each_part([&](int i, auto take_part) {
      double sum = 0.0, two = 0.0;
      int between = 0;
      // (of 64 blocks, those that stay for sure are put together first: their masses take most of the time; those between are few)
      constexpr int kOwnList = kFewGroups / 2 / kWaves;
      constexpr int kOwnSure = 2 * kWide / kWaves;
      float* const sure_ones = reinterpret_cast<float*>(s.wide) + ask.wave() * kOwnSure;
      uint2* const own_list = reinterpret_cast<uint2*>(s.groups) + ask.wave() * kOwnList;
      static_assert(kOwnSure >= 64 * E, "room for all of 64 blocks");
      auto rank = [](uint64_t in) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0)); };
      take_part([&](int block, const float (&x)[E]) {
        int n = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float at = (ref - x[e]) * to_bin;
          const bool sure = at < (float)begin, in = !sure && at < (float)(end + 1);
          const uint64_t all_sure = __ballot(sure), all_in = __ballot(in);
          if (sure) sure_ones[n + rank(all_sure)] = x[e];
          n += __popcll(all_sure);
          if (all_in) {
            const int to = between + rank(all_in);
            if (in && to < kOwnList) own_list[to] = make_uint2(as_u32(x[e]), (uint32_t)(row.number(block) + e));
            between += __popcll(all_in);
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        for (int j = ask.lane(); j < n; j += 128) {
          const float l = sure_ones[j], o = j + 64 < n ? sure_ones[j + 64] : -INFINITY;
          sum += mass(l);
          two += mass(o);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      });
      sum = sum_wave(sum + two);
      const int all_of = between;
      int to = 0;
      if (ask.lane() == 0) to = atomicAdd(&s.taken, all_of <= kOwnList ? all_of : kList + 1);
      to = __builtin_amdgcn_readfirstlane(to);
      if (all_of <= kOwnList && to + all_of <= kList)
        for (int j = ask.lane(); j < all_of; j += 64) {
          const uint2 one = own_list[j];
          s.logit[to + j] = as_f32(one.x);
          s.number[to + j] = (int)one.y;
        }
      if (ask.lane() == 0) part[i] = Part(sum, 0.0, to, all_of);
    });
    __syncthreads();
    const int n = s.taken;
    if (n > kList) return false;
    const int from = from_part(), to = to_part();
    for (int i = from; i < to; ++i) sure += part[i].mass;
    double sure_all;
    ask.before(sure, sure_all);
    // (in the first place that is not before all of them there is one token at least above: `above` counts as one where any mass lies above)
    border = border_of(n, begin > 0 && sure_all > 0.0 ? 1 : 0, sure_all);
    for (int i = from; i < to; ++i) {  // the parts with those of their tokens that were between
      const Part y = part[i];
      double sum = y.mass;
      int equal = 0;
      for (int j = 0; j < y.many; ++j) {
        const float l = s.logit[y.first + j];
        equal += l == border.last;
        if (l > border.last) sum += mass(l);
      }
      part[i] = Part(sum, 0.0, 0, equal);
    }
    __syncthreads();
    return true;
  }

  // The mass of each part above the last token that stays, and how many of its tokens are that one's equals.
  __device__ __forceinline__ void add_up(const Border& x) {
    each_part([&](int i, auto take_part) {
      double sum = 0.0;
      int same = 0;
      take_part([&](int, const float (&y)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          same += y[e] == x.last;
          if (y[e] > x.last) {
            const double w = mass(y[e]);
            sum += w >= (double)lim.m ? w : 0.0;
          }
        }
      });
      sum = sum_wave(sum);
      same = upto_lane(same);
      if (ask.lane() == 63) part[i] = Part(sum, 0.0, 0, same);
    });
    __syncthreads();
  }

  __device__ __forceinline__ bool draw_few() {
    const int floor = floor_of();
    if (floor == kBins - 1 && prm.V > kFew) return false;
    __syncthreads();
    const int n = list_down_to(floor);
    if (n < 0) return false;
    // (a floor that min_p sets is below all that stay; so is the last bin)
    const bool all_there = floor != mass_floor || floor == kBins - 1;
    return n <= kCounted ? draw_counted(n, all_there) : draw_listed(n, all_there);
  }

  template <bool LIMITS>
  __device__ __forceinline__ void draw() {
    sum_up();
    if (lim.greedy) {
      if (top > -INFINITY) greedy();
    } else if (top > -INFINITY) {
      Where where;
      bool drawn = false;
      if (!LIMITS || !lim.some) {
        where = draw_all();
      } else if constexpr (LIMITS) {
        drawn = draw_few();
        if (!drawn) {
          __syncthreads();
          Border x = {-INFINITY, 0};
          bool found = lim.p < 1.f && !lim.k && draw_between(x);
          if (!found && (lim.k || lim.p < 1.f)) {
            __syncthreads();
            x = border_of(-1, 0, 0.0);
          }
          if (found && !(mass(x.last) >= (double)lim.m)) {  // min_p is what ends them
            x = {-INFINITY, 0};
            found = false;
          }
          __syncthreads();
          if (!found) add_up(x);
          where = where_of(x);
        }
      }
      if (!drawn) draw_in(where);
    }
    answer();
  }
};

// Threads of a row with limits, and of one without.
constexpr int kLimited = 512, kFree = 256;
template <typename T, bool LIMITS>
__global__ __launch_bounds__(LIMITS ? kLimited : kFree) void sample_draw_kernel(const SampleParams prm) {
  constexpr int N = LIMITS ? kLimited : kFree;
  typedef std::conditional_t<LIMITS, DrawShared<N>, AskShared<N>> Shared;
  __shared__ Shared shared;
  const int r = blockIdx.x;
  Drawer<T, N, Shared> d(prm, shared, r);
  float u = prm.uniform[r];
  u = u >= 0.f ? fminf(u, 1.f - 0x1p-24f) : u < 0.f ? 0.f : 1.f - 0x1p-24f;
  d.u = (double)u;
  d.template draw<LIMITS>();
}

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

int parts_of(int vocab, int dtype) {  // of a row that may begin anywhere in 16 bytes
  const int each = dtype == MASKKV_BF16 ? 8 : 4;
  return (int)(((int64_t)vocab + 2 * each - 2 + (int64_t)each * kPartBlocks - 1) / (each * kPartBlocks));
}

}  // namespace

size_t sample_workspace_bytes(int64_t rows, int vocab, int dtype) {
  const size_t parts = (size_t)rows * parts_of(vocab, dtype);
  return rows ? pad256(parts * sizeof(Part)) + pad256(parts * kGroups * 4) : 0;
}

int launch_sample(const void* logits, int64_t rows, int vocab, int dtype, int64_t row_bytes, const maskkv_sampling* sampling,
                  int32_t* token, float* prob, float* logprob, void* workspace, hipStream_t stream) {
  SampleParams prm;
  prm.logits = reinterpret_cast<const char*>(logits);
  prm.row_bytes = row_bytes;
  prm.rows = (int)rows;
  prm.V = vocab;
  prm.parts = parts_of(vocab, dtype);
  prm.temperature = sampling->temperature;
  prm.top_k = sampling->top_k;
  prm.top_p = sampling->top_p;
  prm.min_p = sampling->min_p;
  prm.uniform = sampling->uniform;
  prm.token = token;
  prm.prob = prob;
  prm.logprob = logprob;
  const size_t parts = (size_t)rows * prm.parts;
  prm.part = reinterpret_cast<Part*>(workspace);
  prm.group = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + pad256(parts * sizeof(Part)));
  const size_t groups = (parts + 3) / 4;
  if (groups * 256 > 0xFFFFFFFFu) {  // (threads of a launch along a dimension)
    set_error("sample: %lld rows of %d logits are more than a launch can have", (long long)rows, vocab);
    return MASKKV_ESHAPE;
  }
  auto parts_kernel = dtype == MASKKV_BF16 ? &sample_parts_kernel<bf16_t> : &sample_parts_kernel<float>;
  const bool limits = sampling->top_k || sampling->top_p || sampling->min_p;
  auto draw_kernel = dtype == MASKKV_BF16 ? (limits ? &sample_draw_kernel<bf16_t, true> : &sample_draw_kernel<bf16_t, false>)
                                          : (limits ? &sample_draw_kernel<float, true> : &sample_draw_kernel<float, false>);
  hipLaunchKernelGGL(parts_kernel, dim3((unsigned)groups), dim3(256), 0, stream, prm);
  if (int e = check_launch("sample (parts)")) return e;
  hipLaunchKernelGGL(draw_kernel, dim3((unsigned)rows), dim3(limits ? kLimited : kFree), 0, stream, prm);
  return check_launch("sample");
}

}  // namespace maskkv
