// Tokens from logits, with given random numbers: temperature, top-k, top-p, min-p.
//
// Two kernels.  The first reads every row once: a wave takes a part of a row (4 KB) and leaves its largest logit, its mass relative to that
// at the row's temperature and at temperature 1, and, where the row has limits, the largest logit of each group of 128 bytes.  The second
// has a workgroup a row: it adds up the parts and, without limits, reads the one part again in which the wanted mass is reached.  With limits,
// the groups' largest logits say how small a token that stays can be (`floor_of`): few groups reach that, and the tokens of these that do are ranked in
// LDS (`draw_few`).  Where too many do - nearly flat rows, no limit but a small min-p - the last token that stays is found by histograms over the bits of the logits'
// order, and the row is read part by part again (`draw_any`).
//
// Which token is drawn must not depend on roundings: in a flat row of 10^5 tokens an error of 10^-7 of the mass is a hundredth of a token.
// Masses are therefore 64 bits wide from the exponential on: 2^f on [-1/2, 1/2] as 1 + f q(f), q the polynomial of degree 8 through
// (2^f - 1)/f at nine Chebyshev points, off by 4e-14, on a vector unit that does 64-bit operations at the rate of 32-bit ones.
// Histograms add up whole numbers, so that the order in which threads come to them has no part in the result.
#include <type_traits>

#include "kernels.hpp"

namespace maskkv {

namespace {

constexpr int kPartBlocks = 256;  // blocks of 16 bytes of a row's part
constexpr int kLoads = kPartBlocks / 64;
constexpr int kGroupBlocks = 8;   // ... of a group
constexpr int kGroups = kPartBlocks / kGroupBlocks;

struct Part {
  double mass;  // sum of exp((l - top) / temperature)
  float top;    // largest logit
  float plain;  // sum of exp(l - top)
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
  __device__ __forceinline__ double c() const { return 1.4426950408889634074 / (double)T; }
};

// 2^t, t <= 0 (what is below 2^-1100, or NaN, is 0; 2^0 is 1 exactly)
__device__ __forceinline__ double exp2_64(double t) {
  t = fmax(t, -1100.0);
  const double n = rint(t), f = t - n;
  double q = 1.0203121070622722e-07;
  q = fma(q, f, 1.325522487501112e-06);
  q = fma(q, f, 1.5252686846270554e-05);
  q = fma(q, f, 0.00015403455852469646);
  q = fma(q, f, 0.0013333558179043094);
  q = fma(q, f, 0.00961812915940254);
  q = fma(q, f, 0.055504108664760424);
  q = fma(q, f, 0.2402265069581299);
  q = fma(q, f, 0.6931471805599453);
  return ldexp(fma(q, f, 1.0), (int)n);
}
// Mass of a logit relative to the largest one.
__device__ __forceinline__ double mass_of(float l, float top, double c) { return exp2_64(((double)l - (double)top) * c); }

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
      // (NaN counts as -infinity, -0 as 0)
      x[i] = fmaxf(as_f32(sizeof(T) == 4 ? u : i % 2 ? u & 0xFFFF0000u : u << 16), -INFINITY) + 0.f;
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
      x[i] = fmaxf(v, -INFINITY) + 0.f;
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
  double mass = 0.0;
  float plain = 0.f;
  if (ref > -INFINITY) {
    if (prm.logprob) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) plain += fast_exp2((x[j][e] - ref) * kLog2e);
    }
    if (lim.masses) {
      const double c = lim.c();
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) mass += mass_of(x[j][e], ref, c);
    }
  }
  if (prm.logprob) plain = (float)sum_wave((double)plain);
  if (lim.masses) mass = sum_wave(mass);
  if (lane == 0) prm.part[(int64_t)r * prm.parts + i] = Part{mass, top, plain};
}

// ---- a token for every row
constexpr int kDraw = 1024;      // threads
constexpr int kWaves = kDraw / 64;
constexpr int kBins = 1024;      // of the groups' largest logits
constexpr int kFewGroups = 4096; // that are looked into, at most
constexpr int kFew = 2048;       // tokens that are ranked, at most
constexpr int kDigits = 2048;    // values of eleven bits

struct DrawShared {
  double sums[2][kWaves];
  int ints[2][kWaves];
  union {
    struct {
      uint32_t count[kBins];
      unsigned long long mass[kBins];
    } bins;
    struct {
      uint32_t count[kDigits];
      unsigned long long mass[kDigits];
    } digits;
    struct {
      float logit[kFew];
      int number[kFew];
      double mass[kFew];    // in the order of their numbers
      double ranked[kFew];  // in the order of their ranks: the mass before each
    } few;
  };
  uint32_t groups[kFewGroups];
  int found;
  int count;
  double value;
  unsigned long long whole;
  uint32_t key;
};

// What all threads of a workgroup of kDraw ask each other.  `turn` alternates between two places, so that one barrier a question is enough.
struct Ask {
  DrawShared& s;
  int turn = 0;
  __device__ __forceinline__ explicit Ask(DrawShared& shared) : s(shared) {}
  __device__ __forceinline__ int wave() const { return threadIdx.x >> 6; }
  __device__ __forceinline__ int lane() const { return threadIdx.x & 63; }
  // The sum before this thread; of all in `total`.
  __device__ double before(double v, double& total) {
    double upto = v;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
      const double o = __shfl_up(upto, i);
      if (lane() >= i) upto += o;
    }
    turn ^= 1;
    if (lane() == 63) s.sums[turn][wave()] = upto;
    __syncthreads();
    double base = 0.0;
    total = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave()) base = total;
      total += s.sums[turn][w];
    }
    const double o = __shfl_up(upto, 1);
    return base + (lane() ? o : 0.0);
  }
  __device__ int before(int v, int& total) {
    int upto = v;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
      const int o = __shfl_up(upto, i);
      if (lane() >= i) upto += o;
    }
    turn ^= 1;
    if (lane() == 63) s.ints[turn][wave()] = upto;
    __syncthreads();
    int base = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave()) base = total;
      total += s.ints[turn][w];
    }
    return base + upto - v;
  }
  __device__ int least(int v) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) v = min(v, __shfl_xor(v, i));
    turn ^= 1;
    if (lane() == 0) s.ints[turn][wave()] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v = min(v, s.ints[turn][w]);
    return v;
  }
  __device__ float most(float v) {
    v = max_wave(v);
    turn ^= 1;
    if (lane() == 0) s.ints[turn][wave()] = (int)as_u32(v);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v = fmaxf(v, as_f32((uint32_t)s.ints[turn][w]));
    return v;
  }
};

// A logit's place in the order of all, as a whole number.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t u = as_u32(l);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return as_f32(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

constexpr int kNone = 0x7FFFFFFF;

template <typename T>
struct Drawer {
  static constexpr int E = Row<T>::E;
  const SampleParams& prm;
  DrawShared& s;
  Ask ask;
  const Row<T> row;
  const Limits lim;
  const int r;
  Part* const part;
  float top = 0.f, ref = 0.f;  // the largest logit, and what masses are relative to
  double c = 0.0, u = 0.0;
  double masses = 0.0, plain = 0.0;  // of all tokens
  double mine = 0.0;   // of this thread's parts, and before them
  double before = 0.0;

  __device__ Drawer(const SampleParams& p, DrawShared& shared, int number)
      : prm(p), s(shared), ask(shared), row(p, number), lim(p, number), r(number), part(p.part + (int64_t)number * p.parts) {}

  __device__ __forceinline__ float seen(float l) const { return top == INFINITY ? finite_top(l) : l; }
  __device__ __forceinline__ void read(int block, float (&x)[E]) const {
    row.read(block, x);
    if (top == INFINITY) {
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = finite_top(x[e]);
    }
  }
  __device__ __forceinline__ double mass(float l) const { return mass_of(l, ref, c); }
  __device__ __forceinline__ double part_unit(float part_top, double by) const {
    return part_top == top ? 1.0 : part_top == -INFINITY || top == INFINITY ? 0.0 : exp2_64(((double)part_top - (double)ref) * by);
  }
  __device__ __forceinline__ int per() const { return (prm.parts + kDraw - 1) / kDraw; }

  __device__ void answer(int number, double prob) {
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
  __device__ void sum_up() {
    const int from = threadIdx.x * per(), to = min(from + per(), prm.parts);
    float most = -INFINITY;
    for (int i = from; i < to; ++i) most = fmaxf(most, part[i].top);
    top = ask.most(most);
    ref = top == INFINITY ? 0.f : top;
    double own = 0.0;
    for (int i = from; i < to; ++i) {
      const Part x = part[i];
      if (lim.masses) mine += x.mass * part_unit(x.top, c);
      if (prm.logprob) own += x.plain * part_unit(x.top, 1.4426950408889634074);
    }
    if (prm.logprob) ask.before(own, plain);
    if (lim.masses) before = ask.before(mine, masses);
  }

  __device__ void greedy() {
    const int from = threadIdx.x * per(), to = min(from + per(), prm.parts);
    int own = kNone;
    for (int i = to - 1; i >= from; --i)
      if (part[i].top == top) own = i;
    const int i = ask.least(own);
    int at = kNone;
    if (threadIdx.x < kPartBlocks && i * kPartBlocks + (int)threadIdx.x < row.blocks) {
      const int block = i * kPartBlocks + threadIdx.x;
      float x[E];
      row.read(block, x);
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (x[e] == top) at = row.number(block) + e;
    }
    answer(ask.least(at), 1.0);
  }

  // Of the parts' masses (own: of a thread's from `from` on, before: of the ones before) the part in which `target` is exceeded, or the last one with any.
  template <typename F>
  __device__ int part_with(double target, double own, double base, F mass_in, double& base_of_part) {
    const int from = threadIdx.x * per(), to = min(from + per(), prm.parts);
    const bool over = own > 0.0 && base + own > target;
    int who = ask.least(over ? (int)threadIdx.x : kNone);
    if (who == kNone) who = -ask.least(own > 0.0 ? -(int)threadIdx.x : kNone);  // (roundings: the last one)
    if ((int)threadIdx.x == who) {
      int at = from;
      double sum = base, before_it = base;
      for (int i = from; i < to; ++i) {
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

  // The token: in part i, before which the tokens that stay have the mass `base` and `equal` of them are as large as `last`: those
  // above `last` stay, and of its equals the first `left`.
  __device__ void draw_in(int i, double base, double target, double total, float last, int equal, int left) {
    const int block = i * kPartBlocks + threadIdx.x;
    const bool has = threadIdx.x < kPartBlocks && block < row.blocks;
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = -INFINITY;
    if (has) read(block, x);
    int same = 0, all;
#pragma unroll
    for (int e = 0; e < E; ++e) same += x[e] == last;
    int nth = equal + ask.before(same, all);
    double m[E], own = 0.0, unused;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool stays = x[e] > last || (x[e] == last && nth < left);
      nth += x[e] == last;
      const double w = mass(x[e]);
      m[e] = stays && x[e] > -INFINITY && w >= (double)lim.m ? w : 0.0;
      own += m[e];
    }
    const double from = base + ask.before(own, unused);
    int who = ask.least(own > 0.0 && from + own > target ? (int)threadIdx.x : kNone);
    if (who == kNone) who = -ask.least(own > 0.0 ? -(int)threadIdx.x : kNone);
    if ((int)threadIdx.x == who) {
      double sum = from;
      int at = 0;
      bool done = false;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (m[e] > 0.0 && !done) {
          at = e;
          sum += m[e];
          done = sum > target;
          s.value = m[e];
        }
      }
      s.found = row.number(block) + at;
    }
    __syncthreads();
    answer(s.found, s.value / total);
  }

  __device__ void draw_all() {
    double base;
    const double target = u * masses;
    const int i = part_with(target, mine, before, [&](int j) { return part[j].mass * part_unit(part[j].top, c); }, base);
    draw_in(i, base, target, masses, -INFINITY, 0, 0);
  }

  // ---- few tokens stay
  float slope = 0.f;
  int mass_floor = 0;  // what top-p alone asks for
  __device__ __forceinline__ int bin_of(float l) const { return (int)fminf((ref - l) * slope, kBins - 1.f); }

  // The lowest of the bins of logits in which a token that stays can be (from the largest logit down to the smallest of the groups' largest in
  // equal steps).  With a top-k as many groups' largest logits lie above; with a top-p, so much of their mass.
  __device__ int floor_of() {
    const int groups = (row.blocks + kGroupBlocks - 1) / kGroupBlocks;
    const float* group = prm.group + (int64_t)r * prm.parts * kGroups;
    float least = INFINITY;
    for (int i = threadIdx.x; i < groups; i += kDraw) {
      const float l = seen(group[i]);
      least = l > -INFINITY ? fminf(least, l) : least;
    }
    for (int i = threadIdx.x; i < kBins; i += kDraw) {
      s.bins.count[i] = 0;
      s.bins.mass[i] = 0;
    }
    least = -ask.most(-least);
    slope = least < ref ? (kBins - 1) / (ref - least) : 0.f;
    for (int i = threadIdx.x; i < groups; i += kDraw) {
      const float l = seen(group[i]);
      if (l == -INFINITY) continue;
      atomicAdd(&s.bins.count[bin_of(l)], 1u);
      if (lim.masses && lim.p < 1.f) atomicAdd(&s.bins.mass[bin_of(l)], (unsigned long long)(mass(l) * 0x1p40));
    }
    __syncthreads();
    int floor = kBins - 1;
    {
      const int own = s.bins.count[threadIdx.x];
      int all;
      const int upto = ask.before(own, all) + own;
      if (lim.k) floor = min(floor, ask.least(upto >= lim.k ? (int)threadIdx.x : kNone));
    }
    if (lim.masses && lim.p < 1.f) {
      const double own = (double)s.bins.mass[threadIdx.x] * 0x1p-40;
      double all;
      const double upto = ask.before(own, all) + own;
      floor = min(floor, ask.least(upto >= masses * (double)lim.p * (1.0 + 1e-9) ? (int)threadIdx.x : kNone));
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

  // False: too many.
  __device__ bool draw_few(int floor) {
    const int groups = (row.blocks + kGroupBlocks - 1) / kGroupBlocks;
    const float* group = prm.group + (int64_t)r * prm.parts * kGroups;
    int chosen = 0;  // groups, in their order
    for (int base = 0; base < groups; base += kDraw) {
      const int i = base + threadIdx.x;
      const float l = i < groups ? seen(group[i]) : -INFINITY;
      const bool in = l > -INFINITY && bin_of(l) <= floor;
      int all;
      const int at = chosen + ask.before((int)in, all);
      chosen += all;
      if (chosen > kFewGroups) return false;
      if (in) s.groups[at] = i;
    }
    __syncthreads();
    int n = 0;
    for (int base = 0; base < chosen; base += kDraw / kGroupBlocks) {
      const int g = base + threadIdx.x / kGroupBlocks;
      float x[E];
      int own = 0, block = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = -INFINITY;
      if (g < chosen) {
        block = s.groups[g] * kGroupBlocks + threadIdx.x % kGroupBlocks;
        if (block < row.blocks) read(block, x);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) own += x[e] > -INFINITY && bin_of(x[e]) <= floor;
      int all;
      int at = n + ask.before(own, all);
      n += all;
      if (n > kFew) return false;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (x[e] > -INFINITY && bin_of(x[e]) <= floor) {
          s.few.logit[at] = x[e];
          s.few.number[at] = row.number(block) + e;
          ++at;
        }
    }
    __syncthreads();
    constexpr int kOwn = kFew / kDraw;
    float l[kOwn];
    int rank[kOwn];
    double m[kOwn];
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {  // (thread t has the tokens kOwn * t on)
      const int i = threadIdx.x * kOwn + q;
      l[q] = i < n ? s.few.logit[i] : -INFINITY;
      m[q] = i < n ? mass(l[q]) : 0.0;
      rank[q] = 0;
    }
    if ((int)threadIdx.x * kOwn < n) {
      for (int j = 0; j < n; ++j) {
        const float o = s.few.logit[j];
#pragma unroll
        for (int q = 0; q < kOwn; ++q) rank[q] += o > l[q] || (o == l[q] && j < (int)threadIdx.x * kOwn + q);
      }
    }
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
      const int i = threadIdx.x * kOwn + q;
      if (i >= n) continue;
      s.few.mass[i] = m[q];
      s.few.ranked[rank[q]] = lim.k && rank[q] >= lim.k ? 0.0 : m[q];
    }
    __syncthreads();
    double own[kOwn], sum = 0.0, ranked;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
      const int i = threadIdx.x * kOwn + q;
      own[q] = i < n ? s.few.ranked[i] : 0.0;
      sum += own[q];
    }
    double at = ask.before(sum, ranked);
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
      const int i = threadIdx.x * kOwn + q;
      if (i < n) s.few.ranked[i] = at;
      at += own[q];
    }
    __syncthreads();
    const double limit = (double)lim.p * (lim.k ? ranked : masses);
    // (roundings: the last one that stays may not be among these)
    if (lim.p < 1.f && !lim.k && floor == mass_floor && !(ranked >= limit)) return false;
    double stay[kOwn], mine_all = 0.0, total;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
      const int i = threadIdx.x * kOwn + q;
      bool in = i < n && (!lim.k || rank[q] < lim.k) && m[q] >= (double)lim.m;
      if (lim.p < 1.f) in = in && (rank[q] == 0 || s.few.ranked[rank[q]] < limit);
      stay[q] = in ? m[q] : 0.0;
      mine_all += stay[q];
    }
    const double from = ask.before(mine_all, total), target = u * total;
    int who = ask.least(mine_all > 0.0 && from + mine_all > target ? (int)threadIdx.x : kNone);
    if (who == kNone) who = -ask.least(mine_all > 0.0 ? -(int)threadIdx.x : kNone);
    if ((int)threadIdx.x == who) {
      double upto = from;
      bool done = false;
#pragma unroll
      for (int q = 0; q < kOwn; ++q)
        if (stay[q] > 0.0 && !done) {
          upto += stay[q];
          done = upto > target;
          s.found = s.few.number[threadIdx.x * kOwn + q];
          s.value = stay[q];
        }
    }
    __syncthreads();
    answer(s.found, s.value / total);
    return true;
  }

  // ---- any number of them stays
  // The last token in rank that stays when `goal` tokens (by_mass: tokens before which less than `goal` of the mass lies) do: its logit's key, and how many tokens
  // and how much mass lie above, and how many are equal.
  struct Last {
    uint32_t key;
    int above, equal;
    double mass_above;
  };
  __device__ Last last_of(bool by_mass, int goal, double goal_mass, double unit) {
    Last x = {0, 0, 0, 0.0};
    unsigned long long above = 0;
    constexpr int kShifts[] = {21, 10, 0};
    const unsigned long long whole_goal = by_mass ? (unsigned long long)fmin(ceil(goal_mass * unit), 0x1p62) : 0;
#pragma unroll
    for (int level = 0; level < (sizeof(T) == 2 ? 2 : 3); ++level) {
      const int shift = kShifts[level], bits = level == 2 ? 10 : 11;
      __syncthreads();
      for (int i = threadIdx.x; i < kDigits; i += kDraw) {
        s.digits.count[i] = 0;
        s.digits.mass[i] = 0;
      }
      __syncthreads();
      for (int block = threadIdx.x; block < row.blocks; block += kDraw) {
        float v[E];
        read(block, v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint32_t key = key_of(v[e]);
          if (v[e] == -INFINITY || (level && key >> (shift + bits) != x.key >> (shift + bits))) continue;
          const int digit = key >> shift & ((1 << bits) - 1);
          atomicAdd(&s.digits.count[digit], 1u);
          if (lim.p < 1.f) atomicAdd(&s.digits.mass[digit], (unsigned long long)rint(mass(v[e]) * unit));
        }
      }
      __syncthreads();
      // two digits a thread, the largest first
      const int high = kDigits - 1 - 2 * (int)threadIdx.x, low = high - 1;
      const int n_high = s.digits.count[high], n_low = s.digits.count[low];
      const unsigned long long m_high = s.digits.mass[high], m_low = s.digits.mass[low];
      int all;
      const int n_before = x.above + ask.before(n_high + n_low, all);
      const unsigned long long m_before = above + before_whole(m_high + m_low);
      int found = kNone;
      if (by_mass) {
        if (n_low && m_before + m_high + m_low >= whole_goal) found = 2 * threadIdx.x + 1;
        if (n_high && m_before + m_high >= whole_goal) found = 2 * threadIdx.x;
      } else {
        if (n_low && n_before + n_high + n_low >= goal) found = 2 * threadIdx.x + 1;
        if (n_high && n_before + n_high >= goal) found = 2 * threadIdx.x;
      }
      int first = ask.least(found);
      if (first == kNone) first = -ask.least(n_low ? -(2 * (int)threadIdx.x + 1) : n_high ? -2 * (int)threadIdx.x : kNone);  // (the last one there is)
      if (first / 2 == (int)threadIdx.x) {
        const bool is_low = first % 2;
        s.key = x.key | (uint32_t)(is_low ? low : high) << shift;
        s.found = n_before + (is_low ? n_high : 0);
        s.count = is_low ? n_low : n_high;
        s.whole = m_before + (is_low ? m_high : 0);
      }
      __syncthreads();
      x.key = s.key;
      x.above = s.found;
      x.equal = s.count;
      above = s.whole;
    }
    if (sizeof(T) == 2 && !(x.key & 0x80000000u)) x.key |= (1u << kShifts[1]) - 1;  // (of bf16 the low bits are all alike)
    x.mass_above = (double)above / unit;
    return x;
  }
  // (whole numbers: in any order)
  __device__ unsigned long long before_whole(unsigned long long v) {
    unsigned long long upto = v;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
      const unsigned long long o = __shfl_up(upto, i);
      if (ask.lane() >= i) upto += o;
    }
    ask.turn ^= 1;
    unsigned long long* sums = reinterpret_cast<unsigned long long*>(s.sums[ask.turn]);
    if (ask.lane() == 63) sums[ask.wave()] = upto;
    __syncthreads();
    unsigned long long base = 0;
    for (int w = 0; w < ask.wave(); ++w) base += sums[w];
    return base + upto - v;
  }

  __device__ void draw_any() {
    float last = -INFINITY;  // those above stay, and the first `left` of its equals
    int left = 0;
    // masses as whole numbers: of so many units, so that those of all tokens fit
    const double unit = ldexp(1.0, 62 - (32 - __builtin_clz((unsigned)prm.V)));
    double all = masses;
    if (lim.k) {
      const Last x = last_of(false, lim.k, 0.0, unit);
      last = logit_of(x.key);
      left = min(lim.k - x.above, x.equal);
      all = x.mass_above + left * mass(last);
    }
    if (lim.p < 1.f) {
      const double goal = (double)lim.p * all;
      const Last x = last_of(true, 0, goal, unit);
      const float l = logit_of(x.key);
      const double room = ceil((goal - x.mass_above) / mass(l));
      int n = room < x.equal ? (int)fmax(room, 0.0) : x.equal;
      if (x.above == 0 && n < 1) n = 1;
      if (lim.k && l == last) n = min(n, left);
      if (!lim.k || l >= last) {
        last = l;
        left = n;
      }
    }
    __syncthreads();
    // the mass of each part that stays for sure, and how many of its tokens are equal to the last one
    for (int i = threadIdx.x >> 6; i < prm.parts; i += kWaves) {
      double sum = 0.0;
      int same = 0;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int block = i * kPartBlocks + j * 64 + (threadIdx.x & 63);
        if (block >= row.blocks) continue;
        float x[E];
        read(block, x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          same += x[e] == last;
          if (x[e] > last) {
            const double w = mass(x[e]);
            sum += w >= (double)lim.m ? w : 0.0;
          }
        }
      }
      sum = sum_wave(sum);
#pragma unroll
      for (int j = 1; j < 64; j *= 2) same += __shfl_xor(same, j);
      if ((threadIdx.x & 63) == 0) part[i] = Part{sum, as_f32((uint32_t)same), 0.f};
    }
    __syncthreads();
    const int from = threadIdx.x * per(), to = min(from + per(), prm.parts);
    int same = 0, unused;
    for (int i = from; i < to; ++i) same += (int)as_u32(part[i].top);
    const int same_before = ask.before(same, unused);
    double each = last > -INFINITY ? mass(last) : 0.0;
    if (!(each >= (double)lim.m)) each = 0.0;
    int nth = same_before;
    double own = 0.0, total;
    for (int i = from; i < to; ++i) {
      const Part x = part[i];
      const int n = (int)as_u32(x.top), stay = min(max(left - nth, 0), n);
      own += x.mass + stay * each;
      nth += n;
    }
    const double base = ask.before(own, total), target = u * total;
    double base_of_part;
    int walked = same_before;
    const int i = part_with(target, own, base, [&](int j) {
      const Part x = part[j];
      const int n = (int)as_u32(x.top), stay = min(max(left - walked, 0), n);
      walked += n;
      return x.mass + stay * each;
    }, base_of_part);
    int equal = 0;  // in the parts before
    for (int j = threadIdx.x; j < i; j += kDraw) equal += (int)as_u32(part[j].top);
    int equal_all;
    ask.before(equal, equal_all);
    draw_in(i, base_of_part, target, total, last, equal_all, left);
  }

  __device__ void draw() {
    sum_up();
    if (top == -INFINITY) return answer(-1, 0.0);
    if (lim.greedy) return greedy();
    if (!lim.some) return draw_all();
    const int floor = floor_of();
    __syncthreads();
    if (!draw_few(floor)) {
      __syncthreads();
      draw_any();
    }
  }
};

template <typename T>
__global__ __launch_bounds__(kDraw) void sample_draw_kernel(const SampleParams prm) {
  __shared__ DrawShared shared;
  const int r = blockIdx.x;
  Drawer<T> d(prm, shared, r);
  float u = prm.uniform[r];
  u = u >= 0.f ? fminf(u, 1.f - 0x1p-24f) : u < 0.f ? 0.f : 1.f - 0x1p-24f;
  d.u = (double)u;
  d.c = d.lim.greedy ? 0.0 : d.lim.c();
  d.draw();
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
  auto draw_kernel = dtype == MASKKV_BF16 ? &sample_draw_kernel<bf16_t> : &sample_draw_kernel<float>;
  hipLaunchKernelGGL(parts_kernel, dim3((unsigned)groups), dim3(256), 0, stream, prm);
  if (int e = check_launch("sample (parts)")) return e;
  hipLaunchKernelGGL(draw_kernel, dim3((unsigned)rows), dim3(kDraw), 0, stream, prm);
  return check_launch("sample");
}

}  // namespace maskkv
