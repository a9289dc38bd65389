// C ABI of the MaskKV library: argument validation and marshalling only; all arithmetic is in the kernels.
#include <math.h>
#include <mutex>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "kernels.hpp"

namespace maskkv {

static thread_local char g_err[512] = "";

void set_error(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
}

int check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return MASKKV_OK;
  set_error("%s: %s", what, hipGetErrorString(e));
  return MASKKV_EHIP;
}

namespace {

int elem_bytes(const maskkv_desc* d) { return d->dtype == MASKKV_BF16 ? 2 : 4; }

int check_desc(const maskkv_desc* d, Lens* lens) {
  if (!d) {
    set_error("desc is NULL");
    return MASKKV_EINVAL;
  }
  if (d->dtype != MASKKV_F32 && d->dtype != MASKKV_BF16) {
    set_error("dtype %d is neither MASKKV_F32 nor MASKKV_BF16", d->dtype);
    return MASKKV_EDTYPE;
  }
  if (d->d != 64 && d->d != 128) {
    set_error("head_dim %d unsupported (64 or 128)", d->d);
    return MASKKV_ESHAPE;
  }
  if (d->B < 1 || d->B > MASKKV_MAX_BATCH) {
    set_error("B = %d outside 1..%d", d->B, MASKKV_MAX_BATCH);
    return MASKKV_ESHAPE;
  }
  if (d->H < 1 || d->H > 65535 || (int64_t)d->B * d->H > 65535) {
    set_error("H = %d (B*H = %lld) outside 1..65535", d->H, (long long)d->B * d->H);
    return MASKKV_ESHAPE;
  }
  if (d->n_resp < 1 || d->n_query < 1 || d->P_max < 0 || d->q_per_kv < 0 || d->q_per_kv > 64) {
    set_error("n_resp = %d, n_query = %d must be >= 1, P_max = %d >= 0, q_per_kv = %d in 0..64", d->n_resp, d->n_query,
              d->P_max, d->q_per_kv);
    return MASKKV_EINVAL;
  }
  if ((int64_t)d->n_query * query_heads_per_kv(d) > (1 << 20) || (int64_t)d->n_resp * query_heads_per_kv(d) > (1 << 20)) {
    set_error("more than 2^20 query rows per key/value head (n_query %d, n_resp %d, q_per_kv %d)", d->n_query,
              d->n_resp, d->q_per_kv);
    return MASKKV_ESHAPE;
  }
  if ((int64_t)d->P_max + d->n_resp > (1 << 30)) {
    set_error("sequence length %lld too large", (long long)d->P_max + d->n_resp);
    return MASKKV_ESHAPE;
  }
  for (int b = 0; b < MASKKV_MAX_BATCH; ++b) lens->P[b] = 0;
  for (int b = 0; b < d->B; ++b) {
    const int p = d->prompt_len ? d->prompt_len[b] : d->P_max;
    if (p < 0 || p > d->P_max) {
      set_error("prompt_len[%d] = %d outside 0..P_max = %d", b, p, d->P_max);
      return MASKKV_EINVAL;
    }
    lens->P[b] = p;
  }
  return MASKKV_OK;
}

int make_view(const maskkv_desc* d, const maskkv_tensor* t, const char* name, View* v) {
  if (!t || !t->ptr) {
    set_error("%s is NULL", name);
    return MASKKV_EINVAL;
  }
  const int64_t eb = elem_bytes(d);
  if (t->stride_t < d->d || t->stride_h < 0 || t->stride_b < 0) {
    set_error("%s: strides (b=%lld, h=%lld, t=%lld) invalid for head_dim %d", name, (long long)t->stride_b,
              (long long)t->stride_h, (long long)t->stride_t, d->d);
    return MASKKV_EINVAL;
  }
  if (t->stride_t * eb > (int64_t)1 << 24) {  // kernels keep row offsets inside a tile of up to 128 rows in 32 bits
    set_error("%s: token stride of %lld bytes exceeds the supported 16 MiB", name, (long long)(t->stride_t * eb));
    return MASKKV_EINVAL;
  }
  if (((uintptr_t)t->ptr & 15) || ((t->stride_b * eb) & 15) || ((t->stride_h * eb) & 15) || ((t->stride_t * eb) & 15)) {
    set_error("%s: pointer and strides must be multiples of 16 bytes", name);
    return MASKKV_EINVAL;
  }
  v->ptr = reinterpret_cast<char*>(t->ptr);
  v->stride_h = t->stride_h * eb;
  v->stride_t = t->stride_t * eb;
  for (int b = 0; b < MASKKV_MAX_BATCH; ++b) v->boff[b] = 0;
  for (int b = 0; b < d->B; ++b) {
    const int64_t s = t->seq_start ? t->seq_start[b] : 0;
    if (s < 0) {
      set_error("%s: seq_start[%d] negative", name, b);
      return MASKKV_EINVAL;
    }
    v->boff[b] = ((int64_t)b * t->stride_b + s * t->stride_t) * eb;
  }
  return MASKKV_OK;
}

int check_workspace(const char* what, void* ws, size_t have, size_t need) {
  if (need == 0) return MASKKV_OK;
  if (!ws || have < need) {
    set_error("%s: workspace of %zu bytes given, %zu needed", what, ws ? have : (size_t)0, need);
    return MASKKV_EWORKSPACE;
  }
  if ((uintptr_t)ws & 255) {
    set_error("%s: workspace must be 256-byte aligned", what);
    return MASKKV_EWORKSPACE;
  }
  return MASKKV_OK;
}

// A packed array of `rows` rows: its pointer is there (unless there are no rows) and a multiple of 16 bytes.
int check_packed(const char* what, const char* name, const void* p, int64_t rows) {
  if (rows > 0 && !p) {
    set_error("%s: %s is NULL", what, name);
    return MASKKV_EINVAL;
  }
  if ((uintptr_t)p & 15) {
    set_error("%s: %s must be 16-byte aligned", what, name);
    return MASKKV_EINVAL;
  }
  return MASKKV_OK;
}

// (Kernels count rows in 32 bits, also a tile's worth past the last one.)
int check_capacity(const char* what, const char* name, int64_t capacity) {
  if (capacity >= 0 && capacity <= MASKKV_MX_MAX_ROWS) return MASKKV_OK;
  set_error("%s: %s %lld outside 0..%d", what, name, (long long)capacity, MASKKV_MX_MAX_ROWS);
  return MASKKV_EINVAL;
}

int check_mx(const char* what, const char* name, const maskkv_mx_cache* c, int64_t rows, bool keys_only, MxCache* out) {
  *out = MxCache{};
  if (!c) {
    set_error("%s: %s is NULL", what, name);
    return MASKKV_EINVAL;
  }
  if (int e = check_packed(what, "k_codes", c->k_codes, rows)) return e;
  if (int e = check_packed(what, "k_scales", c->k_scales, rows)) return e;
  out->k_codes = reinterpret_cast<char*>(c->k_codes);
  out->k_scales = reinterpret_cast<char*>(c->k_scales);
  if (keys_only) return MASKKV_OK;
  if (int e = check_packed(what, "v_codes", c->v_codes, rows)) return e;
  if (int e = check_packed(what, "v_scales", c->v_scales, rows)) return e;
  out->v_codes = reinterpret_cast<char*>(c->v_codes);
  out->v_scales = reinterpret_cast<char*>(c->v_scales);
  return MASKKV_OK;
}

constexpr int kMostTokens = 1 << 25;  // of a sequence, in maskkv_rotate (a launch has fewer than 2^32 threads along a dimension)

// The angle of the farthest position has to be a number.
bool is_frequency(double f) { return isfinite(f * 2147483648.0); }

int check_rotary_shape(const char* what, int32_t width, int32_t most, int32_t layout) {
  if (width < 2 || width > most || (width & 1)) {
    set_error("%s: width %d must be even and in 2..%d", what, width, most);
    return MASKKV_EINVAL;
  }
  if (layout != MASKKV_ROTARY_HALVES && layout != MASKKV_ROTARY_PAIRS) {
    set_error("%s: layout %d unknown", what, layout);
    return MASKKV_EINVAL;
  }
  return MASKKV_OK;
}

float pick_scale(const maskkv_desc* d, float scale) { return scale > 0.f ? scale : 1.0f / sqrtf((float)d->d); }

// ---- static scratch of maskkv_score_static: one copy per GPU for the life of the process
constexpr size_t kStaticScratchBytes = MASKKV_STATIC_SCRATCH_BYTES;
constexpr int kMaxDevices = 64;
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];
static std::mutex g_scratch_mutex;
static void* g_scratch_ptr[kMaxDevices];  // device address of `scratch` on each GPU (null: not asked for yet)

// Device address of this GPU's copy of `scratch` (the array's name is only a host-side handle: kernels are always
// given this pointer).  Resolved once per device, with that device current.
int static_scratch(void** ptr) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess || dev < 0 || dev >= kMaxDevices) {
    set_error("score_static: hipGetDevice: %s (device %d)", hipGetErrorString(e), dev);
    (void)hipGetLastError();
    return MASKKV_EHIP;
  }
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !p) {
      set_error("score_static: hipGetSymbolAddress: %s", hipGetErrorString(e));
      (void)hipGetLastError();
      return MASKKV_EHIP;
    }
    g_scratch_ptr[dev] = p;
  }
  *ptr = g_scratch_ptr[dev];
  return MASKKV_OK;
}

}  // namespace
}  // namespace maskkv

namespace maskkv {

// maskkv_score with optional stage marks (see kernels.hpp).
int score_entry(const maskkv_desc* desc, const maskkv_tensor* Q_mask, const maskkv_tensor* K_full, float scale,
                float* scores, int64_t score_stride, float* prompt_mass, void* workspace, size_t workspace_bytes,
                void* stream, void* const* events) {
  Lens lens;
  View q, k;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, Q_mask, "Q_mask", &q)) return e;
  if (int e = make_view(desc, K_full, "K_full", &k)) return e;
  if (!scores || score_stride < desc->P_max) {
    set_error("scores is NULL or score_stride %lld < P_max %d", (long long)score_stride, desc->P_max);
    return MASKKV_EINVAL;
  }
  const SweepPlan plan = score_sweep_plan(desc, lens);
  if (int e = check_workspace("score", workspace, workspace_bytes, score_workspace_bytes(desc, lens, plan))) return e;
  return launch_score(desc, q, k, lens, pick_scale(desc, scale), scores, score_stride, prompt_mass, workspace,
                      reinterpret_cast<hipStream_t>(stream), events, plan);
}

int score_plan(const maskkv_desc* desc, SweepPlan* plan, RowsSplit* split) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  *plan = score_sweep_plan(desc, lens);
  *split = score_split(desc, lens, *plan);
  return MASKKV_OK;
}

int attend_mx_plan_entry(const maskkv_desc* desc, int64_t capacity, AttendMxPlan* plan) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = check_capacity("attend_mx", "capacity", capacity)) return e;
  *plan = attend_mx_plan(desc, capacity);
  return MASKKV_OK;
}

int attend_tree_plan_entry(const maskkv_desc* desc, int64_t capacity, AttendTreePlan* plan) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = check_capacity("attend_tree", "capacity", capacity)) return e;
  *plan = attend_tree_plan(desc, capacity);
  return MASKKV_OK;
}

}  // namespace maskkv

using namespace maskkv;

extern "C" {

int maskkv_version(void) { return MASKKV_VERSION; }

const char* maskkv_strerror(int status) {
  switch (status) {
    case MASKKV_OK: return "ok";
    case MASKKV_EINVAL: return "invalid argument";
    case MASKKV_ESHAPE: return "unsupported shape";
    case MASKKV_EDTYPE: return "unsupported dtype";
    case MASKKV_EWORKSPACE: return "workspace missing, too small or misaligned";
    case MASKKV_EHIP: return "HIP launch failed";
    case MASKKV_ECAPACITY: return "output capacity too small";
    default: return "unknown status";
  }
}

const char* maskkv_last_error(void) { return g_err; }

int maskkv_score_workspace_bytes(const maskkv_desc* desc, size_t* bytes) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (!bytes) {
    set_error("bytes is NULL");
    return MASKKV_EINVAL;
  }
  *bytes = score_workspace_bytes(desc, lens, score_sweep_plan(desc, lens));
  return MASKKV_OK;
}

int maskkv_score(const maskkv_desc* desc, const maskkv_tensor* Q_mask, const maskkv_tensor* K_full, float scale,
                 float* scores, int64_t score_stride, float* prompt_mass, void* workspace, size_t workspace_bytes,
                 void* stream) {
  return score_entry(desc, Q_mask, K_full, scale, scores, score_stride, prompt_mass, workspace, workspace_bytes,
                     stream, nullptr);
}

int maskkv_score_given_lse(const maskkv_desc* desc, const maskkv_tensor* Q_mask, const maskkv_tensor* K_full,
                           float scale, const float* row_lse, float* scores, int64_t score_stride,
                           float* prompt_mass, void* workspace, size_t workspace_bytes, void* stream) {
  Lens lens;
  View q, k;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, Q_mask, "Q_mask", &q)) return e;
  if (int e = make_view(desc, K_full, "K_full", &k)) return e;
  if (!row_lse || !scores || score_stride < desc->P_max) {
    set_error("row_lse or scores is NULL, or score_stride %lld < P_max %d", (long long)score_stride, desc->P_max);
    return MASKKV_EINVAL;
  }
  const SweepPlan plan = score_sweep_plan(desc, lens);  // (the workspace is asked for as for maskkv_score)
  if (int e = check_workspace("score_given_lse", workspace, workspace_bytes, score_workspace_bytes(desc, lens, plan)))
    return e;
  return launch_score(desc, q, k, lens, pick_scale(desc, scale), scores, score_stride, prompt_mass, workspace,
                      reinterpret_cast<hipStream_t>(stream), nullptr, SweepPlan{}, row_lse);
}

int maskkv_score_static(const maskkv_desc* desc, const maskkv_tensor* Q_mask, const maskkv_tensor* K_full, float scale,
                        float* scores, int64_t score_stride, float* prompt_mass, void* stream) {
  Lens lens;
  View q, k;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, Q_mask, "Q_mask", &q)) return e;
  if (int e = make_view(desc, K_full, "K_full", &k)) return e;
  if (!scores || score_stride < desc->P_max) {
    set_error("scores is NULL or score_stride %lld < P_max %d", (long long)score_stride, desc->P_max);
    return MASKKV_EINVAL;
  }
  // (the single sweep needs more scratch than the two passes: a description that only the latter fit takes them)
  SweepPlan plan = score_sweep_plan(desc, lens);
  if (score_workspace_bytes(desc, lens, plan) > kStaticScratchBytes) plan = SweepPlan{};
  const size_t need = score_workspace_bytes(desc, lens, plan);
  if (need > kStaticScratchBytes) {
    set_error("score_static: this description needs %zu bytes of scratch, the static array holds %zu; use maskkv_score "
              "with a caller workspace", need, kStaticScratchBytes);
    return MASKKV_EWORKSPACE;
  }
  void* ws = nullptr;
  if (int e = static_scratch(&ws)) return e;
  return launch_score(desc, q, k, lens, pick_scale(desc, scale), scores, score_stride, prompt_mass, ws,
                      reinterpret_cast<hipStream_t>(stream), nullptr, plan);
}

int maskkv_select_workspace_bytes(const maskkv_desc* desc, size_t* bytes) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (!bytes) {
    set_error("bytes is NULL");
    return MASKKV_EINVAL;
  }
  *bytes = select_workspace_bytes(desc);
  return MASKKV_OK;
}

// Validation of maskkv_select: everything the host can know.
static int check_select(const maskkv_desc* desc, const Lens& lens, const float* scores, int64_t score_stride,
                        int pool_window, int pool_mode, const int32_t* budgets, const int32_t* budgets_host,
                        const int32_t* idx, const int32_t* cu_budget, int64_t capacity) {
  if (!scores || !budgets || !cu_budget || score_stride < desc->P_max) {
    set_error("select: scores, budgets or cu_budget NULL, or score_stride %lld < P_max %d", (long long)score_stride,
              desc->P_max);
    return MASKKV_EINVAL;
  }
  if (pool_window < 1 || pool_window > 63 || (pool_window & 1) == 0) {
    set_error("pool_window %d must be odd and in 1..63", pool_window);
    return MASKKV_EINVAL;
  }
  if (pool_mode != MASKKV_POOL_MEAN && pool_mode != MASKKV_POOL_MAX) {
    set_error("pool_mode %d unknown", pool_mode);
    return MASKKV_EINVAL;
  }
  if (capacity < 0 || capacity > 0x7FFFFFFF || (capacity > 0 && !idx)) {
    set_error("select: capacity %lld invalid or idx NULL", (long long)capacity);
    return MASKKV_EINVAL;
  }
  if (desc->P_max > select_max_prompt()) {
    set_error("select: prompts above %lld tokens are not supported (P_max = %d)", (long long)select_max_prompt(),
              desc->P_max);
    return MASKKV_ESHAPE;
  }
  int64_t worst = 0;  // the prefix sums of the clamped budgets are 32-bit
  for (int b = 0; b < desc->B; ++b) worst += (int64_t)desc->H * lens.P[b];
  if (worst > 0x7FFFFFFF) {
    set_error("select: B*H*P = %lld kept rows in the worst case do not fit 32-bit offsets", (long long)worst);
    return MASKKV_ESHAPE;
  }
  if (budgets_host) {
    int64_t sum = 0;
    for (int b = 0; b < desc->B; ++b)
      for (int h = 0; h < desc->H; ++h) {
        const int32_t k = budgets_host[b * desc->H + h];
        if (k < 0) {
          set_error("select: budget %d of (sequence %d, head %d) is negative", k, b, h);
          return MASKKV_EINVAL;
        }
        sum += k < lens.P[b] ? k : lens.P[b];
      }
    if (sum > capacity) {
      set_error("select: the budgets keep %lld rows, capacity is %lld", (long long)sum, (long long)capacity);
      return MASKKV_ECAPACITY;
    }
  }
  return MASKKV_OK;
}

int maskkv_select(const maskkv_desc* desc, const float* scores, int64_t score_stride, int pool_window, int pool_mode,
                  const int32_t* budgets, const int32_t* budgets_host, int32_t* idx, int32_t* cu_budget,
                  int64_t capacity, void* workspace, size_t workspace_bytes, void* stream) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = check_select(desc, lens, scores, score_stride, pool_window, pool_mode, budgets, budgets_host, idx,
                           cu_budget, capacity))
    return e;
  if (int e = check_workspace("select", workspace, workspace_bytes, select_workspace_bytes(desc))) return e;
  return launch_select(desc, lens, scores, score_stride, pool_window, pool_mode, budgets, idx, cu_budget, capacity,
                       workspace, reinterpret_cast<hipStream_t>(stream));
}

int maskkv_compact(const maskkv_desc* desc, const maskkv_tensor* K, const maskkv_tensor* V, const int32_t* idx,
                   const int32_t* cu_budget, int64_t capacity, void* Kc, void* Vc, void* stream) {
  Lens lens;
  View k, v;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, K, "K", &k)) return e;
  if (int e = make_view(desc, V, "V", &v)) return e;
  if (!cu_budget || capacity < 0 || capacity > 0x7FFFFFFF || (capacity > 0 && (!idx || !Kc || !Vc))) {
    set_error("compact: cu_budget NULL, capacity %lld invalid, or idx/Kc/Vc NULL", (long long)capacity);
    return MASKKV_EINVAL;
  }
  if (((uintptr_t)Kc & 15) || ((uintptr_t)Vc & 15)) {
    set_error("compact: Kc and Vc must be 16-byte aligned");
    return MASKKV_EINVAL;
  }
  return launch_compact(desc, lens, k, v, idx, cu_budget, capacity, Kc, Vc, reinterpret_cast<hipStream_t>(stream));
}

int maskkv_attend_workspace_bytes(const maskkv_desc* desc, int full, size_t* bytes) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (!bytes) {
    set_error("bytes is NULL");
    return MASKKV_EINVAL;
  }
  *bytes = attend_workspace_bytes(desc, full != 0);
  return MASKKV_OK;
}

int maskkv_attend(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const void* Kc, const void* Vc,
                  const int32_t* cu_budget, int64_t capacity, const maskkv_tensor* K_resp,
                  const maskkv_tensor* V_resp, float scale, const maskkv_tensor* O, float* lse, void* workspace,
                  size_t workspace_bytes, void* stream) {
  Lens lens;
  View q, k2, v2, o;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, Q_resp, "Q_resp", &q)) return e;
  if (int e = make_view(desc, K_resp, "K_resp", &k2)) return e;
  if (int e = make_view(desc, V_resp, "V_resp", &v2)) return e;
  if (int e = make_view(desc, O, "O", &o)) return e;
  if (!cu_budget || capacity < 0 || capacity > 0x7FFFFFFF || (capacity > 0 && (!Kc || !Vc))) {
    set_error("attend: cu_budget NULL, capacity %lld invalid, or Kc/Vc NULL", (long long)capacity);
    return MASKKV_EINVAL;
  }
  if (((uintptr_t)Kc & 15) || ((uintptr_t)Vc & 15)) {
    set_error("attend: Kc and Vc must be 16-byte aligned");
    return MASKKV_EINVAL;
  }
  if (int e = check_workspace("attend", workspace, workspace_bytes, attend_workspace_bytes(desc, false))) return e;
  return launch_attend(desc, lens, false, q, Kc, Vc, cu_budget, capacity, k2, v2, pick_scale(desc, scale), o, lse,
                       workspace, reinterpret_cast<hipStream_t>(stream));
}

int maskkv_attend_full(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const maskkv_tensor* K_full,
                       const maskkv_tensor* V_full, float scale, const maskkv_tensor* O, float* lse, void* workspace,
                       size_t workspace_bytes, void* stream) {
  Lens lens;
  View q, k2, v2, o;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, Q_resp, "Q_resp", &q)) return e;
  if (int e = make_view(desc, K_full, "K_full", &k2)) return e;
  if (int e = make_view(desc, V_full, "V_full", &v2)) return e;
  if (int e = make_view(desc, O, "O", &o)) return e;
  if (int e = check_workspace("attend_full", workspace, workspace_bytes, attend_workspace_bytes(desc, true))) return e;
  return launch_attend(desc, lens, true, q, nullptr, nullptr, nullptr, 0, k2, v2, pick_scale(desc, scale), o, lse,
                       workspace, reinterpret_cast<hipStream_t>(stream));
}

int maskkv_compact_mx(const maskkv_desc* desc, const maskkv_tensor* K, const maskkv_tensor* V, const int32_t* idx,
                      const int32_t* cu_budget, int64_t capacity, const maskkv_mx_cache* cache, void* stream) {
  Lens lens;
  View k, v;
  MxCache mx;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, K, "K", &k)) return e;
  if (int e = make_view(desc, V, "V", &v)) return e;
  if (int e = check_capacity("compact_mx", "capacity", capacity)) return e;
  if (!cu_budget || (capacity > 0 && !idx)) {
    set_error("compact_mx: cu_budget or idx is NULL");
    return MASKKV_EINVAL;
  }
  if (int e = check_mx("compact_mx", "cache", cache, capacity, false, &mx)) return e;
  return launch_compact_mx(desc, lens, k, v, idx, cu_budget, capacity, mx, reinterpret_cast<hipStream_t>(stream));
}

int maskkv_expand_mx(const maskkv_desc* desc, const maskkv_mx_cache* cache, const int32_t* cu_budget, int64_t capacity,
                     void* Kc, void* Vc, void* stream) {
  Lens lens;
  MxCache mx;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = check_capacity("expand_mx", "capacity", capacity)) return e;
  if (!cu_budget) {
    set_error("expand_mx: cu_budget is NULL");
    return MASKKV_EINVAL;
  }
  if (int e = check_mx("expand_mx", "cache", cache, capacity, false, &mx)) return e;
  if (int e = check_packed("expand_mx", "Kc", Kc, capacity)) return e;
  if (int e = check_packed("expand_mx", "Vc", Vc, capacity)) return e;
  return launch_expand_mx(desc, mx, cu_budget, capacity, Kc, Vc, reinterpret_cast<hipStream_t>(stream));
}

int maskkv_attend_mx_workspace_bytes(const maskkv_desc* desc, int64_t capacity, size_t* bytes) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = check_capacity("attend_mx", "capacity", capacity)) return e;
  if (!bytes) {
    set_error("bytes is NULL");
    return MASKKV_EINVAL;
  }
  *bytes = attend_mx_workspace_bytes(desc, capacity);
  return MASKKV_OK;
}

int maskkv_attend_mx(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const maskkv_mx_cache* cache,
                     const int32_t* cu_budget, int64_t capacity, const maskkv_tensor* K_resp, const maskkv_tensor* V_resp,
                     float scale, const maskkv_tensor* O, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  Lens lens;
  View q, k2, v2, o;
  MxCache mx;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, Q_resp, "Q_resp", &q)) return e;
  if (int e = make_view(desc, K_resp, "K_resp", &k2)) return e;
  if (int e = make_view(desc, V_resp, "V_resp", &v2)) return e;
  if (int e = make_view(desc, O, "O", &o)) return e;
  if (int e = check_capacity("attend_mx", "capacity", capacity)) return e;
  if (!cu_budget) {
    set_error("attend_mx: cu_budget is NULL");
    return MASKKV_EINVAL;
  }
  if (int e = check_mx("attend_mx", "cache", cache, capacity, false, &mx)) return e;
  if (int e = check_workspace("attend_mx", workspace, workspace_bytes, attend_mx_needs(desc, capacity))) return e;
  return launch_attend_mx(desc, q, mx, cu_budget, capacity, k2, v2, pick_scale(desc, scale), o, lse, workspace,
                          reinterpret_cast<hipStream_t>(stream));
}

// Both forms of maskkv_accumulate: over Kc, or over the keys of `cache`.
static int accumulate_entry(const char* what, const maskkv_desc* desc, const maskkv_tensor* Q_resp, const void* Kc,
                            const maskkv_mx_cache* cache, bool mx, const int32_t* cu_budget, int64_t capacity, float scale,
                            const float* row_lse, float decay, const float* weights_in, float* weights_out, void* stream) {
  Lens lens;
  View q;
  MxCache keys{};
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, Q_resp, "Q_resp", &q)) return e;
  if (int e = check_capacity(what, "capacity", capacity)) return e;
  if (int e = mx ? check_mx(what, "cache", cache, capacity, true, &keys) : check_packed(what, "Kc", Kc, capacity)) return e;
  if (!(decay >= 0.f && decay <= 1.f)) {
    set_error("%s: decay %g outside [0, 1]", what, (double)decay);
    return MASKKV_EINVAL;
  }
  if (!cu_budget || !row_lse || (capacity > 0 && (!weights_out || (decay > 0.f && !weights_in)))) {
    set_error("%s: cu_budget, row_lse, weights_out or (with a decay above 0) weights_in is NULL", what);
    return MASKKV_EINVAL;
  }
  const uintptr_t in = (uintptr_t)weights_in, out = (uintptr_t)weights_out, bytes = (uintptr_t)capacity * 4;
  if (decay > 0.f && in != out && in < out + bytes && out < in + bytes) {
    set_error("%s: weights_in and weights_out overlap without being the same", what);
    return MASKKV_EINVAL;
  }
  return launch_accumulate(desc, q, mx ? nullptr : Kc, keys, cu_budget, capacity, pick_scale(desc, scale), row_lse, decay,
                           weights_in, weights_out, reinterpret_cast<hipStream_t>(stream));
}

int maskkv_accumulate(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const void* Kc, const int32_t* cu_budget,
                      int64_t capacity, float scale, const float* row_lse, float decay, const float* weights_in,
                      float* weights_out, void* stream) {
  return accumulate_entry("accumulate", desc, Q_resp, Kc, nullptr, false, cu_budget, capacity, scale, row_lse, decay,
                          weights_in, weights_out, stream);
}

int maskkv_accumulate_mx(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const maskkv_mx_cache* cache,
                         const int32_t* cu_budget, int64_t capacity, float scale, const float* row_lse, float decay,
                         const float* weights_in, float* weights_out, void* stream) {
  return accumulate_entry("accumulate_mx", desc, Q_resp, nullptr, cache, true, cu_budget, capacity, scale, row_lse, decay,
                          weights_in, weights_out, stream);
}

// Both forms of maskkv_evict; `moved` says which rows move with the ones that stay.
static int evict_entry(const char* what, const maskkv_desc* desc, const float* weights, const int32_t* cu_budget,
                       int64_t capacity, const int32_t* budgets, const MovedRows& moved, const int32_t* idx, int32_t* idx_out,
                       int32_t* rows, float* weights_out, int32_t* cu_out, int64_t capacity_out, void* stream) {
  // (An empty array may have no address: positions are asked for on both sides or on neither only where both caches have room for rows.)
  if (!cu_budget || !budgets || !cu_out || (capacity > 0 && !weights) || (capacity_out > 0 && !rows) ||
      (capacity > 0 && capacity_out > 0 && !idx != !idx_out)) {
    set_error("%s: cu_budget, budgets, cu_out, weights or rows is NULL, or only one of idx and idx_out is", what);
    return MASKKV_EINVAL;
  }
  if (desc->P_max > select_max_prompt()) {
    set_error("%s: heads of more than %lld rows are not supported (P_max = %d)", what, (long long)select_max_prompt(), desc->P_max);
    return MASKKV_ESHAPE;
  }
  const int64_t heads = (int64_t)desc->B * desc->H;
  struct Span {
    const void* p;
    int64_t bytes;
  };
  Span in[kMoved + 4] = {{weights, capacity * 4}, {idx, capacity * 4}, {cu_budget, (heads + 1) * 4}, {budgets, heads * 4}};
  Span out[kMoved + 4] = {{weights_out, capacity_out * 4}, {idx_out, capacity_out * 4}, {rows, capacity_out * 4},
                          {cu_out, (heads + 1) * 4}};
  for (int i = 0; i < kMoved; ++i) {
    in[4 + i] = {moved.from[i], moved.bytes[i] * capacity};
    out[4 + i] = {moved.to[i], moved.bytes[i] * capacity_out};
  }
  auto meet = [](const Span& a, const Span& b) {
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + (uint64_t)b.bytes && y < x + (uint64_t)a.bytes;
  };
  for (int o = 0; o < kMoved + 4; ++o) {
    for (int i = 0; i < kMoved + 4; ++i)
      if (meet(out[o], in[i]) || (i < o && meet(out[o], out[i]))) {
        set_error("%s: an output overlaps an input or another output (the smaller cache needs buffers of its own)", what);
        return MASKKV_EINVAL;
      }
  }
  return launch_evict(desc, weights, cu_budget, capacity, budgets, moved, idx, idx_out, rows, weights_out, cu_out, capacity_out,
                      reinterpret_cast<hipStream_t>(stream));
}

int maskkv_evict(const maskkv_desc* desc, const float* weights, const int32_t* cu_budget, int64_t capacity,
                 const int32_t* budgets, const void* Kc, const void* Vc, const int32_t* idx, void* Kc_out, void* Vc_out,
                 int32_t* idx_out, int32_t* rows, float* weights_out, int32_t* cu_out, int64_t capacity_out, void* stream) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = check_capacity("evict", "capacity", capacity)) return e;
  if (int e = check_capacity("evict", "capacity_out", capacity_out)) return e;
  if (int e = check_packed("evict", "Kc", Kc, capacity)) return e;
  if (int e = check_packed("evict", "Vc", Vc, capacity)) return e;
  if (int e = check_packed("evict", "Kc_out", Kc_out, capacity_out)) return e;
  if (int e = check_packed("evict", "Vc_out", Vc_out, capacity_out)) return e;
  const int row = desc->d * elem_bytes(desc);
  const MovedRows moved = {{(const char*)Kc, (const char*)Vc}, {(char*)Kc_out, (char*)Vc_out}, {row, row}};
  return evict_entry("evict", desc, weights, cu_budget, capacity, budgets, moved, idx, idx_out, rows, weights_out, cu_out,
                     capacity_out, stream);
}

int maskkv_evict_mx(const maskkv_desc* desc, const float* weights, const int32_t* cu_budget, int64_t capacity,
                    const int32_t* budgets, const maskkv_mx_cache* cache, const int32_t* idx,
                    const maskkv_mx_cache* cache_out, int32_t* idx_out, int32_t* rows, float* weights_out,
                    int32_t* cu_out, int64_t capacity_out, void* stream) {
  Lens lens;
  MxCache from, to;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = check_capacity("evict_mx", "capacity", capacity)) return e;
  if (int e = check_capacity("evict_mx", "capacity_out", capacity_out)) return e;
  if (int e = check_mx("evict_mx", "cache", cache, capacity, false, &from)) return e;
  if (int e = check_mx("evict_mx", "cache_out", cache_out, capacity_out, false, &to)) return e;
  const MovedRows moved = {{from.k_codes, from.v_codes, from.k_scales, from.v_scales},
                           {to.k_codes, to.v_codes, to.k_scales, to.v_scales},
                           {desc->d / 2, desc->d / 2, desc->d / 32, desc->d / 32}};
  return evict_entry("evict_mx", desc, weights, cu_budget, capacity, budgets, moved, idx, idx_out, rows, weights_out, cu_out,
                     capacity_out, stream);
}

int maskkv_attend_tree_workspace_bytes(const maskkv_desc* desc, int64_t capacity, size_t* bytes) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = check_capacity("attend_tree", "capacity", capacity)) return e;
  if (!bytes) {
    set_error("bytes is NULL");
    return MASKKV_EINVAL;
  }
  *bytes = attend_tree_workspace_bytes(desc, capacity);
  return MASKKV_OK;
}

int maskkv_attend_tree(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const void* Kc, const void* Vc,
                       const int32_t* cu_budget, int64_t capacity, const maskkv_tensor* K_resp, const maskkv_tensor* V_resp,
                       const uint32_t* mask, float scale, const maskkv_tensor* O, float* lse, void* workspace,
                       size_t workspace_bytes, void* stream) {
  Lens lens;
  View q, k2, v2, o;
  if (int e = check_desc(desc, &lens)) return e;
  if (int e = make_view(desc, Q_resp, "Q_resp", &q)) return e;
  if (int e = make_view(desc, K_resp, "K_resp", &k2)) return e;
  if (int e = make_view(desc, V_resp, "V_resp", &v2)) return e;
  if (int e = make_view(desc, O, "O", &o)) return e;
  if (int e = check_capacity("attend_tree", "capacity", capacity)) return e;
  if (!cu_budget || !mask) {
    set_error("attend_tree: cu_budget or mask is NULL");
    return MASKKV_EINVAL;
  }
  if (((uintptr_t)mask & 3) || ((uintptr_t)cu_budget & 3)) {
    set_error("attend_tree: cu_budget and mask must be 4-byte aligned");
    return MASKKV_EINVAL;
  }
  if (int e = check_packed("attend_tree", "Kc", Kc, capacity)) return e;
  if (int e = check_packed("attend_tree", "Vc", Vc, capacity)) return e;
  if (int e = check_workspace("attend_tree", workspace, workspace_bytes, attend_tree_needs(desc, capacity))) return e;
  return launch_attend_tree(desc, q, Kc, Vc, cu_budget, capacity, k2, v2, mask, pick_scale(desc, scale), o, lse, workspace,
                            reinterpret_cast<hipStream_t>(stream));
}

int maskkv_tree_mask(const int32_t* parents, int32_t B, int32_t n, uint32_t* mask, void* stream) {
  if (B < 0 || B > 65535 || n < 0 || n > 1 << 20) {
    set_error("tree_mask: B %d outside 0..65535 or n %d outside 0..2^20", B, n);
    return MASKKV_ESHAPE;
  }
  if (B == 0 || n == 0) return MASKKV_OK;
  if (!parents || !mask || ((uintptr_t)parents & 3) || ((uintptr_t)mask & 3)) {
    set_error("tree_mask: parents or mask is NULL or not 4-byte aligned");
    return MASKKV_EINVAL;
  }
  return launch_tree_mask(parents, B, n, mask, reinterpret_cast<hipStream_t>(stream));
}

// Rows and tokens of maskkv_sample.
static int check_sample(int64_t rows, int32_t vocab, int32_t dtype) {
  if (dtype != MASKKV_F32 && dtype != MASKKV_BF16) {
    set_error("dtype %d is neither MASKKV_F32 nor MASKKV_BF16", dtype);
    return MASKKV_EDTYPE;
  }
  if (rows < 0 || rows > 1 << 20 || vocab < 1 || vocab > 1 << 24) {
    set_error("sample: rows %lld outside 0..2^20 or vocab %d outside 1..2^24", (long long)rows, vocab);
    return MASKKV_ESHAPE;
  }
  return MASKKV_OK;
}

int maskkv_sample_workspace_bytes(int64_t rows, int32_t vocab, int32_t dtype, size_t* bytes) {
  if (int e = check_sample(rows, vocab, dtype)) return e;
  if (!bytes) {
    set_error("bytes is NULL");
    return MASKKV_EINVAL;
  }
  *bytes = sample_workspace_bytes(rows, vocab, dtype);
  return MASKKV_OK;
}

int maskkv_sample(const void* logits, int64_t rows, int32_t vocab, int32_t dtype, int64_t row_stride,
                  const maskkv_sampling* sampling, int32_t* token, float* prob, float* logprob, void* workspace,
                  size_t workspace_bytes, void* stream) {
  if (int e = check_sample(rows, vocab, dtype)) return e;
  const int64_t eb = dtype == MASKKV_BF16 ? 2 : 4;
  if (!sampling || row_stride < vocab || row_stride > INT64_MAX / (1 << 23)) {
    set_error("sample: sampling is NULL, or row_stride %lld is below vocab %d or too large", (long long)row_stride, vocab);
    return MASKKV_EINVAL;
  }
  if (rows == 0) return MASKKV_OK;
  if (!logits || !token || !sampling->uniform) {
    set_error("sample: logits, token or uniform is NULL");
    return MASKKV_EINVAL;
  }
  if ((uintptr_t)logits & (eb - 1)) {
    set_error("sample: logits must be aligned to an element");
    return MASKKV_EINVAL;
  }
  // (an entry a row is read by scalar loads, which leave out the lowest bits of an address)
  for (const void* p : {(const void*)sampling->temperature, (const void*)sampling->top_k, (const void*)sampling->top_p, (const void*)sampling->min_p,
                        (const void*)sampling->uniform, (const void*)token, (const void*)prob, (const void*)logprob})
    if ((uintptr_t)p & 3) {
      set_error("sample: the arrays of an entry a row must be 4-byte aligned");
      return MASKKV_EINVAL;
    }
  if (int e = check_workspace("sample", workspace, workspace_bytes, sample_workspace_bytes(rows, vocab, dtype))) return e;
  return launch_sample(logits, rows, vocab, dtype, row_stride * eb, sampling, token, prob, logprob, workspace,
                       reinterpret_cast<hipStream_t>(stream));
}

int maskkv_rotary_frequencies(int32_t width, int32_t layout, double base, int32_t scaling, double factor, double trained,
                              double slow, double fast, maskkv_rotary* rotary) {
  if (int e = check_rotary_shape("rotary_frequencies", width, 128, layout)) return e;
  if (!rotary || !(base > 0.0) || !isfinite(base)) {
    set_error("rotary_frequencies: rotary is NULL or base %g is not a positive number", base);
    return MASKKV_EINVAL;
  }
  const bool bands = scaling == MASKKV_ROTARY_BANDS;
  if (scaling != MASKKV_ROTARY_PLAIN && scaling != MASKKV_ROTARY_LINEAR && scaling != MASKKV_ROTARY_BASE && !bands) {
    set_error("rotary_frequencies: scaling %d unknown", scaling);
    return MASKKV_EINVAL;
  }
  if (scaling != MASKKV_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) {
    set_error("rotary_frequencies: factor %g is not a number of 1 or more", factor);
    return MASKKV_EINVAL;
  }
  if (bands && (!(trained > 0.0) || !isfinite(trained) || !(slow >= 0.0) || !(fast > slow) || !isfinite(fast))) {
    set_error("rotary_frequencies: trained %g must be above 0 and slow %g, fast %g be 0 <= slow < fast", trained, slow, fast);
    return MASKKV_EINVAL;
  }
  if (scaling == MASKKV_ROTARY_BASE && width > 2) base *= pow(factor, width / (width - 2.0));
  maskkv_rotary r = {width, layout, bands ? 1.0 + 0.1 * log(factor) : 1.0, {}};
  for (int i = 0; i < width / 2; ++i) {
    double f = pow(base, -2.0 * i / width);
    if (scaling == MASKKV_ROTARY_LINEAR) f /= factor;
    if (bands) {
      const double turns = trained * f / 6.283185307179586476925;
      const double keep = fmin(fmax((turns - slow) / (fast - slow), 0.0), 1.0);
      f *= keep + (1.0 - keep) / factor;
    }
    if (!is_frequency(f)) {
      set_error("rotary_frequencies: base %g is beyond the range of frequencies", base);
      return MASKKV_EINVAL;
    }
    r.freq[i] = f;
  }
  *rotary = r;
  return MASKKV_OK;
}

// Whether rows of two views with the same strides share bytes: of all their heads, and of the first n[b] tokens of each sequence.
static bool rows_meet(const maskkv_desc* desc, const View& x, const View& y, int heads, const int32_t* n) {
  const int64_t row = (int64_t)desc->d * elem_bytes(desc), sh = x.stride_h, st = x.stride_t;
  auto end = [&](int b) { return (heads - 1) * sh + (n[b] - 1) * st + row; };  // of a sequence's rows, from its first one's begin
  int64_t lo[2] = {INT64_MAX, INT64_MAX}, hi[2] = {INT64_MIN, INT64_MIN};
  for (int v = 0; v < 2; ++v)
    for (int b = 0; b < desc->B; ++b) {
      if (n[b] < 1) continue;
      const int64_t at = (int64_t)(uintptr_t)(v ? y : x).ptr + (v ? y : x).boff[b];
      lo[v] = at < lo[v] ? at : lo[v];
      hi[v] = at + end(b) > hi[v] ? at + end(b) : hi[v];
    }
  if (lo[0] >= hi[1] || lo[1] >= hi[0]) return false;
  for (int a = 0; a < desc->B; ++a)
    for (int b = 0; b < desc->B; ++b) {
      if (n[a] < 1 || n[b] < 1) continue;
      const int64_t far = (int64_t)(uintptr_t)x.ptr + x.boff[a] - (int64_t)(uintptr_t)y.ptr - y.boff[b];
      if (far >= end(b) || -far >= end(a)) continue;
      // (a token's heads side by side with other rows, or each head with other heads: where the first rows lie tells)
      auto apart = [&](int64_t period, int64_t bytes) {
        const int64_t m = (far % period + period) % period;
        return m >= bytes && m + bytes <= period;
      };
      if (apart(st, (heads - 1) * sh + row) || (sh > 0 && st % sh == 0 && apart(sh, row))) continue;
      for (int64_t dh = 1 - heads; dh < heads; ++dh) {  // (of two heads so far apart: the tokens whose rows begin nearest to each other)
        const int64_t x0 = far + dh * sh, least = 1 - n[b], most = n[a] - 1;
        int64_t dt = -x0 / st;
        for (dt -= 1; dt * st + x0 <= -row; ++dt) {}
        dt = dt < least ? least : dt;
        if (dt <= most && x0 + dt * st > -row && x0 + dt * st < row) return true;
      }
    }
  return false;
}

// One of maskkv_rotate's inputs with its output, of so many heads and tokens: both views, or neither.
static int check_turned(const maskkv_desc* desc, const maskkv_tensor* in, const maskkv_tensor* out, const char* name, int heads, int n_tokens, const int32_t* token_len,
                        View* from, View* to) {
  if (!in != !out) {
    set_error("rotate: only one of %s and %s_out is NULL", name, name);
    return MASKKV_EINVAL;
  }
  if (!in) return MASKKV_OK;
  if (int e = make_view(desc, in, name, from)) return e;
  if (int e = make_view(desc, out, name, to)) return e;
  // (a stride that no element is behind says nothing)
  const bool strides = (from->stride_t == to->stride_t || n_tokens <= 1) && (from->stride_h == to->stride_h || heads == 1);
  bool same = strides, begin = false;
  int32_t n[MASKKV_MAX_BATCH];
  for (int b = 0; b < desc->B; ++b) {
    n[b] = token_len ? token_len[b] : n_tokens;
    const bool there = from->ptr + from->boff[b] == to->ptr + to->boff[b];
    same = same && there;
    begin = begin || (there && n[b] > 0);
  }
  if (same || !(strides ? rows_meet(desc, *from, *to, heads, n) : begin)) return MASKKV_OK;
  set_error("rotate: %s_out overlaps %s and is not the same view", name, name);
  return MASKKV_EINVAL;
}

int maskkv_rotate(const maskkv_desc* desc, const maskkv_rotary* rotary, const int32_t* positions, int32_t n_tokens,
                  const int32_t* token_len, const maskkv_tensor* Q, const maskkv_tensor* Q_out, const maskkv_tensor* K,
                  const maskkv_tensor* K_out, void* stream) {
  Lens lens;
  View q, qo, k, ko;
  if (int e = check_desc(desc, &lens)) return e;
  if (!rotary) {
    set_error("rotate: rotary is NULL");
    return MASKKV_EINVAL;
  }
  if (int e = check_rotary_shape("rotate", rotary->width, desc->d, rotary->layout)) return e;
  bool finite = isfinite((float)rotary->amplitude);
  for (int i = 0; i < rotary->width / 2; ++i) finite = finite && is_frequency(rotary->freq[i]);
  if (!finite) {
    set_error("rotate: a frequency times 2^31 or the amplitude is not a finite number");
    return MASKKV_EINVAL;
  }
  if (n_tokens < 0 || n_tokens > kMostTokens) {
    set_error("rotate: n_tokens %d outside 0..%d", n_tokens, kMostTokens);
    return MASKKV_EINVAL;
  }
  if (!Q && !K) {
    set_error("rotate: neither Q nor K is given");
    return MASKKV_EINVAL;
  }
  for (int b = 0; token_len && b < desc->B; ++b)
    if (token_len[b] < 0 || token_len[b] > n_tokens) {
      set_error("rotate: token_len[%d] = %d outside 0..n_tokens = %d", b, token_len[b], n_tokens);
      return MASKKV_EINVAL;
    }
  if (int e = check_turned(desc, Q, Q_out, "Q", desc->H * query_heads_per_kv(desc), n_tokens, token_len, &q, &qo)) return e;
  if (int e = check_turned(desc, K, K_out, "K", desc->H, n_tokens, token_len, &k, &ko)) return e;
  if (n_tokens == 0) return MASKKV_OK;
  if (!positions || ((uintptr_t)positions & 3)) {
    set_error("rotate: positions is NULL or not 4-byte aligned");
    return MASKKV_EINVAL;
  }
  return launch_rotate(desc, rotary, positions, n_tokens, token_len, Q ? &q : nullptr, &qo, K ? &k : nullptr, &ko,
                       reinterpret_cast<hipStream_t>(stream));
}

int maskkv_head_budgets(const maskkv_desc* desc, const float* prompt_mass, int32_t k_l, float alpha, int32_t* budgets,
                        void* stream) {
  Lens lens;
  if (int e = check_desc(desc, &lens)) return e;
  if (!prompt_mass || !budgets || k_l < 0 || !(alpha >= 0.f && alpha <= 1.f)) {
    set_error("head_budgets: NULL pointer, k_l %d < 0 or alpha %g outside [0, 1]", k_l, (double)alpha);
    return MASKKV_EINVAL;
  }
  return launch_head_budgets(desc, prompt_mass, k_l, alpha, budgets, reinterpret_cast<hipStream_t>(stream));
}

int maskkv_layer_importance_workspace_bytes(size_t* bytes) {
  if (!bytes) {
    set_error("bytes is NULL");
    return MASKKV_EINVAL;
  }
  *bytes = layer_importance_workspace_bytes();
  return MASKKV_OK;
}

int maskkv_layer_importance(const void* h_in, const void* h_out, int64_t n_tokens, int32_t hidden, int32_t dtype,
                            int64_t row_stride, float* importance, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (dtype != MASKKV_F32 && dtype != MASKKV_BF16) {
    set_error("dtype %d is neither MASKKV_F32 nor MASKKV_BF16", dtype);
    return MASKKV_EDTYPE;
  }
  const int64_t eb = dtype == MASKKV_BF16 ? 2 : 4;
  if (!h_in || !h_out || !importance || n_tokens < 1 || hidden < 8 || (hidden & 7) || row_stride < hidden) {
    set_error("layer_importance: NULL pointer, n_tokens %lld < 1, hidden %d not a positive multiple of 8, or "
              "row_stride %lld < hidden", (long long)n_tokens, hidden, (long long)row_stride);
    return MASKKV_EINVAL;
  }
  if (((uintptr_t)h_in & 15) || ((uintptr_t)h_out & 15) || ((row_stride * eb) & 15) || ((hidden * eb) & 15)) {
    set_error("layer_importance: pointers, rows and row stride must be multiples of 16 bytes");
    return MASKKV_EINVAL;
  }
  if (int e = check_workspace("layer_importance", workspace, workspace_bytes, layer_importance_workspace_bytes()))
    return e;
  return launch_layer_importance(h_in, h_out, n_tokens, hidden, dtype, row_stride * eb, importance, workspace,
                                 reinterpret_cast<hipStream_t>(stream));
}

int maskkv_value_shift(const void* V_now, const void* V_prev, int64_t n_tokens, int32_t width, int32_t dtype,
                       int64_t row_stride, float delta, float* cos, int32_t* refresh, int32_t* count, void* stream) {
  if (dtype != MASKKV_F32 && dtype != MASKKV_BF16) {
    set_error("dtype %d is neither MASKKV_F32 nor MASKKV_BF16", dtype);
    return MASKKV_EDTYPE;
  }
  const int64_t eb = dtype == MASKKV_BF16 ? 2 : 4;
  if (!V_now || !V_prev || !cos || !refresh || !count || n_tokens < 1 || n_tokens > 0x7FFFFFFF || width < 8 ||
      (width & 7) || row_stride < width || !(delta == delta)) {
    set_error("value_shift: NULL pointer, n_tokens %lld outside 1..2^31-1, width %d not a positive multiple of 8, "
              "row_stride %lld < width, or delta is NaN", (long long)n_tokens, width, (long long)row_stride);
    return MASKKV_EINVAL;
  }
  if (((uintptr_t)V_now & 15) || ((uintptr_t)V_prev & 15) || ((row_stride * eb) & 15)) {
    set_error("value_shift: pointers and row stride must be multiples of 16 bytes");
    return MASKKV_EINVAL;
  }
  return launch_value_shift(V_now, V_prev, n_tokens, width, dtype, row_stride * eb, delta, cos, refresh, count,
                            reinterpret_cast<hipStream_t>(stream));
}

int maskkv_layer_budgets(const float* importance, int32_t n_layers, int64_t k_p, float beta, const int32_t* boundary,
                         int32_t n_boundary, int64_t* k_l) {
  if (!importance || !k_l || n_layers < 1 || k_p < 0 || !(beta >= 0.f && beta <= 1.f) || n_boundary < 0 ||
      (n_boundary > 0 && !boundary)) {
    set_error("layer_budgets: NULL pointer, n_layers %d < 1, k_p %lld < 0, beta %g outside [0, 1] or bad boundary list",
              n_layers, (long long)k_p, (double)beta);
    return MASKKV_EINVAL;
  }
  // group membership: 1 = boundary
  int first_last[2] = {0, n_layers - 1};
  const int32_t* bl = boundary ? boundary : first_last;
  const int nbl = boundary ? n_boundary : (n_layers > 1 ? 2 : 1);
  int n_b = 0;
  double imp_b = 0.0, imp_m = 0.0;
  for (int l = 0; l < n_layers; ++l) {
    if (!(importance[l] >= 0.f)) {
      set_error("layer_budgets: importance[%d] = %g is negative or NaN", l, (double)importance[l]);
      return MASKKV_EINVAL;
    }
    bool is_b = false;
    for (int i = 0; i < nbl; ++i) {
      if (bl[i] < 0 || bl[i] >= n_layers) {
        set_error("layer_budgets: boundary layer %d outside 0..%d", bl[i], n_layers - 1);
        return MASKKV_EINVAL;
      }
      is_b = is_b || bl[i] == l;
    }
    if (is_b) {
      ++n_b;
      imp_b += (double)importance[l];
    } else {
      imp_m += (double)importance[l];
    }
    k_l[l] = is_b ? 1 : 0;  // remembered until the shares are known
  }
  if (!(imp_b + imp_m > 0.0)) {
    set_error("layer_budgets: the importances sum to zero");
    return MASKKV_EINVAL;
  }
  const int n_m = n_layers - n_b;
  const int64_t k_base = (int64_t)floor((double)beta * (double)k_p / (double)n_layers);
  const double k_imp = (double)(k_p - (int64_t)n_layers * k_base);
  const double part_b = k_imp * imp_b / (imp_b + imp_m);
  const double part_m = k_imp - part_b;
  const int64_t share_b = n_b > 0 ? (int64_t)floor(part_b / n_b) : 0;
  const int64_t share_m = n_m > 0 ? (int64_t)floor(part_m / n_m) : 0;
  for (int l = 0; l < n_layers; ++l) k_l[l] = k_base + (k_l[l] ? share_b : share_m);
  return MASKKV_OK;
}

}  // extern "C"
