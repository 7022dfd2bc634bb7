// Entry points of the operators that need no context: argument checks, device, launch.
#include <cfloat>
#include <cstdio>
#include <cstdlib>

#include "kernels.h"
#include "moe_ep.h"

using namespace moe_ep;

namespace {

const char* set_why(const char** why, const char* msg) { if (why) *why = msg; return msg; }
int refuse(const char** why, const char* msg) { set_why(why, msg); return MOE_EP_EINVAL; }

thread_local char t_text[192];   // a message that names a pointer or a HIP error; the calling thread's until its next call

int hip_failed(const char** why, const char* what, hipError_t e)
{
    (void)hipGetLastError();
    snprintf(t_text, sizeof t_text, "%s: %s", what, hipGetErrorString(e));
    set_why(why, t_text);
    return MOE_EP_EHIP;
}

// The call's device is current while this lives; the caller's is afterwards.
struct DeviceScope {
    int before = -1;
    hipError_t error = hipSuccess;
    explicit DeviceScope(int device)
    {
        error = hipGetDevice(&before);
        if (error != hipSuccess) { before = -1; return; }
        if (before == device) before = -1;
        else if ((error = hipSetDevice(device)) != hipSuccess) before = -1;
    }
    ~DeviceScope() { if (before >= 0) (void)hipSetDevice(before); }
};

bool checks_pointers()
{
    static const bool on = [] { const char* v = getenv("MOE_EP_CHECK_POINTERS"); return !v || atoi(v) != 0; }();
    return on;
}

// rows of row_bytes, row_stride bytes apart
struct Span { const void* p; size_t rows, row_stride, row_bytes; const char* name; bool written; };
size_t extent(const Span& s) { return s.rows ? (s.rows - 1) * s.row_stride + s.row_bytes : 0; }

// whether some row of one lies on some row of the other; rows of the same distance may lie side by side
bool meet(const Span& s, const Span& t)
{
    const Span &a = s.p <= t.p ? s : t, &b = s.p <= t.p ? t : s;
    const size_t off = (size_t)(static_cast<const char*>(b.p) - static_cast<const char*>(a.p));
    if (off >= extent(a)) return false;
    if (a.row_stride != b.row_stride || a.rows < 2 || b.rows < 2) return true;
    const size_t at = off % a.row_stride;
    return at < a.row_bytes || at + b.row_bytes > a.row_stride;
}

// a result that lies on something else of its call, or NULL: needs no GPU
const char* overlap(const Span* sp, int n)
{
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j) {
            if (!sp[i].written || i == j || !sp[i].p || !sp[j].p || !meet(sp[i], sp[j])) continue;
            snprintf(t_text, sizeof t_text, "%s must not overlap %s", sp[i].name, sp[j].name);
            return t_text;
        }
    return nullptr;
}
// a buffer that the device cannot read or write, or NULL
const char* out_of_reach(const Span* sp, int n, int device)
{
    for (int i = 0; i < n && checks_pointers(); ++i) {
        if (!sp[i].p) continue;
        if (const char* bad = check_span(sp[i].p, extent(sp[i]), false, nullptr, device)) {
            snprintf(t_text, sizeof t_text, "%s %s", sp[i].name, bad);
            return t_text;
        }
    }
    return nullptr;
}

bool off_alignment(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

constexpr long long kMostStride = 1ll << 22, kMostFeatures = 1 << 20, kMostRows = 1 << 30;

}  // namespace

extern "C" {

int moe_ep_validate_routing(const moe_ep_routing* r, const char** why)
{
    set_why(why, "ok");
    if (!r) return refuse(why, "rule is NULL");
    if (r->n_experts < 1 || r->n_experts > 512) return refuse(why, "n_experts must be in 1..512");
    const int groups = r->n_groups == 0 ? 1 : r->n_groups;
    if (groups < 1 || groups > 64 || r->n_experts % groups) return refuse(why, "n_groups must be in 0..64 and divide n_experts");
    if (groups > 1 && (r->top_groups < 1 || r->top_groups > groups)) return refuse(why, "top_groups must be in 1..n_groups");
    const int reach = groups > 1 ? r->n_experts / groups * r->top_groups : r->n_experts;
    if (r->top_k < 1 || r->top_k > 64 || r->top_k > reach) return refuse(why, "top_k must be in 1..64 and at most the experts of top_groups groups");
    if (r->score != MOE_EP_SCORE_SOFTMAX && r->score != MOE_EP_SCORE_SIGMOID) return refuse(why, "unknown score");
    if (r->group_score != MOE_EP_GROUP_MAX && r->group_score != MOE_EP_GROUP_TOP2) return refuse(why, "unknown group_score");
    if (r->renormalise != 0 && r->renormalise != 1) return refuse(why, "renormalise must be 0 or 1");
    if (r->score_type != MOE_EP_BF16 && r->score_type != MOE_EP_F32) return refuse(why, "score_type must be MOE_EP_BF16 or MOE_EP_F32");
    if (r->score_stride != 0 && (r->score_stride < r->n_experts || r->score_stride > kMostStride)) return refuse(why, "score_stride must be 0 or in n_experts..2^22");
    if (!(r->scale > 0.f && r->scale <= FLT_MAX)) return refuse(why, "scale must be a positive number");
    if (r->device < 0) return refuse(why, "device must be >= 0");
    return MOE_EP_OK;
}

int moe_ep_route(const moe_ep_routing* r, const void* scores, const float* bias, const uint8_t* token_mask, int32_t n_tokens,
                 int32_t* idx, float* w, void* stream, const char** why)
{
    if (moe_ep_validate_routing(r, why) != MOE_EP_OK) return MOE_EP_EINVAL;
    if (n_tokens < 0 || n_tokens > kMostRows) return refuse(why, "n_tokens must be in 0..2^30");
    if (n_tokens == 0) return MOE_EP_OK;
    if (!scores || !idx || !w) return refuse(why, "scores, idx and w must not be NULL");
    const int size = r->score_type == MOE_EP_BF16 ? 2 : 4;
    const long long stride = r->score_stride ? r->score_stride : r->n_experts;
    if (off_alignment(scores, size) || off_alignment(bias, 4) || off_alignment(idx, 4) || off_alignment(w, 4))
        return refuse(why, "scores, bias, idx and w must be aligned to their elements");
    const size_t out = (size_t)n_tokens * r->top_k * 4;
    const Span sp[] = {{scores, (size_t)n_tokens, (size_t)stride * size, (size_t)r->n_experts * size, "scores", false},
                       {bias, 1, 0, (size_t)r->n_experts * 4, "bias", false},
                       {token_mask, 1, 0, (size_t)n_tokens, "token_mask", false},
                       {idx, 1, 0, out, "idx", true},
                       {w, 1, 0, out, "w", true}};
    if (const char* bad = overlap(sp, 5)) return refuse(why, bad);
    DeviceScope device(r->device);
    if (device.error != hipSuccess) return hip_failed(why, "selecting the device", device.error);
    if (const char* bad = out_of_reach(sp, 5, r->device)) return refuse(why, bad);
    const int groups = r->n_groups == 0 ? 1 : r->n_groups;
    const RouteArgs a{scores, bias, token_mask, idx, w, stride, n_tokens, r->n_experts, r->top_k, groups, groups > 1 ? r->top_groups : 1,
                      r->score_type == MOE_EP_BF16, r->score == MOE_EP_SCORE_SIGMOID, r->group_score == MOE_EP_GROUP_TOP2, r->renormalise != 0, r->scale};
    const hipError_t e = launch_route(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_EP_OK : hip_failed(why, "launch", e);
}

int moe_ep_validate_linear(const moe_ep_linear_config* c, const char** why)
{
    set_why(why, "ok");
    if (!c) return refuse(why, "cfg is NULL");
    if (c->in_features < 1 || c->in_features > kMostFeatures) return refuse(why, "in_features must be in 1..2^20");
    if (c->out_features < 1 || c->out_features > kMostFeatures) return refuse(why, "out_features must be in 1..2^20");
    if (c->weight_type != MOE_EP_BF16 && c->weight_type != MOE_EP_F32) return refuse(why, "weight_type must be MOE_EP_BF16 or MOE_EP_F32");
    if (c->out_type != MOE_EP_BF16 && c->out_type != MOE_EP_F32) return refuse(why, "out_type must be MOE_EP_BF16 or MOE_EP_F32");
    if (c->activation < 0 || c->activation >= kActCount) return refuse(why, "unknown activation");
    const auto fits = [](long long stride, long long cols) { return stride == 0 || (stride >= cols && stride <= kMostStride); };
    if (!fits(c->x_stride, c->in_features)) return refuse(why, "x_stride must be 0 or in in_features..2^22");
    if (!fits(c->weight_stride, c->in_features)) return refuse(why, "weight_stride must be 0 or in in_features..2^22");
    if (!fits(c->residual_stride, c->out_features)) return refuse(why, "residual_stride must be 0 or in out_features..2^22");
    if (!fits(c->out_stride, c->out_features)) return refuse(why, "out_stride must be 0 or in out_features..2^22");
    if (c->device < 0) return refuse(why, "device must be >= 0");
    return MOE_EP_OK;
}

int moe_ep_linear(const moe_ep_linear_config* c, const void* x, const void* weight, const float* bias, const void* residual,
                  int32_t n_rows, void* out, void* stream, const char** why)
{
    if (moe_ep_validate_linear(c, why) != MOE_EP_OK) return MOE_EP_EINVAL;
    if (n_rows < 0 || n_rows > kMostRows) return refuse(why, "n_rows must be in 0..2^30");
    if (n_rows == 0) return MOE_EP_OK;
    if (!x || !weight || !out) return refuse(why, "x, weight and out must not be NULL");
    const int K = c->in_features, N = c->out_features;
    const int ws = c->weight_type == MOE_EP_F32 ? 4 : 2, os = c->out_type == MOE_EP_F32 ? 4 : 2;
    const long long ldx = c->x_stride ? c->x_stride : K, ldw = c->weight_stride ? c->weight_stride : K;
    const long long ldr = c->residual_stride ? c->residual_stride : N, ldo = c->out_stride ? c->out_stride : N;
    if (off_alignment(x, 2) || off_alignment(weight, ws) || off_alignment(bias, 4) || off_alignment(residual, os) || off_alignment(out, os))
        return refuse(why, "x, weight, bias, residual and out must be aligned to their elements");
    // an element of the residual is read by the lane that writes the result in its place: the same buffer may be both
    const bool in_place = residual == out && ldr == ldo;
    const size_t rows = (size_t)n_rows;
    const Span sp[] = {{x, rows, (size_t)ldx * 2, (size_t)K * 2, "x", false},
                       {weight, (size_t)N, (size_t)ldw * ws, (size_t)K * ws, "weight", false},
                       {bias, 1, 0, (size_t)N * 4, "bias", false},
                       {in_place ? nullptr : residual, rows, (size_t)ldr * os, (size_t)N * os, "residual", false},
                       {out, rows, (size_t)ldo * os, (size_t)N * os, "out", true}};
    if (const char* bad = overlap(sp, 5)) return refuse(why, bad);
    DeviceScope device(c->device);
    if (device.error != hipSuccess) return hip_failed(why, "selecting the device", device.error);
    if (const char* bad = out_of_reach(sp, 5, c->device)) return refuse(why, bad);
    LinearArgs a{};
    a.x = static_cast<const uint16_t*>(x); a.w = weight; a.bias = bias; a.residual = residual; a.out = out;
    a.ldx = ldx; a.ldw = ldw; a.ldr = ldr; a.ldo = ldo;
    a.R = n_rows; a.N = N; a.K = K; a.act = c->activation;
    a.w32 = ws == 4; a.out32 = os == 4;
    int n_cu = 0;
    hipError_t e = hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, c->device);
    if (e == hipSuccess) e = launch_linear(a, n_cu, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_EP_OK : hip_failed(why, "launch", e);
}

}  // extern "C"
