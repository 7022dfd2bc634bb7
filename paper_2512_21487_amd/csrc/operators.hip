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
// A buffer that the device cannot read or write, or NULL.  Buffers often lie in one allocation: one that lies in an allocation that another of this call's was found in is not asked
// about again (0.2 us each).
const char* out_of_reach(const Span* sp, int n, int device)
{
    constexpr int kMost = 16;
    Allocation known[kMost];
    int count = 0;
    for (int i = 0; i < n && checks_pointers(); ++i) {
        if (!sp[i].p) continue;
        const char* const p = static_cast<const char*>(sp[i].p);
        const size_t bytes = extent(sp[i]);
        bool in = false;
        for (int k = 0; k < count && !in; ++k) in = p >= known[k].base && (size_t)(p - known[k].base) <= known[k].size && known[k].size - (size_t)(p - known[k].base) >= bytes;
        if (in) continue;
        Allocation found{nullptr, 0};
        if (const char* bad = check_span(p, bytes, false, nullptr, device, &found)) {
            snprintf(t_text, sizeof t_text, "%s %s", sp[i].name, bad);
            return t_text;
        }
        if (found.base && count < kMost) known[count++] = found;
    }
    return nullptr;
}

bool off_alignment(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

constexpr long long kMostStride = 1ll << 22, kMostFeatures = 1 << 20, kMostRows = 1 << 30, kMostAdapters = 1 << 20;

// A product's arguments as its kernels read them, and what it reads and writes
struct Product {
    static constexpr int kSpans = 5;
    LinearArgs args{};
    Span spans[kSpans];
    bool aligned;
    Product(const moe_ep_linear_config& c, const void* x, const void* weight, const float* bias, const void* residual, int32_t n_rows, void* out)
    {
        const int K = c.in_features, N = c.out_features;
        const int ws = c.weight_type == MOE_EP_F32 ? 4 : 2, os = c.out_type == MOE_EP_F32 ? 4 : 2;
        const long long ldx = c.x_stride ? c.x_stride : K, ldw = c.weight_stride ? c.weight_stride : K;
        const long long ldr = c.residual_stride ? c.residual_stride : N, ldo = c.out_stride ? c.out_stride : N;
        aligned = !off_alignment(x, 2) && !off_alignment(weight, ws) && !off_alignment(bias, 4) && !off_alignment(residual, os) && !off_alignment(out, os);
        // an element of the residual is read by the lane that writes the result in its place: the same buffer may be both
        const bool in_place = residual == out && ldr == ldo;
        const size_t rows = (size_t)n_rows;
        spans[0] = {x, rows, (size_t)ldx * 2, (size_t)K * 2, "x", false};
        spans[1] = {weight, (size_t)N, (size_t)ldw * ws, (size_t)K * ws, "weight", false};
        spans[2] = {bias, 1, 0, (size_t)N * 4, "bias", false};
        spans[3] = {in_place ? nullptr : residual, rows, (size_t)ldr * os, (size_t)N * os, "residual", false};
        spans[4] = {out, rows, (size_t)ldo * os, (size_t)N * os, "out", true};
        args.x = static_cast<const uint16_t*>(x); args.w = weight; args.bias = bias; args.residual = residual; args.out = out;
        args.ldx = ldx; args.ldw = ldw; args.ldr = ldr; args.ldo = ldo;
        args.R = n_rows; args.N = N; args.K = K; args.act = c.activation;
        args.w32 = ws == 4; args.out32 = os == 4;
    }
};

// What the workspace holds: x A^T of every row; behind it, of up to kGathered rows, x W^T in fp32 and the groups' table, of more the lists of the row tiles, a bit for every row of a tile and, where rows are
// not on 16 bytes, copies of x and of W that are.  A tile has 16 to 256 rows: (R / t + 1)
// (1 + t (1 + t / 32)) numbers are at most those of t = 256 and one more for 16 rows.
struct AdapterWorkspace {
    size_t low, wide, table, lists, none, x, w;
    AdapterWorkspace(const moe_ep_linear_config& c, const moe_ep_adapter_config& ad, int32_t n_rows)
    {
        const int few = n_rows < kGathered ? n_rows : kGathered;
        low = (size_t)n_rows * adapter_pitch(adapter_width(ad.rank)) * 2;
        wide = ((size_t)few * c.out_features * 4 + 15) / 16 * 16;
        table = (size_t)adapter_groups(few, ad.n_adapters) * kGroupEntry * 4;
        lists = (((size_t)n_rows * 9 + n_rows / 16 + adapter_list(256) + 1) * 4 + 15) / 16 * 16;
        none = n_rows > kGathered ? (((size_t)n_rows + 15) / 16 * (((size_t)c.out_features + 31) / 32) * 2 + 15) / 16 * 16 : 0;
        const int K = c.in_features;
        const size_t row = (size_t)adapter_pitch_of(K) * 2;
        x = n_rows > kGathered && rows_off_16(K, c.x_stride ? c.x_stride : K) ? n_rows * row : 0;
        w = n_rows > kGathered && rows_off_16(K, c.weight_stride ? c.weight_stride : K) ? c.out_features * row : 0;
    }
    size_t bytes() const { return low + (wide + table > lists + none + x + w ? wide + table : lists + none + x + w); }   // of more rows not fewer: that holds of each
};

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
    const Product p(*c, x, weight, bias, residual, n_rows, out);
    if (!p.aligned) return refuse(why, "x, weight, bias, residual and out must be aligned to their elements");
    if (const char* bad = overlap(p.spans, Product::kSpans)) return refuse(why, bad);
    DeviceScope device(c->device);
    if (device.error != hipSuccess) return hip_failed(why, "selecting the device", device.error);
    if (const char* bad = out_of_reach(p.spans, Product::kSpans, c->device)) return refuse(why, bad);
    int n_cu = 0;
    hipError_t e = hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, c->device);
    if (e == hipSuccess) e = launch_linear(p.args, n_cu, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_EP_OK : hip_failed(why, "launch", e);
}

int moe_ep_validate_linear_adapters(const moe_ep_linear_config* c, const moe_ep_adapter_config* ad, const char** why)
{
    if (moe_ep_validate_linear(c, why) != MOE_EP_OK) return MOE_EP_EINVAL;
    if (c->weight_type != MOE_EP_BF16) return refuse(why, "weight_type must be MOE_EP_BF16 beside adapters");
    if (!ad) return refuse(why, "adapters is NULL");
    if (ad->n_adapters < 1 || ad->n_adapters > kMostAdapters) return refuse(why, "n_adapters must be in 1..2^20");
    if (ad->rank < 8 || ad->rank > kRankMost || ad->rank % 8) return refuse(why, "rank must be a multiple of 8 in 8..128");
    return MOE_EP_OK;
}

size_t moe_ep_linear_adapters_workspace_bytes(const moe_ep_linear_config* c, const moe_ep_adapter_config* ad, int32_t n_rows)
{
    if (moe_ep_validate_linear_adapters(c, ad, nullptr) != MOE_EP_OK || n_rows < 1 || n_rows > kMostRows) return 0;
    return AdapterWorkspace(*c, *ad, n_rows).bytes();
}

int moe_ep_linear_adapters(const moe_ep_linear_config* c, const moe_ep_adapter_config* ad, const void* x, const void* weight, const float* bias,
                           const void* residual, const int32_t* index, const void* down, const void* up, const float* scale, int32_t n_rows, void* out,
                           void* workspace, size_t workspace_bytes, void* stream, const char** why)
{
    if (moe_ep_validate_linear_adapters(c, ad, why) != MOE_EP_OK) return MOE_EP_EINVAL;
    if (n_rows < 0 || n_rows > kMostRows) return refuse(why, "n_rows must be in 0..2^30");
    if (n_rows == 0) return MOE_EP_OK;
    if (!x || !weight || !out) return refuse(why, "x, weight and out must not be NULL");
    if (!index || !down || !up || !workspace) return refuse(why, "index, down, up and workspace must not be NULL");
    const Product p(*c, x, weight, bias, residual, n_rows, out);
    if (!p.aligned || off_alignment(index, 4) || off_alignment(down, 2) || off_alignment(scale, 4))
        return refuse(why, "x, weight, bias, residual, index, down, scale and out must be aligned to their elements");
    if (off_alignment(up, 16) || off_alignment(workspace, 16)) return refuse(why, "up and workspace must be aligned to 16 bytes");
    const size_t need = moe_ep_linear_adapters_workspace_bytes(c, ad, n_rows);
    if (workspace_bytes < need) {
        snprintf(t_text, sizeof t_text, "workspace has %zu bytes, the call needs %zu", workspace_bytes, need);
        return refuse(why, t_text);
    }
    const size_t n = (size_t)ad->n_adapters, each = (size_t)ad->rank * 2;
    constexpr int kSpans = Product::kSpans + 5;
    Span sp[kSpans];
    for (int i = 0; i < Product::kSpans; ++i) sp[i] = p.spans[i];
    Span* const mine = sp + Product::kSpans;
    mine[0] = {index, 1, 0, (size_t)n_rows * 4, "index", false};
    mine[1] = {down, 1, 0, n * each * (size_t)c->in_features, "down", false};
    mine[2] = {up, 1, 0, n * each * (size_t)c->out_features, "up", false};
    mine[3] = {scale, 1, 0, n * 4, "scale", false};
    mine[4] = {workspace, 1, 0, need, "workspace", true};
    if (const char* bad = overlap(sp, kSpans)) return refuse(why, bad);
    DeviceScope device(c->device);
    if (device.error != hipSuccess) return hip_failed(why, "selecting the device", device.error);
    if (const char* bad = out_of_reach(sp, kSpans, c->device)) return refuse(why, bad);
    int n_cu = 0;
    hipError_t e = hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, c->device);
    if (e != hipSuccess) return hip_failed(why, "launch", e);
    AdapterArgs a{};
    a.index = index; a.down = static_cast<const uint16_t*>(down); a.up = static_cast<const uint16_t*>(up); a.scale = scale;
    a.low = static_cast<uint16_t*>(workspace);
    a.n = ad->n_adapters; a.rank = ad->rank; a.width = adapter_width(a.rank);
    const AdapterWorkspace parts(*c, *ad, n_rows);
    char* const behind = static_cast<char*>(workspace) + parts.low;
    if (n_rows <= kGathered)
        e = launch_linear_grouped(p.args, a, reinterpret_cast<float*>(behind), reinterpret_cast<int32_t*>(behind + parts.wide), n_cu, static_cast<hipStream_t>(stream));
    else {
        a.lists = reinterpret_cast<int32_t*>(behind);
        a.none = reinterpret_cast<uint16_t*>(behind + parts.lists);
        char* const copies = behind + parts.lists + parts.none;
        e = launch_linear_adapters(p.args, a, parts.x ? reinterpret_cast<uint16_t*>(copies) : nullptr, parts.w ? reinterpret_cast<uint16_t*>(copies + parts.x) : nullptr, n_cu,
                                   static_cast<hipStream_t>(stream));
    }
    return e == hipSuccess ? MOE_EP_OK : hip_failed(why, "launch", e);
}

int moe_ep_validate_norm(const moe_ep_norm_config* c, const char** why)
{
    set_why(why, "ok");
    if (!c) return refuse(why, "cfg is NULL");
    if (c->features < 1 || c->features > kNormMost) return refuse(why, "features must be in 1..32768");
    if (c->norm_after < 0 || c->norm_after >= kNormCount) return refuse(why, "unknown norm_after");
    if (c->norm_before < 0 || c->norm_before >= kNormCount) return refuse(why, "unknown norm_before");
    const auto type = [](int t) { return t == MOE_EP_BF16 || t == MOE_EP_F32; };
    if (!type(c->block_type)) return refuse(why, "block_type must be MOE_EP_BF16 or MOE_EP_F32");
    if (!type(c->stream_type)) return refuse(why, "stream_type must be MOE_EP_BF16 or MOE_EP_F32");
    if (!type(c->out_type)) return refuse(why, "out_type must be MOE_EP_BF16 or MOE_EP_F32");
    if (!type(c->weight_type)) return refuse(why, "weight_type must be MOE_EP_BF16 or MOE_EP_F32");
    if (!type(c->gate_type)) return refuse(why, "gate_type must be MOE_EP_BF16 or MOE_EP_F32");
    if (c->gate_form < 0 || c->gate_form >= kGateCount) return refuse(why, "unknown gate_form");
    if (c->gate_per_row != 0 && c->gate_per_row != 1) return refuse(why, "gate_per_row must be 0 or 1");
    const bool norms = c->norm_after != MOE_EP_NORM_NONE || c->norm_before != MOE_EP_NORM_NONE;
    if (norms && !(c->eps >= 1e-20f && c->eps <= 1.0f)) return refuse(why, "eps must be in 1e-20..1");
    const auto finite = [](float f) { return f >= -FLT_MAX && f <= FLT_MAX; };
    if (!finite(c->block_scale)) return refuse(why, "block_scale must be finite");
    if (!finite(c->residual_scale)) return refuse(why, "residual_scale must be finite");
    if (!finite(c->weight_offset)) return refuse(why, "weight_offset must be finite");
    const auto fits = [](long long stride, long long cols) { return stride == 0 || (stride >= cols && stride <= kMostStride); };
    if (!fits(c->block_stride, c->features)) return refuse(why, "block_stride must be 0 or in features..2^22");
    if (!fits(c->residual_stride, c->features)) return refuse(why, "residual_stride must be 0 or in features..2^22");
    if (!fits(c->gate_stride, c->gate_per_row ? 1 : c->features)) return refuse(why, "gate_stride must be 0 or in features (of one gate a row: 1)..2^22");
    if (!fits(c->sum_stride, c->features)) return refuse(why, "sum_stride must be 0 or in features..2^22");
    if (!fits(c->out_stride, c->features)) return refuse(why, "out_stride must be 0 or in features..2^22");
    if (c->device < 0) return refuse(why, "device must be >= 0");
    return MOE_EP_OK;
}

int moe_ep_norm(const moe_ep_norm_config* c, const void* block, const void* residual, const void* gate, const void* after_weight, const void* after_bias,
                const void* before_weight, const void* before_bias, int32_t n_rows, void* sum, void* out, void* stream, const char** why)
{
    if (moe_ep_validate_norm(c, why) != MOE_EP_OK) return MOE_EP_EINVAL;
    if (n_rows < 0 || n_rows > kMostRows) return refuse(why, "n_rows must be in 0..2^30");
    if (n_rows == 0) return MOE_EP_OK;
    const bool before = c->norm_before != MOE_EP_NORM_NONE;
    if (!block) return refuse(why, "block must not be NULL");
    if (before != (out != nullptr)) return refuse(why, "out must be given exactly where there is a norm_before");
    if (!before && (before_weight || before_bias)) return refuse(why, "before_weight and before_bias need a norm_before");
    if (!sum && !out) return refuse(why, "sum and out must not both be NULL");
    const int M = c->features;
    const auto size = [](int type) { return type == MOE_EP_F32 ? 4 : 2; };
    const int bs = size(c->block_type), ss = size(c->stream_type), os = size(c->out_type), ws = size(c->weight_type), gs = size(c->gate_type);
    const auto apart = [](long long stride, int cols) { return stride ? stride : (long long)cols; };
    const int gate_cols = c->gate_per_row ? 1 : M;
    const long long ldb = apart(c->block_stride, M), ldr = apart(c->residual_stride, M), ldg = apart(c->gate_stride, gate_cols);
    const long long lds = apart(c->sum_stride, M), ldo = apart(c->out_stride, M);
    if (off_alignment(block, bs) || off_alignment(residual, ss) || off_alignment(gate, gs) || off_alignment(sum, ss) || off_alignment(out, os) ||
        off_alignment(after_weight, ws) || off_alignment(after_bias, ws) || off_alignment(before_weight, ws) || off_alignment(before_bias, ws))
        return refuse(why, "every pointer must be aligned to its elements");
    // a lane reads its elements of a row before it writes in their place, and no other lane does either
    const bool stream_in_place = residual == sum && ldr == lds, block_in_place = block == out && ldb == ldo && bs == os;
    const size_t rows = (size_t)n_rows, vector = (size_t)M * ws;
    const Span sp[] = {{block, rows, (size_t)ldb * bs, (size_t)M * bs, "block", false},
                       {residual, rows, (size_t)ldr * ss, (size_t)M * ss, "residual", false},
                       {gate, rows, (size_t)ldg * gs, (size_t)gate_cols * gs, "gate", false},
                       {after_weight, 1, 0, vector, "after_weight", false},
                       {after_bias, 1, 0, vector, "after_bias", false},
                       {before_weight, 1, 0, vector, "before_weight", false},
                       {before_bias, 1, 0, vector, "before_bias", false},
                       {sum, rows, (size_t)lds * ss, (size_t)M * ss, "sum", true},
                       {out, rows, (size_t)ldo * os, (size_t)M * os, "out", true}};
    constexpr int kSpans = sizeof sp / sizeof *sp, kSum = kSpans - 2, kOut = kSpans - 1;
    Span others[kSpans];
    for (int i = 0; i < kSpans; ++i) others[i] = sp[i];
    if (stream_in_place) others[1].p = nullptr;
    others[kOut].written = false;
    if (const char* bad = overlap(others, kSpans)) return refuse(why, bad);        // of sum with everything, out among it
    others[1].p = residual;
    others[kOut].written = true;
    others[kSum].written = false;
    if (block_in_place) others[0].p = nullptr;
    if (const char* bad = overlap(others, kSpans)) return refuse(why, bad);        // and of out
    DeviceScope device(c->device);
    if (device.error != hipSuccess) return hip_failed(why, "selecting the device", device.error);
    if (const char* bad = out_of_reach(sp, kSpans, c->device)) return refuse(why, bad);
    NormArgs a{};
    a.block = block; a.residual = residual; a.gate = gate; a.sum = sum; a.out = out;
    a.after_weight = after_weight; a.after_bias = after_bias; a.before_weight = before_weight; a.before_bias = before_bias;
    a.ldb = ldb; a.ldr = ldr; a.ldg = ldg; a.lds = lds; a.ldo = ldo;
    a.R = n_rows; a.M = M; a.after = c->norm_after; a.before = c->norm_before; a.gate_form = c->gate_form;
    a.block32 = bs == 4; a.stream32 = ss == 4; a.out32 = os == 4; a.weight32 = ws == 4; a.gate32 = gs == 4; a.gate_per_row = c->gate_per_row != 0;
    a.eps = c->eps; a.block_scale = c->block_scale; a.residual_scale = c->residual_scale; a.offset = c->weight_offset;
    int n_cu = 0;
    hipError_t e = hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, c->device);
    if (e == hipSuccess) e = launch_norm(a, n_cu, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_EP_OK : hip_failed(why, "launch", e);
}

}  // extern "C"
