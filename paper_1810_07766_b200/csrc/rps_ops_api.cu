// C ABI of the training operators (include/rps_ops.h): argument checks, the layout of the lent workspaces, and the order
// of the launches.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "rps_ops_kernels.h"

namespace {

using namespace rps_ops;

thread_local char g_error[256] = "";

int fail(int code, const char* format, ...)
{
    va_list args;
    va_start(args, format);
    vsnprintf(g_error, sizeof(g_error), format, args);
    va_end(args);
    return code;
}

int cuda_status(cudaError_t err, const char* where)
{
    if (err == cudaSuccess) return RPS_OK;
    return fail(RPS_ECUDA, "%s: %s", where, cudaGetErrorString(err));
}

#define RPS_TRY(call)                                              \
    do {                                                           \
        const int status_ = cuda_status((call), __func__);         \
        if (status_ != RPS_OK) return status_;                     \
    } while (0)

int start()
{
    g_error[0] = '\0';
    return RPS_OK;
}

// Hands out 256-byte aligned parts of a workspace; with base 0 it only counts.
struct Carver {
    unsigned char* base;
    size_t used = 0;
    template <typename T>
    T* take(int64_t count)
    {
        T* at = reinterpret_cast<T*>(base + used);
        used += (size_t)round_up(count * (int64_t)sizeof(T), 256);
        return at;
    }
};

bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

bool aligned_matrix(const void* p, int64_t row, int64_t worker) { return aligned(p, 16) && row % 8 == 0 && worker % 8 == 0; }

// A piece of the vocabulary is as wide as lets dl (and the weight, where it has to be laid out anew) of one piece stay within this.
constexpr int64_t kPieceBytes = 512ll << 20;
constexpr int64_t kMaxSize = (1ll << 24) - 1;

int check_output_strides(const char* name, int n, int64_t rows, int64_t cols, int64_t row, int64_t worker)
{
    if (row < cols) return fail(RPS_EINVAL, "%s: a row stride of %lld is less than the %lld columns", name, (long long)row, (long long)cols);
    if (row >= 1ll << 31) return fail(RPS_EINVAL, "%s: a row stride of %lld", name, (long long)row);
    if (n > 1 && worker < (rows - 1) * row + cols && (worker < cols || row < (n - 1) * worker + cols))
        return fail(RPS_EINVAL, "%s: the workers' parts overlap (worker stride %lld)", name, (long long)worker);
    return RPS_OK;
}

int check_common(int dtype, int n)
{
    if (dtype != RPS_F32 && dtype != RPS_BF16) return fail(RPS_EINVAL, "dtype %d is neither RPS_F32 nor RPS_BF16", dtype);
    if (n < 1 || n > RPS_MAX_WORKERS) return fail(RPS_EINVAL, "n = %d workers; 1..%d are possible", n, (int)RPS_MAX_WORKERS);
    return RPS_OK;
}

int check_workspace(const void* workspace, size_t have, size_t want)
{
    if (have < want) return fail(RPS_EINVAL, "a workspace of %zu bytes is needed, %zu were given", want, have);
    if (want > 0 && (workspace == nullptr || !aligned(workspace, 256))) return fail(RPS_EINVAL, "the workspace is NULL or not 256-byte aligned");
    return RPS_OK;
}

// ------------------------------------------------------------------------------------------------------------ loss

struct LcePlan {
    LceParams p{};
    ProductParams product{};
    bool lay_out_weight = false;
    int64_t piece = 0;
    bf16* weight = nullptr;
    bf16* dl = nullptr;
    float* hidden_parts = nullptr;
    float* weight_parts = nullptr;
    ProductShape hidden_shape{}, weight_shape{};
    size_t bytes = 0;
};

int check_lce(const rps_lce_desc* d)
{
    if (d == nullptr) return fail(RPS_EINVAL, "desc is NULL");
    if (int rc = check_common(d->dtype, d->n)) return rc;
    if (d->reduction < RPS_REDUCE_NONE || d->reduction > RPS_REDUCE_MEAN) return fail(RPS_EINVAL, "reduction %d", d->reduction);
    if (d->tokens < 0 || d->tokens > kMaxSize) return fail(RPS_EINVAL, "tokens = %lld", (long long)d->tokens);
    if (d->vocab < 1 || d->vocab >= 1ll << 30) return fail(RPS_EINVAL, "vocab = %lld", (long long)d->vocab);
    if (d->cols < 1 || d->cols > kMaxSize) return fail(RPS_EINVAL, "cols = %lld", (long long)d->cols);
    if (d->hidden_row < d->cols || d->weight_row < d->cols || d->hidden_worker < 0 || d->weight_worker < 0)
        return fail(RPS_EINVAL, "strides of hidden (%lld, %lld) or weight (%lld, %lld)", (long long)d->hidden_worker,
                    (long long)d->hidden_row, (long long)d->weight_worker, (long long)d->weight_row);
    return RPS_OK;
}

LcePlan plan_lce(const rps_lce_desc& d, const void* weight, bool backward, void* workspace)
{
    LcePlan plan;
    LceParams& p = plan.p;
    p.n = d.n, p.f32 = d.dtype == RPS_F32, p.planes = p.f32 ? 3 : 1, p.reduction = d.reduction, p.backward = backward;
    p.tokens = d.tokens, p.tokens_padded = round_up(d.tokens > 0 ? d.tokens : 1, kTokenTile);
    p.vocab = d.vocab, p.cols = d.cols, p.cols_padded = round_up(d.cols, 8), p.ignore_index = d.ignore_index;
    p.hidden_row = d.hidden_row, p.hidden_worker = d.hidden_worker;
    plan.lay_out_weight = p.f32 || !aligned_matrix(weight, d.weight_row, d.weight_worker);
    plan_lce_dot(&p);
    if (p.dot_rows > 0) {
        Carver c{static_cast<unsigned char*>(workspace)};
        p.count = c.take<int>(p.n);
        p.rows = c.take<int>(p.n * p.tokens);
        p.target = c.take<int>(p.n * p.tokens_padded);
        if (backward) {
            p.info = c.take<float2>(p.n * p.tokens_padded);
            p.scale = c.take<float>(p.n);
            p.dot_dl = c.take<float>(p.n * p.vocab * p.dot_rows);
            p.dot_parts = c.take<float>(p.dot_ranges * p.n * p.dot_rows * round_up(p.cols, 4));
        } else {
            p.done = c.take<int>(p.n);
            p.sums = c.take<float>(p.n * lce_merge_blocks(p.tokens));
            p.stat_tiles = p.dot_blocks;
            p.part = c.take<float2>(p.n * p.stat_tiles * p.tokens_padded);
            p.hit = c.take<float>(p.n * p.tokens_padded);
        }
        plan.bytes = c.used;
        return plan;
    }
    const int64_t whole = round_up(d.vocab, kVocabTile);
    plan.piece = whole;
    const auto narrow = [&](int64_t bytes_per_column) {
        const int64_t most = kPieceBytes / bytes_per_column / kVocabTile * kVocabTile;
        if (plan.piece > most) plan.piece = most > kVocabTile ? most : kVocabTile;
    };
    if (backward) narrow(p.n * p.planes * p.tokens_padded * 2);
    if (plan.lay_out_weight) narrow(p.n * p.planes * p.cols_padded * 2);
    ProductParams& g = plan.product;
    // in several pieces the tiles are whole, so that the pieces' statistics lie side by side
    g.shaped(product_shape(d.tokens, d.vocab, d.cols, d.n, p.planes, false));
    if (plan.piece < whole)
        g.tile_cols = kVocabTile;
    else
        plan.piece = round_up(d.vocab, g.tile_cols);  // dl is written in whole tiles
    p.stat_tiles = ceil_div(d.vocab, g.tile_cols);

    Carver c{static_cast<unsigned char*>(workspace)};
    p.count = c.take<int>(p.n);
    p.rows = c.take<int>(p.n * p.tokens);
    p.target = c.take<int>(p.n * p.tokens_padded);
    p.packed = c.take<bf16>(p.n * p.planes * p.tokens_padded * p.cols_padded);
    if (plan.lay_out_weight) plan.weight = c.take<bf16>(p.n * p.planes * plan.piece * p.cols_padded);
    if (backward) {
        p.info = c.take<float2>(p.n * p.tokens_padded);
        plan.dl = c.take<bf16>(p.n * p.planes * p.tokens_padded * plan.piece);
        p.scale = c.take<float>(p.n);
        plan.hidden_shape = product_shape(d.tokens, d.cols, plan.piece < d.vocab ? plan.piece : d.vocab, p.n, p.planes, true);
        if (plan.piece < d.vocab || plan.hidden_shape.splits > 1)
            plan.hidden_parts = c.take<float>(plan.hidden_shape.splits * p.n * p.tokens_padded * round_up(p.cols, plan.hidden_shape.tile_cols));
        plan.weight_shape = product_shape(plan.piece < d.vocab ? plan.piece : d.vocab, d.cols, d.tokens, p.n, p.planes, true);
        if (plan.weight_shape.splits > 1) plan.weight_parts = c.take<float>(plan.weight_shape.splits * p.n * plan.piece * round_up(p.cols, plan.weight_shape.tile_cols));
    } else {
        p.done = c.take<int>(p.n);
        p.sums = c.take<float>(p.n * lce_merge_blocks(p.tokens));
        p.part = c.take<float2>(p.n * p.stat_tiles * p.tokens_padded);
        p.hit = c.take<float>(p.n * p.tokens_padded);
    }
    plan.bytes = c.used;

    g.workers = p.n, g.planes = p.planes, g.count = p.count;
    g.vocab = (int)p.vocab, g.stat_tiles = (int)p.stat_tiles, g.target = p.target;
    g.part = const_cast<float2*>(p.part), g.hit = const_cast<float*>(p.hit), g.info = p.info, g.dl = plan.dl;
    g.tokens_padded = p.tokens_padded, g.piece = plan.piece, g.rows = p.rows, g.tokens = p.tokens;
    g.scale = p.scale;
    return plan;
}

Operand hidden_operand(const LceParams& p)
{
    const int64_t plane = p.tokens_padded * p.cols_padded;
    return {p.packed, p.planes * plane, plane, p.cols_padded, p.tokens_padded, p.cols_padded};
}

// The piece's rows of the weight as an operand, laid out anew where the tensor cores cannot read them as they are.
int weight_operand(const rps_lce_desc& d, const LcePlan& plan, const void* weight, int64_t v0, int64_t rows, Operand* out, cudaStream_t stream)
{
    const LceParams& p = plan.p;
    if (!plan.lay_out_weight) {
        *out = {static_cast<const bf16*>(weight) + v0 * d.weight_row, d.weight_worker, 0, d.weight_row, rows, d.cols};
        return RPS_OK;
    }
    const int64_t plane = plan.piece * p.cols_padded;
    PlanesParams q{};
    q.src = static_cast<const unsigned char*>(weight) + v0 * d.weight_row * (p.f32 ? 4 : 2);
    q.f32 = p.f32, q.n = p.n, q.planes = p.planes;
    q.rows = rows, q.cols = d.cols, q.src_row = d.weight_row, q.src_worker = d.weight_worker;
    q.dst = plan.weight, q.dst_row = p.cols_padded, q.dst_plane = plane, q.dst_worker = p.planes * plane;
    *out = {plan.weight, p.planes * plane, plane, p.cols_padded, rows, p.cols_padded};
    return cuda_status(launch_planes(q, stream), "laying the weight out");
}

}  // namespace

extern "C" const char* rps_ops_last_error(void) { return g_error; }

extern "C" int rps_ops_check(void* cuda_stream)
{
    start();
    int gave_up = 0, norm_gave_up = 0;
    RPS_TRY(read_gave_up(&gave_up, static_cast<cudaStream_t>(cuda_stream)));
    RPS_TRY(read_norm_gave_up(&norm_gave_up, static_cast<cudaStream_t>(cuda_stream)));
    return gave_up == 0 && norm_gave_up == 0 ? RPS_OK : fail(RPS_ECUDA, "a wait inside a kernel gave up; the outputs of the calls since the last check are not valid");
}

extern "C" int rps_lce_workspace(const rps_lce_desc* desc, const void* weight, int backward, size_t* bytes)
{
    start();
    if (bytes == nullptr) return fail(RPS_EINVAL, "bytes is NULL");
    if (int rc = check_lce(desc)) return rc;
    *bytes = plan_lce(*desc, weight, backward != 0, nullptr).bytes;
    return RPS_OK;
}

extern "C" int rps_lce_forward(const rps_lce_desc* desc, const void* hidden, const void* weight, const int64_t* targets,
                               float* loss, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    start();
    if (int rc = check_lce(desc)) return rc;
    const rps_lce_desc& d = *desc;
    if (weight == nullptr || (d.tokens > 0 && (hidden == nullptr || targets == nullptr || lse == nullptr)) ||
        (loss == nullptr && (d.tokens > 0 || d.reduction != RPS_REDUCE_NONE)))
        return fail(RPS_EINVAL, "NULL array");
    LcePlan plan = plan_lce(d, weight, false, workspace);
    if (int rc = check_workspace(workspace, workspace_bytes, plan.bytes)) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    LceParams& p = plan.p;
    p.targets = targets, p.hidden = hidden, p.loss = loss, p.lse = lse;
    if (p.dot_rows > 0) {
        p.weight = weight, p.weight_row = d.weight_row, p.weight_worker = d.weight_worker;
        RPS_TRY(launch_lce_dot(p, stream));
        RPS_TRY(launch_lce_merge(p, stream));
        return RPS_OK;
    }
    RPS_TRY(launch_lce_rows(p, stream));
    if (d.tokens == 0) return RPS_OK;
    ProductParams g = plan.product;
    g.a = hidden_operand(p);
    g.m = (int)d.tokens, g.k = (int)d.cols;
    for (int64_t v0 = 0; v0 < d.vocab; v0 += plan.piece) {
        const int64_t rows = d.vocab - v0 < plan.piece ? d.vocab - v0 : plan.piece;
        if (int rc = weight_operand(d, plan, weight, v0, rows, &g.b, stream)) return rc;
        g.v0 = (int)v0, g.n = (int)rows;
        RPS_TRY(launch_product(Product::kLse, g, stream));
    }
    RPS_TRY(launch_lce_merge(p, stream));
    return RPS_OK;
}

extern "C" int rps_lce_backward(const rps_lce_desc* desc, const void* hidden, const void* weight, const int64_t* targets,
                                const float* lse, const float* dloss, void* dhidden, void* dweight, void* workspace,
                                size_t workspace_bytes, void* cuda_stream)
{
    start();
    if (int rc = check_lce(desc)) return rc;
    const rps_lce_desc& d = *desc;
    if (int rc = check_output_strides("dweight", d.n, d.vocab, d.cols, d.dweight_row, d.dweight_worker)) return rc;
    if (weight == nullptr || dweight == nullptr || (d.tokens > 0 && (hidden == nullptr || targets == nullptr || lse == nullptr || dhidden == nullptr)) ||
        (dloss == nullptr && (d.tokens > 0 || d.reduction != RPS_REDUCE_NONE)))
        return fail(RPS_EINVAL, "NULL array");
    LcePlan plan = plan_lce(d, weight, true, workspace);
    if (int rc = check_workspace(workspace, workspace_bytes, plan.bytes)) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    LceParams& p = plan.p;
    p.targets = targets, p.hidden = hidden, p.lse_in = lse, p.dloss = dloss, p.dhidden = dhidden;
    if (p.dot_rows > 0) {
        p.weight = weight, p.weight_row = d.weight_row, p.weight_worker = d.weight_worker;
        p.dweight = dweight, p.dweight_row = d.dweight_row, p.dweight_worker = d.dweight_worker;
        RPS_TRY(launch_lce_dot(p, stream));
        RPS_TRY(launch_lce_dot_grads(p, stream));
        ProductParams g{};
        g.workers = p.n, g.planes = p.planes, g.count = p.count, g.rows = p.rows, g.tokens = p.tokens, g.scale = p.scale;
        g.m = (int)d.tokens, g.n = (int)d.cols, g.splits = p.dot_ranges;
        g.parts = p.dot_parts, g.part_rows = p.dot_rows, g.part_row = round_up(d.cols, 4);
        g.out = dhidden, g.out_row = d.cols, g.out_worker = d.tokens * d.cols;
        RPS_TRY(launch_join(Product::kDhidden, g, stream));
        return RPS_OK;
    }
    RPS_TRY(launch_lce_rows(p, stream));
    const Operand h = hidden_operand(p);
    for (int64_t v0 = 0; v0 < d.vocab; v0 += plan.piece) {
        const int64_t rows = d.vocab - v0 < plan.piece ? d.vocab - v0 : plan.piece;
        const int64_t tiled = round_up(rows, plan.product.tile_cols);  // dl is written (zeros behind the last row) in whole tiles
        Operand weight_rows;
        if (int rc = weight_operand(d, plan, weight, v0, rows, &weight_rows, stream)) return rc;
        const int64_t plane = p.tokens_padded * plan.piece;
        const Operand dl{plan.dl, p.planes * plane, plane, plan.piece, p.tokens_padded, tiled};
        ProductParams g = plan.product;
        g.v0 = (int)v0;
        if (d.tokens > 0) {
            g.a = h, g.b = weight_rows, g.m = (int)d.tokens, g.n = (int)rows, g.k = (int)d.cols;
            RPS_TRY(launch_product(Product::kDlogits, g, stream));
            g.a = dl, g.n = (int)d.cols, g.k = (int)rows, g.shaped(plan.hidden_shape);
            g.parts = plan.hidden_parts, g.part_rows = p.tokens_padded, g.part_row = round_up(d.cols, g.tile_cols), g.add = v0 > 0;
            g.out = dhidden, g.out_row = d.cols, g.out_worker = d.tokens * d.cols;
            RPS_TRY(launch_product(Product::kDhidden, g, stream));
            if (g.parts != nullptr && v0 + rows == d.vocab) RPS_TRY(launch_join(Product::kDhidden, g, stream));
        }
        g.a = dl, g.b = h, g.m = (int)rows, g.n = (int)d.cols, g.k = (int)d.tokens, g.shaped(plan.weight_shape);
        g.parts = plan.weight_parts, g.part_rows = plan.piece, g.part_row = round_up(d.cols, g.tile_cols), g.add = 0;
        g.out = static_cast<unsigned char*>(dweight) + v0 * d.dweight_row * (p.f32 ? 4 : 2), g.out_row = d.dweight_row, g.out_worker = d.dweight_worker;
        RPS_TRY(launch_product(Product::kDweight, g, stream));
        if (g.parts != nullptr) RPS_TRY(launch_join(Product::kDweight, g, stream));
    }
    return RPS_OK;
}

// ------------------------------------------------------------------------------------------------------------ norm

namespace {

int check_norm(const rps_norm_desc* d)
{
    if (d == nullptr) return fail(RPS_EINVAL, "desc is NULL");
    if (int rc = check_common(d->dtype, d->n)) return rc;
    if (d->cols < 1) return fail(RPS_EINVAL, "cols = %lld", (long long)d->cols);
    if (d->cols > RPS_MAX_NORM_COLS) return fail(RPS_ELIMIT, "cols = %lld; rows of up to %d are held", (long long)d->cols, (int)RPS_MAX_NORM_COLS);
    if (d->tokens < 0 || d->n * d->tokens >= 1ll << 31) return fail(RPS_EINVAL, "tokens = %lld", (long long)d->tokens);
    if (d->gates < 1 || (d->tokens > 0 ? d->tokens % d->gates != 0 : d->gates != 1))
        return fail(RPS_EINVAL, "gates = %lld does not divide tokens = %lld", (long long)d->gates, (long long)d->tokens);
    if (d->post_worker < 0 || d->pre_worker < 0 || d->gate_worker < 0) return fail(RPS_EINVAL, "negative stride between workers");
    if (d->wait_limit_ms < 0 || d->withhold_sums < 0 || d->withhold_sums > 1)
        return fail(RPS_EINVAL, "wait_limit_ms = %d, withhold_sums = %d", d->wait_limit_ms, d->withhold_sums);
    if (!std::isfinite(d->scale) || !std::isfinite(d->eps) || d->eps < 0) return fail(RPS_EINVAL, "scale = %g, eps = %g", d->scale, d->eps);
    return RPS_OK;
}

NormParams norm_params(const rps_norm_desc& d)
{
    NormParams p{};
    p.f32 = d.dtype == RPS_F32, p.n = d.n, p.tokens = d.tokens, p.cols = d.cols, p.gates = d.gates;
    p.rows_per_gate = d.tokens / d.gates;
    p.post_worker = d.post_worker, p.pre_worker = d.pre_worker, p.gate_worker = d.gate_worker;
    p.scale = (float)d.scale, p.eps = (float)d.eps;
    p.pitch = rps_pack_pitch(d.cols), p.groups = ceil_div(d.cols, RPS_PACK_GROUP);
    p.wait_limit_ms = d.wait_limit_ms, p.withhold_sums = d.withhold_sums;
    if (d.tokens > 0) plan_norm_backward(&p);
    return p;
}

}  // namespace

extern "C" int rps_norm_forward(const rps_norm_desc* desc, const void* x, const void* f, const void* gate, const void* post,
                                const void* pre, void* h, void* y, float* r_f, float* r_h, int8_t* f_codes,
                                float* f_scales, int8_t* h_codes, float* h_scales, void* cuda_stream)
{
    start();
    if (int rc = check_norm(desc)) return rc;
    if (desc->tokens == 0) return RPS_OK;
    if (!x || !f || !gate || !post || !pre || !h || !y) return fail(RPS_EINVAL, "NULL array");
    if ((r_f == nullptr) != (r_h == nullptr)) return fail(RPS_EINVAL, "r_f and r_h go together");
    const int packed = (f_codes != nullptr) + (f_scales != nullptr) + (h_codes != nullptr) + (h_scales != nullptr);
    if (packed != 0 && packed != 4) return fail(RPS_EINVAL, "f_codes, f_scales, h_codes and h_scales go together");
    if (!aligned(f_codes, 16) || !aligned(h_codes, 16) || !aligned(f_scales, 16) || !aligned(h_scales, 16))
        return fail(RPS_EINVAL, "codes and scales have to be 16-byte aligned");
    NormParams p = norm_params(*desc);
    p.x = x, p.f = f, p.gate = gate, p.post = post, p.pre = pre, p.h = h, p.y = y, p.r_f = r_f, p.r_h = r_h;
    p.f_codes = f_codes, p.f_scales = f_scales, p.h_codes = h_codes, p.h_scales = h_scales;
    RPS_TRY(launch_norm_forward(p, static_cast<cudaStream_t>(cuda_stream)));
    return RPS_OK;
}

extern "C" int rps_norm_workspace(const rps_norm_desc* desc, size_t* bytes)
{
    start();
    if (bytes == nullptr) return fail(RPS_EINVAL, "bytes is NULL");
    if (int rc = check_norm(desc)) return rc;
    const NormParams p = norm_params(*desc);
    *bytes = (size_t)round_up(p.n * p.blocks * 3 * p.cols * 4, 256);
    return RPS_OK;
}

extern "C" int rps_norm_backward(const rps_norm_desc* desc, const void* dh, const void* dy, const void* f,
                                 const float* f_scales, const void* h, const float* h_scales, const float* r_f,
                                 const float* r_h, const void* gate, const void* post, const void* pre, void* dx, void* df,
                                 void* dgate, void* dpost, void* dpre, void* workspace, size_t workspace_bytes,
                                 void* cuda_stream)
{
    start();
    if (int rc = check_norm(desc)) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!dgate || !dpost || !dpre) return fail(RPS_EINVAL, "NULL array");
    if (desc->tokens == 0) {
        const size_t bytes = (size_t)desc->n * desc->cols * (desc->dtype == RPS_F32 ? 4 : 2);
        RPS_TRY(cudaMemsetAsync(dgate, 0, bytes, stream));
        RPS_TRY(cudaMemsetAsync(dpost, 0, bytes, stream));
        RPS_TRY(cudaMemsetAsync(dpre, 0, bytes, stream));
        return RPS_OK;
    }
    if (!dy || !f || !h || !r_f || !r_h || !gate || !post || !pre || !dx || !df) return fail(RPS_EINVAL, "NULL array");
    if ((f_scales == nullptr) != (h_scales == nullptr)) return fail(RPS_EINVAL, "f and h are both packed or neither");
    if (f_scales != nullptr && (!aligned(f, 16) || !aligned(h, 16) || !aligned(f_scales, 16) || !aligned(h_scales, 16)))
        return fail(RPS_EINVAL, "codes and scales have to be 16-byte aligned");
    NormParams p = norm_params(*desc);
    if (int rc = check_workspace(workspace, workspace_bytes, (size_t)round_up(p.n * p.blocks * 3 * p.cols * 4, 256))) return rc;
    p.packed = f_scales != nullptr;
    p.dh = dh, p.dy = dy, p.f = f, p.h_in = h, p.f_scales = const_cast<float*>(f_scales), p.h_scales = const_cast<float*>(h_scales);
    p.r_f = const_cast<float*>(r_f), p.r_h = const_cast<float*>(r_h), p.gate = gate, p.post = post, p.pre = pre;
    p.dx = dx, p.df = df, p.dgate = dgate, p.dpost = dpost, p.dpre = dpre, p.partial = static_cast<float*>(workspace);
    RPS_TRY(launch_norm_backward(p, stream));
    return RPS_OK;
}

// ------------------------------------------------------------------------------------------------------------ 8 bits

namespace {

int check_pack(int dtype, int64_t rows, int64_t cols, const void* x, int64_t x_row, const void* codes, const void* scales)
{
    if (int rc = check_common(dtype, 1)) return rc;
    if (rows < 0 || rows >= 1ll << 31) return fail(RPS_EINVAL, "rows = %lld", (long long)rows);
    if (cols < 1 || cols > kMaxSize) return fail(RPS_EINVAL, "cols = %lld", (long long)cols);
    if (x_row < cols) return fail(RPS_EINVAL, "a row stride of %lld is less than the %lld columns", (long long)x_row, (long long)cols);
    if (rows > 0 && (x == nullptr || codes == nullptr || scales == nullptr)) return fail(RPS_EINVAL, "NULL array");
    if (!aligned(codes, 16) || !aligned(scales, 16)) return fail(RPS_EINVAL, "codes and scales have to be 16-byte aligned");
    return RPS_OK;
}

PackParams pack_params(int dtype, int64_t rows, int64_t cols, int64_t x_row)
{
    PackParams p{};
    p.f32 = dtype == RPS_F32, p.rows = rows, p.cols = cols, p.x_row = x_row;
    p.pitch = rps_pack_pitch(cols), p.groups = ceil_div(cols, RPS_PACK_GROUP);
    return p;
}

}  // namespace

extern "C" int64_t rps_pack_pitch(int64_t cols) { return round_up(cols, 16); }

extern "C" int rps_pack(int dtype, int64_t rows, int64_t cols, const void* x, int64_t x_row, int8_t* codes, float* scales,
                        void* cuda_stream)
{
    start();
    if (int rc = check_pack(dtype, rows, cols, x, x_row, codes, scales)) return rc;
    if (rows == 0) return RPS_OK;
    PackParams p = pack_params(dtype, rows, cols, x_row);
    p.x = x, p.codes = codes, p.scales = scales;
    RPS_TRY(launch_pack(p, static_cast<cudaStream_t>(cuda_stream)));
    return RPS_OK;
}

extern "C" int rps_unpack(int dtype, int64_t rows, int64_t cols, const int8_t* codes, const float* scales, void* x,
                          int64_t x_row, void* cuda_stream)
{
    start();
    if (int rc = check_pack(dtype, rows, cols, x, x_row, codes, scales)) return rc;
    if (rows == 0) return RPS_OK;
    PackParams p = pack_params(dtype, rows, cols, x_row);
    p.out = x, p.codes = const_cast<int8_t*>(codes), p.scales = const_cast<float*>(scales);
    RPS_TRY(launch_unpack(p, static_cast<cudaStream_t>(cuda_stream)));
    return RPS_OK;
}

namespace {

struct WgradPlan {
    Operand dy{}, x{};
    PlanesParams lay_out{};
    PackParams unpack{};
    bool lay_out_dy = false;
    ProductShape shape{};
    float* parts = nullptr;
    size_t bytes = 0;
};

int check_wgrad(const rps_wgrad_desc* d)
{
    if (d == nullptr) return fail(RPS_EINVAL, "desc is NULL");
    if (int rc = check_common(d->dtype, d->n)) return rc;
    if (d->tokens < 0 || d->tokens > kMaxSize) return fail(RPS_EINVAL, "tokens = %lld", (long long)d->tokens);
    if (d->outs < 1 || d->outs > kMaxSize || d->cols < 1 || d->cols > kMaxSize)
        return fail(RPS_EINVAL, "outs = %lld, cols = %lld", (long long)d->outs, (long long)d->cols);
    if (d->n * d->tokens >= 1ll << 31) return fail(RPS_EINVAL, "n * tokens = %lld", (long long)(d->n * d->tokens));
    if (d->wait_limit_ms < 0 || d->withhold_copies < 0 || d->withhold_copies > 1)
        return fail(RPS_EINVAL, "wait_limit_ms = %d, withhold_copies = %d", d->wait_limit_ms, d->withhold_copies);
    if (d->dy_row < d->outs || d->dy_worker < 0) return fail(RPS_EINVAL, "strides of dy (%lld, %lld)", (long long)d->dy_worker, (long long)d->dy_row);
    return check_output_strides("dweight", d->n, d->outs, d->cols, d->dweight_row, d->dweight_worker);
}

WgradPlan plan_wgrad(const rps_wgrad_desc& d, const void* dy, void* workspace)
{
    WgradPlan plan;
    const int planes = d.dtype == RPS_F32 ? 3 : 1;
    const int64_t tokens = d.tokens > 0 ? d.tokens : 1;
    plan.lay_out_dy = d.dtype == RPS_F32 || !aligned_matrix(dy, d.dy_row, d.dy_worker);
    Carver c{static_cast<unsigned char*>(workspace)};
    const int64_t x_row = round_up(d.cols, 8), x_plane = tokens * x_row;
    bf16* x = c.take<bf16>(d.n * planes * x_plane);
    plan.x = {x, planes * x_plane, x_plane, x_row, d.tokens, x_row};
    PackParams& u = plan.unpack;
    u = pack_params(d.dtype, d.n * d.tokens, d.cols, d.cols);
    u.planes_out = x, u.planes = planes, u.tokens = tokens, u.dst_row = x_row, u.dst_plane = x_plane, u.dst_worker = planes * x_plane;
    plan.dy = {static_cast<const bf16*>(dy), d.dy_worker, 0, d.dy_row, d.tokens, d.outs};
    if (plan.lay_out_dy) {
        const int64_t row = round_up(d.outs, 8), plane = tokens * row;
        bf16* to = c.take<bf16>(d.n * planes * plane);
        plan.dy = {to, planes * plane, plane, row, d.tokens, row};
        PlanesParams& q = plan.lay_out;
        q.src = dy, q.f32 = d.dtype == RPS_F32, q.n = d.n, q.planes = planes, q.rows = d.tokens, q.cols = d.outs;
        q.src_row = d.dy_row, q.src_worker = d.dy_worker, q.dst = to, q.dst_row = row, q.dst_plane = plane, q.dst_worker = planes * plane;
    }
    plan.shape = product_shape(d.outs, d.cols, d.tokens, d.n, planes, true);
    if (plan.shape.splits > 1) plan.parts = c.take<float>(plan.shape.splits * d.n * round_up(d.outs, kVocabTile) * round_up(d.cols, plan.shape.tile_cols));
    plan.bytes = c.used;
    return plan;
}

}  // namespace

extern "C" int rps_wgrad_workspace(const rps_wgrad_desc* desc, const void* dy, size_t* bytes)
{
    start();
    if (bytes == nullptr) return fail(RPS_EINVAL, "bytes is NULL");
    if (int rc = check_wgrad(desc)) return rc;
    *bytes = plan_wgrad(*desc, dy, nullptr).bytes;
    return RPS_OK;
}

extern "C" int rps_packed_wgrad(const rps_wgrad_desc* desc, const void* dy, const int8_t* codes, const float* scales,
                                void* dweight, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    start();
    if (int rc = check_wgrad(desc)) return rc;
    const rps_wgrad_desc& d = *desc;
    if (dweight == nullptr || (d.tokens > 0 && (dy == nullptr || codes == nullptr || scales == nullptr))) return fail(RPS_EINVAL, "NULL array");
    if (!aligned(codes, 16) || !aligned(scales, 16)) return fail(RPS_EINVAL, "codes and scales have to be 16-byte aligned");
    WgradPlan plan = plan_wgrad(d, dy, workspace);
    if (int rc = check_workspace(workspace, workspace_bytes, plan.bytes)) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (d.tokens > 0) {
        plan.unpack.codes = const_cast<int8_t*>(codes), plan.unpack.scales = const_cast<float*>(scales);
        RPS_TRY(launch_unpack_planes(plan.unpack, stream));
        if (plan.lay_out_dy) RPS_TRY(launch_planes(plan.lay_out, stream));
    }
    ProductParams g{};
    g.a = plan.dy, g.b = plan.x, g.workers = d.n, g.planes = d.dtype == RPS_F32 ? 3 : 1;
    g.m = (int)d.outs, g.n = (int)d.cols, g.k = (int)d.tokens, g.shaped(plan.shape), g.wait_limit_ms = d.wait_limit_ms, g.withhold_copies = d.withhold_copies;
    g.out = dweight, g.out_row = d.dweight_row, g.out_worker = d.dweight_worker;
    g.parts = plan.parts, g.part_rows = round_up(d.outs, kVocabTile), g.part_row = round_up(d.cols, g.tile_cols);
    RPS_TRY(launch_product(Product::kDweight, g, stream));
    if (g.parts != nullptr) RPS_TRY(launch_join(Product::kDweight, g, stream));
    return RPS_OK;
}
