// C ABI of the operators on the workers' sequences (include/rps_ops.h): argument checks, the layout of the lent workspaces, and the order of the
// launches.
#include <cmath>

#include "rps_ops_host.h"

namespace {

using namespace rps_ops;

// ------------------------------------------------------------------------------------------------------- embedding
int check_embed(const rps_embed_desc* d)
{
    if (d == nullptr) return fail(RPS_EINVAL, "desc is NULL");
    if (int rc = check_common(d->dtype, d->n)) return rc;
    if (d->accumulate < 0 || d->accumulate > 1 || d->reserved != 0) return fail(RPS_EINVAL, "accumulate = %d, reserved = %d", d->accumulate, d->reserved);
    if (d->tokens < 0 || d->tokens > kMaxSize || d->n * d->tokens >= 1ll << 31) return fail(RPS_EINVAL, "tokens = %lld", (long long)d->tokens);
    if (d->vocab < 1 || d->vocab >= 1ll << 30) return fail(RPS_EINVAL, "vocab = %lld", (long long)d->vocab);
    if (d->cols < 1 || d->cols > kMaxSize) return fail(RPS_EINVAL, "cols = %lld", (long long)d->cols);
    if (!std::isfinite(d->scale)) return fail(RPS_EINVAL, "scale = %g", d->scale);
    return RPS_OK;
}

EmbedParams embed_params(const rps_embed_desc& d)
{
    EmbedParams p{};
    p.f32 = d.dtype == RPS_F32, p.n = d.n, p.accumulate = d.accumulate, p.scale = (float)d.scale;
    p.count = d.tokens, p.vocab = d.vocab, p.cols = d.cols, p.ignore_index = d.ignore_index;
    p.weight_row = d.weight_row, p.weight_worker = d.weight_worker, p.dweight_row = d.dweight_row, p.dweight_worker = d.dweight_worker;
    return p;
}

size_t plan_embed_workspace(EmbedParams* prm, void* workspace)
{
    EmbedParams& p = *prm;
    if (p.count == 0) return 0;
    plan_embed(prm);
    Carver c{static_cast<unsigned char*>(workspace)};
    for (int i = 0; i < (p.sort_blocks > 0 ? 2 : 1); ++i) p.keys[i] = c.take<uint32_t>(p.n * p.count), p.from[i] = c.take<uint32_t>(p.n * p.count);
    if (p.sort_blocks > 0) p.counts = c.take<uint32_t>(p.n * 256 * p.sort_blocks);
    if (p.tiles > 1) p.parts = c.take<float>(p.n * p.tiles * 2 * p.part_row);
    return c.used;
}

}  // namespace

extern "C" int rps_embed_forward(const rps_embed_desc* desc, const int64_t* tokens, const void* weight, void* out, void* cuda_stream)
{
    start();
    if (int rc = check_embed(desc)) return rc;
    if (desc->weight_row < desc->cols || desc->weight_worker < 0)
        return fail(RPS_EINVAL, "strides of weight (%lld, %lld)", (long long)desc->weight_worker, (long long)desc->weight_row);
    if (desc->tokens == 0) return RPS_OK;
    if (tokens == nullptr || weight == nullptr || out == nullptr) return fail(RPS_EINVAL, "NULL array");
    EmbedParams p = embed_params(*desc);
    p.tokens = tokens, p.weight = weight, p.out = out;
    RPS_TRY(launch_embed_lookup(p, static_cast<cudaStream_t>(cuda_stream)));
    return RPS_OK;
}

extern "C" int rps_embed_workspace(const rps_embed_desc* desc, size_t* bytes)
{
    start();
    if (bytes == nullptr) return fail(RPS_EINVAL, "bytes is NULL");
    if (int rc = check_embed(desc)) return rc;
    EmbedParams p = embed_params(*desc);
    *bytes = plan_embed_workspace(&p, nullptr);
    return RPS_OK;
}

extern "C" int rps_embed_backward(const rps_embed_desc* desc, const int64_t* tokens, const void* dout, void* dweight, void* workspace,
                                  size_t workspace_bytes, void* cuda_stream)
{
    start();
    if (int rc = check_embed(desc)) return rc;
    if (int rc = check_output_strides("dweight", desc->n, desc->vocab, desc->cols, desc->dweight_row, desc->dweight_worker)) return rc;
    if (dweight == nullptr || (desc->tokens > 0 && (tokens == nullptr || dout == nullptr))) return fail(RPS_EINVAL, "NULL array");
    EmbedParams p = embed_params(*desc);
    if (int rc = check_workspace(workspace, workspace_bytes, plan_embed_workspace(&p, workspace))) return rc;
    p.tokens = tokens, p.dout = dout, p.dweight = dweight;
    RPS_TRY(launch_embed_gradient(p, static_cast<cudaStream_t>(cuda_stream)));
    return RPS_OK;
}
