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
    if (!std::isfinite((float)d->scale)) return fail(RPS_EINVAL, "scale = %g", d->scale);
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

// ------------------------------------------------------------------------------------------------- linear attention
namespace {

int check_attention(const rps_linear_attention_desc* d)
{
    if (d == nullptr) return fail(RPS_EINVAL, "desc is NULL");
    if (int rc = check_common(d->dtype, d->n)) return rc;
    if (d->reserved != 0) return fail(RPS_EINVAL, "reserved = %d", d->reserved);
    if (d->wait_limit_ms < 0 || d->withhold_copies < 0 || d->withhold_copies > 1)
        return fail(RPS_EINVAL, "wait_limit_ms = %d, withhold_copies = %d", d->wait_limit_ms, d->withhold_copies);
    if (d->heads < 1 || d->heads > 65535) return fail(RPS_EINVAL, "heads = %d", d->heads);
    if (d->sequences < 0 || d->sequences >= 1ll << 28 || d->n * d->sequences * d->heads >= 1ll << 28) return fail(RPS_EINVAL, "sequences = %lld", (long long)d->sequences);
    if (d->tokens < 0 || d->tokens >= 1ll << 31) return fail(RPS_EINVAL, "tokens = %lld", (long long)d->tokens);
    if (d->key_cols < 1 || d->value_cols < 1) return fail(RPS_EINVAL, "key_cols = %lld, value_cols = %lld", (long long)d->key_cols, (long long)d->value_cols);
    if (d->key_cols > RPS_MAX_HEAD_COLS || d->value_cols > RPS_MAX_HEAD_COLS)
        return fail(RPS_ELIMIT, "key_cols = %lld, value_cols = %lld; heads of up to %d are possible", (long long)d->key_cols, (long long)d->value_cols,
                    (int)RPS_MAX_HEAD_COLS);
    for (const rps_axis_strides* s : {&d->q, &d->k, &d->v, &d->dout})
        if (s->worker < 0 || s->sequence < 0 || s->token < 0 || s->head < 0) return fail(RPS_EINVAL, "a negative stride");
    if (!std::isfinite((float)d->scale)) return fail(RPS_EINVAL, "scale = %g", d->scale);
    return RPS_OK;
}

MixOperand operand(const void* base, const rps_axis_strides& s) { return {base, s.worker, s.sequence, s.token, s.head}; }

MixParams mix_params(const rps_linear_attention_desc& d, const float* log_decay, const int64_t* lengths)
{
    MixParams p{};
    p.f32 = d.dtype == RPS_F32, p.n = d.n, p.heads = d.heads, p.sequences = d.sequences, p.tokens = d.tokens;
    p.log_decay = log_decay, p.lengths = lengths, p.wait_limit_ms = d.wait_limit_ms, p.withhold_copies = d.withhold_copies;
    return p;
}

// The forms of a call, of arrays that may be NULL where only sizes count.
MixParams forward_params(const rps_linear_attention_desc& d, const void* q, const void* k, const void* v, const float* log_decay, const int64_t* lengths,
                         const float* state_in, void* out, float* state_out)
{
    MixParams p = mix_params(d, log_decay, lengths);
    const float scale = (float)d.scale;
    p.terms = 1;
    p.term[0] = {operand(q, d.q), operand(k, d.k), operand(v, d.v), out, (int)d.key_cols, (int)d.value_cols, 0, state_in, state_out, d.value_cols, 1, scale, scale, 1.0f, (int)d.key_cols, (int)d.value_cols};
    plan_mix(&p);
    return p;
}

MixParams backward_params(const rps_linear_attention_desc& d, const void* dout, const float* dstate_out, const void* q, const void* k, const void* v, const float* log_decay,
                          const int64_t* lengths, const float* state_in, void* dq, void* dk, void* dv, float* dstate_in)
{
    MixParams p = mix_params(d, log_decay, lengths);
    const float scale = (float)d.scale;
    const int kc = (int)d.key_cols, vc = (int)d.value_cols;
    p.terms = 3;
    p.term[0] = {operand(dout, d.dout), operand(v, d.v), operand(k, d.k), dq, vc, kc, 0, state_in, nullptr, 1, vc, scale, scale, 1.0f, vc, kc};
    p.term[1] = {operand(v, d.v), operand(dout, d.dout), operand(q, d.q), dk, vc, kc, 1, dstate_out, nullptr, 1, vc, scale, 1.0f, scale, vc, kc};
    p.term[2] = {operand(k, d.k), operand(q, d.q), operand(dout, d.dout), dv, kc, vc, 1, dstate_out, dstate_in, vc, 1, scale, 1.0f, scale, kc, vc};
    plan_mix(&p);
    return p;
}

size_t mix_workspace(MixParams* p, void* workspace)
{
    Carver c{static_cast<unsigned char*>(workspace)};
    if (p->segments > 1) p->segment_states = c.take<float>(p->terms * p->units * p->segments * p->state_room);
    if (p->copies_bytes > 0) p->copies = c.take<unsigned char>(p->copies_bytes);
    return c.used;
}

}  // namespace

extern "C" int rps_linear_attention_workspace(const rps_linear_attention_desc* desc, int backward, size_t* bytes)
{
    start();
    if (bytes == nullptr) return fail(RPS_EINVAL, "bytes is NULL");
    if (int rc = check_attention(desc)) return rc;
    MixParams p = backward != 0 ? backward_params(*desc, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr)
                                : forward_params(*desc, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr);
    *bytes = mix_workspace(&p, nullptr);
    return RPS_OK;
}

extern "C" int rps_linear_attention_forward(const rps_linear_attention_desc* desc, const void* q, const void* k, const void* v, const float* log_decay,
                                            const int64_t* lengths, const float* state_in, void* out, float* state_out, void* workspace,
                                            size_t workspace_bytes, void* cuda_stream)
{
    start();
    if (int rc = check_attention(desc)) return rc;
    if (desc->sequences == 0) return RPS_OK;
    if (log_decay == nullptr || (desc->tokens > 0 && (q == nullptr || k == nullptr || v == nullptr || out == nullptr))) return fail(RPS_EINVAL, "NULL array");
    MixParams p = forward_params(*desc, q, k, v, log_decay, lengths, state_in, out, state_out);
    if (int rc = check_workspace(workspace, workspace_bytes, mix_workspace(&p, workspace))) return rc;
    RPS_TRY(launch_mix(p, static_cast<cudaStream_t>(cuda_stream)));
    return RPS_OK;
}

extern "C" int rps_linear_attention_backward(const rps_linear_attention_desc* desc, const void* dout, const float* dstate_out, const void* q, const void* k,
                                             const void* v, const float* log_decay, const int64_t* lengths, const float* state_in, void* dq, void* dk,
                                             void* dv, float* dstate_in, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    start();
    if (int rc = check_attention(desc)) return rc;
    if (desc->sequences == 0) return RPS_OK;
    if (log_decay == nullptr || (desc->tokens > 0 && (!dout || !q || !k || !v || !dq || !dk || !dv))) return fail(RPS_EINVAL, "NULL array");
    MixParams p = backward_params(*desc, dout, dstate_out, q, k, v, log_decay, lengths, state_in, dq, dk, dv, dstate_in);
    if (int rc = check_workspace(workspace, workspace_bytes, mix_workspace(&p, workspace))) return rc;
    RPS_TRY(launch_mix(p, static_cast<cudaStream_t>(cuda_stream)));
    return RPS_OK;
}

extern "C" int rps_linear_attention_step(const rps_linear_attention_desc* desc, const void* q, const void* k, const void* v, const float* log_decay,
                                         const float* state_in, void* out, float* state_out, void* cuda_stream)
{
    start();
    if (int rc = check_attention(desc)) return rc;
    if (desc->tokens != 1) return fail(RPS_EINVAL, "tokens = %lld; a step takes 1", (long long)desc->tokens);
    if (desc->sequences == 0) return RPS_OK;
    if (!q || !k || !v || !log_decay || !state_in || !out || !state_out) return fail(RPS_EINVAL, "NULL array");
    const MixParams p = forward_params(*desc, q, k, v, log_decay, nullptr, state_in, out, state_out);
    RPS_TRY(launch_mix_step(p, static_cast<cudaStream_t>(cuda_stream)));
    return RPS_OK;
}
