// Linear attention with a decay for each head: its chunked form for sequences and its recurrent form for single tokens.
//
// With W the state before a chunk of C tokens (rows i of x, y, z) and r the head's decay, one form
//
//   out_i = sum_{j<=i} r^(i-j) (x_i . y_j) z_j + r^(i+1) x_i W,    W' = r^C W + sum_j r^(C-1-j) y_j^T z_j
//
// gives the forward pass (x, y, z = q, k, v) and every gradient: dq (dout, v, k, with W transposed), and in reversed time, where the state is that of
// the gradient and a token's own factor comes one step later (`late`), dk (v, dout, q) and dv (k, q, dout).  The three gradients go
// through one launch, so that the third reads what the others have brought into L2.
//
// Where there are too few heads of sequences to fill the SMs, sequences are cut into segments: one launch makes each segment's own sum of y^T z,
// one adds them up in order into the states that segments begin with, and the main one then runs all segments at once (y and z are read twice).
//
// The kernel here takes fp32 operands (bf16 ones: rps_mix_tensor.cu; where TMA cannot copy them, copies of theirs; rps_mix_mma.cu in short sequences of narrow
// heads or of what TMA cannot copy).  A CTA has a sequence's head and 64 columns of z, chunk by chunk of 64 tokens; all products are of fp32 in registers, 4 x 4 results to a
// thread with two 16-byte reads of shared memory for every 16 to 32 multiplications.  148 heads of 512 tokens x 64 take 95 us forward, 444 take 234: 40 % of
// the multiplications' rate; what else a chunk needs of issue slots and its barriers bound it.  (8 x 8 results in 64 threads: 163 and 261, 8 x 4
// in 128 104 and 194, but 4 x 3 sequences of 333 x 5 x 48 x 40, forward and backward, 164 us instead of 129.  Six products of bf16 parts on the
// tensor cores, mma.sync, whose operands every warp had to cut for itself: 117 for the 148 heads, 193 for the latter.)
#include <algorithm>

#include "rps_mix.cuh"
#include "rps_tma.cuh"

namespace rps_ops {
namespace {

using rps::LaunchState;

constexpr int kC = kMixChunk, kTile = 64;  // tokens of a chunk; columns of z of a CTA
constexpr int kThreads = 256;              // 16 x 16, with 4 x 4 results each

// Shared memory, in floats: rows of x and y, of z and of what is made, none of which meet a bank twice in a read.  MT: 64 columns of x and y each.
template <int MT>
struct Shape {
    static constexpr int kRowA = MT * 64 + 4, kRow = kTile + 4, kStages = MT;  // two CTAs share an SM where one stage is all there is
    static constexpr int kStage = kC * (2 * kRowA + kRow);
    static constexpr int kBytes = (kStages * kStage + kC * kRow + MT * 64 * kRow + kC + 4) * 4;
};

__device__ __forceinline__ float4 four(const float* p) { return *reinterpret_cast<const float4*>(p); }

// Four values into columns c.. of a row of `cols`.
template <int ALIGN>
__device__ __forceinline__ void store_four(float* row, int c, int cols, const float (&v)[4])
{
    if constexpr (ALIGN == 16) {
        if (c < cols) *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < cols) row[c + j] = v[j];
    }
}

// STATES: no output, only each segment's own sum.
template <int MT, int ALIGN, bool STATES>
__global__ void __launch_bounds__(kThreads, MT == 1 ? 2 : 1) rps_mix_kernel(const __grid_constant__ MixParams prm)
{
    after_the_kernel_before();
    using S = Shape<MT>;
    constexpr int W = 4;
    extern __shared__ __align__(16) float shared[];
    float* const scores = shared + S::kStages * S::kStage;
    float* const state = scores + kC * S::kRow;
    float* const powers = state + MT * 64 * S::kRow;  // r^0 .. r^64

    const MixTerm& term = prm.term[blockIdx.y];
    const int a = term.a, b = term.b, a4 = (a + 3) / 4 * 4;
    const int64_t item = blockIdx.x / prm.columns;
    const int col0 = (int)(blockIdx.x - item * prm.columns) * kTile;
    if (col0 >= b) return;
    const int segment = (int)(item % prm.segments);
    const int64_t unit = item / prm.segments;
    if (STATES && segment + 1 == prm.segments) return;
    const Place at = place_of(prm, unit);
    const int warp = threadIdx.x / 32, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int cols = min(kTile, b - col0);
    const int64_t i0 = segment * prm.segment_tokens, i1 = min(at.length, i0 + prm.segment_tokens);
    const int late = term.reversed;
    const float log_decay = __ldg(prm.log_decay + at.w * prm.heads + at.head);
    if (threadIdx.x <= kC) powers[threadIdx.x] = (float)power(log_decay, threadIdx.x);

    const float* const x = first_token<float>(term.x, at);
    const float* const y = first_token<float>(term.y, at);
    const float* const z = first_token<float>(term.z, at);
    float* const out = static_cast<float*>(term.out) + ((at.w * prm.sequences + at.sequence) * prm.tokens * prm.heads + at.head) * b + col0;
    // a chunk's rows; behind the last token zeros
    const auto load = [&](int64_t i, int stage) {
        float* const to = shared + stage * S::kStage;
        const auto rows = [&](float* tile, int row_length, const float* from, int64_t stride, int c0, int limit, int width) {
            const int across = (width + W - 1) / W;
            for (int u = threadIdx.x; u < kC * across; u += kThreads) {
                const int r = u / across, c = (u - r * across) * W;
                const int64_t at_row = i + r, token = late ? at.length - 1 - at_row : at_row;
                const bool there = at_row < i1;
                copy_slice<float, ALIGN>(rps::smem_addr(tile + r * row_length + c), from + (there ? token : 0) * stride, c0 + c, there ? limit : 0);
            }
        };
        if (!STATES) rows(to, S::kRowA, x, term.x.token, 0, a, a);
        rows(to + kC * S::kRowA, S::kRowA, y, term.y.token, 0, a, a);
        rows(to + 2 * kC * S::kRowA, S::kRow, z, term.z.token, col0, b, kTile);
        copies_sent();
    };

    // W: rows 64 m + 4 ty + i, columns 4 tx + j
    float w[MT][4][4];
    const float* init = nullptr;
    int64_t init_a = b, init_b = 1;
    if (!STATES && prm.segments > 1)
        init = prm.segment_states + ((blockIdx.y * prm.units + unit) * prm.segments + segment) * prm.state_room;
    else if (!STATES && term.state_in != nullptr)
        init = term.state_in + unit * a * b, init_a = term.state_a, init_b = term.state_b;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = m * 64 + ty * 4 + i, col = col0 + tx * 4 + j;
                w[m][i][j] = init != nullptr && row < a && col < b ? __ldg(init + row * init_a + col * init_b) : 0.0f;
            }
    bool zero = init == nullptr;  // so far
    const auto publish = [&] {  // W where the products read it
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(state + (m * 64 + ty * 4 + i) * S::kRow + tx * 4) = make_float4(w[m][i][0], w[m][i][1], w[m][i][2], w[m][i][3]);
    };
    if (!STATES && !zero) publish();
    if (S::kStages == 2 && i0 < i1) load(i0, 0);

    int stage = 0;
    for (int64_t i = i0; i < i1; i += kC) {
        if constexpr (S::kStages == 1) {
            load(i, 0);
            copies_arrived<0>();
        } else if (i + kC < i1) {
            load(i + kC, stage ^ 1);
            copies_arrived<1>();
        } else {
            copies_arrived<0>();
        }
        __syncthreads();
        const float* const tx_rows = shared + stage * S::kStage;
        const float* const ty_rows = tx_rows + kC * S::kRowA;
        const float* const tz_rows = ty_rows + kC * S::kRowA;
        const int inside = (int)min((int64_t)kC, i1 - i);
        if constexpr (!STATES) {
            const float* const own = tx_rows + ty * 4 * S::kRowA;
            // x . y of these rows with tokens tx + 16 j, the blocks of 16 up to this warp's rows
            {
                float s[4][4] = {};
                for (int k = 0; k < a4; k += 4) {
                    float4 l[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) l[q] = four(own + q * S::kRowA + k);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j > warp / 2) break;
                        const float4 r = four(ty_rows + (tx + 16 * j) * S::kRowA + k);
#pragma unroll
                        for (int q = 0; q < 4; ++q) s[q][j] = fmaf(l[q].x, r.x, fmaf(l[q].y, r.y, fmaf(l[q].z, r.z, fmaf(l[q].w, r.w, s[q][j]))));
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j > warp / 2) break;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int apart = ty * 4 + q - (tx + 16 * j);
                        scores[(ty * 4 + q) * S::kRow + tx + 16 * j] = apart >= 0 ? s[q][j] * (term.score_scale * powers[max(apart, 0)]) : 0.0f;
                    }
                }
            }
            float o[4][4] = {};
            const auto add = [&](const float4& l, const float4 (&r)[4], float (&sum)[4]) {
                const float f[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    sum[0] = fmaf(f[k], r[k].x, sum[0]), sum[1] = fmaf(f[k], r[k].y, sum[1]), sum[2] = fmaf(f[k], r[k].z, sum[2]), sum[3] = fmaf(f[k], r[k].w, sum[3]);
            };
            if (!zero) {
                for (int k = 0; k < a4; k += 4) {
                    float4 r[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) r[q] = four(state + (k + q) * S::kRow + tx * 4);
#pragma unroll
                    for (int q = 0; q < 4; ++q) add(four(own + q * S::kRowA + k), r, o[q]);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float factor = term.state_scale * powers[ty * 4 + q + 1 - late];
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[q][j] *= factor;
                }
            }
            __syncwarp();  // a warp's rows of scores are its own
            for (int k = 0; k < warp * 8 + 8; k += 4) {
                float4 r[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) r[q] = four(tz_rows + (k + q) * S::kRow + tx * 4);
#pragma unroll
                for (int q = 0; q < 4; ++q) add(four(scores + (ty * 4 + q) * S::kRow + k), r, o[q]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t row = i + ty * 4 + q, token = late ? at.length - 1 - row : row;
                if (row < i1) store_four<ALIGN>(out + token * prm.heads * b, tx * 4, cols, o[q]);
            }
        }
        // W
        const float whole = powers[inside];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m * 64 + warp * 8 >= a) break;
            float u[4][4] = {};
#pragma unroll 4
            for (int k = 0; k < inside; ++k) {
                const float factor = term.update_scale * powers[inside - 1 - k + late];
                const float4 l = four(ty_rows + k * S::kRowA + m * 64 + ty * 4);
                float4 r = four(tz_rows + k * S::kRow + tx * 4);
                r = make_float4(r.x * factor, r.y * factor, r.z * factor, r.w * factor);
                const float f[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    u[q][0] = fmaf(f[q], r.x, u[q][0]), u[q][1] = fmaf(f[q], r.y, u[q][1]), u[q][2] = fmaf(f[q], r.z, u[q][2]), u[q][3] = fmaf(f[q], r.w, u[q][3]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[m][q][j] = m * 64 + ty * 4 + q < a ? fmaf(whole, w[m][q][j], u[q][j]) : 0.0f;
        }
        zero = false;
        __syncthreads();
        if (!STATES && i + kC < i1) publish();
        if (S::kStages == 2) stage ^= 1;
    }

    float* to = nullptr;
    int64_t to_a = b, to_b = 1;
    if (STATES)
        to = prm.segment_states + ((blockIdx.y * prm.units + unit) * prm.segments + segment + 1) * prm.state_room;
    else if (segment + 1 == prm.segments && term.state_out != nullptr)
        to = term.state_out + unit * a * b, to_a = term.state_a, to_b = term.state_b;
    if (to != nullptr) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int row = m * 64 + ty * 4 + i, col = col0 + tx * 4 + j;
                    if (row < a && col < b) to[row * to_a + col * to_b] = w[m][i][j];
                }
    }
    if constexpr (!STATES) {
        // rows behind the sequence's last token
        const int64_t t1 = min(prm.tokens, i0 + prm.segment_tokens);
        const float none[4] = {};
        for (int64_t t = max(at.length, i0) + ty; t < t1; t += 16) store_four<ALIGN>(out + t * prm.heads * b, tx * 4, cols, none);
    }
}

// The states that segments begin with, out of the segments' own sums: slot s + 1 holds that of segment s, slot 0 becomes the first state.
constexpr int kJoinThreads = 256;

// Tokens of segment s; `end_aligned`: it is the first chunk of a sequence that is not full, not the last.
__device__ __forceinline__ int64_t segment_length(const MixParams& prm, int64_t length, int s, bool end_aligned)
{
    const int64_t first = s * prm.segment_tokens;
    if (!end_aligned) return max((int64_t)0, min(prm.segment_tokens, length - first));
    const int64_t whole = (length + kMixTensorChunk - 1) / kMixTensorChunk * kMixTensorChunk, missing = whole - length;
    return max((int64_t)0, min(prm.segment_tokens, whole - first) - (s == 0 ? missing : 0));
}

__global__ void __launch_bounds__(kJoinThreads) rps_mix_join_kernel(const __grid_constant__ MixParams prm)
{
    after_the_kernel_before();
    const MixTerm& term = prm.term[blockIdx.y];
    const int64_t unit = blockIdx.x / prm.join_blocks;
    const int e = (int)(blockIdx.x - unit * prm.join_blocks) * kJoinThreads + threadIdx.x, row = e / term.b, col = e - row * term.b;
    __shared__ float decay[kMixSegments];
    const Place at = place_of(prm, unit);
    const float log_decay = __ldg(prm.log_decay + at.w * prm.heads + at.head);
    for (int s = threadIdx.x; s + 1 < prm.segments; s += kJoinThreads)
        decay[s] = (float)power(log_decay, segment_length(prm, at.length, s, prm.tensor && !term.reversed));
    __syncthreads();
    if (e >= term.a * term.b) return;
    float* slot = prm.segment_states + (blockIdx.y * prm.units + unit) * prm.segments * prm.state_room + e;
    const bool there = term.state_in != nullptr && row < term.rows && col < term.cols;
    float w = there ? __ldg(term.state_in + unit * term.rows * term.cols + row * term.state_a + col * term.state_b) : 0.0f;
    slot[0] = w;
    for (int s0 = 0; s0 + 1 < prm.segments; s0 += 8) {
        float own[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) own[j] = s0 + j + 1 < prm.segments ? __ldcg(slot + (s0 + j + 1) * prm.state_room) : 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (s0 + j + 1 >= prm.segments) break;
            w = fmaf(decay[s0 + j], w, own[j]);
            slot[(s0 + j + 1) * prm.state_room] = w;
        }
    }
}

// ----------------------------------------------------------------------------------------------------- single tokens
// state' = r state + k^T v, out = scale q state': bound by the state, read and written once.  A CTA to a head of a sequence; VEC columns to a thread,
// 2^log_across threads to a row of the state.
constexpr int kStepThreads = 256;

template <typename T, int VEC>
__global__ void __launch_bounds__(kStepThreads) rps_mix_step_kernel(const __grid_constant__ MixParams prm, int log_across)
{
    after_the_kernel_before();
    __shared__ float q[kMixMaxCols], k[kMixMaxCols], v[kMixMaxCols];
    __shared__ float sums[kStepThreads * VEC];
    const MixTerm& term = prm.term[0];
    const int64_t unit = blockIdx.x;
    const Place at = place_of(prm, unit);
    const int a = term.a, b = term.b, across = 1 << log_across, down = kStepThreads >> log_across;
    const int row0 = threadIdx.x >> log_across, c = (threadIdx.x & (across - 1)) * VEC;
    const float decay = (float)power(__ldg(prm.log_decay + at.w * prm.heads + at.head), 1);
    for (int i = threadIdx.x; i < a; i += kStepThreads) {
        q[i] = to_float(first_token<T>(term.x, at)[i]) * term.score_scale;
        k[i] = to_float(first_token<T>(term.y, at)[i]);
    }
    for (int i = threadIdx.x; i < b; i += kStepThreads) v[i] = to_float(first_token<T>(term.z, at)[i]);
    __syncthreads();
    const float* from = term.state_in + unit * a * b + c;
    float* to = term.state_out + unit * a * b + c;
    float sum[VEC], mine[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] = 0.0f, mine[j] = c + j < b ? v[c + j] : 0.0f;
    if (c < b) {
        constexpr int kAtATime = 8;
        for (int r0 = row0; r0 < a; r0 += down * kAtATime) {
            float s[kAtATime][VEC];
#pragma unroll
            for (int i = 0; i < kAtATime; ++i) {
                const int r = r0 + i * down;
                if constexpr (VEC == 4) {
                    const float4 f = r < a ? __ldcs(reinterpret_cast<const float4*>(from + r * b)) : make_float4(0, 0, 0, 0);
                    s[i][0] = f.x, s[i][1] = f.y, s[i][2] = f.z, s[i][3] = f.w;
                } else {
                    s[i][0] = r < a ? __ldcs(from + r * b) : 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < kAtATime; ++i) {
                const int r = r0 + i * down;
                if (r >= a) break;
                const float kr = k[r], qr = q[r];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    s[i][j] = fmaf(kr, mine[j], decay * s[i][j]);
                    sum[j] = fmaf(qr, s[i][j], sum[j]);
                }
                if constexpr (VEC == 4)
                    __stcs(reinterpret_cast<float4*>(to + r * b), make_float4(s[i][0], s[i][1], s[i][2], s[i][3]));
                else
                    __stcs(to + r * b, s[i][0]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) sums[(row0 << log_across) * VEC + c + j] = sum[j];
    __syncthreads();
    if ((int)threadIdx.x < b) {
        float all = 0.0f;
        for (int r = 0; r < down; ++r) all += sums[(r << log_across) * VEC + threadIdx.x];
        static_cast<T*>(term.out)[unit * b + threadIdx.x] = from_float<T>(all);
    }
}

// ------------------------------------------------------------------------------------------------------------ copies
// Rows of bf16 into another layout: columns past `from_cols` become zeros, those past `to_cols` are left out.
struct MixMove {
    MixOperand from, to;
    int from_cols, to_cols, from_pairs, to_pairs;  // pairs: two columns lie within 4 aligned bytes
};

struct MixMoves {
    MixMove move[4];
    int count, log_across;  // 2^log_across threads to a row, two columns to a thread
    int64_t blocks;         // CTAs of a sequence's tokens
    int head_blocks;
    bool all;               // tokens that take no part as well
};

constexpr int kMoveThreads = 256, kMoveTokens = 4, kMoveHeads = 4;  // of a thread, all under way at once

__global__ void __launch_bounds__(kMoveThreads) rps_mix_move_kernel(const __grid_constant__ MixParams prm, const __grid_constant__ MixMoves moves)
{
    after_the_kernel_before();
    const MixMove& m = moves.move[blockIdx.y];
    const int64_t part = blockIdx.x / moves.head_blocks, s = part / moves.blocks;
    const int h0 = (int)(blockIdx.x - part * moves.head_blocks) * kMoveHeads, heads = min(kMoveHeads, prm.heads - h0);
    const int c = (threadIdx.x & ((1 << moves.log_across) - 1)) * 2, down = kMoveThreads >> moves.log_across;
    const Place at = place_of(prm, s * prm.heads + h0);
    const int64_t t0 = (part - s * moves.blocks) * down * kMoveTokens + (threadIdx.x >> moves.log_across), limit = moves.all ? prm.tokens : at.length;
    if (c >= m.to_cols) return;
    const bf16* const from = first_token<bf16>(m.from, at) + t0 * m.from.token + c;
    bf16* const to = const_cast<bf16*>(first_token<bf16>(m.to, at)) + t0 * m.to.token + c;
    uint32_t v[kMoveTokens][kMoveHeads], next[kMoveTokens][kMoveHeads];
    const auto load = [&](uint32_t(&to)[kMoveTokens][kMoveHeads], const auto* first, bool there) {
#pragma unroll
        for (int i = 0; i < kMoveTokens; ++i)
#pragma unroll
            for (int h = 0; h < kMoveHeads; ++h) {
                const auto* p = first + ((int64_t)i * down * m.from.token + h * m.from.head) * (int64_t)sizeof(bf16) / (int64_t)sizeof(*first);
                to[i][h] = there && t0 + i * down < limit && h < heads ? __ldg(p) : 0;
            }
    };
    if (m.from_pairs) {
        load(v, reinterpret_cast<const uint32_t*>(from), c < m.from_cols);
    } else {
        load(v, reinterpret_cast<const unsigned short*>(from), c < m.from_cols), load(next, reinterpret_cast<const unsigned short*>(from) + 1, c + 1 < m.from_cols);
#pragma unroll
        for (int i = 0; i < kMoveTokens; ++i)
#pragma unroll
            for (int h = 0; h < kMoveHeads; ++h) v[i][h] |= next[i][h] << 16;
    }
#pragma unroll
    for (int i = 0; i < kMoveTokens; ++i)
#pragma unroll
        for (int h = 0; h < kMoveHeads; ++h) {
            bf16* p = to + (int64_t)i * down * m.to.token + h * m.to.head;
            if (t0 + i * down >= limit || h >= heads) continue;
            if (m.to_pairs) {
                *reinterpret_cast<uint32_t*>(p) = v[i][h];
            } else {
                *reinterpret_cast<unsigned short*>(p) = (unsigned short)v[i][h];
                if (c + 1 < m.to_cols) reinterpret_cast<unsigned short*>(p)[1] = (unsigned short)(v[i][h] >> 16);
            }
        }
}

// -------------------------------------------------------------------------------------------------------------- host
cudaError_t launch_moves(const MixParams& prm, MixMoves& moves, cudaStream_t stream)
{
    if (moves.count == 0) return cudaSuccess;
    int widest = 0;
    for (int i = 0; i < moves.count; ++i) {
        MixMove& m = moves.move[i];
        const auto pairs = [&](const MixOperand& o, int cols) { return alignment<bf16>(o.base, cols, o.token | o.head | o.sequence | o.worker) >= 4; };
        m.from_pairs = pairs(m.from, m.from_cols), m.to_pairs = pairs(m.to, m.to_cols);
        widest = std::max(widest, m.to_cols);
    }
    moves.log_across = 0;
    while (2 << moves.log_across < widest) ++moves.log_across;
    moves.blocks = ceil_div(prm.tokens, (kMoveThreads >> moves.log_across) * kMoveTokens);
    moves.head_blocks = (int)ceil_div(prm.heads, kMoveHeads);
    return launch_after(rps_mix_move_kernel, dim3((unsigned)(prm.n * prm.sequences * moves.blocks * moves.head_blocks), (unsigned)moves.count), kMoveThreads, 0, stream, 1,
                        prm, moves);
}

// Of the terms of a call the arrays that are distinct: a forward call's x, y, z, and a backward one's (dout, v, k), (v, dout, q), (k, q, dout).
constexpr int kOperands[3][3] = {{0, 1, 2}, {1, 0, 3}, {2, 3, 0}};

// `p` with copies that TMA can copy in place of what it cannot, and how they are made; the bytes that they take.
size_t with_copies(MixParams* prm, MixMoves* in, MixMoves* out)
{
    MixParams& p = *prm;
    const int64_t rows = p.n * p.sequences * p.tokens * p.heads;
    unsigned char* at = p.copies;
    size_t bytes = 0;
    const auto dense = [&](const void* base, int64_t cols) -> MixOperand {
        return {base, p.sequences * p.tokens * p.heads * cols, p.tokens * p.heads * cols, p.heads * cols, cols};
    };
    const auto room = [&](int cols) {
        const MixOperand o = dense(at == nullptr ? nullptr : at + bytes, round_up(cols, 8));
        bytes += round_up(rows * round_up(cols, 8) * 2, 256);
        return o;
    };
    MixOperand copy[4];
    bool copied[4] = {}, known[4] = {};
    in->count = out->count = 0, in->all = false, out->all = true;
    for (int i = 0; i < p.terms; ++i) {
        MixTerm& t = p.term[i];
        MixOperand* const operands[3] = {&t.x, &t.y, &t.z};
        for (int j = 0; j < 3; ++j) {
            const int which = kOperands[i][j], cols = j < 2 ? t.a : t.b;
            MixOperand& o = *operands[j];
            if (!known[which]) {
                known[which] = true, copied[which] = !mix_fits_tensor(p, o, cols);
                if (copied[which]) copy[which] = room(cols), in->move[in->count++] = {o, copy[which], cols, (int)round_up(cols, 8)};
            }
            if (copied[which]) o = copy[which];
        }
        if (t.b % 8 != 0) {
            const MixOperand o = room(t.b);
            out->move[out->count++] = {o, dense(t.out, t.b), (int)round_up(t.b, 8), t.b};
            t.out = const_cast<void*>(o.base);
        }
        t.a = (int)round_up(t.a, 8), t.b = (int)round_up(t.b, 8);
    }
    return bytes;
}

cudaError_t launch_join(const MixParams& prm, cudaStream_t stream)
{
    return launch_after(rps_mix_join_kernel, dim3((unsigned)(prm.units * prm.join_blocks), (unsigned)prm.terms), kJoinThreads, 0, stream, 1, prm);
}

template <int MT, int ALIGN, bool STATES>
cudaError_t launch_kernel(const MixParams& prm, cudaStream_t stream)
{
    static LaunchState granted;
    const cudaError_t err = rps::grant_smem(granted, rps_mix_kernel<MT, ALIGN, STATES>, Shape<MT>::kBytes);
    if (err != cudaSuccess) return err;
    return launch_after(rps_mix_kernel<MT, ALIGN, STATES>, dim3((unsigned)(prm.units * prm.segments * prm.columns), (unsigned)prm.terms), kThreads, Shape<MT>::kBytes, stream, 1,
                        prm);
}

template <int MT, int ALIGN>
cudaError_t launch_either(const MixParams& prm, bool states, cudaStream_t stream)
{
    return states ? launch_kernel<MT, ALIGN, true>(prm, stream) : launch_kernel<MT, ALIGN, false>(prm, stream);
}

cudaError_t launch_f32(const MixParams& prm, bool states, cudaStream_t stream)
{
    int widest = 0;
    for (int i = 0; i < prm.terms; ++i) widest = std::max(widest, prm.term[i].a);
    const bool wide = mix_alignment<float>(prm) == 16;
    if (widest <= 64) return wide ? launch_either<1, 16>(prm, states, stream) : launch_either<1, 4>(prm, states, stream);
    return wide ? launch_either<2, 16>(prm, states, stream) : launch_either<2, 4>(prm, states, stream);
}

}  // namespace

// From so many tokens of a sequence on, bf16 arrays that TMA cannot copy as they lie go by way of copies that it can, for the tensor cores' fifth
// generation.  By way of copies / as they lie (us): 64 sequences of 16 x 61, 64 tokens 99 / 57 forward, 321 / 205 with backward; 128 tokens 121 / 107,
// 375 / 431; 256 tokens 177 / 230, 545 / 863; 27 of 212 tokens x 18 x (14, 117) 115 / 113, 318 / 446; 2 of 3841 x 14 x (85, 98) 125 / 347, 345 / 1361.
int64_t copied_tokens(const MixParams& prm) { return prm.terms == 1 ? 193 : 128; }

// Short sequences of narrow heads, which TMA could copy, go through the fourth generation's tensor cores all the same: a chunk of 64 tokens is less padded
// than one of 128, and two CTAs share an SM, where the other kernel's takes all of its tensor memory.  That one / this (us), 2048 heads of 64
// columns: 8 tokens 103 / 54 forward, 420 / 191 with backward; 64 tokens 117 / 72, 437 / 245; 128 tokens 114 / 103, 441 / 386; 192 tokens 148 / 142,
// 588 / 534; 256 tokens 148 / 180, 590 / 682.  256 heads of 64 tokens 65 / 38 with backward, 16 heads of 128 40 / 38.  Wider heads: 2048 of
// 128 columns 152 / 187 with 8 tokens, 159 / 228 with 64.  (A call that is to withhold copies goes to the kernel that makes them.)
bool short_and_narrow(const MixParams& p)
{
    return p.tokens <= 3 * kMixChunk && std::max(p.term[0].a, p.term[0].b) <= kTile && p.copies_bytes == 0 && p.withhold_copies == 0;
}

// Sequences are cut into as many segments as take the least time by this count, in microseconds: a round of CTAs takes 6 to begin and end with and
// for each 128 tokens, as measured, on the tensor cores 4 (2.5 for heads of 64, 4.3 of 128); in fp32 37, or with up to 64 columns, where two CTAs share an SM, 21 for one
// and 35 for both; the segments' own sums, made first, 0.6 of that; joining them 6.
void plan_mix(MixParams* prm)
{
    MixParams& p = *prm;
    p.units = (int64_t)p.n * p.sequences * p.heads;
    p.columns = 1, p.state_room = 0;
    for (int i = 0; i < p.terms; ++i) {
        p.columns = std::max(p.columns, (int)ceil_div(p.term[i].b, kTile));
        p.state_room = std::max<int64_t>(p.state_room, round_up(p.term[i].a * p.term[i].b, 4));
    }
    if (!p.f32 && p.tokens < 1ll << 30 && p.tokens >= copied_tokens(p)) {
        MixParams q = p;
        MixMoves in, out;
        q.copies = nullptr;
        p.copies_bytes = with_copies(&q, &in, &out);
        for (int i = 0; i < q.terms; ++i) p.state_room = std::max<int64_t>(p.state_room, q.term[i].a * q.term[i].b);
    }
    p.join_blocks = (int)ceil_div(p.state_room, kJoinThreads);
    const int64_t chunks = std::max<int64_t>(1, ceil_div(p.tokens, kMixTensorChunk)), ctas = p.units * p.terms * (p.f32 ? p.columns : 1);
    const bool narrow = std::max(p.term[0].a, p.term[0].b) <= kTile;
    const auto rounds = [&](int64_t count, double chunks_each) {
        if (!p.f32 || !narrow) return (double)ceil_div(count, kSms) * ((p.f32 ? 37.0 : 4.0) * chunks_each + 6.0);
        const int64_t both = count / (2 * kSms), rest = count - both * 2 * kSms;
        return (double)both * (35.0 * chunks_each + 6.0) + (rest == 0 ? 0.0 : (rest <= kSms ? 21.0 : 35.0) * chunks_each + 6.0);
    };
    int64_t best = 1;
    double least = 0.0;
    for (int64_t s = 1; s <= std::min<int64_t>(chunks, kMixSegments); ++s) {
        const int64_t each = ceil_div(chunks, s);
        if (s > 1 && (ceil_div(chunks, each) != s || ctas * s > 4 * kSms)) continue;
        const double cost = rounds(ctas * s, (double)each) + (s > 1 ? rounds(ctas * (s - 1), 0.6 * (double)each) + 6.0 : 0.0);
        if (s == 1 || cost < least) best = s, least = cost;
    }
    p.segment_tokens = ceil_div(chunks, best) * kMixTensorChunk;
    p.segments = (int)best;
}

cudaError_t launch_mix(const MixParams& prm, cudaStream_t stream)
{
    MixParams p = prm;
    MixMoves in, out;
    in.count = out.count = 0;
    if (p.copies_bytes > 0) {
        with_copies(&p, &in, &out);
        if (!mix_fits_tensor(p)) p = prm, in.count = out.count = 0;  // what needs no copy lies at an odd address
    }
    p.tensor = !p.f32 && mix_fits_tensor(p) && !short_and_narrow(p);
    const auto launch = p.f32 ? launch_f32 : p.tensor ? launch_mix_tensor : launch_mix_mma;
    cudaError_t err = launch_moves(p, in, stream);
    if (err == cudaSuccess && p.segments > 1) {
        err = launch(p, true, stream);
        if (err == cudaSuccess) err = launch_join(p, stream);
    }
    if (err == cudaSuccess) err = launch(p, false, stream);
    return err == cudaSuccess ? launch_moves(p, out, stream) : err;
}

cudaError_t launch_mix_step(const MixParams& prm, cudaStream_t stream)
{
    const MixTerm& t = prm.term[0];
    const bool wide = t.b % 4 == 0 && (reinterpret_cast<uintptr_t>(t.state_in) | reinterpret_cast<uintptr_t>(t.state_out)) % 16 == 0;
    int log = 0;
    while ((wide ? 4 : 1) << log < t.b) ++log;
    const dim3 grid((unsigned)prm.units);
    if (prm.f32)
        return wide ? launch_after(rps_mix_step_kernel<float, 4>, grid, kStepThreads, 0, stream, 1, prm, log)
                    : launch_after(rps_mix_step_kernel<float, 1>, grid, kStepThreads, 0, stream, 1, prm, log);
    return wide ? launch_after(rps_mix_step_kernel<bf16, 4>, grid, kStepThreads, 0, stream, 1, prm, log)
                : launch_after(rps_mix_step_kernel<bf16, 1>, grid, kStepThreads, 0, stream, 1, prm, log);
}

}  // namespace rps_ops
