// Parameter blocks and launch wrappers of the training operators (include/rps_ops.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "rps_ops.h"

namespace rps_ops {

using bf16 = __nv_bfloat16;

// Of a B200.  Plans are made without asking the device, so that workspaces have the sizes that the calls then count on; a launch that has to know
// how many there are asks sm_count.
constexpr int kSms = 148;

inline int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Launches a kernel so that its CTAs may be placed while the kernel before it in the stream drains (programmatic stream
// serialization).  Each of these kernels begins with after_the_kernel_before(): nothing is read or written in global memory ahead of
// it, and every CTA passes it, so that a kernel's end implies the end of all before it.
template <typename Kernel, typename... Args>
cudaError_t launch_after(Kernel kernel, dim3 grid, int threads, size_t shared, cudaStream_t stream, int cluster, const Args&... args)
{
    cudaLaunchConfig_t config{};
    config.gridDim = grid, config.blockDim = dim3((unsigned)threads), config.dynamicSmemBytes = shared, config.stream = stream;
    cudaLaunchAttribute attributes[2] = {};
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = (unsigned)cluster, attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    config.attrs = attributes, config.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&config, kernel, args...);
}

// ---------------------------------------------------------------------------------------------------- products
// Token rows are padded to whole tiles, and the vocabulary goes through the loss in whole tiles.
constexpr int kTokenTile = 256;
constexpr int kTokenBlock = 64;  // of tokens as a summed axis
constexpr int kVocabTile = 256;

// An operand of a product: bf16 [worker][plane][rows][row stride].  fp32 values lie in three planes whose sum they are.
struct Operand {
    const bf16* base;
    int64_t worker, plane, row;  // strides
    int64_t rows, cols;          // what exists; zero outside
};

enum class Product {
    kLse,      // A = hidden [m][k], B = weight [n][k]: softmax statistics of each row over a tile of columns
    kDlogits,  // the same product: dl = g (exp(l - lse) - [v == target]) into planes
    kTopLse,   // kLse of logits times `sharpness`, and the logits of each row's entries
    kTopDlogits,  // kDlogits of them, less the probabilities of the row's entries instead of a target's one
    kDhidden,  // A = dl [m][k], B = weight [k][n]: a sum over pieces of the vocabulary, then scattered to the tokens' rows
    kDweight   // A = dl or dy [k][m], B = hidden or x [k][n]
};

constexpr int kTopBuckets = 64;

// How a product is cut: columns of its tiles, runs of its summed axis, and CTAs that make a tile (1 or 2).
struct ProductShape {
    int tile_cols, splits, ctas;
};

struct ProductParams {
    Operand a, b;
    int workers, planes;  // three planes: fp32 operands and results, one: bf16
    int m, n, k;        // upper bounds where the token count (m, or k in kDweight) is the device's to say
    const int* count;   // [worker] tokens that take part, or NULL: all
    // kLse, kDlogits
    int v0, vocab;          // first row of the vocabulary in this piece; all of it
    int stat_tiles;         // softmax statistics are kept for every tile's columns
    const int* target;      // [worker][tokens_padded]
    float2* part;           // [worker][stat_tiles][tokens_padded]: running maximum and sum
    float* hit;             // [worker][tokens_padded]: the target's logit
    const float2* info;     // [worker][tokens_padded]: lse, g
    bf16* dl;               // [worker][plane][tokens_padded][piece]
    // kTopLse, kTopDlogits: up to `top` entries of each token, by rising row of the weight (behind the last: the largest int)
    int top, bucket_rows;      // kTopBuckets buckets of this many rows of the weight each
    float sharpness;
    const unsigned short* entry_bucket;  // [worker][tokens][kTopBuckets]: first entry in the bucket or behind it
    const int* entry_id;       // [worker][tokens][top]
    const float* entry_weight; // their probabilities
    float* entry_logit;        // written by kTopLse
    int64_t tokens_padded, piece;
    // kDhidden, kDweight: the result, scaled and in the caller's type, or (part != NULL) fp32 parts of it that launch_join adds up
    void* out;
    int64_t out_row, out_worker;
    const float* scale;     // [worker], or NULL: factor of the result
    const int* rows;        // kDhidden: [worker][tokens]: token of each row
    int64_t tokens;
    // The summed axis may be cut into `splits` runs of blocks, each with its own part [split][worker][part_rows][part_row]; over several
    // pieces of the vocabulary a part goes on growing (`add`).
    int splits, tile_cols, ctas;  // product_shape
    void shaped(const ProductShape& s) { tile_cols = s.tile_cols, splits = s.splits, ctas = s.ctas; }
    int wait_limit_ms, withhold_copies;  // 0: the default; see rps_wgrad_desc
    int a_rows;                   // rows of A that a CTA copies (launch_product's to set)
    int add;
    float* parts;
    int64_t part_rows, part_row;  // multiples of the tile
};

ProductShape product_shape(int64_t m, int64_t n, int64_t k, int workers, int planes, bool may_split);

cudaError_t launch_product(Product which, const ProductParams& prm, cudaStream_t stream);
cudaError_t launch_join(Product which, const ProductParams& prm, cudaStream_t stream);  // the parts into `out`
cudaError_t read_gave_up(int* value, cudaStream_t stream);  // whether a wait in a product gave up, and clears it; synchronises
cudaError_t read_norm_gave_up(int* value, cudaStream_t stream);  // the same of a norm
cudaError_t sm_count(int* out);                             // of the current device

// ---------------------------------------------------------------------------------------------------- the loss
struct LceParams {
    int n, planes, f32, reduction, backward;
    int64_t tokens, tokens_padded, vocab, cols, cols_padded, ignore_index;
    const int64_t* targets;
    int* rows;        // [n][tokens]: tokens that take part in their order, then the others
    int* count;       // [n]
    int* target;      // [n][tokens_padded]: targets of the rows, -1 for one that names no row of weight
    float2* info;     // [n][tokens_padded] (backward): lse and the factor of the row's dl
    float* scale;     // [n] (backward): the factor that a worker's rows share, applied to the sums of products
    const float* lse_in;
    const float* dloss;
    const void* hidden;
    int64_t hidden_row, hidden_worker;
    bf16* packed;     // [n][planes][tokens_padded][cols_padded]
    void* dhidden;    // backward: the rows of ignored tokens are cleared along the way
    // forward's end
    const float2* part;
    const float* hit;
    int64_t stat_tiles;  // as ProductParams
    float factor, sharpness;  // of the loss's gradient, and of the logits: 1 but for distillation
    // distillation (top > 0): see ProductParams
    int top;
    const int* entry_id;
    const float *entry_weight, *entry_logit;
    float* loss;
    float* lse;
    float* sums;      // [n][lce_merge_blocks(tokens)]
    int* done;        // [n]
    // a few tokens (dot_rows > 0): see rps_lce_dot.cu
    int dot_rows, dot_blocks;          // room for tokens in dot_dl; CTAs of each worker that make logits
    int dot_ranges, dot_wide, dot_high;  // of the gradients: ranges of the vocabulary; warps of a CTA along a row and over rows
    const void* weight;
    int64_t weight_row, weight_worker;
    void* dweight;
    int64_t dweight_row, dweight_worker;
    float* dot_dl;                     // [n][vocab][dot_rows]
    float* dot_parts;                  // [ranges][n][dot_rows][round_up(cols, 4)]: of dhidden
};
// Whether so few tokens go through dot products, and how; the rest of prm is set.
void plan_lce_dot(LceParams* prm);
cudaError_t launch_lce_dot(const LceParams& prm, cudaStream_t stream);         // statistics, or (backward) dl
cudaError_t launch_lce_dot_grads(const LceParams& prm, cudaStream_t stream);   // dweight, and dhidden's parts

// Distillation's teacher: its entries' probabilities, sorted by row of the weight, and which tokens have any.
struct TeacherParams {
    int n, top, top_f32;
    int64_t tokens, vocab, ignore_index;
    float sharpness;
    const int64_t* ids;     // [n][tokens][top]
    const void* logits;
    int bucket_rows;
    unsigned short* entry_bucket;  // as ProductParams
    int* entry_id;
    float* entry_weight;
    int64_t* targets;       // [n][tokens]: 0, kNoTeacher for a token without entries, -1 for one whose entries are no distribution
};
constexpr int64_t kNoTeacher = -100;
cudaError_t launch_teacher(const TeacherParams& prm, cudaStream_t stream);

// Which tokens take part, and their rows laid out.
cudaError_t launch_lce_rows(const LceParams& prm, cudaStream_t stream);
int64_t lce_merge_blocks(int64_t tokens);
cudaError_t launch_lce_merge(const LceParams& prm, cudaStream_t stream);  // the loss, or (top > 0) the divergence from the teacher

// Lays the rows of a matrix of each worker out as planes; columns past `cols` become zero.
struct PlanesParams {
    const void* src;
    int f32, n, planes;
    int64_t rows, cols, src_row, src_worker;
    bf16* dst;
    int64_t dst_row, dst_plane, dst_worker;
};
cudaError_t launch_planes(const PlanesParams& prm, cudaStream_t stream);

// ---------------------------------------------------------------------------------------------------- 8 bits
struct PackParams {
    int f32;
    int64_t rows, cols, x_row, pitch, groups;
    const void* x;
    void* out;
    int8_t* codes;
    float* scales;
    // unpacking into planes: rows of one worker are `tokens`
    bf16* planes_out;
    int planes;
    int64_t tokens, dst_row, dst_plane, dst_worker;
};
cudaError_t launch_pack(const PackParams& prm, cudaStream_t stream);
cudaError_t launch_unpack(const PackParams& prm, cudaStream_t stream);
cudaError_t launch_unpack_planes(const PackParams& prm, cudaStream_t stream);

// ---------------------------------------------------------------------------------------------------- norm
struct NormParams {
    int f32, n, packed;
    int cluster;  // CTAs that share a row
    int64_t tokens, cols, gates, rows_per_gate;
    int64_t post_worker, pre_worker, gate_worker;
    float scale, eps;
    const void *x, *f, *h_in, *gate, *post, *pre, *dh, *dy;
    void *h, *y, *dx, *df, *dgate, *dpost, *dpre;
    float *r_f, *r_h;
    int8_t *f_codes, *h_codes;
    float *f_scales, *h_scales;
    int64_t pitch, groups;
    // backward: each worker's tokens are cut over blocks that lie inside one gate group (chunks > 0: `chunks` blocks a group),
    // or hold whole groups (chunks == 0)
    int64_t rows_per_block, blocks, chunks;
    float* partial;  // [n][blocks][3][cols]: dpost, dpre, dgate
    int wait_limit_ms, withhold_sums;  // 0: the default; see rps_norm_desc
};
void plan_norm_backward(NormParams* prm);
cudaError_t launch_norm_forward(const NormParams& prm, cudaStream_t stream);
cudaError_t launch_norm_backward(const NormParams& prm, cudaStream_t stream);

// ---------------------------------------------------------------------------------------------------- embedding
struct EmbedParams {
    int f32, n, accumulate;
    float scale;
    int64_t count, vocab, cols, ignore_index;  // count: tokens of a worker
    const int64_t* tokens;
    const void* weight;
    int64_t weight_row, weight_worker;
    void* out;
    const void* dout;
    void* dweight;
    int64_t dweight_row, dweight_worker;
    // backward (plan_embed): the tokens sorted by row, in one of two places each
    int key_bits, digit_bits, sorted;  // sorted: which place
    int64_t sort_blocks;               // CTAs that sort a worker's tokens; 0: a cluster of eight, in shared memory (few: each of those that sum)
    uint32_t *keys[2], *from[2];       // [n][count]
    uint32_t* counts;                  // [n][256][sort_blocks]
    int64_t tile, tiles, part_row;     // sorted tokens of a tile; of a worker
    float* parts;                      // [n][tiles][2][part_row]: sums of runs that cross tiles: from the tile before, into the next
};
void plan_embed(EmbedParams* prm);
cudaError_t launch_embed_lookup(const EmbedParams& prm, cudaStream_t stream);
cudaError_t launch_embed_gradient(const EmbedParams& prm, cudaStream_t stream);

// ---------------------------------------------------------------------------------------------------- linear attention
constexpr int kMixChunk = 64, kMixTensorChunk = 128, kMixMaxCols = RPS_MAX_HEAD_COLS, kMixSegments = 64;

// [worker][sequence][token][head][cols]; strides
struct MixOperand {
    const void* base;
    int64_t worker, sequence, token, head;
};

// One form (rps_mix.cu).
struct MixTerm {
    MixOperand x, y, z;
    void* out;              // [worker][sequence][token][head][b], dense
    int a, b, reversed;     // columns of x and y, and of z; whether time runs backwards
    const float* state_in;  // a * b of each unit, or NULL: zeros
    float* state_out;       // or NULL
    int64_t state_a, state_b;  // strides of the states' elements
    float score_scale, state_scale, update_scale;  // of x . y, of x W, and of what is added to W
    int rows, cols;         // of the states: a and b, but where a and b are columns of copies (plan_mix)
};

struct MixParams {
    int f32, n, heads, terms;
    int64_t sequences, tokens;
    const int64_t* lengths;   // [n][sequences], or NULL
    const float* log_decay;   // [n][heads]
    MixTerm term[3];
    int wait_limit_ms, withhold_copies;  // 0: the default; see rps_linear_attention_desc
    // plan_mix
    int64_t units, segment_tokens, state_room;  // segment_tokens: a multiple of kMixTensorChunk
    int columns, segments, join_blocks, tensor;
    float* segment_states;    // [term][unit][segment][state_room] (segments > 1)
    size_t copies_bytes;      // of copies of the operands and results that TMA cannot copy as they lie, with columns in eights (0: none are made)
    unsigned char* copies;
};
void plan_mix(MixParams* prm);
cudaError_t launch_mix(const MixParams& prm, cudaStream_t stream);
bool mix_fits_tensor(const MixParams& prm);  // whether rps_mix_tensor.cu takes it
bool mix_fits_tensor(const MixParams& prm, const MixOperand& o, int cols);  // an operand, at a 16-byte aligned address
cudaError_t launch_mix_tensor(const MixParams& prm, bool states, cudaStream_t stream);  // states: the segments' own sums
cudaError_t launch_mix_mma(const MixParams& prm, bool states, cudaStream_t stream);     // bf16 that it does not
cudaError_t read_mix_gave_up(int* value, cudaStream_t stream);
cudaError_t launch_mix_step(const MixParams& prm, cudaStream_t stream);

// ---------------------------------------------------------------------------------------------------- device helpers
#ifdef __CUDACC__
// A flag in device memory.
inline cudaError_t read_and_clear(int& flag, int* value, cudaStream_t stream)
{
    const int zero = 0;
    cudaError_t err = cudaMemcpyFromSymbolAsync(value, flag, sizeof(int), 0, cudaMemcpyDeviceToHost, stream);
    if (err == cudaSuccess) err = cudaStreamSynchronize(stream);
    if (err == cudaSuccess && *value != 0) err = cudaMemcpyToSymbolAsync(flag, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, stream);
    if (err == cudaSuccess) err = cudaStreamSynchronize(stream);
    return err;
}

__device__ __forceinline__ void after_the_kernel_before()
{
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
}

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<bf16>(bf16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 from_float<bf16>(float v) { return __float2bfloat16_rn(v); }

// Two values as bf16, rounded to nearest; what would round to infinity becomes the largest number.
__device__ __forceinline__ uint32_t nearest_two_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ uint32_t two_bf16(float lo, float hi)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// An fp32 value is the sum of three bf16 values exactly: each is the nearest to what the ones before it leave, so that what the last two
// leave out of a product has no sign in common with it.  (Cut off instead of rounded, the parts are up to twice as large, and the products of
// parts that are not made reach 2^-21 of the result, always with its sign; rounded 2^-24.)  An infinity or a NaN is the third one, after
// zeros: of the products made the third part takes part in that with the other operand's first one alone, so that an infinity times a
// number is an infinity, and none meets a part that happens to be zero.  Two values at a time, as words.
__device__ __forceinline__ void split_two(float a, float b, uint32_t (&parts)[3])
{
    const bool finite_a = fabsf(a) <= 3.402823466e38f, finite_b = fabsf(b) <= 3.402823466e38f;
    float x = finite_a ? a : 0.0f, y = finite_b ? b : 0.0f;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        parts[q] = nearest_two_bf16(x, y);
        x -= __uint_as_float(parts[q] << 16), y -= __uint_as_float(parts[q] & 0xFFFF0000u);
    }
    parts[2] = two_bf16(finite_a ? x : a, finite_b ? y : b);
}
#endif

}  // namespace rps_ops
