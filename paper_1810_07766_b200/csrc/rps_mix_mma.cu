// Linear attention's form (rps_mix.cu) for bf16 operands in short sequences of narrow heads, and for those that TMA cannot copy: odd numbers of columns or
// strides in short sequences (of long ones copies are made, plan_mix), and odd addresses.
//
// A CTA has a sequence's head and 64 columns of z, chunk by chunk of 64 tokens; W stays in its registers as fp32.  Products go through the tensor cores by
// mma.sync: tiles are 64 x 64 with 16 rows to a warp, and every operand is scaled or masked in registers on its way from one product to the next.
// Operands are used as they are; what is made here is rounded to bf16 where it is multiplied once more on its way to a bf16 result (the masked
// products, W), and kept in three parts where it is summed into a state (r^(C-1-j) y_j).  Bound by the latency of a chunk's way through its four warps.
// (37 x 4 heads of 512 tokens x 60, forward and backward: 163 us; multiplied in fp32 registers, as fp32 operands are, 416.)
#include <algorithm>

#include "rps_mix.cuh"
#include "rps_tma.cuh"

namespace rps_ops {
namespace {

constexpr int kC = kMixChunk, kTile = 64, kThreads = 128;  // tokens of a chunk; columns of z of a CTA

// ------------------------------------------------------------------------------------------------------ instructions
__device__ __forceinline__ void multiply(float (&sum)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(sum[0]), "+f"(sum[1]), "+f"(sum[2]), "+f"(sum[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <bool TRANSPOSED>
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t addr)
{
    if constexpr (TRANSPOSED)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// A 16 x 16 operand (rows x summed axis), as parts whose sum it is, and two 16 x 8 ones (summed axis x columns).
template <int PARTS>
struct Left {
    uint32_t part[PARTS][4];
};
struct Right {
    uint32_t word[2][2];
};

// How operands come out of tiles in shared memory.  ROW: elements from a row to the next, chosen so that a warp's reads meet no bank twice.
struct Tile {
    // [row][summed axis]
    template <int ROW>
    static __device__ __forceinline__ void left(Left<1>& a, const bf16* tile, int row, int k)
    {
        const int lane = threadIdx.x % 32;
        load_matrices<false>(a.part[0], rps::smem_addr(tile + (row + lane % 16) * ROW + k + lane / 16 * 8));
    }
    // [column][summed axis]
    template <int ROW>
    static __device__ __forceinline__ void right_across(Right& b, const bf16* tile, int k, int col)
    {
        const int lane = threadIdx.x % 32;
        uint32_t r[4];
        load_matrices<false>(r, rps::smem_addr(tile + (col + lane % 8 + lane / 16 * 8) * ROW + k + lane / 8 % 2 * 8));
        b.word[0][0] = r[0], b.word[0][1] = r[1], b.word[1][0] = r[2], b.word[1][1] = r[3];
    }
    // [summed axis][column]
    template <int ROW>
    static __device__ __forceinline__ void right(Right& b, const bf16* tile, int k, int col)
    {
        const int lane = threadIdx.x % 32;
        uint32_t r[4];
        load_matrices<true>(r, rps::smem_addr(tile + (k + lane % 16) * ROW + col + lane / 16 * 8));
        b.word[0][0] = r[0], b.word[0][1] = r[1], b.word[1][0] = r[2], b.word[1][1] = r[3];
    }
    // [summed axis][row], times a factor for each step of the summed axis: the lane's are at k + 2 (lane % 4) + {0, 1, 8, 9}
    template <int ROW>
    static __device__ __forceinline__ void left_across(Left<3>& a, const bf16* tile, int k, int row, const float (&factor)[4])
    {
        const int lane = threadIdx.x % 32;
        uint32_t r[4];
        load_matrices<true>(r, rps::smem_addr(tile + (k + lane % 8 + lane / 16 * 8) * ROW + row + lane / 8 % 2 * 8));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t word[3];
            const Pair scale(factor[i / 2 * 2], factor[i / 2 * 2 + 1]);
            cut_in_parts(Pair(__uint_as_float(r[i] << 16), __uint_as_float(r[i] & 0xFFFF0000u)), scale, scale * Pair(kBelow), word[0], word[1], word[2]);
            word[1] = keep_infinities(word[0], word[1]), word[2] = keep_infinities(word[0], word[2]);
#pragma unroll
            for (int q = 0; q < 3; ++q) a.part[q][i] = word[q];
        }
    }
    static __device__ __forceinline__ void store_two(bf16* at, float a, float b) { *reinterpret_cast<uint32_t*>(at) = two_bf16(a, b); }
};

// Products of parts, the smallest first; TILES tiles of 8 columns side by side, of which the first `tiles` are wanted.
template <int PARTS, int TILES>
__device__ __forceinline__ void multiply_parts(float (&sum)[TILES][4], const Left<PARTS>& a, const Right (&b)[TILES / 2], int tiles)
{
#pragma unroll
    for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
        for (int n = 0; n < TILES; ++n)
            if (n < tiles) multiply(sum[n], a.part[p], b[n / 2].word[n % 2][0], b[n / 2].word[n % 2][1]);
}

// ------------------------------------------------------------------------------------------------------------ kernel
// MT: 64 columns of x and y each.  STATES: no output, only each segment's own sum.
template <int MT>
struct Shape {
    static constexpr int kRowA = MT * 64 + 8, kRowB = kTile + 8;
    static constexpr int kStage = kC * (2 * kRowA + kRowB);  // elements: x, y, z
    static constexpr int kBytes = (2 * kStage + MT * 64 * kRowB) * 2 + (kC + 4) * 4;
};

template <int MT, int ALIGN, bool STATES>
__global__ void __launch_bounds__(kThreads) rps_mix_mma_kernel(const __grid_constant__ MixParams prm)
{
    after_the_kernel_before();
    using S = Shape<MT>;
    using T = bf16;
    constexpr int W = Slice<T>::kWidth, NT = 8;  // tiles of 8 columns of a warp
    extern __shared__ __align__(128) unsigned char raw[];
    T* const stages = reinterpret_cast<T*>(raw);
    T* const state = stages + 2 * S::kStage;
    float* const powers = reinterpret_cast<float*>(state + MT * 64 * S::kRowB);  // r^0 .. r^64

    const MixTerm& term = prm.term[blockIdx.y];
    const int a = term.a, b = term.b, a16 = (a + 15) / 16 * 16;
    const int64_t item = blockIdx.x / prm.columns;
    const int col0 = (int)(blockIdx.x - item * prm.columns) * kTile;
    if (col0 >= b) return;
    const int segment = (int)(item % prm.segments);
    const int64_t unit = item / prm.segments;
    if (STATES && segment + 1 == prm.segments) return;
    const Place at = place_of(prm, unit);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, wr = warp, g = lane / 4, t2 = lane % 4 * 2;
    const int cols = min(kTile, b - col0), tiles = min(NT, (cols + 7) / 8);
    const int64_t i0 = segment * prm.segment_tokens, i1 = min(at.length, i0 + prm.segment_tokens);
    const int late = term.reversed;
    const float log_decay = __ldg(prm.log_decay + at.w * prm.heads + at.head);
    if (threadIdx.x <= kC) powers[threadIdx.x] = (float)power(log_decay, threadIdx.x);

    const T* const x = first_token<T>(term.x, at);
    const T* const y = first_token<T>(term.y, at);
    const T* const z = first_token<T>(term.z, at);
    // a chunk's rows; behind the last token zeros
    const auto load = [&](int64_t i, int stage) {
        T* const to = stages + stage * S::kStage;
        const auto rows = [&](T* tile, int row_length, const T* from, int64_t stride, int c0, int limit, int width) {
            const int across = (width + W - 1) / W;
            for (int u = threadIdx.x; u < kC * across; u += kThreads) {
                const int r = u / across, c = (u - r * across) * W;
                const int64_t at_row = i + r, token = late ? at.length - 1 - at_row : at_row;
                const bool there = at_row < i1;
                copy_slice<T, ALIGN>(rps::smem_addr(tile + r * row_length + c), from + (there ? token : 0) * stride, c0 + c, there ? limit : 0);
            }
        };
        if (!STATES) rows(to, S::kRowA, x, term.x.token, 0, a, a16);
        rows(to + kC * S::kRowA, S::kRowA, y, term.y.token, 0, a, a16);
        rows(to + 2 * kC * S::kRowA, S::kRowB, z, term.z.token, col0, b, kTile);
        copies_sent();
    };

    // W: rows 16 (wr + 4 m) + g and + 8, columns 8 n + t2 and + 1
    float w[MT][NT][4];
    bool zero = true;  // so far
    const float* init = prm.segments > 1 && !STATES ? prm.segment_states + ((blockIdx.y * prm.units + unit) * prm.segments + segment) * prm.state_room : nullptr;
    int64_t init_a = b, init_b = 1;
    if (!STATES && prm.segments == 1 && term.state_in != nullptr) init = term.state_in + unit * a * b, init_a = term.state_a, init_b = term.state_b;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = (wr + 4 * m) * 16 + g + e / 2 * 8, col = col0 + n * 8 + t2 + e % 2;
                w[m][n][e] = init != nullptr && row < a && col < b ? __ldg(init + row * init_a + col * init_b) : 0.0f;
            }
    if (init != nullptr) zero = false;
    const auto publish = [&] {  // W where the products read it
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; e += 2)
                    Tile::store_two(state + ((wr + 4 * m) * 16 + g + e / 2 * 8) * S::kRowB + n * 8 + t2, w[m][n][e], w[m][n][e + 1]);
    };
    if (i0 < i1) load(i0, 0);
    if (!STATES && !zero) publish();

    int stage = 0;
    for (int64_t i = i0; i < i1; i += kC, stage ^= 1) {
        if (i + kC < i1) {
            load(i + kC, stage ^ 1);
            copies_arrived<1>();
        } else {
            copies_arrived<0>();
        }
        __syncthreads();
        T* const tx = stages + stage * S::kStage;
        const T* const ty = tx + kC * S::kRowA;
        const T* const tz = ty + kC * S::kRowA;
        const int inside = (int)min((int64_t)kC, i1 - i);
        if constexpr (!STATES) {
            const int row0 = wr * 16;
            // x . y of these rows with the tokens up to them
            float p[8][4];
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[n][e] = 0.0f;
            const int keys = 2 * wr + 2;
            for (int k = 0; k < a16; k += 16) {
                Left<1> left;
                Tile::left<S::kRowA>(left, tx, row0, k);
                Right right[4];
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (2 * n < keys) Tile::right_across<S::kRowA>(right[n], ty, k, n * 16);
                multiply_parts<1, 8>(p, left, right, keys);
            }
            float out[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) out[n][e] = 0.0f;
            if (!zero) {
                for (int k = 0; k < a16; k += 16) {
                    Left<1> left;
                    Tile::left<S::kRowA>(left, tx, row0, k);
                    Right right[NT / 2];
#pragma unroll
                    for (int n = 0; n < NT / 2; ++n)
                        if (2 * n < tiles) Tile::right<S::kRowB>(right[n], state, k, 2 * n * 8);
                    multiply_parts<1, NT>(out, left, right, tiles);
                }
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float factor = term.state_scale * powers[row0 + g + e / 2 * 8 + 1 - late];
#pragma unroll
                    for (int n = 0; n < NT; ++n) out[n][e] *= factor, out[n][e + 1] *= factor;
                }
            }
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int apart = row0 + g + e / 2 * 8 - (n * 8 + t2 + e % 2);
                    p[n][e] = apart >= 0 ? p[n][e] * (term.score_scale * powers[max(apart, 0)]) : 0.0f;
                }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k > wr) break;
                Left<1> left;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    left.part[0][i] = two_bf16(p[2 * k + i / 2][i % 2 * 2], p[2 * k + i / 2][i % 2 * 2 + 1]);
                }
                Right right[NT / 2];
#pragma unroll
                for (int n = 0; n < NT / 2; ++n)
                    if (2 * n < tiles) Tile::right<S::kRowB>(right[n], tz, k * 16, 2 * n * 8);
                multiply_parts<1, NT>(out, left, right, tiles);
            }
            // out through this warp's rows of x, which have been read
            __syncwarp();
            T* const own = tx + row0 * S::kRowA;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; e += 2) Tile::store_two(own + (g + e / 2 * 8) * S::kRowA + n * 8 + t2, out[n][e], out[n][e + 1]);
            __syncwarp();
            constexpr int kAcross = NT * 8 / W, kDown = 32 / kAcross;
            const int c = lane % kAcross * W;
#pragma unroll
            for (int r = lane / kAcross; r < 16; r += kDown) {
                const int64_t row = i + row0 + r, token = late ? at.length - 1 - row : row;
                if (row < i1)
                    store_slice<T, ALIGN>(static_cast<T*>(term.out) + (((at.w * prm.sequences + at.sequence) * prm.tokens + token) * prm.heads + at.head) * b + col0, c,
                                          cols, *reinterpret_cast<const uint4*>(own + r * S::kRowA + c));
            }
        }
        // W
        const float whole = powers[inside];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if ((wr + 4 * m) * 16 >= a16) break;
            float u[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) u[n][e] = 0.0f;
#pragma unroll
            for (int k = 0; k < kC; k += 16) {
                if (k >= inside) break;
                float factor[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    const int left = inside - 1 - (k + t2 + f % 2 + f / 2 * 8);
                    factor[f] = left >= 0 ? term.update_scale * powers[left + late] : 0.0f;
                }
                Left<3> left;
                Tile::left_across<S::kRowA>(left, ty, k, (wr + 4 * m) * 16, factor);
                Right right[NT / 2];
#pragma unroll
                for (int n = 0; n < NT / 2; ++n)
                    if (2 * n < tiles) Tile::right<S::kRowB>(right[n], tz, k, 2 * n * 8);
                multiply_parts<3, NT>(u, left, right, tiles);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)  // rows behind the heads' columns stay zeros: an infinite z makes NaN of their part of u
                    w[m][n][e] = (wr + 4 * m) * 16 + g + e / 2 * 8 < a ? fmaf(whole, w[m][n][e], u[n][e]) : 0.0f;
        }
        zero = false;
        __syncthreads();
        if (!STATES && i + kC < i1) publish();
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
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = (wr + 4 * m) * 16 + g + e / 2 * 8, col = col0 + n * 8 + t2 + e % 2;
                    if (row < a && col < b) to[row * to_a + col * to_b] = w[m][n][e];
                }
    }
    if constexpr (!STATES) {
        // rows behind the sequence's last token
        const int64_t t1 = min(prm.tokens, i0 + prm.segment_tokens);
        for (int64_t t = max(at.length, i0) + warp; t < t1; t += 4)
            for (int c = lane * W; c < cols; c += 32 * W)
                store_slice<T, ALIGN>(static_cast<T*>(term.out) + (((at.w * prm.sequences + at.sequence) * prm.tokens + t) * prm.heads + at.head) * b + col0, c, cols,
                                      make_uint4(0, 0, 0, 0));
    }
}

// -------------------------------------------------------------------------------------------------------------- host
template <int MT, int ALIGN, bool STATES>
cudaError_t launch_kernel(const MixParams& prm, cudaStream_t stream)
{
    static rps::LaunchState granted;
    const cudaError_t err = rps::grant_smem(granted, rps_mix_mma_kernel<MT, ALIGN, STATES>, Shape<MT>::kBytes);
    if (err != cudaSuccess) return err;
    return launch_after(rps_mix_mma_kernel<MT, ALIGN, STATES>, dim3((unsigned)(prm.units * prm.segments * prm.columns), (unsigned)prm.terms), kThreads, Shape<MT>::kBytes, stream,
                        1, prm);
}

template <int MT, int ALIGN>
cudaError_t launch_either(const MixParams& prm, bool states, cudaStream_t stream)
{
    return states ? launch_kernel<MT, ALIGN, true>(prm, stream) : launch_kernel<MT, ALIGN, false>(prm, stream);
}

}  // namespace

cudaError_t launch_mix_mma(const MixParams& prm, bool states, cudaStream_t stream)
{
    int widest = 0;
    for (int i = 0; i < prm.terms; ++i) widest = std::max(widest, prm.term[i].a);
    const int align = mix_alignment<bf16>(prm);
    if (widest <= 64) return align == 16 ? launch_either<1, 16>(prm, states, stream) : align == 4 ? launch_either<1, 4>(prm, states, stream) : launch_either<1, 2>(prm, states, stream);
    return align == 16 ? launch_either<2, 16>(prm, states, stream) : align == 4 ? launch_either<2, 4>(prm, states, stream) : launch_either<2, 2>(prm, states, stream);
}

}  // namespace rps_ops
