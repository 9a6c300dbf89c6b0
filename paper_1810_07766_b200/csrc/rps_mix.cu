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
// A CTA takes a sequence's head and 64 columns of z, chunk by chunk; W stays in its registers as fp32.  Where there are too few of those to fill
// the SMs, sequences are cut into segments: one launch makes each segment's own sum of y^T z, one adds them up in order into the states that
// segments begin with, and the main one then runs all segments at once (y and z are read twice).
//
// Products go through the tensor cores (mma.sync: tiles are 64 x 64 with 16 rows to a warp, and every operand is scaled or masked in registers
// on its way from one product to the next).  bf16 operands are used as they are; what is made here is rounded to bf16 where it is multiplied
// once more on its way to a bf16 result (the masked products, W), and kept in three parts where it is summed into a state (r^(C-1-j) y_j).
// fp32 operands are three bf16 parts each, of whose products six are made (split_two).
#include <algorithm>

#include "rps_mix.cuh"
#include "rps_tma.cuh"

namespace rps_ops {
namespace {

using rps::LaunchState;

constexpr int kC = kMixChunk, kTile = 64;  // tokens of a chunk; columns of z of a CTA

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

// A 16 x 16 operand (rows x summed axis) and two 16 x 8 ones (summed axis x columns), as parts whose sum they are.
template <int PARTS>
struct Left {
    uint32_t part[PARTS][4];
};
template <int PARTS>
struct Right {
    uint32_t part[PARTS][2][2];
};

// Two values as PARTS words.
template <int PARTS>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&word)[PARTS])
{
    if constexpr (PARTS == 1) {
        word[0] = two_bf16(a, b);
    } else {
        split_two(a, b, word);
    }
}

// How tiles lie in shared memory, and how operands come out of them.  ROW: elements from a row to the next, chosen so that a warp's
// reads meet no bank twice.
template <typename T>
struct Tile;

template <>
struct Tile<bf16> {
    static constexpr int kPad = 8, kParts = 1;
    // [row][summed axis]
    template <int ROW>
    static __device__ __forceinline__ void left(Left<1>& a, const bf16* tile, int row, int k)
    {
        const int lane = threadIdx.x % 32;
        load_matrices<false>(a.part[0], rps::smem_addr(tile + (row + lane % 16) * ROW + k + lane / 16 * 8));
    }
    // [column][summed axis]
    template <int ROW>
    static __device__ __forceinline__ void right_across(Right<1>& b, const bf16* tile, int k, int col)
    {
        const int lane = threadIdx.x % 32;
        uint32_t r[4];
        load_matrices<false>(r, rps::smem_addr(tile + (col + lane % 8 + lane / 16 * 8) * ROW + k + lane / 8 % 2 * 8));
        b.part[0][0][0] = r[0], b.part[0][0][1] = r[1], b.part[0][1][0] = r[2], b.part[0][1][1] = r[3];
    }
    // [summed axis][column]
    template <int ROW>
    static __device__ __forceinline__ void right(Right<1>& b, const bf16* tile, int k, int col)
    {
        const int lane = threadIdx.x % 32;
        uint32_t r[4];
        load_matrices<true>(r, rps::smem_addr(tile + (k + lane % 16) * ROW + col + lane / 16 * 8));
        b.part[0][0][0] = r[0], b.part[0][0][1] = r[1], b.part[0][1][0] = r[2], b.part[0][1][1] = r[3];
    }
    // [summed axis][row], times a factor for each step of the summed axis: the lane's are at k + 2 (lane % 4) + {0, 1, 8, 9}
    template <int ROW, int PARTS>
    static __device__ __forceinline__ void left_across(Left<PARTS>& a, const bf16* tile, int k, int row, const float (&factor)[4])
    {
        const int lane = threadIdx.x % 32;
        uint32_t r[4];
        load_matrices<true>(r, rps::smem_addr(tile + (k + lane % 8 + lane / 16 * 8) * ROW + row + lane / 8 % 2 * 8));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t word[PARTS];
            split_pair<PARTS>(__uint_as_float(r[i] << 16) * factor[i / 2 * 2], __uint_as_float(r[i] & 0xFFFF0000u) * factor[i / 2 * 2 + 1], word);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) a.part[q][i] = word[q];
        }
    }
    static __device__ __forceinline__ void store_two(bf16* at, float a, float b) { *reinterpret_cast<uint32_t*>(at) = two_bf16(a, b); }
};

template <>
struct Tile<float> {
    static constexpr int kPad = 4, kParts = 3;
    static __device__ __forceinline__ void split(float a, float b, uint32_t& first, uint32_t& second, uint32_t& third)
    {
        uint32_t word[3];
        split_two(a, b, word);
        first = word[0], second = word[1], third = word[2];
    }
    template <int ROW>
    static __device__ __forceinline__ void left(Left<3>& a, const float* tile, int row, int k)
    {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = *reinterpret_cast<const float2*>(tile + (row + lane / 4 + i % 2 * 8) * ROW + k + lane % 4 * 2 + i / 2 * 8);
            split(v.x, v.y, a.part[0][i], a.part[1][i], a.part[2][i]);
        }
    }
    template <int ROW>
    static __device__ __forceinline__ void right_across(Right<3>& b, const float* tile, int k, int col)
    {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float2 v = *reinterpret_cast<const float2*>(tile + (col + n * 8 + lane / 4) * ROW + k + lane % 4 * 2 + i * 8);
                split(v.x, v.y, b.part[0][n][i], b.part[1][n][i], b.part[2][n][i]);
            }
    }
    template <int ROW>
    static __device__ __forceinline__ void right(Right<3>& b, const float* tile, int k, int col)
    {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float* at = tile + (k + lane % 4 * 2 + i * 8) * ROW + col + n * 8 + lane / 4;
                split(at[0], at[ROW], b.part[0][n][i], b.part[1][n][i], b.part[2][n][i]);
            }
    }
    template <int ROW, int PARTS>
    static __device__ __forceinline__ void left_across(Left<PARTS>& a, const float* tile, int k, int row, const float (&factor)[4])
    {
        static_assert(PARTS == 3, "fp32 values are three parts");
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float* at = tile + (k + lane % 4 * 2 + i / 2 * 8) * ROW + row + lane / 4 + i % 2 * 8;
            split(at[0] * factor[i / 2 * 2], at[ROW] * factor[i / 2 * 2 + 1], a.part[0][i], a.part[1][i], a.part[2][i]);
        }
    }
    static __device__ __forceinline__ void store_two(float* at, float a, float b) { *reinterpret_cast<float2*>(at) = make_float2(a, b); }
};

// Products of parts, the smallest first; TILES tiles of 8 columns side by side, of which the first `tiles` are wanted.
template <int LEFT, int RIGHT, int TILES>
__device__ __forceinline__ void multiply_parts(float (&sum)[TILES][4], const Left<LEFT>& a, const Right<RIGHT> (&b)[TILES / 2], int tiles)
{
#pragma unroll
    for (int order = LEFT + RIGHT - 2; order >= 0; --order) {
        if (order > 2) continue;  // what these would add is below 2^-24 of the result
#pragma unroll
        for (int p = 0; p < LEFT; ++p) {
            const int q = order - p;
            if (q < 0 || q >= RIGHT) continue;
#pragma unroll
            for (int n = 0; n < TILES; ++n)
                if (n < tiles) multiply(sum[n], a.part[p], b[n / 2].part[q][n % 2][0], b[n / 2].part[q][n % 2][1]);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------ kernel
// MT: 64 columns of x and y each; WN: warps that share a chunk's 16 rows.  STATES: no output, only each segment's own sum.
template <typename T, int MT, int WN>
struct Shape {
    static constexpr int kThreads = 128 * WN, kTiles = 8 / WN;              // tiles of 8 columns of a warp
    static constexpr int kRowA = MT * 64 + Tile<T>::kPad, kRowB = kTile + Tile<T>::kPad;
    static constexpr int kStage = kC * (2 * kRowA + kRowB);                  // elements: x, y, z
    static constexpr int kBytes = (2 * kStage + MT * 64 * kRowB) * (int)sizeof(T) + (kC + 4) * 4;
};

template <typename T, int MT, int WN, int ALIGN, bool STATES>
__global__ void __launch_bounds__(Shape<T, MT, WN>::kThreads) rps_mix_kernel(const __grid_constant__ MixParams prm)
{
    after_the_kernel_before();
    using S = Shape<T, MT, WN>;
    constexpr int W = Slice<T>::kWidth, kParts = Tile<T>::kParts, kStateParts = 3, NT = S::kTiles;
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
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, wr = warp % 4, wn = warp / 4, g = lane / 4, t2 = lane % 4 * 2;
    const int cols = min(kTile, b - col0), tiles = max(0, min(NT, (cols + 7) / 8 - wn * NT));  // of this warp
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
            for (int u = threadIdx.x; u < kC * across; u += S::kThreads) {
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

    // W: rows 16 (wr + 4 m) + g and + 8, columns (wn NT + n) 8 + t2 and + 1
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
                const int row = (wr + 4 * m) * 16 + g + e / 2 * 8, col = col0 + (wn * NT + n) * 8 + t2 + e % 2;
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
                    Tile<T>::store_two(state + ((wr + 4 * m) * 16 + g + e / 2 * 8) * S::kRowB + (wn * NT + n) * 8 + t2, w[m][n][e], w[m][n][e + 1]);
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
                Left<kParts> left;
                Tile<T>::template left<S::kRowA>(left, tx, row0, k);
                Right<kParts> right[4];
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (2 * n < keys) Tile<T>::template right_across<S::kRowA>(right[n], ty, k, n * 16);
                multiply_parts<kParts, kParts, 8>(p, left, right, keys);
            }
            float out[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) out[n][e] = 0.0f;
            if (!zero) {
                for (int k = 0; k < a16; k += 16) {
                    Left<kParts> left;
                    Tile<T>::template left<S::kRowA>(left, tx, row0, k);
                    Right<kParts> right[NT / 2];
#pragma unroll
                    for (int n = 0; n < NT / 2; ++n)
                        if (2 * n < tiles) Tile<T>::template right<S::kRowB>(right[n], state, k, (wn * NT + 2 * n) * 8);
                    multiply_parts<kParts, kParts, NT>(out, left, right, tiles);
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
                Left<kParts> left;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t word[kParts];
                    split_pair<kParts>(p[2 * k + i / 2][i % 2 * 2], p[2 * k + i / 2][i % 2 * 2 + 1], word);
#pragma unroll
                    for (int q = 0; q < kParts; ++q) left.part[q][i] = word[q];
                }
                Right<kParts> right[NT / 2];
#pragma unroll
                for (int n = 0; n < NT / 2; ++n)
                    if (2 * n < tiles) Tile<T>::template right<S::kRowB>(right[n], tz, k * 16, (wn * NT + 2 * n) * 8);
                multiply_parts<kParts, kParts, NT>(out, left, right, tiles);
            }
            // out through this warp's rows of x, which have been read (by all warps that share them)
            if constexpr (WN > 1)
                asm volatile("bar.sync %0, %1;" ::"r"(1 + wr), "n"(32 * WN) : "memory");
            else
                __syncwarp();
            T* const own = tx + row0 * S::kRowA;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; e += 2) Tile<T>::store_two(own + (g + e / 2 * 8) * S::kRowA + (wn * NT + n) * 8 + t2, out[n][e], out[n][e + 1]);
            __syncwarp();
            constexpr int kAcross = NT * 8 / W, kDown = 32 / kAcross;
            const int c = wn * NT * 8 + lane % kAcross * W;
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
                Left<kStateParts> left;
                Tile<T>::template left_across<S::kRowA, kStateParts>(left, ty, k, (wr + 4 * m) * 16, factor);
                Right<kParts> right[NT / 2];
#pragma unroll
                for (int n = 0; n < NT / 2; ++n)
                    if (2 * n < tiles) Tile<T>::template right<S::kRowB>(right[n], tz, k, (wn * NT + 2 * n) * 8);
                multiply_parts<kStateParts, kParts, NT>(u, left, right, tiles);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[m][n][e] = fmaf(whole, w[m][n][e], u[n][e]);
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
                    const int row = (wr + 4 * m) * 16 + g + e / 2 * 8, col = col0 + (wn * NT + n) * 8 + t2 + e % 2;
                    if (row < a && col < b) to[row * to_a + col * to_b] = w[m][n][e];
                }
    }
    if constexpr (!STATES) {
        // rows behind the sequence's last token
        const int64_t t1 = min(prm.tokens, i0 + prm.segment_tokens);
        for (int64_t t = max(at.length, i0) + warp; t < t1; t += 4 * WN)
            for (int c = lane * W; c < cols; c += 32 * W)
                store_slice<T, ALIGN>(static_cast<T*>(term.out) + (((at.w * prm.sequences + at.sequence) * prm.tokens + t) * prm.heads + at.head) * b + col0, c, cols,
                                      make_uint4(0, 0, 0, 0));
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
    float w = term.state_in != nullptr ? __ldg(term.state_in + unit * term.a * term.b + row * term.state_a + col * term.state_b) : 0.0f;
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

// -------------------------------------------------------------------------------------------------------------- host
template <typename T, int MT, int WN, int ALIGN, bool STATES>
cudaError_t launch_kernel(const MixParams& prm, cudaStream_t stream)
{
    static LaunchState granted;
    using S = Shape<T, MT, WN>;
    const cudaError_t err = rps::grant_smem(granted, rps_mix_kernel<T, MT, WN, ALIGN, STATES>, S::kBytes);
    if (err != cudaSuccess) return err;
    return launch_after(rps_mix_kernel<T, MT, WN, ALIGN, STATES>, dim3((unsigned)(prm.units * prm.segments * prm.columns), (unsigned)prm.terms), S::kThreads, S::kBytes,
                        stream, 1, prm);
}

cudaError_t launch_join(const MixParams& prm, cudaStream_t stream)
{
    return launch_after(rps_mix_join_kernel, dim3((unsigned)(prm.units * prm.join_blocks), (unsigned)prm.terms), kJoinThreads, 0, stream, 1, prm);
}

template <typename T, int MT, int WN, int ALIGN>
cudaError_t run(const MixParams& prm, cudaStream_t stream)
{
    if (prm.segments > 1) {
        cudaError_t err = launch_kernel<T, MT, WN, ALIGN, true>(prm, stream);
        if (err == cudaSuccess) err = launch_join(prm, stream);
        if (err != cudaSuccess) return err;
    }
    return launch_kernel<T, MT, WN, ALIGN, false>(prm, stream);
}

template <typename T>
int operand_alignment(const MixOperand& o, int64_t cols)
{
    return std::min({alignment<T>(o.base, cols, o.token), alignment<T>(o.base, cols, o.head), alignment<T>(o.base, cols, o.sequence), alignment<T>(o.base, cols, o.worker)});
}

template <typename T, int WN>
cudaError_t mix(const MixParams& prm, cudaStream_t stream)
{
    int align = 16, widest = 0;
    for (int i = 0; i < prm.terms; ++i) {
        const MixTerm& t = prm.term[i];
        align = std::min({align, operand_alignment<T>(t.x, t.a), operand_alignment<T>(t.y, t.a), operand_alignment<T>(t.z, t.b), alignment<T>(t.out, t.b, t.b)});
        widest = std::max(widest, t.a);
    }
    if (widest <= 64) return align == 16 ? run<T, 1, WN, 16>(prm, stream) : align == 4 ? run<T, 1, WN, 4>(prm, stream) : run<T, 1, WN, sizeof(T)>(prm, stream);
    return align == 16 ? run<T, 2, WN, 16>(prm, stream) : align == 4 ? run<T, 2, WN, 4>(prm, stream) : run<T, 2, WN, sizeof(T)>(prm, stream);
}

}  // namespace

// Sequences are cut into as many segments as take the least time by this count of chunks of 128 tokens: a round of CTAs (one to an SM) takes its
// segment's chunks and one more to begin and end with; the segments' own sums, made first, 0.6 of a chunk each; joining them 3.
void plan_mix(MixParams* prm)
{
    MixParams& p = *prm;
    p.units = (int64_t)p.n * p.sequences * p.heads;
    p.columns = 1, p.state_room = 0;
    for (int i = 0; i < p.terms; ++i) {
        p.columns = std::max(p.columns, (int)ceil_div(p.term[i].b, kTile));
        p.state_room = std::max<int64_t>(p.state_room, round_up(p.term[i].a * p.term[i].b, 4));
    }
    p.join_blocks = (int)ceil_div(p.state_room, kJoinThreads);
    const int64_t chunks = std::max<int64_t>(1, ceil_div(p.tokens, kMixTensorChunk)), ctas = p.units * p.terms * (p.f32 ? p.columns : 1);
    int64_t best = 1;
    double least = 0.0;
    for (int64_t s = 1; s <= std::min<int64_t>(chunks, kMixSegments); ++s) {
        const int64_t each = ceil_div(chunks, s);
        if (s > 1 && (ceil_div(chunks, each) != s || ctas * s > 4 * kSms)) continue;
        const double cost = (double)ceil_div(ctas * s, kSms) * (double)(each + 1) + (s > 1 ? (double)ceil_div(ctas * (s - 1), kSms) * (0.6 * (double)each + 1.0) + 3.0 : 0.0);
        if (s == 1 || cost < least) best = s, least = cost;
    }
    p.segment_tokens = ceil_div(chunks, best) * kMixTensorChunk;
    p.segments = (int)best;
}

cudaError_t launch_mix(const MixParams& prm, cudaStream_t stream)
{
    if (prm.f32) return mix<float, 2>(prm, stream);
    if (!mix_fits_tensor(prm)) return mix<bf16, 1>(prm, stream);
    MixParams p = prm;
    p.tensor = 1;
    if (p.segments > 1) {
        cudaError_t err = launch_mix_tensor(p, true, stream);
        if (err == cudaSuccess) err = launch_join(p, stream);
        if (err != cudaSuccess) return err;
    }
    return launch_mix_tensor(p, false, stream);
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
