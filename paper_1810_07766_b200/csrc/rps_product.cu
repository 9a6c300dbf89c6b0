// Matrix products of the training operators on the tensor cores, with their epilogues.
//
// A pair of CTAs (a cluster of two, on neighbouring SMs) makes one 256 x 256 tile: each CTA stages 128 rows of A and half of B's 256
// columns, one thread of the first CTA issues the pair's tcgen05.mma, and each CTA's tensor memory holds its 128 rows of the
// result in fp32.  Tensor memory has room for two tiles, so the epilogue of one runs under the products of the next.  The
// pairs are persistent and take the tiles round robin.
//
// Roles in a CTA: warp 0 copies (TMA boxes of 64 columns, 128-byte swizzle, a ring of kStages), warp 1 issues the products
// (first CTA only) and owns the tensor memory, warps 2..9 are the epilogue: two for each quarter of the 128 rows, each with
// half of the columns, a row to a lane, so that a row's softmax statistics need no exchange between lanes.
//
// Operands are read as they lie in memory: with the summed axis contiguous, or (dl and W in dH = dl W, dl and H in dW = dl^T H) with
// the other one contiguous, which the descriptors of the shared-memory tiles express; nothing is transposed.
//
// fp32 operands are three bf16 parts each (24 significant bits); of the nine products of parts the six that reach 2^-24
// of the result are made, the smallest first, into the same accumulator.
#include <mutex>

#include "rps_ops_kernels.h"
#include "rps_tma.cuh"

namespace rps_ops {
namespace {

using rps::mbar_arrive_expect_tx;
using rps::mbar_init;
using rps::smem_addr;

constexpr int kTileM = 256, kTileN = 256, kDepth = 64;  // of a pair; 64 bf16 are one 128-byte swizzled line
constexpr int kHalf = kTileN / 2;  // columns of a warp of the epilogue
constexpr int kStages = 6;
constexpr int kOperandBytes = 128 * kDepth * 2;  // one operand's part of a stage in one CTA
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 32 * (2 + kEpilogueWarps);
// The tensor cores cut an fp32 sum off after each step of 16 instead of rounding it, a bias that grows with the number of steps
// (relative error of a 512-long sum of random terms: 5e-7).  Where fp32 accuracy is asked for, the summed axis goes
// through in segments whose sums the epilogue adds in fp32, rounded: every 512 of fp32 operands' leading parts, and every 1024 for
// the softmax statistics of bf16 operands.  An extra segment costs the epilogue about 600 cycles under at least 4096 of products.
constexpr int kSegmentF32 = 8, kSegmentStatistics = 16;  // in blocks of kDepth
constexpr uint64_t kWaitNs = 2000000000ull;

static_assert(kTileM == kTokenTile && kTileN == kVocabTile, "operands are padded to whole tiles");

// Rows leave through shared memory: a lane holds one row, and 32 lanes writing 16 bytes of 32 rows each would touch 32 lines at a time and
// half a sector of each.  Instead 64 bytes of each of the warp's 32 rows are laid down (parts of 16 bytes, exchanged by the row's
// number so that neither side has bank conflicts) and written out as 4 lanes to a row; rows that are not 16-byte aligned go out
// element by element, still in the order of memory.  (Gradient of 8 fp32 weights of 10001 x 650, rows of 2600 bytes: 453 -> XXX us.)
struct Staging {
    uint4 part[32][4];
    int64_t at[32];
};

struct Control {
    Staging staging[kEpilogueWarps];
    uint64_t full[kStages], empty[kStages], sum_full[2], sum_empty[2];
    uint32_t tensor_memory;
    int start[RPS_MAX_WORKERS + 1];  // first tile of each worker
};

constexpr int kSharedBytes = 1024 + kStages * kStageBytes + (int)sizeof(Control);

// Set when a bounded wait gave up (rps_ops_check).
__device__ int g_gave_up = 0;

struct Maps {
    CUtensorMap a, b;
};

// ------------------------------------------------------------------------------------------------------ instructions
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive;\n\tbarrier.cluster.wait;" ::: "memory");
}

// The address of the first CTA's copy of a shared variable.
__device__ __forceinline__ uint32_t in_first_cta(uint32_t addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}

__device__ __forceinline__ void arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Waits for the phase with the given parity; what the pair did before it is then visible.  Gives up after kWaitNs.
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity), "r"(rps::kSuspendHintNs)
        : "memory");
    return done != 0;
}

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity)
{
    if (try_wait(bar, parity)) return true;
    const uint64_t start = rps::global_timer_ns();
#pragma unroll 1
    while (!try_wait(bar, parity))
        if (rps::global_timer_ns() - start > kWaitNs) return false;
    return true;
}

// One box into this CTA's shared memory; its bytes are counted on the first CTA's barrier.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, int plane, int worker, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, "
        "%5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(plane), "r"(worker), "r"(bar)
        : "memory");
}

// Descriptor of a shared-memory tile with the 128-byte swizzle: start address and the two strides in units of 16 bytes, the
// constant 1 at bit 46, layout 2 (128-byte swizzle) at bit 61.  Summed axis contiguous: `stride` leads from 8 rows to the
// next 8.  Other axis contiguous: `stride` leads from 8 steps of the summed axis to the next 8, `lead` from one 64-wide box to the next.
__device__ __forceinline__ uint64_t tile_descriptor(uint32_t addr, uint32_t lead, uint32_t stride)
{
    return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)((lead >> 4) & 0x3FFF) << 16 | (uint64_t)((stride >> 4) & 0x3FFF) << 32 | 1ull << 46 |
           2ull << 61;
}

// fp32 sums of bf16 products, 256 x 256 over the pair.
__host__ __device__ constexpr uint32_t instruction_descriptor(bool a_other, bool b_other)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | (a_other ? 1u : 0u) << 15 | (b_other ? 1u : 0u) << 16 | (uint32_t)(kTileN / 8) << 17 |
           (uint32_t)(kTileM / 16) << 24;
}

__device__ __forceinline__ void multiply(uint32_t sum, uint64_t a, uint64_t b, uint32_t descriptor, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(sum),
        "l"(a), "l"(b), "r"(descriptor), "r"((uint32_t)add)
        : "memory");
}

// Arrives on the barrier at this offset in both CTAs once the products issued so far are done.
__device__ __forceinline__ void commit_to_pair(uint32_t bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
        : "memory");
}

// 16 columns of this lane's row.
__device__ __forceinline__ void load_sums(float* v, uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
          "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(addr)
        : "memory");
}

// 128 columns of this lane's row: taken over, or added to those of the segments before.
__device__ __forceinline__ void take_sums(float (&v)[kHalf], uint32_t addr, bool add)
{
    __syncwarp();
    if (!add) {
#pragma unroll
        for (int c = 0; c < kHalf; c += 16) load_sums(v + c, addr + c);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        return;
    }
#pragma unroll
    for (int c = 0; c < kHalf; c += 16) {
        float r[16];
        load_sums(r, addr + c);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
        for (int j = 0; j < 16; ++j) v[c + j] += r[j];
    }
}

// --------------------------------------------------------------------------------------------------------- epilogues
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t two_bf16(float lo, float hi)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// Part q of an fp32 value.
__device__ __forceinline__ float part_of(float v, int q)
{
    const float lead = leading_bits(v), rest = rest_of(v, lead), mid = leading_bits(rest);
    return q == 0 ? lead : q == 1 ? mid : rest - mid;
}

// `at`: offset of this lane's row in `out`, or -1 if it is not to be written; `cols` of the 128 columns exist.  ADD: to what is there
// (fp32, wide).  PART: not the values but that part of them.
template <bool ADD, bool PART, typename T>
__device__ __forceinline__ void store_rows(Staging& stage, const float (&v)[kHalf], T* out, int64_t at, int cols, bool wide, int part = 0)
{
    constexpr int kChunk = 64 / sizeof(T), kPart = 16 / sizeof(T);  // columns
    const int lane = threadIdx.x % 32;
    __syncwarp();
    stage.at[lane] = at;
#pragma unroll
    for (int c = 0; c < kHalf / kChunk; ++c) {
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float* f = v + c * kChunk + q * kPart;
            uint4 word;
            if constexpr (sizeof(T) == 4)
                word = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            else
                word = PART ? make_uint4(two_bf16(part_of(f[0], part), part_of(f[1], part)), two_bf16(part_of(f[2], part), part_of(f[3], part)),
                                         two_bf16(part_of(f[4], part), part_of(f[5], part)), two_bf16(part_of(f[6], part), part_of(f[7], part)))
                            : make_uint4(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7]));
            stage.part[lane][q ^ (lane >> 1 & 3)] = word;
        }
        __syncwarp();
        if (wide) {
            const int col = c * kChunk + lane % 4 * kPart;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = lane / 4 + 8 * i;
                uint4 word = stage.part[r][lane % 4 ^ (r >> 1 & 3)];
                const int64_t row_at = stage.at[r];
                T* to = out + row_at + col;
                if (row_at < 0 || col >= cols) continue;
                if constexpr (ADD) {
                    const float4 old = *reinterpret_cast<const float4*>(to);
                    word = make_uint4(__float_as_uint(__uint_as_float(word.x) + old.x), __float_as_uint(__uint_as_float(word.y) + old.y),
                                      __float_as_uint(__uint_as_float(word.z) + old.z), __float_as_uint(__uint_as_float(word.w) + old.w));
                }
                if (col + kPart <= cols) {
                    *reinterpret_cast<uint4*>(to) = word;
                } else {
                    const T* e = reinterpret_cast<const T*>(&word);
#pragma unroll
                    for (int k = 0; k < kPart; ++k)
                        if (col + k < cols) to[k] = e[k];
                }
            }
        } else {
            constexpr int kRows = 32 / kChunk;  // rows that the warp writes at a time, an element to a lane: 2 of fp32, 1 of bf16
            const int col = lane % kChunk;
#pragma unroll 4
            for (int r0 = 0; r0 < 32; r0 += kRows) {
                const int r = r0 + lane / kChunk;
                const int64_t to = stage.at[r];
                const T e = reinterpret_cast<const T*>(&stage.part[r][col / kPart ^ (r >> 1 & 3)])[col % kPart];
                if (to >= 0 && c * kChunk + col < cols) out[to + c * kChunk + col] = e;
            }
        }
    }
}

// One row's 128 columns of a tile.
template <Product WHICH>
__device__ __forceinline__ void epilogue(const ProductParams& prm, int w, int row, int n0, int count, float (&v)[kHalf], bool wide, Staging& stage)
{
    const int cols = prm.n - n0;
    if (cols <= 0 && WHICH != Product::kDlogits) return;
    if constexpr (WHICH == Product::kLse) {
        if (row >= count) return;
        if (cols < kHalf) {
#pragma unroll
            for (int j = 0; j < kHalf; ++j)
                if (j >= cols) v[j] = -INFINITY;
        }
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kHalf; ++j) top = fmaxf(top, v[j]);
        const float at = top == -INFINITY ? 0.0f : top * kLog2e;
        const int t = prm.target[w * prm.tokens_padded + row] - prm.v0 - n0;
        if (t >= 0 && t < kHalf) {
            float hit = 0.0f;
#pragma unroll
            for (int j = 0; j < kHalf; ++j)
                if (j == t) hit = v[j];
            prm.hit[w * prm.tokens_padded + row] = hit;
        }
#pragma unroll
        for (int j = 0; j < kHalf; ++j) sum += exp2_fast(fmaf(v[j], kLog2e, -at));
        prm.part[((int64_t)w * prm.stat_tiles + (prm.v0 + n0) / kStatCols) * prm.tokens_padded + row] = make_float2(top, sum);
    } else if constexpr (WHICH == Product::kDlogits) {
        const bool in = row < count;
        const float2 info = in ? prm.info[w * prm.tokens_padded + row] : make_float2(0.0f, 0.0f);
        const int t = in ? prm.target[w * prm.tokens_padded + row] - prm.v0 - n0 : -1;
        const int64_t at_dl = ((int64_t)w * prm.planes * prm.tokens_padded + row) * prm.piece + n0;
        const float at = info.x * kLog2e;
#pragma unroll
        for (int j = 0; j < kHalf; ++j) {
            const float p = exp2_fast(fmaf(v[j], kLog2e, -at)) - (j == t ? 1.0f : 0.0f);
            v[j] = in && j < cols ? info.y * p : 0.0f;
        }
        if (prm.planes == 1) {
            store_rows<false, false>(stage, v, prm.dl, at_dl, kHalf, true);
        } else {
#pragma unroll 1
            for (int q = 0; q < 3; ++q) store_rows<false, true>(stage, v, prm.dl + q * prm.tokens_padded * prm.piece, at_dl, kHalf, true, q);
        }
    } else {
        constexpr bool kHidden = WHICH == Product::kDhidden;
        const bool in = row < (kHidden ? count : prm.m);
        if constexpr (kHidden) {
            const int64_t at = in ? (w * prm.tokens_padded + row) * prm.acc_row + n0 : -1;
            if (!prm.last) {
                if (prm.first)
                    store_rows<false, false>(stage, v, prm.acc, at, kHalf, true);
                else
                    store_rows<true, false>(stage, v, prm.acc, at, kHalf, true);
                return;
            }
            if (!prm.first && in) {
                const float* acc = prm.acc + at;
#pragma unroll
                for (int j = 0; j < kHalf; j += 4) {
                    const float4 a = *reinterpret_cast<const float4*>(acc + j);
                    v[j] += a.x, v[j + 1] += a.y, v[j + 2] += a.z, v[j + 3] += a.w;
                }
            }
        }
        const float g = prm.scale != nullptr ? prm.scale[w] : 1.0f;
        const int64_t at = !in ? -1 : w * prm.out_worker + (kHidden ? (int64_t)prm.rows[w * prm.tokens + row] : (int64_t)(prm.v0 + row)) * prm.out_row + n0;
#pragma unroll
        for (int j = 0; j < kHalf; ++j) v[j] *= g;
        if (prm.out_f32)
            store_rows<false, false>(stage, v, static_cast<float*>(prm.out), at, cols, wide);
        else
            store_rows<false, false>(stage, v, static_cast<bf16*>(prm.out), at, cols, wide);
    }
}

// ------------------------------------------------------------------------------------------------------------ kernel
template <Product WHICH>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    rps_product_kernel(const __grid_constant__ ProductParams prm, const __grid_constant__ Maps maps)
{
    constexpr bool kAOther = WHICH == Product::kDweight;                                  // A's rows are contiguous, not the summed axis
    constexpr bool kBOther = WHICH == Product::kDweight || WHICH == Product::kDhidden;
    constexpr bool kRowsFirst = WHICH != Product::kDweight;                               // order of the tiles: see below
    extern __shared__ unsigned char raw[];
    const uint32_t base = (smem_addr(raw) + 1023) / 1024 * 1024;
    unsigned char* const stages = raw + (base - smem_addr(raw));
    Control& control = *reinterpret_cast<Control*>(stages + kStages * kStageBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();

    if (warp == 0 && lane == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&control.full[s]), 1);
            mbar_init(smem_addr(&control.empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_addr(&control.sum_full[s]), 1);
            mbar_init(smem_addr(&control.sum_empty[s]), 2 * kEpilogueWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&control.tensor_memory)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    const int n_tiles = (prm.n + kTileN - 1) / kTileN;
    if (warp == 2) {
        // tiles of each worker: where the tokens are rows, only those that hold a token that takes part
        int total = 0;
        for (int w = 0; w < prm.workers; ++w) {
            const int rows = WHICH != Product::kDweight && prm.count != nullptr ? prm.count[w] : prm.m;
            if (lane == 0) control.start[w] = total;
            total += (rows + kTileM - 1) / kTileM * n_tiles;
        }
        if (lane == 0) control.start[prm.workers] = total;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tensor_memory = control.tensor_memory;

    const int total = control.start[prm.workers], pairs = gridDim.x / 2;
    struct Tile {
        int w, m0, n0, blocks, count, first_segment;  // blocks up to the end of the first segment
    };
    const int segment = prm.planes == 3 ? kSegmentF32 : WHICH == Product::kLse ? kSegmentStatistics : 0;  // 0: one segment
    int worker = 0;
    const auto tile_at = [&](int tile) {
        while (tile >= control.start[worker + 1]) ++worker;
        Tile t;
        t.w = worker;
        tile -= control.start[worker];
        const int m_tiles = (control.start[worker + 1] - control.start[worker]) / n_tiles;
        // kLse, kDlogits: all rows of a column of tiles before the next one, so that the weight is read from memory once; kDweight: all
        // columns of a row of tiles, for dl's sake
        const int m = kRowsFirst ? tile % m_tiles : tile / n_tiles, n = kRowsFirst ? tile / m_tiles : tile % n_tiles;
        t.m0 = m * kTileM, t.n0 = n * kTileN;
        t.count = prm.count != nullptr ? prm.count[worker] : (WHICH == Product::kDweight ? prm.k : prm.m);
        const int k = WHICH == Product::kDweight ? t.count : prm.k;
        const int depth = (k + kDepth - 1) / kDepth;
        t.blocks = depth * (prm.planes == 1 ? 1 : 6);
        // of fp32 operands the five products that are small against the sixth are one segment with its beginning
        t.first_segment = segment == 0 ? t.blocks : min(t.blocks, segment + (prm.planes == 1 ? 0 : 5 * depth));
        return t;
    };
    bool fine = true;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0, issued = 0;
            uint32_t phase = 0;
            for (int tile = blockIdx.x / 2; tile < total && fine; tile += pairs) {
                const Tile t = tile_at(tile);
                const int depth = prm.planes == 1 ? t.blocks : t.blocks / 6;
                const int m0 = t.m0 + rank * 128, n0 = t.n0 + rank * 128;
                const int wa = prm.a.worker != 0 ? t.w : 0, wb = prm.b.worker != 0 ? t.w : 0;
                for (int kb = 0; kb < t.blocks; ++kb) {
                    fine = wait(smem_addr(&control.empty[stage]), phase ^ 1);
                    if (!fine) break;
                    const int product = kb / depth, k0 = (kb - product * depth) * kDepth;
                    // parts of A and B: (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
                    const int pa = prm.planes == 1 ? 0 : (0x001012 >> (4 * product)) & 3;
                    const int pb = prm.planes == 1 ? 0 : (0x010210 >> (4 * product)) & 3;
                    const uint32_t bar = in_first_cta(smem_addr(&control.full[stage]));
                    if (rank == 0) mbar_arrive_expect_tx(smem_addr(&control.full[stage]), 2 * kStageBytes);
                    const uint32_t a = base + stage * kStageBytes, b = a + kOperandBytes;
                    if (kAOther) {
                        load_box(a, &maps.a, m0, k0, pa, wa, bar);
                        load_box(a + kOperandBytes / 2, &maps.a, m0 + 64, k0, pa, wa, bar);
                    } else {
                        load_box(a, &maps.a, k0, m0, pa, wa, bar);
                    }
                    if (kBOther) {
                        load_box(b, &maps.b, n0, k0, pb, wb, bar);
                        load_box(b + kOperandBytes / 2, &maps.b, n0 + 64, k0, pb, wb, bar);
                    } else {
                        load_box(b, &maps.b, k0, n0, pb, wb, bar);
                    }
                    ++issued;
                    if (++stage == kStages) stage = 0, phase ^= 1;
                }
            }
            if (fine) {
                // the pair's arrivals on this CTA's barriers: all have come before it may end
                for (int i = 0; i < kStages && fine; ++i) {
                    fine = wait(smem_addr(&control.empty[stage]), phase ^ 1);
                    if (++stage == kStages) stage = 0, phase ^= 1;
                }
            } else if (rank == 0) {
                // copies still on their way when a wait gave up: the last kStages of them at most
                for (int i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
                    wait(smem_addr(&control.full[i % kStages]), i / kStages & 1);
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            constexpr uint32_t descriptor = instruction_descriptor(kAOther, kBOther);
            // one product covers 16 of the summed axis: 32 bytes further along swizzled rows, or 16 rows of 128 bytes further
            constexpr uint32_t a_step = kAOther ? 2048 : 32, b_step = kBOther ? 2048 : 32;
            int stage = 0, made = 0;
            uint32_t phase = 0;
            for (int tile = blockIdx.x / 2; tile < total && fine; tile += pairs) {
                const Tile t = tile_at(tile);
                int end = t.first_segment;
                for (int kb = 0; kb < t.blocks && fine; end = min(end + segment, t.blocks)) {
                    const int buffer = made & 1, begin = kb;
                    fine = wait(smem_addr(&control.sum_empty[buffer]), (made >> 1 & 1) ^ 1);
                    if (!fine) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    for (; kb < end; ++kb) {
                        fine = wait(smem_addr(&control.full[stage]), phase);
                        if (!fine) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t a = base + stage * kStageBytes, b = a + kOperandBytes;
#pragma unroll
                        for (int k = 0; k < kDepth / 16; ++k)
                            multiply(tensor_memory + buffer * kTileN, tile_descriptor(a + k * a_step, kAOther ? kOperandBytes / 2 : 16, 1024),
                                     tile_descriptor(b + k * b_step, kBOther ? kOperandBytes / 2 : 16, 1024), descriptor, kb > begin || k > 0);
                        commit_to_pair(smem_addr(&control.empty[stage]));
                        if (++stage == kStages) stage = 0, phase ^= 1;
                    }
                    if (!fine) break;
                    commit_to_pair(smem_addr(&control.sum_full[buffer]));
                    ++made;
                }
            }
        }
    } else {
        const int quarter = warp % 4, half = (warp - 2) / 4;
        const bool wide = (reinterpret_cast<uintptr_t>(prm.out) | (prm.out_row | prm.out_worker) * (prm.out_f32 ? 4 : 2)) % 16 == 0;
        int made = 0;
        for (int tile = blockIdx.x / 2; tile < total && fine; tile += pairs) {
            const Tile t = tile_at(tile);
            float v[kHalf];
            if (t.blocks == 0) {
#pragma unroll
                for (int j = 0; j < kHalf; ++j) v[j] = 0.0f;
            }
            int end = t.first_segment;
            for (int kb = 0; kb < t.blocks; kb = end, end = min(end + segment, t.blocks)) {
                const int buffer = made & 1;
                fine = __all_sync(0xFFFFFFFFu, wait(smem_addr(&control.sum_full[buffer]), made >> 1 & 1));
                if (!fine) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                take_sums(v, tensor_memory + ((uint32_t)(quarter * 32) << 16) + buffer * kTileN + half * kHalf, kb > 0);
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_cluster(in_first_cta(smem_addr(&control.sum_empty[buffer])));
                ++made;
            }
            if (!fine) break;
            epilogue<WHICH>(prm, t.w, t.m0 + (int)rank * 128 + quarter * 32 + lane, t.n0 + half * kHalf, t.count, v, wide, control.staging[warp - 2]);
        }
    }
    if (!fine && lane == 0) atomicExch(&g_gave_up, 1);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    __syncwarp();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tensor_memory) : "memory");
}

// ------------------------------------------------------------------------------------------------------------- host
// Boxes of 64 contiguous columns and box_rows rows of one plane of one worker.
bool encode_operand(CUtensorMap* map, const Operand& o, int planes, int workers, int box_rows)
{
    rps::EncodeTiledFn encode = rps::encode_tiled_fn();
    if (encode == nullptr) return false;
    const cuuint64_t row = (cuuint64_t)o.row * 2;
    // an axis of one element takes any stride
    const cuuint64_t plane = planes > 1 ? (cuuint64_t)o.plane * 2 : row, worker = o.worker != 0 ? (cuuint64_t)o.worker * 2 : plane;
    const cuuint64_t dims[4] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)planes, (cuuint64_t)(o.worker != 0 ? workers : 1)};
    const cuuint64_t strides[3] = {row, plane, worker};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1}, steps[4] = {1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<bf16*>(o.base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <Product WHICH>
cudaError_t launch(const ProductParams& prm, cudaStream_t stream)
{
    static rps::LaunchState state;
    cudaError_t err = rps::grant_smem(state, rps_product_kernel<WHICH>, kSharedBytes);
    if (err != cudaSuccess) return err;
    int sms = 0;
    if ((err = sm_count(&sms)) != cudaSuccess) return err;
    Maps maps{};
    constexpr bool a_other = WHICH == Product::kDweight, b_other = WHICH == Product::kDweight || WHICH == Product::kDhidden;
    ProductParams p = prm;
    if (p.k == 0) {  // nothing is read: the kernel writes zeros
        p.count = nullptr;
    } else if (!encode_operand(&maps.a, p.a, p.planes, p.workers, a_other ? 64 : 128) || !encode_operand(&maps.b, p.b, p.planes, p.workers, b_other ? 64 : 128)) {
        return cudaErrorInvalidValue;
    }
    const int64_t tiles = ceil_div(p.m, kTileM) * ceil_div(p.n, kTileN) * p.workers;
    const int pairs = (int)(tiles < sms / 2 ? tiles : sms / 2);
    rps_product_kernel<WHICH><<<2 * pairs, kThreads, kSharedBytes, stream>>>(p, maps);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_product(Product which, const ProductParams& prm, cudaStream_t stream)
{
    switch (which) {
        case Product::kLse: return launch<Product::kLse>(prm, stream);
        case Product::kDlogits: return launch<Product::kDlogits>(prm, stream);
        case Product::kDhidden: return launch<Product::kDhidden>(prm, stream);
        default: return launch<Product::kDweight>(prm, stream);
    }
}

cudaError_t read_gave_up(int* value, cudaStream_t stream)
{
    const int zero = 0;
    cudaError_t err = cudaMemcpyFromSymbolAsync(value, g_gave_up, sizeof(int), 0, cudaMemcpyDeviceToHost, stream);
    if (err == cudaSuccess) err = cudaStreamSynchronize(stream);
    if (err == cudaSuccess && *value != 0) err = cudaMemcpyToSymbolAsync(g_gave_up, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, stream);
    if (err == cudaSuccess) err = cudaStreamSynchronize(stream);
    return err;
}

cudaError_t sm_count(int* out)
{
    static std::mutex lock;
    static int counts[rps::kMaxDevices] = {};
    int dev = 0;
    cudaError_t err = rps::current_device(&dev);
    if (err != cudaSuccess) return err;
    std::lock_guard<std::mutex> hold(lock);
    if (counts[dev] == 0 && (err = cudaDeviceGetAttribute(&counts[dev], cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return err;
    *out = counts[dev];
    return cudaSuccess;
}

}  // namespace rps_ops
