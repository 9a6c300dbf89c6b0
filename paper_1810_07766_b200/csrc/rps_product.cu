// Matrix products of the training operators on the tensor cores, with their epilogues.
//
// A pair of CTAs (a cluster of two, on neighbouring SMs) makes one 256 x 256 tile (or, product_shape, a CTA alone one of 128 x 256): each CTA stages 128 rows of A and half of B's 256
// columns, one thread of the first CTA issues the pair's tcgen05.mma, and each CTA's tensor memory holds its 128 rows of the
// result in fp32.  Tensor memory has room for two tiles, so the epilogue of one runs under the products of the next.  The
// pairs are persistent and take the tiles round robin.
//
// Roles in a CTA: warp 0 copies (TMA boxes of 64 columns, 128-byte swizzle, a ring of 6 to 24 stages), warp 1 issues the products
// (first CTA only) and owns the tensor memory, the others are the epilogue, a row to a lane, so that a row's softmax statistics need
// no exchange between lanes.  bf16 operands have 16 such warps of 64 columns, which work on 32 columns at a time straight out of tensor
// memory; fp32 operands 8 of 128 columns, held in registers while their segments (below) are added.  (With 8 warps of 128 columns
// in registers for bf16, too few to issue while another waits, a tile's end took 4.2 us where it is all there is, instead of 2.9.)
//
// Operands are read as they lie in memory: with the summed axis contiguous, or (dl and W in dH = dl W, dl and H in dW = dl^T H) with
// the other one contiguous, which the descriptors of the shared-memory tiles express; nothing is transposed.
//
// fp32 operands are three bf16 parts each (24 significant bits); of the nine products of parts six are made, and the others are below 2^-24 of
// the result (split_two).  The three parts of a block lie in three stages of the ring, so each is copied once for its three products.
#include <algorithm>
#include <atomic>
#include <mutex>
#include <type_traits>

#include "rps_cluster.cuh"
#include "rps_rows.cuh"

namespace rps_ops {
namespace {

using rps::mbar_arrive_expect_tx;
using rps::mbar_init;
using rps::smem_addr;

constexpr int kTileN = 256, kDepth = 64;  // columns of a tile at most, and of the summed axis at a time; 64 bf16 are one 128-byte swizzled line
constexpr int kOperandBytes = 128 * kDepth * 2;  // 128 rows of an operand in a stage
constexpr int kBoxBytes = 64 * kDepth * 2;       // 64 columns of an operand whose summed axis is not the contiguous one
constexpr int kRingBytes = 6 * 2 * kOperandBytes;
constexpr int kMostStages = 24;                  // of narrower tiles and fewer rows more stages fit
// Warps of the epilogue: two (fp32) or four (bf16) for each quarter of a CTA's 128 rows.
template <int PLANES>
struct Epilogue {
    static constexpr int kParts = PLANES == 3 ? 2 : 4;
    static constexpr int kWarps = 4 * kParts;
    // Warps 0 and 1 issue copies and products; with fp32 the epilogue's are groups of four, whose registers are shared out anew.
    static constexpr int kFirst = PLANES == 3 ? 4 : 2, kThreads = 32 * (kFirst + kWarps);
    static constexpr int kCols = kTileN / kParts;  // of a warp, at most
};
constexpr int kMostEpilogueWarps = Epilogue<1>::kWarps;
// Registers of a thread with fp32, whose 128 columns a row left too few of the 168 that all threads alike can have, and what is spilled is far
// away: nearly all of the SM's memory is shared memory here.  (The gradient above 219 -> 186 us, 3 of 5534 x 1020 32 -> 28.)
constexpr int kLaunchRegisters = 168, kIssueRegisters = 72, kEpilogueRegisters = 216;
static_assert(4 * kIssueRegisters + Epilogue<3>::kWarps * kEpilogueRegisters <= Epilogue<3>::kThreads / 32 * kLaunchRegisters, "the block's own");
// The tensor cores cut an fp32 sum off after each step of 16 instead of rounding it, a bias that grows with the number of steps
// (relative error of a 512-long sum of random terms: 5e-7).  Where fp32 accuracy is asked for, the summed axis goes
// through in segments whose sums the epilogue adds in fp32, rounded: every 2 blocks of fp32 operands (48 steps), and every 16 blocks (64
// steps) for the softmax statistics of bf16 operands.  Adding a segment takes the epilogue about 600 cycles under the 6144 or 8192
// cycles of the products of the next one.  (Segments of 4 blocks for dl, whose tiles' ends then hold the next products up less: 8 x 500
// x 10001 x 650 fp32 256 -> 238 us, errors of the gradients 6e-7 -> 9e-7; not taken.)
constexpr int kSegmentF32 = 2, kSegmentStatistics = 16;  // in blocks of kDepth
// bf16 results are rounded to 2^-9 of their size anyhow, but not after any number of steps: of a sum of terms of one sign each step cuts off 1e-7 of
// what it ends at (measured over 2^19 tokens: 3.2e-3 in one run, 1.3e-4 in runs of 2048 steps, which are these).
constexpr int kSegmentBf16 = 512;  // LONG: a kernel of its own, as the sums between segments take the registers of the others' epilogue

static_assert(kTileN == kVocabTile && kTokenTile % 256 == 0 && kTokenBlock == kDepth, "operands are padded to whole tiles");

// Rows leave through shared memory: a lane holds one row, and 32 lanes writing 16 bytes of 32 rows each would touch 32 lines at a time and
// half a sector of each.  Instead 64 bytes of each of the warp's 32 rows are laid down (parts of 16 bytes, exchanged by the row's
// number so that neither side has bank conflicts) and written out as 4 lanes to a row; rows that are not 16-byte aligned go out
// element by element, still in the order of memory.  (Gradient of 8 fp32 weights of 10001 x 650, rows of 2600 bytes: 453 -> 186 us.)
struct Staging {
    uint4 part[32][4];
};
struct StagingWithOffsets : Staging {  // fp32, whose 8 warps leave room for the rows' offsets; bf16 makes them anew from the rows' numbers
    int64_t at[32];
};

struct Control {
    union {
        Staging staging[kMostEpilogueWarps];
        StagingWithOffsets staging_f32[Epilogue<3>::kWarps];
    };
    uint64_t full[kMostStages], empty[kMostStages], sum_full[2], sum_empty[2];
    uint64_t statistics[4][4];  // kLse, of each quarter of the rows and four tiles in turn: the warps' parts are there
    uint32_t tensor_memory;
    int count[RPS_MAX_WORKERS];      // tokens of each worker that take part
    int start[RPS_MAX_WORKERS + 1];  // first tile of each worker
};

template <int PLANES>
__device__ __forceinline__ auto& staging_of(Control& control)
{
    if constexpr (PLANES == 3)
        return control.staging_f32;
    else
        return control.staging;
}

constexpr int kSharedBytes = 1024 + kRingBytes + (int)sizeof(Control);
// The products read 128 rows of A whatever part of them a stage holds; behind the last stage lies Control.
static_assert(sizeof(Control) >= kOperandBytes, "reads past the ring stay in shared memory");

// Set when a bounded wait gave up (rps_ops_check).
__device__ int g_gave_up = 0;

struct Maps {
    CUtensorMap a, b;
};

// ------------------------------------------------------------------------------------------------------ instructions
// The address of the first CTA's copy of a shared variable.
__device__ __forceinline__ uint32_t in_first_cta(uint32_t addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}

// Says that tensor memory has been read.  Relaxed: what has to come before it are the loads of tensor memory, which
// tcgen05.fence::before_thread_sync orders; a release would wait for the stores of the tile before as well (4.6 -> 4.2 us a tile of stores).
__device__ __forceinline__ void arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}


// One box into this CTA's shared memory; its bytes are counted on the first CTA's barrier.
template <int CTAS>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, int plane, int worker, uint32_t bar)
{
    if constexpr (CTAS == 2)
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, "
            "%5}], [%6];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(plane), "r"(worker), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(plane), "r"(worker), "r"(bar)
            : "memory");
}

// Descriptor of a shared-memory tile with the 128-byte swizzle: start address and two strides in units of 16 bytes, the constant 1 at
// bit 46, layout 2 (128-byte swizzle) at bit 61.  Summed axis contiguous: the stride at bit 32 leads from 8 rows to the next 8.
// Other axis contiguous: it leads from 8 steps of the summed axis to the next 8, and the one at bit 16 from one 64-wide box to the
// next.  The upper word is the same for all, and in the lower one tiles and their parts lie a constant apart.
constexpr uint32_t kDescriptorHigh = 1024 / 16 | 1u << 14 | 2u << 29;

__device__ __forceinline__ uint32_t descriptor_low(uint32_t addr, bool other) { return addr >> 4 | (uint32_t)(other ? kBoxBytes / 16 : 1) << 16; }

// fp32 sums of bf16 products, rows x tile_n.
__device__ __forceinline__ uint32_t instruction_descriptor(bool a_other, bool b_other, int rows, int tile_n)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | (a_other ? 1u : 0u) << 15 | (b_other ? 1u : 0u) << 16 | (uint32_t)(tile_n / 8) << 17 | (uint32_t)(rows / 16) << 24;
}

// `a`, `b`: lower words of the descriptors.
template <int CTAS>
__device__ __forceinline__ void multiply(uint32_t sum, uint32_t a, uint32_t b, uint32_t descriptor, bool add)
{
    if constexpr (CTAS == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(sum),
            "r"(a), "r"(b), "n"(kDescriptorHigh), "r"(descriptor), "r"((uint32_t)add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(sum),
            "r"(a), "r"(b), "n"(kDescriptorHigh), "r"(descriptor), "r"((uint32_t)add)
            : "memory");
}

// Arrives on the barrier at this offset (in both CTAs of a pair) once the products issued so far are done.
template <int CTAS>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (CTAS == 2)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// All 512 columns of tensor memory, for the whole kernel.
template <int CTAS>
__device__ __forceinline__ void take_tensor_memory(uint32_t address_to)
{
    if constexpr (CTAS == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(address_to) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(address_to) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}

template <int CTAS>
__device__ __forceinline__ void free_tensor_memory(uint32_t address)
{
    if constexpr (CTAS == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(address) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(address) : "memory");
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

// COLS columns of this lane's row: taken over, or added to those of the segments before.  (Of a narrower tile the last ones are whatever
// tensor memory holds; they are not stored.)
template <int COLS>
__device__ __forceinline__ void take_sums(float (&v)[COLS], uint32_t addr, bool add, int width)
{
    __syncwarp();
    if (!add) {
#pragma unroll
        for (int c = 0; c < COLS; c += 16) load_sums(v + c, addr + c);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        return;
    }
#pragma unroll
    for (int c = 0; c < COLS; c += 16) {
        if (c >= width) break;
        float r[16];
        load_sums(r, addr + c);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
        for (int j = 0; j < 16; ++j) v[c + j] += r[j];
    }
}

// --------------------------------------------------------------------------------------------------------- epilogues
__device__ __forceinline__ void store_element(float* to, float e) { __stcg(to, e); }
__device__ __forceinline__ void store_element(bf16* to, bf16 e) { __stcg(reinterpret_cast<unsigned short*>(to), __bfloat16_as_ushort(e)); }

// Where a warp's rows go: lane's row `index` (-1: not written) of rows `stride` apart, from `out` on, which is this warp's first column.
template <typename T>
struct Rows {
    T* out;
    int stride;
    int index;
    int cols;   // that exist
    bool wide;  // rows are 16-byte aligned
    int top;    // kDweight: the warp's first row, the others follow it
    int rows;   // of them that exist
};

// Offset of row r of the warp, -1 if it is not written; all lanes ask.
template <typename T>
__device__ __forceinline__ int64_t row_offset(const Staging&, const Rows<T>& to, int r)
{
    const int index = __shfl_sync(0xFFFFFFFFu, to.index, r);
    return index < 0 ? -1 : (int64_t)index * to.stride;
}
template <typename T>
__device__ __forceinline__ int64_t row_offset(const StagingWithOffsets& stage, const Rows<T>&, int r)
{
    return stage.at[r];
}
template <typename T>
__device__ __forceinline__ void set_offsets(Staging&, const Rows<T>&)
{
}
template <typename T>
__device__ __forceinline__ void set_offsets(StagingWithOffsets& stage, const Rows<T>& to)
{
    __syncwarp();
    stage.at[threadIdx.x % 32] = to.index < 0 ? -1 : (int64_t)to.index * to.stride;
}

// 64 bytes of each of the warp's rows, from column `c` on.  Loads come before stores, several at a time.  ADD, WHOLE, RUN: see store_rows.
template <bool ADD, bool WHOLE, bool RUN, typename T, typename Stage>
__device__ __forceinline__ void store_chunk(Stage& stage, const uint4 (&mine)[4], const Rows<T>& to, int c)
{
    constexpr int kChunk = 64 / sizeof(T), kPart = 16 / sizeof(T);  // columns
    const int lane = threadIdx.x % 32;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 4; ++q) stage.part[lane][q ^ (lane >> 1 & 3)] = mine[q];
    __syncwarp();
    if (WHOLE || to.wide) {
        const int col = c + lane % 4 * kPart;
        uint4 word[4];
        int64_t row[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = lane / 4 + 8 * i;
            word[i] = stage.part[r][lane % 4 ^ (r >> 1 & 3)];
            row[i] = row_offset(stage, to, r);
        }
        if (col >= to.cols) return;
        if constexpr (ADD) {
            float4 old[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) old[i] = row[i] < 0 ? make_float4(0, 0, 0, 0) : __ldcg(reinterpret_cast<const float4*>(to.out + row[i] + col));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                word[i] = make_uint4(__float_as_uint(__uint_as_float(word[i].x) + old[i].x), __float_as_uint(__uint_as_float(word[i].y) + old[i].y),
                                     __float_as_uint(__uint_as_float(word[i].z) + old[i].z), __float_as_uint(__uint_as_float(word[i].w) + old[i].w));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (row[i] < 0) continue;
            T* at = to.out + row[i] + col;
            if (WHOLE || col + kPart <= to.cols) {
                __stcg(reinterpret_cast<uint4*>(at), word[i]);
            } else {
                const T* e = reinterpret_cast<const T*>(&word[i]);
#pragma unroll
                for (int k = 0; k < kPart; ++k)
                    if (col + k < to.cols) store_element(at + k, e[k]);
            }
        }
    } else {
        // an element to a lane, rows kRows at a time (2 of fp32, 1 of bf16)
        constexpr int kRows = 32 / kChunk, kAtATime = 8;
        const int col = lane % kChunk, below = lane / kChunk;
        const bool there = c + col < to.cols;
        if constexpr (RUN) {
            T* at = to.out + (int64_t)(to.top + below) * to.stride + c + col;
#pragma unroll 1
            for (int r0 = 0; r0 < 32; r0 += kRows * kAtATime) {
                T e[kAtATime];
#pragma unroll
                for (int i = 0; i < kAtATime; ++i) {
                    const int r = r0 + i * kRows + below;
                    e[i] = reinterpret_cast<const T*>(&stage.part[r][col / kPart ^ (r >> 1 & 3)])[col % kPart];
                }
#pragma unroll
                for (int i = 0; i < kAtATime; ++i, at += (int64_t)kRows * to.stride)
                    if (r0 + i * kRows + below < to.rows && there) store_element(at, e[i]);
            }
        } else {
#pragma unroll 1
            for (int r0 = 0; r0 < 32; r0 += kRows * kAtATime) {
                T e[kAtATime];
                int64_t row[kAtATime];
#pragma unroll
                for (int i = 0; i < kAtATime; ++i) {
                    const int r = r0 + i * kRows + below;
                    row[i] = row_offset(stage, to, r);
                    e[i] = reinterpret_cast<const T*>(&stage.part[r][col / kPart ^ (r >> 1 & 3)])[col % kPart];
                }
#pragma unroll
                for (int i = 0; i < kAtATime; ++i)
                    if (row[i] >= 0 && there) store_element(to.out + row[i] + c + col, e[i]);
            }
        }
    }
}

// The warp's rows.  WHOLE: they are 16-byte aligned and `cols` a multiple of 16 bytes.  ADD: to what is there (fp32, WHOLE).  RUN: they follow
// one another from to.top on, so that a row's place needs no looking up (3 bf16 gradients of 5534 x 2047: 52 -> 33 us).
template <bool ADD, bool WHOLE, bool RUN, typename T, int COLS, typename Stage>
__device__ __forceinline__ void store_rows(Stage& stage, const float (&v)[COLS], const Rows<T>& to)
{
    constexpr int kChunk = 64 / sizeof(T), kPart = 16 / sizeof(T);
    if (WHOLE || !RUN || to.wide) set_offsets(stage, to);
#pragma unroll
    for (int c = 0; c < COLS; c += kChunk) {
        if (c >= to.cols) break;
        uint4 mine[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float* f = v + c + q * kPart;
            if constexpr (sizeof(T) == 4)
                mine[q] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            else
                mine[q] = make_uint4(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7]));
        }
        store_chunk<ADD, WHOLE, RUN>(stage, mine, to, c);
    }
}

// fp32 values as three planes of bf16 parts, as split_two makes them but for infinities (of an infinite dloss alone), whose first parts are the largest
// number: what they are summed into is infinite or NaN.
template <int COLS, typename Stage>
__device__ __forceinline__ void store_parts(Stage& stage, float (&v)[COLS], Rows<bf16> to, int64_t plane)
{
    set_offsets(stage, to);
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
        if (c >= to.cols) break;
        Rows<bf16> part_to = to;
#pragma unroll
        for (int q = 0; q < 3; ++q, part_to.out += plane) {
            uint4 mine[4];
            uint32_t* word = reinterpret_cast<uint32_t*>(mine);
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                float &f0 = v[c + j], &f1 = v[c + j + 1];
                if (q < 2) {
                    word[j / 2] = nearest_two_bf16(f0, f1);
                    f0 -= __uint_as_float(word[j / 2] << 16), f1 -= __uint_as_float(word[j / 2] & 0xFFFF0000u);
                } else {
                    word[j / 2] = two_bf16(f0, f1);
                }
            }
            store_chunk<false, true, false>(stage, mine, part_to, c);
        }
    }
}

// What the epilogue needs to know of a row, read while the products are still on their way.
struct RowInfo {
    int target;   // kLse, kDlogits: less the first column of this warp
    float2 info;  // kDlogits: lse and g
    int index;    // of the row where it is stored, -1 if it is not
    float scale;
};

template <Product WHICH>
__device__ __forceinline__ RowInfo row_info(const ProductParams& prm, int w, int row, int n0, int count)
{
    RowInfo r{};
    const bool in = row < (WHICH == Product::kDweight ? prm.m : count);
    if constexpr (WHICH == Product::kLse || WHICH == Product::kDlogits) {
        r.target = in ? __ldg(prm.target + w * prm.tokens_padded + row) - prm.v0 - n0 : -1;
        if (WHICH == Product::kDlogits && in) r.info = __ldg(prm.info + w * prm.tokens_padded + row);
        // the product with dl over the tokens reads whole blocks of them: zeros behind the last one
        r.index = row < (count + kDepth - 1) / kDepth * kDepth ? row : -1;
    } else {
        r.index = !in ? -1 : WHICH == Product::kDhidden && prm.parts == nullptr ? __ldg(prm.rows + w * prm.tokens + row) : row;
        r.scale = prm.scale != nullptr ? __ldg(prm.scale + w) : 1.0f;
    }
    return r;
}

// kLse: a warp's columns of one row of a tile, `width` of them.  `turn`: tiles that the warp has had.  False if a wait gave up.
template <int PLANES, int COLS>
__device__ __forceinline__ bool statistics(const ProductParams& prm, int w, int row, int n0, int width, int count, const RowInfo& info, float (&v)[COLS],
                                           Control& control, int quarter, int part, int turn, uint64_t limit_ns)
{
    constexpr int kParts = Epilogue<PLANES>::kParts;
    const int cols = min(width, prm.n - n0);
    // in runs of 32 columns, as a narrow tile has fewer
    const int t = info.target;
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
        if (c >= cols) break;
        if (cols - c < 32) {
#pragma unroll
            for (int j = c; j < c + 32; ++j)
                if (j >= cols) v[j] = -INFINITY;
        }
#pragma unroll
        for (int j = c; j < c + 32; ++j) top = fmaxf(top, v[j]);
    }
    const float at = top == -INFINITY ? 0.0f : top;
    Pair total(0.0f);
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
        if (c >= cols) break;
        if (t >= c && t < min(c + 32, cols)) {
            float hit = 0.0f;
#pragma unroll
            for (int j = c; j < c + 32; ++j)
                if (j == t) hit = v[j];
            prm.hit[w * prm.tokens_padded + row] = hit;
        }
#pragma unroll
        for (int j = c; j < c + 32; j += 2) total = total + exp_of_difference(Pair(v[j], v[j + 1]), at);
    }
    sum = total.sum();
    // The warps of these rows put theirs together.  There is room for four tiles' in turn, as none of them can be more than two tiles
    // ahead of another: tensor memory holds two.
    static_assert(sizeof(control.staging) >= 4 * kParts * 128 * sizeof(float2), "unused here otherwise");
    float2* row_statistics = reinterpret_cast<float2*>(control.staging) + (turn & 3) * kParts * 128;
    const uint32_t there = smem_addr(&control.statistics[quarter][turn & 3]);
    const int lane = threadIdx.x % 32, r = quarter * 32 + lane;
    row_statistics[part * 128 + r] = make_float2(top, sum);
    __syncwarp();
    if (lane == 0) rps::mbar_arrive(there);
    if (part != 0) return true;
    if (!__all_sync(0xFFFFFFFFu, wait_for(there, turn >> 2 & 1, limit_ns))) return false;
    if (row >= count) return true;
    for (int k = 1; k < kParts; ++k) {
        const float2 p = row_statistics[k * 128 + r];
        const float m = fmaxf(top, p.x), from = m == -INFINITY ? 0.0f : m;
        sum = fmaf(sum, exp_of_difference(top, from), p.y * exp_of_difference(p.x, from));
        top = m;
    }
    prm.part[((int64_t)w * prm.stat_tiles + (prm.v0 + n0) / prm.tile_cols) * prm.tokens_padded + row] = make_float2(top, sum);
    return true;
}

// The other products: columns n0.. of one row of a tile, `width` (at most COLS) of them.
template <Product WHICH, int PLANES, int COLS, typename Stage>
__device__ __forceinline__ void store_columns(const ProductParams& prm, int w, int split, int row, int n0, int width, int count, int target,
                                              const RowInfo& info, float (&v)[COLS], bool wide, Stage& stage)
{
    const int cols = min(width, prm.n - n0);
    if constexpr (WHICH == Product::kDlogits) {
        const bool in = row < count;
#pragma unroll
        for (int c = 0; c < COLS; c += 32) {
            if (c >= width) break;
#pragma unroll
            for (int j = c; j < c + 32; ++j) {
                const float p = exp_of_difference(v[j], info.info.x) - (j == target ? 1.0f : 0.0f);
                v[j] = in && j < cols ? info.info.y * p : 0.0f;
            }
        }
        const int64_t plane = prm.tokens_padded * prm.piece;
        const Rows<bf16> to{prm.dl + w * PLANES * plane + n0, (int)prm.piece, info.index, width, true, 0, 0};
        if constexpr (PLANES == 1)
            store_rows<false, true, false>(stage, v, to);
        else
            store_parts(stage, v, to, plane);
    } else {
        if (cols <= 0) return;
        if (prm.parts != nullptr) {
            const Rows<float> to{prm.parts + ((int64_t)split * prm.workers + w) * prm.part_rows * prm.part_row + n0, (int)prm.part_row, info.index, width,
                                 true, 0, 0};
            if (prm.add)
                store_rows<true, true, false>(stage, v, to);
            else
                store_rows<false, true, false>(stage, v, to);
            return;
        }
#pragma unroll
        for (int j = 0; j < COLS; ++j) v[j] *= info.scale;
        using T = std::conditional_t<PLANES == 3, float, bf16>;
        const int top = row - (int)(threadIdx.x % 32);
        store_rows<false, false, WHICH == Product::kDweight>(
            stage, v, Rows<T>{static_cast<T*>(prm.out) + w * prm.out_worker + n0, (int)prm.out_row, info.index, cols, wide, top, min(32, prm.m - top)});
    }
}

// ------------------------------------------------------------------------------------------------------------ kernel
template <Product WHICH, int PLANES, int CTAS, bool LONG>
__global__ void __launch_bounds__(Epilogue<PLANES>::kThreads, 1)
    rps_product_kernel(const __grid_constant__ ProductParams prm, const __grid_constant__ Maps maps)
{
    constexpr bool kAOther = WHICH == Product::kDweight;                                  // A's rows are contiguous, not the summed axis
    constexpr bool kBOther = WHICH == Product::kDweight || WHICH == Product::kDhidden;
    constexpr bool kRowsFirst = WHICH != Product::kDweight;                               // order of the tiles: see below
    constexpr int kRows = 128 * CTAS;  // of a tile
    extern __shared__ unsigned char raw[];
    const uint32_t base = (smem_addr(raw) + 1023) / 1024 * 1024;
    unsigned char* const ring = raw + (base - smem_addr(raw));
    Control& control = *reinterpret_cast<Control*>(ring + kRingBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = CTAS == 2 ? cluster_rank() : 0;

    if (warp == 0 && lane == 0) {
        for (int s = 0; s < kMostStages; ++s) {
            mbar_init(smem_addr(&control.full[s]), 1);
            mbar_init(smem_addr(&control.empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_addr(&control.sum_full[s]), 1);
            mbar_init(smem_addr(&control.sum_empty[s]), CTAS * Epilogue<PLANES>::kWarps);
        }
        for (int s = 0; s < 16; ++s) mbar_init(smem_addr(&control.statistics[s / 4][s % 4]), Epilogue<PLANES>::kParts);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) take_tensor_memory<CTAS>(smem_addr(&control.tensor_memory));
    if (warp == 0 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b) : "memory");
    }
    const int tile_n = prm.tile_cols, own_n = tile_n / CTAS;  // columns of B that a CTA copies
    const int n_tiles = (prm.n + tile_n - 1) / tile_n;
    const uint32_t a_bytes = prm.a_rows * kDepth * 2, b_bytes = kBOther ? (own_n + 63) / 64 * (kBoxBytes) : own_n * kDepth * 2;
    const int stages = min(kMostStages, (int)(kRingBytes / (a_bytes + b_bytes)));
    after_the_kernel_before();
    if (warp == 2) {
        // tiles of each worker (a lane to a worker): where the tokens are rows, only those that hold a token that takes part
        int total = 0;
        for (int w0 = 0; w0 < prm.workers; w0 += 32) {
            const int w = w0 + lane;
            int count = 0, tiles = 0;
            if (w < prm.workers) {
                count = prm.count != nullptr ? __ldg(prm.count + w) : (WHICH == Product::kDweight ? prm.k : prm.m);
                tiles = ((WHICH == Product::kDweight ? prm.m : count) + kRows - 1) / kRows * n_tiles;
                control.count[w] = count;
            }
            int upto = tiles;
#pragma unroll
            for (int s = 1; s < 32; s *= 2) {
                const int n = __shfl_up_sync(0xFFFFFFFFu, upto, s);
                if (lane >= s) upto += n;
            }
            if (w < prm.workers) control.start[w + 1] = total + upto;
            total += __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
        if (lane == 0) control.start[0] = 0;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CTAS == 2) cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tensor_memory = control.tensor_memory;

    const int tiles = control.start[prm.workers], groups = gridDim.x / CTAS, total = tiles * prm.splits;
    struct Tile {
        int w, split, m0, n0, count, first, blocks;  // blocks of the summed axis: the first one and how many
    };
    const auto tile_at = [&](int item) {
        Tile t;
        t.split = item / tiles;
        int tile = item - t.split * tiles;
        t.w = 0;
        while (tile >= control.start[t.w + 1]) ++t.w;
        tile -= control.start[t.w];
        const int m_tiles = (control.start[t.w + 1] - control.start[t.w]) / n_tiles;
        // kLse, kDlogits: all rows of a column of tiles before the next one, so that the weight is read from memory once; kDweight: all
        // columns of a row of tiles, for dl's sake
        const int m = kRowsFirst ? tile % m_tiles : tile / n_tiles, n = kRowsFirst ? tile / m_tiles : tile % n_tiles;
        t.m0 = m * kRows, t.n0 = n * tile_n;
        t.count = control.count[t.w];
        const int k = WHICH == Product::kDweight ? t.count : prm.k;
        const int depth = (k + kDepth - 1) / kDepth, run = (depth + prm.splits - 1) / prm.splits;
        t.first = t.split * run;
        t.blocks = max(0, min(depth - t.first, run));
        return t;
    };
    // blocks to a segment
    const int segment = PLANES == 3 ? kSegmentF32 : WHICH == Product::kLse ? kSegmentStatistics : LONG ? kSegmentBf16 : 1 << 30;
    bool fine = true;
    const uint64_t limit_ns = prm.wait_limit_ms > 0 ? (uint64_t)prm.wait_limit_ms * 1000000u : rps::kDefaultWaitLimitNs;
    const auto wait = [&](uint32_t bar, uint32_t parity) { return wait_for(bar, parity, limit_ns); };

    if (warp < Epilogue<PLANES>::kFirst) {
        if constexpr (PLANES == 3) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegisters));
        if (warp == 0) {
            if (lane == 0) {
                int stage = 0, issued = 0;
                uint32_t phase = 0;
                for (int tile = blockIdx.x / CTAS; tile < total && fine; tile += groups) {
                    const Tile t = tile_at(tile);
                    const int m0 = t.m0 + rank * 128, n0 = t.n0 + rank * own_n;
                    const int wa = prm.a.worker != 0 ? t.w : 0, wb = prm.b.worker != 0 ? t.w : 0;
                    // a CTA's part that holds no row or column of the result is not copied: what the products read in its place reaches
                    // only results that are not stored
                    const int rows = WHICH == Product::kDweight ? prm.m : t.count;
                    const bool copy_a = m0 < rows, copy_b = n0 < prm.n;
                    const uint32_t bytes = (CTAS == 2 && t.m0 + 128 < rows ? 2 : 1) * a_bytes + (CTAS == 2 && t.n0 + own_n < prm.n ? 2 : 1) * b_bytes;
                    for (int i = 0; i < t.blocks * PLANES && prm.withhold_copies == 0; ++i) {
                        fine = wait(smem_addr(&control.empty[stage]), phase ^ 1);
                        if (!fine) break;
                        const int kb = PLANES == 1 ? i : i / 3, plane = i - kb * PLANES, k0 = (t.first + kb) * kDepth;
                        const uint32_t bar = in_first_cta(smem_addr(&control.full[stage]));
                        if (rank == 0) mbar_arrive_expect_tx(smem_addr(&control.full[stage]), bytes);
                        const uint32_t a = base + stage * (a_bytes + b_bytes), b = a + a_bytes;
                        if (copy_a) {
                            if (kAOther) {
                                load_box<CTAS>(a, &maps.a, m0, k0, plane, wa, bar);
                                load_box<CTAS>(a + kBoxBytes, &maps.a, m0 + 64, k0, plane, wa, bar);
                            } else {
                                load_box<CTAS>(a, &maps.a, k0, m0, plane, wa, bar);
                            }
                        }
                        if (copy_b) {
                            if (kBOther) {
                                for (int c = 0; c < own_n; c += 64) load_box<CTAS>(b + c / 64 * kBoxBytes, &maps.b, n0 + c, k0, plane, wb, bar);
                            } else {
                                load_box<CTAS>(b, &maps.b, k0, n0, plane, wb, bar);
                            }
                        }
                        ++issued;
                        if (++stage == stages) stage = 0, phase ^= 1;
                    }
                }
                if (fine) {
                    // the pair's arrivals on this CTA's barriers: all have come before it may end
                    for (int i = 0; i < stages && fine; ++i) {
                        fine = wait(smem_addr(&control.empty[stage]), phase ^ 1);
                        if (++stage == stages) stage = 0, phase ^= 1;
                    }
                } else if (rank == 0) {
                    // copies still on their way when a wait gave up: those of the last round of the ring at most
                    for (int i = issued > stages ? issued - stages : 0; i < issued; ++i)
                        wait(smem_addr(&control.full[i % stages]), i / stages & 1);
                }
            }
        } else if (warp == 1) {
            if (rank == 0 && lane == 0) {
                const uint32_t descriptor = instruction_descriptor(kAOther, kBOther, kRows, tile_n);
                // one product covers 16 of the summed axis: 32 bytes further along swizzled rows, or 16 rows of 128 bytes further
                constexpr uint32_t a_step = (kAOther ? 2048 : 32) / 16, b_step = (kBOther ? 2048 : 32) / 16;
                const uint32_t a_first = descriptor_low(base, kAOther), b_first = descriptor_low(base + a_bytes, kBOther), stage_step = (a_bytes + b_bytes) / 16;
                int stage = 0, made = 0;
                uint32_t phase = 0;
                for (int tile = blockIdx.x / CTAS; tile < total && fine; tile += groups) {
                    const Tile t = tile_at(tile);
                    for (int kb = 0; kb < t.blocks && fine;) {
                        const int buffer = made & 1, begin = kb, end = min(kb + segment, t.blocks);
                        fine = wait(smem_addr(&control.sum_empty[buffer]), (made >> 1 & 1) ^ 1);
                        if (!fine) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t sum = tensor_memory + buffer * kTileN;
                        const auto block = [&](uint32_t a, uint32_t b, bool add) {
#pragma unroll
                            for (int k = 0; k < kDepth / 16; ++k) multiply<CTAS>(sum, a + k * a_step, b + k * b_step, descriptor, add || k > 0);
                        };
                        for (; kb < end; ++kb) {
                            uint32_t a[PLANES], b[PLANES], freed[PLANES];
#pragma unroll
                            for (int q = 0; q < PLANES; ++q) {
                                fine = fine && wait(smem_addr(&control.full[stage]), phase);
                                a[q] = a_first + stage * stage_step, b[q] = b_first + stage * stage_step, freed[q] = smem_addr(&control.empty[stage]);
                                if (++stage == stages) stage = 0, phase ^= 1;
                            }
                            if (!fine) break;
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                            if constexpr (PLANES == 1) {
                                block(a[0], b[0], kb > begin);
                            } else {  // parts of A and B, the smallest products first, and a stage given back as soon as it has had its last
                                block(a[2], b[0], kb > begin);
                                block(a[0], b[2], true);
                                commit<CTAS>(freed[2]);
                                block(a[1], b[1], true);
                                block(a[1], b[0], true);
                                block(a[0], b[1], true);
                                commit<CTAS>(freed[1]);
                                block(a[0], b[0], true);
                            }
                            commit<CTAS>(freed[0]);
                        }
                        if (!fine) break;
                        commit<CTAS>(smem_addr(&control.sum_full[buffer]));
                        ++made;
                    }
                }
            }
        }
    } else {
        if constexpr (PLANES == 3) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEpilogueRegisters));
        constexpr int kCols = Epilogue<PLANES>::kCols;
        const int quarter = warp % 4, part = (warp - Epilogue<PLANES>::kFirst) / 4, part_n = tile_n / Epilogue<PLANES>::kParts;
        const bool wide = (reinterpret_cast<uintptr_t>(prm.out) | (prm.out_row | prm.out_worker) * (PLANES == 3 ? 4 : 2)) % 16 == 0;
        int made = 0, turn = 0;
        const auto summed = [&] {
            fine = __all_sync(0xFFFFFFFFu, wait(smem_addr(&control.sum_full[made & 1]), made >> 1 & 1));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            return fine;
        };
        const auto taken = [&] {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) arrive_cluster(in_first_cta(smem_addr(&control.sum_empty[made & 1])));
            ++made;
        };
        for (int tile = blockIdx.x / CTAS; tile < total && fine; tile += groups) {
            const Tile t = tile_at(tile);
            const int row = t.m0 + (int)rank * 128 + quarter * 32 + lane, n0 = t.n0 + part * part_n;
            const RowInfo info = row_info<WHICH>(prm, t.w, row, n0, t.count);
            // a warp none of whose rows is wanted only keeps step
            const bool idle = t.m0 + (int)rank * 128 + quarter * 32 >= (WHICH == Product::kDweight ? prm.m : WHICH == Product::kDlogits ? (t.count + kDepth - 1) / kDepth * kDepth : t.count);
            const uint32_t columns = tensor_memory + ((uint32_t)(quarter * 32) << 16) + part * part_n;
            auto& staging = staging_of<PLANES>(control)[warp - Epilogue<PLANES>::kFirst];
            if constexpr (PLANES == 1 && WHICH != Product::kLse && !LONG) {  // one segment
                if (t.blocks > 0 && !summed()) break;
#pragma unroll 1
                for (int c = 0; c < part_n && !idle; c += 32) {
                    float v[32];
                    if (t.blocks > 0) {
                        take_sums(v, columns + (made & 1) * kTileN + c, false, 32);
                        if (c + 32 >= part_n) taken();
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0.0f;
                    }
                    store_columns<WHICH, PLANES>(prm, t.w, t.split, row, n0 + c, min(32, part_n - c), t.count, info.target - c, info, v, wide, staging);
                }
                if (t.blocks > 0 && idle) taken();
            } else {
                float v[kCols];
                if (t.blocks == 0) {
#pragma unroll
                    for (int j = 0; j < kCols; ++j) v[j] = 0.0f;
                }
                for (int kb = 0; kb < t.blocks; kb = min(kb + segment, t.blocks)) {
                    if (!summed()) break;
                    if (!idle) take_sums(v, columns + (made & 1) * kTileN, kb > 0, part_n);
                    taken();
                }
                if (!fine) break;
                if (idle) continue;
                if constexpr (WHICH == Product::kLse)
                    fine = statistics<PLANES>(prm, t.w, row, n0, part_n, t.count, info, v, control, quarter, part, turn++, limit_ns);
                else
                    store_columns<WHICH, PLANES>(prm, t.w, t.split, row, n0, part_n, t.count, info.target, info, v, wide, staging);
            }
        }
    }
    if (!fine && lane == 0) atomicExch(&g_gave_up, 1);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CTAS == 2) cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    __syncwarp();
    if (warp == 1) free_tensor_memory<CTAS>(tensor_memory);
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

// Whether the kernel was compiled to the registers that its epilogue shares out anew: it would wait for ever for those that a smaller launch does not have.
// `known` keeps the number once it has been asked for; a question that fails is asked again.
template <typename Kernel>
cudaError_t check_registers(std::atomic<int>& known, Kernel kernel)
{
    int registers = known.load(std::memory_order_relaxed);
    if (registers == 0) {
        cudaFuncAttributes attributes{};
        const cudaError_t err = cudaFuncGetAttributes(&attributes, kernel);
        if (err != cudaSuccess) return err;
        known.store(registers = attributes.numRegs, std::memory_order_relaxed);
    }
    return registers == kLaunchRegisters ? cudaSuccess : cudaErrorInvalidKernelImage;
}

template <Product WHICH, int PLANES, int CTAS, bool LONG>
cudaError_t launch(const ProductParams& prm, cudaStream_t stream)
{
    static rps::LaunchState state;
    cudaError_t err = rps::grant_smem(state, rps_product_kernel<WHICH, PLANES, CTAS, LONG>, kSharedBytes);
    if (err != cudaSuccess) return err;
    if constexpr (PLANES == 3) {
        static std::atomic<int> registers{0};
        if ((err = check_registers(registers, rps_product_kernel<WHICH, PLANES, CTAS, LONG>)) != cudaSuccess) return err;
    }
    int sms = 0;
    if ((err = sm_count(&sms)) != cudaSuccess) return err;
    Maps maps{};
    constexpr bool a_other = WHICH == Product::kDweight, b_other = WHICH == Product::kDweight || WHICH == Product::kDhidden;
    ProductParams p = prm;
    if (p.splits < 1) p.splits = 1;
    p.a_rows = a_other || p.m > 128 ? 128 : (int)round_up(p.m, 8);
    if (p.k == 0) {  // nothing is read: the kernel writes zeros
        p.count = nullptr;
    } else if (!encode_operand(&maps.a, p.a, p.planes, p.workers, a_other ? 64 : p.a_rows) || !encode_operand(&maps.b, p.b, p.planes, p.workers, b_other ? 64 : p.tile_cols / CTAS)) {
        return cudaErrorInvalidValue;
    }
    const int64_t tiles = ceil_div(p.m, 128 * CTAS) * ceil_div(p.n, p.tile_cols) * p.workers * p.splits;
    const int groups = (int)(tiles < sms / CTAS ? tiles : sms / CTAS);
    return launch_after(rps_product_kernel<WHICH, PLANES, CTAS, LONG>, dim3(CTAS * groups), Epilogue<PLANES>::kThreads, kSharedBytes, stream, CTAS, p, maps);
}

template <Product WHICH, int PLANES>
cudaError_t launch_pairs_or_not(const ProductParams& prm, cudaStream_t stream)
{
    if constexpr (PLANES == 1 && WHICH != Product::kLse) {  // the others have segments in any case
        const int64_t run = ceil_div(ceil_div(prm.k, kDepth), std::max(prm.splits, 1));
        if (run > kSegmentBf16) return prm.ctas == 2 ? launch<WHICH, PLANES, 2, true>(prm, stream) : launch<WHICH, PLANES, 1, true>(prm, stream);
    }
    return prm.ctas == 2 ? launch<WHICH, PLANES, 2, false>(prm, stream) : launch<WHICH, PLANES, 1, false>(prm, stream);
}

}  // namespace

// Pairs of CTAs share B's copies, but a tile of theirs has 256 rows: where its second half would be empty (up to 128 rows), a CTA alone
// makes one.  (4 workers of 42 tokens, 1314 words, 2530 columns fp32: dl W 57 us in pairs, 32 alone.  1024 tokens, 32768 words, 768
// columns fp32: logits 174 us in pairs, 255 alone; 8 workers of 375 tokens, whose last pair of three halves is half empty: 206 and 263.)
//
// A product with fewer tiles than there are pairs (or CTAs) and a long summed axis is cut along it, so that all work.  In
// microseconds: a block takes 0.27 (the six products of parts of fp32: 1.6) and a tile's end 1; a part written and read 0.1 (0.05 of a
// single CTA), the launch that joins them 5.  (48 tiles of 157 fp32 blocks: 312 us whole, 222 + 10 in three runs.  From 74 tiles on
// cutting only evens the last round out, and the board's power, not the idle pairs, bounds it: 120 tiles of 1024 bf16
// blocks took 745 us whole, 740 + 15 in three.)
//
// The tiles' columns are a multiple of 32: as few as their number allows (650 columns are three of 224 instead of 256); and up to two
// rounds so few that rounds x time of a tile is least.  Half of a tile's time is A's, whose copies are the same for any width (a
// quarter of fp32's, where each copy has three products), and half B's.  So 76 tiles of 192 become 114 of 128 (two workers' 1048 x 4735 x 345 fp32: 65 -> 49 us), and a
// small call's tiles so narrow that every place has one.  (Of many rounds the widest are best: 8192 x 8192 x 2048 bf16 in 4 rounds of
// 256 columns 184 us, in 5 of 192 246 us.)  (4 workers of 32 tokens, 1000 words, 256 columns: the four products of a step 39 us with tiles of 256, 32 us with 128 and 64.)
double block_time(int planes, int ctas, double tile)
{
    if (planes == 1) return 0.27 * (0.5 + 0.5 * tile / kTileN);
    if (ctas == 2) return std::max(1.05, 0.45 + 0.0047 * tile);
    return tile <= 128 ? std::max(1.03, 0.86 + 0.0027 * tile) : 0.0133 * tile;
}

ProductShape product_shape(int64_t m, int64_t n, int64_t k, int workers, int planes, bool may_split)
{
    const int64_t halves = ceil_div(m > 0 ? m : 1, 128), whole = ceil_div(halves, 2);
    const int ctas = halves == 1 ? 1 : 2;
    const int64_t places = kSms / ctas, others = (ctas == 1 ? halves : whole) * workers, blocks = ceil_div(k, kDepth);
    const int64_t fewest = ceil_div(n, kTileN);
    ProductShape best{};
    double least = 0.0;
    const auto consider = [&](int64_t across) {
        const int64_t tile = round_up(ceil_div(n, across), 32), tiles = ceil_div(n, tile) * others;
        const double part = (double)tile / kTileN, block = block_time(planes, ctas, (double)tile);
        for (int s = 1; s <= 32 && (s == 1 || (may_split && tiles < places && s * 4 <= blocks)); ++s) {
            const double cost = (double)ceil_div(tiles * s, places) * ((double)ceil_div(blocks, s) * block + part + 0.5) +
                                (s > 1 ? 5.0 + 0.05 * ctas * part * (double)(tiles * s) : 0.0);
            if (best.ctas == 0 || cost < least) best = {(int)tile, s, ctas}, least = cost;
        }
    };
    // whole tiles, halves of them, up to eight more in a row, and one for every place
    consider(fewest);
    if (fewest * others <= 2 * places) {
        for (int64_t a = fewest + 1; a < fewest + 8; ++a) consider(a);
        consider(std::max(fewest, std::min(places / others, n / 32)));
    }
    if (planes == 3 && ctas == 1) consider(2 * fewest);
    return best;
}

namespace {

// Parts of a product added up, scaled and rounded into the result, four columns to a lane.  A warp to a row, the parts in their order;
// TOGETHER (8 parts and more): the eight warps of a CTA share 128 columns of a row, each adding its parts in their order before they
// join (32 parts of 5 rows of 2048: 33 -> 3.6 us).
template <typename T, bool HIDDEN, bool TOGETHER>
__global__ void __launch_bounds__(256) rps_join_kernel(const ProductParams prm)
{
    after_the_kernel_before();
    __shared__ float4 sums[TOGETHER ? 8 : 1][32];
    const int w = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t row = TOGETHER ? blockIdx.x : (int64_t)blockIdx.x * 8 + warp;
    if (row >= (HIDDEN ? (int64_t)prm.count[w] : (int64_t)prm.m)) return;
    const float g = prm.scale != nullptr ? prm.scale[w] : 1.0f;
    T* out = static_cast<T*>(prm.out) + w * prm.out_worker + (HIDDEN ? (int64_t)prm.rows[w * prm.tokens + row] : row) * prm.out_row;
    const float* part = prm.parts + (w * prm.part_rows + row) * prm.part_row;
    const int64_t next = prm.workers * prm.part_rows * prm.part_row;
    const bool wide = (reinterpret_cast<uintptr_t>(out) / sizeof(T)) % 4 == 0;
    for (int c = lane * 4 + (int)blockIdx.z * 128; TOGETHER || c < prm.n; c += 128 * gridDim.z) {
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (c < prm.n) {
#pragma unroll 8
            for (int k = TOGETHER ? warp : 0; k < prm.splits; k += TOGETHER ? 8 : 1) {
                const float4 p = __ldcs(reinterpret_cast<const float4*>(part + k * next + c));
                s.x += p.x, s.y += p.y, s.z += p.z, s.w += p.w;
            }
        }
        if constexpr (TOGETHER) {
            sums[warp][lane] = s;
            __syncthreads();
            if (warp != 0 || c >= prm.n) return;
#pragma unroll
            for (int k = 1; k < 8; ++k) {
                const float4 p = sums[k][lane];
                s.x += p.x, s.y += p.y, s.z += p.z, s.w += p.w;
            }
        }
        const T e[4] = {from_float<T>(s.x * g), from_float<T>(s.y * g), from_float<T>(s.z * g), from_float<T>(s.w * g)};
        if (wide && c + 4 <= prm.n) {
            if constexpr (sizeof(T) == 4)
                *reinterpret_cast<float4*>(out + c) = make_float4(e[0], e[1], e[2], e[3]);
            else
                *reinterpret_cast<uint2*>(out + c) = make_uint2(two_bf16(s.x * g, s.y * g), two_bf16(s.z * g, s.w * g));
        } else {
            for (int k = 0; k < 4; ++k)
                if (c + k < prm.n) out[c + k] = e[k];
        }
        if constexpr (TOGETHER) return;
    }
}

template <typename T, bool HIDDEN>
cudaError_t join(const ProductParams& prm, cudaStream_t stream)
{
    const int64_t rows = ceil_div(prm.m, 8), across = std::min<int64_t>(ceil_div(prm.n, 128), 65535);
    if (prm.splits >= 8 && across * 128 >= prm.n)
        return launch_after(rps_join_kernel<T, HIDDEN, true>, dim3((unsigned)prm.m, (unsigned)prm.workers, (unsigned)across), 256, 0, stream, 1, prm);
    const int64_t along = std::max<int64_t>(1, std::min(across, kSms * 8 / (rows * prm.workers)));  // few rows share their columns out (182 of 2253: 30 -> 5 us)
    return launch_after(rps_join_kernel<T, HIDDEN, false>, dim3((unsigned)rows, (unsigned)prm.workers, (unsigned)along), 256, 0, stream, 1, prm);
}

}  // namespace

cudaError_t launch_join(Product which, const ProductParams& prm, cudaStream_t stream)
{
    const bool hidden = which == Product::kDhidden;
    if (prm.planes == 3) return hidden ? join<float, true>(prm, stream) : join<float, false>(prm, stream);
    return hidden ? join<bf16, true>(prm, stream) : join<bf16, false>(prm, stream);
}

cudaError_t launch_product(Product which, const ProductParams& prm, cudaStream_t stream)
{
    const bool f32 = prm.planes == 3;
    switch (which) {
        case Product::kLse: return f32 ? launch_pairs_or_not<Product::kLse, 3>(prm, stream) : launch_pairs_or_not<Product::kLse, 1>(prm, stream);
        case Product::kDlogits: return f32 ? launch_pairs_or_not<Product::kDlogits, 3>(prm, stream) : launch_pairs_or_not<Product::kDlogits, 1>(prm, stream);
        case Product::kDhidden: return f32 ? launch_pairs_or_not<Product::kDhidden, 3>(prm, stream) : launch_pairs_or_not<Product::kDhidden, 1>(prm, stream);
        default: return f32 ? launch_pairs_or_not<Product::kDweight, 3>(prm, stream) : launch_pairs_or_not<Product::kDweight, 1>(prm, stream);
    }
}

cudaError_t read_gave_up(int* value, cudaStream_t stream) { return read_and_clear(g_gave_up, value, stream); }

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
