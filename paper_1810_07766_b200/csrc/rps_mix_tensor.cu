// Linear attention's form (rps_mix.cu) on the fifth-generation tensor cores, for bf16 operands that TMA can copy: 16-byte aligned, columns in eights.
//
// A CTA takes a segment of a sequence's head in chunks of 128 tokens, rows l in the order of memory whichever way time runs; with the masked decays D,
//
//   P = x y^T,  O = (P o D) z + r^e (x W),  U = (r^f y)^T z,  W' = r^c W + U
//
// are four tcgen05 products of 128 rows, whose sums lie in tensor memory side by side.  The chunks end with the sequence's last token, so it
// is the first one that may begin ahead of the sequence; TMA fills zeros there, and never reads past the last token that takes part.
//
// Roles (groups of four warps): warp 0 copies y and z of the next chunk (and x, once x W has been made) while this one is worked on, warp 1 issues the
// products, warp 2 sends out away, warp 3 brings W's first value; eight (a lane to a row, half of the columns) turn P into
// the masked product, which goes back to tensor memory as the left operand of the next one, and lay O down in shared memory; sixteen make r^f y
// in parts and hold W as fp32 in registers (a lane to a row of W, a quarter of the columns), which they bring up to date out of U and lay down as bf16
// for the next chunk; the first of them sends its last value away.  With up to 64 columns of y and z (OWN) all the parts have places of their own, and twice, so that the next chunk's are made
// while U is; with more, the first takes y's place and the others one after the other a single one.
//
// Each role's code for a chunk is run once by a few warps and then not until the next chunk, so its instructions come from afar: it is kept short (loops
// that are not unrolled, each step written once; 115 KB of code took 454 us forward and backward of 2 x 8 sequences of
// up to 2048 tokens x 16 x 128, the same steps written once 421).
//
// r^f y is three bf16 parts where a state is written (fp32 has 24 bits, and a state sums many terms); where W only goes on into bf16 results, as itself
// rounded to bf16, two.  (One, whose rounding is then as large as those of P o D and W, took dq and dk of heads of 128 from 2.3e-3 to 2.7e-3 of
// their norm off.)
//
// 2 x 8 sequences of 2048 tokens x 16 x 128: 143 us forward, 388 backward (a CTA: some 7 us and 4.3 for every chunk; with heads of 64, 2.5).  That parts go with
// infinities, too (rps_mix.cuh), is 2 % of both.
// What a chunk takes is this kernel's own instructions and the way from one role to the next, not the tensor cores (a fifth) or memory.
#include "rps_mix.cuh"
#include "rps_tensor.cuh"

namespace rps_ops {
namespace {

using rps::mbar_arrive_expect_tx;
using rps::mbar_init;
using rps::smem_addr;

constexpr int kC = kMixTensorChunk;
constexpr int kBox = 64, kBoxBytes = kC * kBox * 2;  // columns of a copy: one swizzled line of 128 bytes a row
constexpr int kStateBox = 32;                        // fp32 columns of a state's copy: the same
constexpr int kOutWarps = 8, kStateWarps = 16, kFirstOut = 4, kFirstState = kFirstOut + kOutWarps;
constexpr int kThreads = 32 * (kFirstState + kStateWarps);
// Registers of a thread, shared out anew among the groups of four warps: those that hold W have more than the 72 that all alike could have.
constexpr int kLaunchRegisters = 72, kIssueRegisters = 40, kOutRegisters = 56, kStateRegisters = 88;
static_assert(4 * kIssueRegisters + kOutWarps * kOutRegisters + kStateWarps * kStateRegisters <= kThreads / 32 * kLaunchRegisters, "the block's own");
// columns of tensor memory: P, and P o D as 16-bit pairs in its place; x W; (P o D) z; U
constexpr int kAtP = 0, kAtState = 128, kAtOut = 256, kAtU = 384;

// Barriers.  Whoever waits for one has to do so before it completes a second time, as a wait only tells even completions from odd ones; those that
// would get further ahead come in pairs that take turns.
struct Control {
    uint64_t full[2], empty[2], x_full, scores, masked, of_state, out_done, out_free, parts[2], parts_used, last_part, update[2];
    uint64_t state_ready, staged[2], left, state_in, state_read, state_out;
    uint32_t tensor_memory;
    float powers[kC + 1];  // r^0 .. r^128
    float near[64];        // score_scale times the decay from a row to a column e - 32 less, zero ahead of time
    alignas(16) float within[32];  // a decay's share of each of 32 columns
};

// How a state reaches a CTA or leaves it: not at all, by TMA, or element by element (in another order, or at an odd address).
enum StateWay { kNoState = 0, kCopied = 1, kByElement = 2 };

struct MixMaps {
    CUtensorMap of[3][4];  // x, y, z and out of each term
    CUtensorMap state[3][2];  // W before and after
    int way[3][2];
};

// Where a CTA's arrays lie in shared memory.
struct Places {
    int a_boxes, b_boxes;
    bool out_in_y;                          // out leaves from y's place, whose first part has been multiplied by then
    uint32_t y_bytes, z_bytes, w_box;
    uint32_t x, y, z, part, w, out, control;  // offsets; two of y and z; W's first and last value takes the place of `part` and `w`
    __host__ __device__ Places(int a, int b, bool own)
    {
        a_boxes = (a + kBox - 1) / kBox, b_boxes = (b + kBox - 1) / kBox;
        out_in_y = a_boxes == 2 && b_boxes == 2;
        y_bytes = a_boxes * kBoxBytes, z_bytes = b_boxes * kBoxBytes, w_box = a_boxes * kBox * kBox * 2;
        x = 0, y = x + y_bytes, z = y + 2 * y_bytes, part = z + 2 * z_bytes, w = part + (own ? 6 : 1) * y_bytes;
        out = w + b_boxes * w_box, control = out + (out_in_y ? 0 : z_bytes);
    }
};

__device__ int g_gave_up = 0;

__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int col, int token, const Place& at, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst), "l"(map), "r"(col),
                 "r"(token), "r"(at.head), "r"(at.sequence), "r"(at.w), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void store_box(uint32_t src, const CUtensorMap* map, int col, int token, const Place& at)
{
    asm volatile("cp.async.bulk.tensor.5d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3, %4, %5}], [%6];" ::"l"(map), "r"(col), "r"(token), "r"(at.head),
                 "r"(at.sequence), "r"(at.w), "r"(src)
                 : "memory");
}

// 32 columns of all rows of a state.
__device__ __forceinline__ void load_state(uint32_t dst, const CUtensorMap* map, int col, int index, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, 0, %3}], [%4];" ::"r"(dst), "l"(map), "r"(col), "r"(index),
                 "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void store_state(uint32_t src, const CUtensorMap* map, int col, int index)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, 0, %2}], [%3];" ::"l"(map), "r"(col), "r"(index), "r"(src) : "memory");
}

// The left operand in tensor memory.
__device__ __forceinline__ void multiply_from_tensor(uint32_t sum, uint32_t a, uint32_t b, uint32_t descriptor, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}" ::"r"(sum),
        "r"(a), "r"(b), "n"(kDescriptorHigh), "r"(descriptor), "r"((uint32_t)add)
        : "memory");
}

// 16 words of this lane's row.
__device__ __forceinline__ void store_words(uint32_t addr, const uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr), "r"(v[0]), "r"(v[1]),
        "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}

__device__ __forceinline__ void tensor_loads_done() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// What this thread wrote to shared memory is there for the tensor cores and TMA.
__device__ __forceinline__ void writes_done() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ uint4 read_shared(uint32_t addr) { return read_slot(addr); }
__device__ __forceinline__ void write_shared(uint32_t addr, const uint4& v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// exp(log_decay * exponent) of exponents up to 128, the argument's own rounding made up for.
__device__ __forceinline__ float small_power(float log_decay, int exponent)
{
    if (!(log_decay <= 0.0f)) return nanf("");
    const float rate = fmaxf(log_decay, -1e4f), e = (float)exponent, argument = rate * e;
    return expf(argument) * (1.0f + fmaf(rate, e, -argument));
}

// CTAs are placed in their order, and sequences may differ in length: the longest ones first, so that the last places to fall free wait for short ones.
// (256 heads of sequences of up to 2048 tokens, lengths spread evenly, forward and backward: 421 us in the order given, 406 so.)  Every CTA finds its
// own: with kMostSorted sequences at most, whose lengths a warp's width of comparisons each sorts in about a microsecond.
constexpr int kMostSorted = 256;

__device__ __forceinline__ int64_t longest_first(const MixParams& prm, int item, unsigned char* shared)
{
    const int sequences = (int)(prm.n * prm.sequences);
    if (prm.lengths == nullptr || sequences > kMostSorted || sequences == 1) return item;
    int64_t* const lengths = reinterpret_cast<int64_t*>(shared);
    int& found = *reinterpret_cast<int*>(lengths + kMostSorted);
    const int rank = item / prm.heads;
    if ((int)threadIdx.x < sequences) lengths[threadIdx.x] = __ldg(prm.lengths + threadIdx.x);
    __syncthreads();
    if ((int)threadIdx.x < sequences) {
        const int64_t mine = lengths[threadIdx.x];
        int before = 0;
        for (int s = 0; s < sequences; ++s) before += lengths[s] > mine || (lengths[s] == mine && s < (int)threadIdx.x);
        if (before == rank) found = threadIdx.x;
    }
    __syncthreads();
    const int64_t unit = (int64_t)found * prm.heads + item % prm.heads;
    __syncthreads();  // the place is used anew
    return unit;
}

template <bool STATES, bool OWN>
__global__ void __launch_bounds__(kThreads, 1) rps_mix_tensor_kernel(const __grid_constant__ MixParams prm, const __grid_constant__ MixMaps maps)
{
    after_the_kernel_before();
    // the terms of a head of a sequence side by side, as they read the same arrays
    const int which = (int)(blockIdx.x % prm.terms), item = (int)(blockIdx.x / prm.terms), segment = item % prm.segments;
    const MixTerm& term = prm.term[which];
    if (STATES && segment + 1 == prm.segments) return;
    extern __shared__ __align__(16) unsigned char raw[];
    const int64_t unit = longest_first(prm, item / prm.segments, raw);
    const uint32_t base = (smem_addr(raw) + 1023) / 1024 * 1024;
    const int a = term.a, b = term.b;
    const Places places(a, b, OWN);
    const int a_boxes = places.a_boxes, b_boxes = places.b_boxes;
    const uint32_t y_bytes = places.y_bytes, z_bytes = places.z_bytes;
    Control& control = *reinterpret_cast<Control*>(raw + (base + places.control - smem_addr(raw)));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const Place at = place_of(prm, unit);
    const bool reversed = term.reversed != 0;

    // the segment's chunks, counted in the order of time
    const int length = (int)at.length, chunks = (length + kC - 1) / kC, missing = chunks * kC - length;  // of the first chunk's rows
    const int per_segment = (int)(prm.segment_tokens / kC), begin = segment * per_segment, count = max(0, min(chunks - begin, per_segment));
    const auto chunk_at = [&](int i) { return reversed ? chunks - 1 - (begin + i) : begin + i; };
    const bool last = segment + 1 == prm.segments;
    const bool third_part = STATES || term.state_out != nullptr;
    // the last chunk's part of W counts only where W is written
    const bool writes_state = STATES || (last && term.state_out != nullptr);
    const auto updates = [&](int i) { return i + 1 < count || writes_state; };
    // U's place: without O's use of tensor memory two take turns, as the next chunk's U does not wait for W there
    const auto u_of = [](int i) { return STATES && (i & 1) ? kAtOut : kAtU; };
    // W before the segment and after it
    const int64_t slot = (which * prm.units + unit) * prm.segments + segment;
    const int way_in = maps.way[which][0], way_out = writes_state ? maps.way[which][1] : kNoState;
    const int state_boxes = (b + kStateBox - 1) / kStateBox;
    const uint32_t state_box_bytes = a_boxes * kBox * kStateBox * 4;

    if (warp == 0 && lane == 0) {
        const auto init = [](uint64_t& bar, int arrivals) { mbar_init(smem_addr(&bar), arrivals); };
        for (int s = 0; s < 2; ++s) {
            init(control.full[s], 1), init(control.empty[s], places.out_in_y && !STATES ? 2 : 1);
            init(control.parts[s], kStateWarps), init(control.update[s], 1), init(control.staged[s], kOutWarps);
        }
        init(control.x_full, 1), init(control.scores, 1), init(control.of_state, 1), init(control.out_done, 1), init(control.parts_used, 1);
        init(control.masked, kOutWarps), init(control.out_free, kOutWarps), init(control.left, 1);
        init(control.last_part, kStateWarps), init(control.state_ready, kStateWarps);
        init(control.state_in, 1), init(control.state_read, kStateWarps), init(control.state_out, kStateWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) take_tensor_memory<1>(smem_addr(&control.tensor_memory));
    const float log_decay = __ldg(prm.log_decay + at.w * prm.heads + at.head);
    if (threadIdx.x <= kC)
        control.powers[threadIdx.x] = small_power(log_decay, threadIdx.x);
    else if (threadIdx.x >= 192 && threadIdx.x < 224)
        control.within[threadIdx.x - 192] = small_power(log_decay, reversed ? threadIdx.x - 192 : 223 - threadIdx.x);
    else if (threadIdx.x >= 256 && threadIdx.x < 320) {
        const int apart = reversed ? 288 - (int)threadIdx.x : (int)threadIdx.x - 288;
        control.near[threadIdx.x - 256] = apart < 0 ? 0.0f : term.score_scale * small_power(log_decay, apart);
    }
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tensor = control.tensor_memory;

    bool fine = true;
    const uint64_t limit_ns = prm.wait_limit_ms > 0 ? (uint64_t)prm.wait_limit_ms * 1000000u : rps::kDefaultWaitLimitNs;
    const auto wait = [&](uint64_t& bar, int turn) { return rps::mbar_wait(smem_addr(&bar), turn & 1, limit_ns); };  // for the turn-th completion
    const auto warp_wait = [&](uint64_t& bar, int turn) {
        fine = __all_sync(0xFFFFFFFFu, wait(bar, turn));
        after_sync();
        return fine;
    };
    const auto warp_arrive = [&](uint64_t& bar) {
        before_sync();
        __syncwarp();
        if (lane == 0) rps::mbar_arrive(smem_addr(&bar));
    };

    if (warp < kFirstOut) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegisters));
        if (warp == 0 && elect_one()) {
            const CUtensorMap* map = maps.of[which];
            int issued = 0;
            for (int i = 0; i < count && prm.withhold_copies == 0; ++i) {
                const int s = i & 1, token = length - kC * (chunks - chunk_at(i));
                if (!(fine = wait(control.empty[s], (i >> 1) + 1))) break;
                uint32_t bar = smem_addr(&control.full[s]);
                mbar_arrive_expect_tx(bar, y_bytes + z_bytes);
                for (int c = 0; c < a_boxes; ++c) load_box(base + places.y + s * y_bytes + c * kBoxBytes, map + 1, c * kBox, token, at, bar);
                for (int c = 0; c < b_boxes; ++c) load_box(base + places.z + s * z_bytes + c * kBoxBytes, map + 2, c * kBox, token, at, bar);
                ++issued;
                if (!STATES) {
                    if (i > 0 && !(fine = wait(control.of_state, i - 1))) break;  // the chunk before has read x
                    bar = smem_addr(&control.x_full);
                    mbar_arrive_expect_tx(bar, y_bytes);
                    for (int c = 0; c < a_boxes; ++c) load_box(base + places.x + c * kBoxBytes, map, c * kBox, token, at, bar);
                }
            }
            // all copies have arrived before the CTA may end
            for (int i = max(0, issued - 2); i < issued; ++i) fine = wait(control.full[i & 1], i >> 1) && fine;
            if (!STATES && issued > 0) fine = wait(control.x_full, issued - 1) && fine;
        }
        if (warp == 1 && elect_one()) {
            const int b16 = (b + 15) / 16 * 16;
            const uint32_t of_scores = instruction_descriptor(false, false, kC, kC), of_state = instruction_descriptor(false, true, kC, b16);
            const uint32_t of_update = instruction_descriptor(true, true, kC, b16);
            const uint32_t x = descriptor_low(base + places.x, false, kBoxBytes), w = descriptor_low(base + places.w, true, places.w_box);
            const uint32_t first_y = descriptor_low(base + places.y, false, kBoxBytes), first_z = descriptor_low(base + places.z, true, kBoxBytes);
            const uint32_t first_part = descriptor_low(base + places.y, true, kBoxBytes), rest = descriptor_low(base + places.part, true, kBoxBytes);
            // along the rows of a tile 16 columns further: 32 bytes, after 64 the next box; along its columns 16 rows of 128 bytes
            constexpr uint32_t along = 32 / 16, across = 2048 / 16, box = kBoxBytes / 16;
            for (int i = 0; i < count; ++i) {
                const int s = i & 1;
                const uint32_t y = first_y + s * (y_bytes / 16), z = first_z + s * (z_bytes / 16);
                if (!(fine = wait(control.full[s], i >> 1))) break;
                if (!STATES) {
                    // P's place holds the left operand of the product for out of the chunk before
                    if (!(fine = wait(control.x_full, i) && (i == 0 || wait(control.out_done, i - 1)))) break;
                    after_sync();
#pragma unroll 1
                    for (int c = 0; c < a_boxes; ++c)
#pragma unroll
                        for (int k = 0; k < 4; ++k) multiply<1>(tensor + kAtP, x + c * box + k * along, y + c * box + k * along, of_scores, c + k > 0);
                    commit<1>(smem_addr(&control.scores));
                    if (!(fine = wait(control.state_ready, i) && wait(control.out_free, i + 1))) break;
                    after_sync();
#pragma unroll 1
                    for (int c = 0; c < a_boxes; ++c)
#pragma unroll
                        for (int k = 0; k < 4; ++k) multiply<1>(tensor + kAtState, x + c * box + k * along, w + (4 * c + k) * across, of_state, c + k > 0);
                    commit<1>(smem_addr(&control.of_state));
                }
                const int parts = !updates(i) ? 0 : third_part ? 3 : 2;
                // the product for out comes when its left operand is there, as a rule while the last part is on its way
                const int before_out = OWN ? parts : min(parts, 2);
                if (parts > 0) {
                    if (!(fine = OWN ? wait(control.parts[s], i >> 1) : wait(control.parts[0], i))) break;
                    after_sync();
                }
#pragma unroll 1
                for (int p = 0; p <= parts; ++p) {
                    if (p == before_out) {
                        if (!OWN && parts == 3) commit<1>(smem_addr(&control.parts_used));
                        if (parts == before_out && parts > 0) commit<1>(smem_addr(&control.update[s]));
                        if (!STATES) {
                            if (!(fine = wait(control.masked, i))) break;
                            after_sync();
#pragma unroll 1
                            for (int c = 0; c < 2; ++c)
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    multiply_from_tensor(tensor + kAtOut, tensor + kAtP + c * 64 + k * 8, z + (4 * c + k) * across, of_state, c + k > 0);
                            commit<1>(smem_addr(&control.out_done));
                        }
                        if (p == parts) break;
                        if (!(fine = wait(control.last_part, i))) break;
                        after_sync();
                    }
                    if (p < parts) {
                        const uint32_t left = OWN ? rest + (s * 3 + p) * box : p == 0 ? first_part + s * (y_bytes / 16) : rest;
#pragma unroll 1
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                multiply<1>(tensor + u_of(i), left + (4 * c + k) * across, z + (4 * c + k) * across, of_update, p + c + k > 0);
                    } else {
                        commit<1>(smem_addr(&control.update[s]));
                    }
                }
                if (!fine) break;
                commit<1>(smem_addr(&control.empty[s]));
            }
        }
        if (!STATES && warp == 2 && elect_one()) {
            for (int i = 0; i < count; ++i) {
                if (!(fine = wait(control.staged[i & 1], i >> 1))) break;
                const int token = length - kC * (chunks - chunk_at(i));
                if (token >= 0) {  // a copy may not begin ahead of the array
                    const uint32_t from = base + (places.out_in_y ? places.y + (i & 1) * y_bytes : places.out);
                    for (int c = 0; c < b_boxes; ++c) store_box(from + c * kBoxBytes, maps.of[which] + 3, c * kBox, token, at);
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                }
                rps::mbar_arrive(smem_addr(places.out_in_y ? &control.empty[i & 1] : &control.left));
            }
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        }
        if (warp == 3 && elect_one()) {
            if (way_in == kCopied && prm.withhold_copies == 0) {
                const uint32_t bar = smem_addr(&control.state_in);
                mbar_arrive_expect_tx(bar, state_boxes * state_box_bytes);
                const int from = (int)(prm.segments > 1 ? slot : unit);
                for (int c = 0; c < state_boxes; ++c) load_state(base + places.part + c * state_box_bytes, &maps.state[which][0], c * kStateBox, from, bar);
                fine = wait(control.state_in, 0);
            }
        }
    } else if (warp < kFirstState) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOutRegisters));
        if constexpr (!STATES) {
            const int quarter = warp % 4, half = (warp - kFirstOut) / 4, row = quarter * 32 + lane;
            const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
            const int first_col = half * b_boxes * 32, last_col = min(b, first_col + b_boxes * 32);
            bf16* const out = static_cast<bf16*>(term.out) + ((at.w * prm.sequences + at.sequence) * prm.tokens * prm.heads + at.head) * b;
            // rows behind the sequence's last token, while the first chunk is on its way
            const int pieces = b / 8, rows = 32 / pieces;
            const int64_t t1 = min(prm.tokens, (segment + 1) * prm.segment_tokens);
            if (lane < rows * pieces)
                for (int64_t t = max(at.length, segment * prm.segment_tokens) + (warp - kFirstOut) * rows + lane / pieces; t < t1; t += kOutWarps * rows)
                    *reinterpret_cast<uint4*>(out + t * prm.heads * b + lane % pieces * 8) = make_uint4(0, 0, 0, 0);
            for (int i = 0; i < count; ++i) {
                const int chunk = chunk_at(i), token = length - kC * (chunks - chunk) + row;
                if (!warp_wait(control.scores, i)) break;
#pragma unroll 1
                for (int c = half * 64; c < half * 64 + 64; c += 32) {
                    uint32_t word[16];
                    const int apart = reversed ? c - quarter * 32 : quarter * 32 - c;  // of the rows' 32 and the columns'
                    if (apart < 0) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) word[j] = 0;
                    } else {
                        float p[32];
                        __syncwarp();
                        load_sums(p, tensor + lanes + kAtP + c), load_sums(p + 16, tensor + lanes + kAtP + c + 16);
                        tensor_loads_done();
                        if (apart == 0) {
                            const float* near = control.near + 32 + lane;
#pragma unroll
                            for (int j = 0; j < 32; ++j) p[j] *= near[-j];
#pragma unroll
                            for (int j = 0; j < 16; ++j) word[j] = two_bf16(p[2 * j], p[2 * j + 1]);
                        } else {
                            // columns that lie wholly on the near side of these rows: a decay is one of the row's distance to them times one of the column's
                            const Pair far(term.score_scale * control.powers[reversed ? c - row : row - c - 31]);
#pragma unroll
                            for (int j = 0; j < 16; j += 2) {
                                const float4 f = *reinterpret_cast<const float4*>(control.within + 2 * j);
                                float lo, hi;
                                (Pair(p[2 * j], p[2 * j + 1]) * far * Pair(f.x, f.y)).get(lo, hi);
                                word[j] = two_bf16(lo, hi);
                                (Pair(p[2 * j + 2], p[2 * j + 3]) * far * Pair(f.z, f.w)).get(lo, hi);
                                word[j + 1] = two_bf16(lo, hi);
                            }
                        }
                    }
                    // pairs of 64 columns in the first half of their places, which have been read by then
                    store_words(tensor + lanes + kAtP + c / 64 * 64 + c % 64 / 2, word);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                warp_arrive(control.masked);
                if (!warp_wait(control.out_done, i)) break;
                // (before out_free: the barrier may not get two phases ahead)
                if (places.out_in_y && updates(i) && !(third_part ? warp_wait(control.parts_used, i) : warp_wait(control.update[i & 1], i >> 1))) break;
                const int first = chunk == 0 ? missing : 0;
                const Pair factor(term.state_scale * control.powers[reversed ? kC - 1 - row : max(row + 1 - first, 0)]);
                const uint32_t stage = base + (places.out_in_y ? places.y + (i & 1) * y_bytes : places.out) + row * 128;
                if (!places.out_in_y && i > 0 && !warp_wait(control.left, i - 1)) break;  // the chunk before has left its place
                if (first_col >= b) warp_arrive(control.out_free);
#pragma unroll 1
                for (int c = first_col; c < last_col; c += 16) {
                    float v[16], u[16];
                    __syncwarp();
                    load_sums(v, tensor + lanes + kAtOut + c), load_sums(u, tensor + lanes + kAtState + c);
                    tensor_loads_done();
                    if (c + 16 >= last_col) warp_arrive(control.out_free);
#pragma unroll
                    for (int j = 0; j < 16; j += 8) {
                        Pair o[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[k] = fma(factor, Pair(u[j + 2 * k], u[j + 2 * k + 1]), Pair(v[j + 2 * k], v[j + 2 * k + 1]));
                        const uint4 word = narrow(o);
                        const int col = c + j;
                        if (first == 0)
                            write_shared(stage + col / kBox * kBoxBytes + ((col % kBox / 8 ^ (row & 7)) << 4), word);
                        else if (token >= 0 && col < b)
                            *reinterpret_cast<uint4*>(out + (int64_t)token * prm.heads * b + col) = word;
                    }
                }
                writes_done();
                warp_arrive(control.staged[i & 1]);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kStateRegisters));
        const int quarter = warp % 4, share = (warp - kFirstState) / 4, row = quarter * 32 + lane, swizzle = row & 7;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        // W: row `row`, columns from col0 on: 32 of them, or 16 where there are no more than 64 in all
        const int width = b_boxes * 16, col0 = share * width;
        const bool there = row < a_boxes * kBox;  // in shared memory
        float w[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) w[j] = 0.0f;
        const uint32_t state_row = base + places.part + col0 / kStateBox * state_box_bytes + row * 128;
        if (way_in == kCopied) {
            if (warp_wait(control.state_in, 0) && there) {
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    if (j >= width || col0 + j >= b) break;
                    const uint4 v = read_shared(state_row + ((col0 % kStateBox / 4 + j / 4 ^ swizzle) << 4));
                    w[j] = __uint_as_float(v.x), w[j + 1] = __uint_as_float(v.y), w[j + 2] = __uint_as_float(v.z), w[j + 3] = __uint_as_float(v.w);
                }
            }
            // the others' columns lie where this thread's are laid down next
            if (fine) {
                warp_arrive(control.state_read);
                warp_wait(control.state_read, 0);
            }
        } else if (way_in == kByElement && row < term.rows) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < width && col0 + j < term.cols) w[j] = __ldg(term.state_in + unit * term.rows * term.cols + row * term.state_a + (col0 + j) * term.state_b);
        }
        const auto publish = [&] {  // W where the products read it
            if (there) {
#pragma unroll
                for (int j = 0; j < 32; j += 8) {
                    if (j >= width) break;
                    const int col = col0 + j;
                    write_shared(base + places.w + col / kBox * places.w_box + row * 128 + ((col % kBox / 8 ^ swizzle) << 4),
                                 make_uint4(two_bf16(w[j], w[j + 1]), two_bf16(w[j + 2], w[j + 3]), two_bf16(w[j + 4], w[j + 5]), two_bf16(w[j + 6], w[j + 7])));
                }
            }
            writes_done();
            warp_arrive(control.state_ready);
        };
        // this thread's columns of a row of y: a quarter of them, in pieces of 8
        constexpr int kPieces = OWN ? 2 : 4;
        const int pieces = a_boxes * 2, piece0 = share * pieces % 8;
        const uint32_t row_at = base + share * pieces / 8 * kBoxBytes + row * 128;
        uint4 third[kPieces];
        // y of chunk i into its parts: where there is but one place for them, the first in y's own
        const auto split = [&](int i) {
            const int s = i & 1, first = chunk_at(i) == 0 ? missing : 0;
            const uint32_t from = row_at + places.y + s * y_bytes, to = row_at + places.part + (OWN ? s * 3 * y_bytes : 0);
            const uint32_t first_to = OWN ? to : from, second_to = to + (OWN ? y_bytes : 0);
            const Pair factor(term.update_scale * control.powers[reversed ? max(row + 1 - first, 0) : kC - 1 - row]);
            const Pair below = factor * Pair(kBelow);
            uint32_t odd = 0;
#pragma unroll
            for (int q = 0; q < kPieces; ++q) {
                if (q >= pieces) break;
                const uint32_t piece = ((piece0 + q) ^ swizzle) << 4;
                Pair v[4];
                widen(read_shared(from + piece), v);
                uint32_t part[3][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    cut_in_parts(v[j], factor, below, part[0][j], part[1][j], part[2][j]);
                    odd |= part[2][j];
                }
                third[q] = make_uint4(part[2][0], part[2][1], part[2][2], part[2][3]);
                write_shared(first_to + piece, make_uint4(part[0][0], part[0][1], part[0][2], part[0][3]));
                write_shared(second_to + piece, make_uint4(part[1][0], part[1][1], part[1][2], part[1][3]));
                if (OWN) write_shared(to + 2 * y_bytes + piece, third[q]);
            }
            // NaN among the third parts; next to values beyond 2^15, which this may take for some, nothing is changed either
            if (has_infinite_exponent(odd)) {
#pragma unroll
                for (int q = 0; q < kPieces; ++q) {
                    if (q >= pieces) break;
                    const uint32_t piece = ((piece0 + q) ^ swizzle) << 4;
                    const uint4 is = read_shared(first_to + piece);
                    write_shared(second_to + piece, keep_infinities(is, read_shared(second_to + piece)));
                    third[q] = keep_infinities(is, third[q]);
                    if (OWN) write_shared(to + 2 * y_bytes + piece, third[q]);
                }
            }
            writes_done();
            warp_arrive(control.parts[OWN ? s : 0]);
        };
        // W of the next chunk: false if a wait gave up.  Rows behind the heads' columns stay zeros: an infinite z makes NaN of their part of U.
        const bool row_of_w = row < term.rows;
        const auto bring_up_to_date = [&](int i) {
            if (!warp_wait(control.update[i & 1], i >> 1)) return false;
            const Pair whole(control.powers[kC - (chunk_at(i) == 0 ? missing : 0)]);
#pragma unroll
            for (int c = 0; c < 32; c += 16) {
                if (c >= width) break;
                float u[16];
                __syncwarp();
                load_sums(u, tensor + lanes + u_of(i) + col0 + c);
                tensor_loads_done();
                if (!row_of_w) continue;
#pragma unroll
                for (int j = 0; j < 16; j += 2) fma(whole, Pair(w[c + j], w[c + j + 1]), Pair(u[j], u[j + 1])).get(w[c + j], w[c + j + 1]);
            }
            before_sync();
            return true;
        };
        if constexpr (OWN) {
            // a chunk's parts are made before the W that goes with them is waited for
            for (int i = 0; fine; ++i) {
                if (i < count && updates(i)) {
                    if (!warp_wait(control.full[i & 1], i >> 1)) break;
                    split(i);
                }
                if (i > 0 && (!updates(i - 1) || !bring_up_to_date(i - 1))) break;
                if (i >= count) break;
                if constexpr (!STATES) {
                    if (i > 0 && !warp_wait(control.of_state, i - 1)) break;  // W's place has been read
                    publish();
                }
            }
        } else {
            for (int i = 0; i < count && fine; ++i) {
                if constexpr (!STATES) {
                    if (i > 0 && !warp_wait(control.of_state, i - 1)) break;
                    publish();
                }
                // y's own place has been read by the product for P; the other was left by the chunk before
                if (!updates(i) || !warp_wait(control.full[i & 1], i >> 1) || (!STATES && !warp_wait(control.scores, i))) break;
                split(i);
                if (third_part) {
                    if (!warp_wait(control.parts_used, i)) break;
#pragma unroll
                    for (int q = 0; q < kPieces; ++q)
                        if (q < pieces) write_shared(row_at + places.part + (((piece0 + q) ^ swizzle) << 4), third[q]);
                    writes_done();
                    warp_arrive(control.last_part);
                }
                if (!bring_up_to_date(i)) break;
            }
        }
        // the last product has read the places that W's last value takes
        if (way_out == kCopied && fine) {
            if (there) {
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    if (j >= width || col0 + j >= b) break;
                    write_shared(state_row + ((col0 % kStateBox / 4 + j / 4 ^ swizzle) << 4),
                                 make_uint4(__float_as_uint(w[j]), __float_as_uint(w[j + 1]), __float_as_uint(w[j + 2]), __float_as_uint(w[j + 3])));
                }
            }
            writes_done();
            warp_arrive(control.state_out);
            // (a warp that has come this far: from the segment's start on a wait for all of it would be longer than for any data)
            if (warp == kFirstState && warp_wait(control.state_out, 0) && elect_one()) {
                const int to = (int)(STATES ? slot + 1 : unit);
                for (int c = 0; c < state_boxes; ++c) store_state(base + places.part + c * state_box_bytes, &maps.state[which][1], c * kStateBox, to);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            }
        } else if (way_out == kByElement && fine && row < term.rows) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < width && col0 + j < term.cols) term.state_out[unit * term.rows * term.cols + row * term.state_a + (col0 + j) * term.state_b] = w[j];
        }
    }
    if (!fine) atomicExch(&g_gave_up, 1);
    before_sync();
    __syncthreads();
    after_sync();
    __syncwarp();
    if (warp == 1) free_tensor_memory<1>(tensor);
}

// -------------------------------------------------------------------------------------------------------------- host
bool fits(const MixParams& prm, const MixOperand& o, int cols) { return reinterpret_cast<uintptr_t>(o.base) % 16 == 0 && mix_fits_tensor(prm, o, cols); }

bool encode(CUtensorMap* map, const MixParams& prm, const MixOperand& o, int cols)
{
    rps::EncodeTiledFn encode = rps::encode_tiled_fn();
    if (encode == nullptr) return false;
    const auto bytes = [](int64_t size, int64_t step) { return (cuuint64_t)(size <= 1 ? 16 : step * 2); };  // an axis of one element takes any stride
    const cuuint64_t dims[5] = {(cuuint64_t)cols, (cuuint64_t)prm.tokens, (cuuint64_t)prm.heads, (cuuint64_t)prm.sequences, (cuuint64_t)prm.n};
    const cuuint64_t strides[4] = {bytes(prm.tokens, o.token), bytes(prm.heads, o.head), bytes(prm.sequences, o.sequence), bytes(prm.n, o.worker)};
    const cuuint32_t box[5] = {kBox, kC, 1, 1, 1}, steps[5] = {1, 1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(o.base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// `states` states of a x b, `apart` elements from one to the next.
bool encode_state(CUtensorMap* map, const float* base, int a, int b, int64_t states, int64_t apart)
{
    rps::EncodeTiledFn encode = rps::encode_tiled_fn();
    if (encode == nullptr) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)b, (cuuint64_t)a, (cuuint64_t)states}, strides[2] = {(cuuint64_t)b * 4, (cuuint64_t)apart * 4};
    const cuuint32_t box[3] = {kStateBox, (cuuint32_t)(ceil_div(a, kBox) * kBox), 1}, steps[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<float*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Shared memory of a CTA: more than half of an SM's, as the tensor memory that a CTA takes is all there is.
size_t shared_bytes(int a, int b, bool own) { return std::max<size_t>(120 << 10, 1024 + Places(a, b, own).control + sizeof(Control)); }
static_assert(sizeof(Control) <= 2048, "shared memory for the widest heads");

template <bool STATES, bool OWN>
cudaError_t launch(const MixParams& prm, const MixMaps& maps, cudaStream_t stream)
{
    static rps::LaunchState granted;
    size_t bytes = 0;
    for (int i = 0; i < prm.terms; ++i) bytes = std::max(bytes, shared_bytes(prm.term[i].a, prm.term[i].b, OWN));
    cudaError_t err = rps::grant_smem(granted, rps_mix_tensor_kernel<STATES, OWN>, (uint32_t)bytes);
    if (err != cudaSuccess) return err;
    static std::atomic<int> registers{0};
    if ((err = check_registers(registers, rps_mix_tensor_kernel<STATES, OWN>, kLaunchRegisters)) != cudaSuccess) return err;
    return launch_after(rps_mix_tensor_kernel<STATES, OWN>, dim3((unsigned)(prm.units * prm.segments * prm.terms)), kThreads, bytes, stream, 1, prm, maps);
}

}  // namespace

// Whether TMA can copy an operand as it lies: axes of more than one element need strides that are multiples of 16 bytes (and not zero).
bool mix_fits_tensor(const MixParams& prm, const MixOperand& o, int cols)
{
    const auto stride = [](int64_t size, int64_t step) { return size <= 1 || (step > 0 && step % 8 == 0 && step < 1ll << 38); };
    return cols % 8 == 0 && stride(prm.tokens, o.token) && stride(prm.heads, o.head) && stride(prm.sequences, o.sequence) && stride(prm.n, o.worker);
}

bool mix_fits_tensor(const MixParams& prm)
{
    if (prm.tokens < 1 || prm.tokens >= 1ll << 30) return false;
    for (int i = 0; i < prm.terms; ++i) {
        const MixTerm& t = prm.term[i];
        if (!fits(prm, t.x, t.a) || !fits(prm, t.y, t.a) || !fits(prm, t.z, t.b) || reinterpret_cast<uintptr_t>(t.out) % 16 != 0) return false;
    }
    return true;
}

cudaError_t launch_mix_tensor(const MixParams& prm, bool states, cudaStream_t stream)
{
    MixMaps maps{};
    for (int i = 0; i < prm.terms; ++i) {
        const MixTerm& t = prm.term[i];
        if (!encode(&maps.of[i][0], prm, t.x, t.a) || !encode(&maps.of[i][1], prm, t.y, t.a) || !encode(&maps.of[i][2], prm, t.z, t.b) ||
            !encode(&maps.of[i][3], prm, {t.out, prm.sequences * prm.tokens * prm.heads * t.b, prm.tokens * prm.heads * t.b, (int64_t)prm.heads * t.b, t.b}, t.b))
            return cudaErrorInvalidValue;
        const bool segmented = prm.segments > 1;
        const int64_t all = prm.terms * prm.units * prm.segments, each = (int64_t)t.a * t.b;
        const auto state = [&](int which, bool in_segments, const float* at) {
            const bool dense = t.state_b == 1 && t.rows == t.a && t.cols == t.b;
            maps.way[i][which] = at == nullptr ? kNoState : in_segments || (dense && reinterpret_cast<uintptr_t>(at) % 16 == 0) ? kCopied : kByElement;
            return maps.way[i][which] != kCopied || encode_state(&maps.state[i][which], at, t.a, t.b, in_segments ? all : prm.units, in_segments ? prm.state_room : each);
        };
        if (!state(0, segmented, states ? nullptr : segmented ? prm.segment_states : t.state_in) || !state(1, states, states ? prm.segment_states : t.state_out))
            return cudaErrorInvalidValue;
    }
    // key and value columns are x's and z's in one term or another
    const bool own = prm.term[0].a <= kBox && prm.term[0].b <= kBox;
    if (states) return own ? launch<true, true>(prm, maps, stream) : launch<true, false>(prm, maps, stream);
    return own ? launch<false, true>(prm, maps, stream) : launch<false, false>(prm, maps, stream);
}

cudaError_t read_mix_gave_up(int* value, cudaStream_t stream) { return read_and_clear(g_gave_up, value, stream); }

}  // namespace rps_ops
