// The step between two blocks of a network: norm, gate, residual scale, residual sum, norm; forward and backward.
//
// Bound by memory: forward reads x, f (and gate) and writes h, y; backward reads dh, dy, f, h (and gate) and writes dx, df
// (and dgate).  So every tensor is touched once.  A row is spread over a CTA of at most 512 threads, 16 bytes of it to a thread (a wider
// row over a cluster of CTAs that exchange their sums through distributed shared memory), so that a row lives in
// registers between its sums and its results.  CTAs walk many rows; each thread copies its own slices of the next kAhead rows into
// shared memory meanwhile (cp.async: no registers, and no barrier, as a thread reads what it copied itself).
//
// Backward needs two means of a row, of a * h and of b * f, where b depends on the first one.  With q = scale * gate * post * f,
//   sum b f = sum q (dh + r_h a) - r_h^3 mean(a h) sum q h,
// so both come out of three sums made in one pass, with one barrier for a row.  The sums over rows (dpost, dpre, and dgate where
// tokens share a gate) stay in the registers of the thread that owns the columns; a block writes its own once, and a
// second kernel adds the blocks' in a fixed order.
#include <algorithm>

#include "rps_cluster.cuh"
#include "rps_kernels.h"
#include "rps_rows.cuh"

namespace rps_ops {
namespace {

constexpr int kMostThreads = 512;
constexpr int kSlots = 4, kAhead = kSlots - 1;      // rows in shared memory: this one and those ahead
// Threads on an SM at once, by registers.  By shared memory (the slots, the sums' 4 KB and 1 KB of the system for each CTA of 228 KB) so many CTAs
// of 256 threads and more fit too; of narrower ones fewer: forward 7 of 8 of 128 threads, 13 of 16 of 64 and 20 of 32 of 32, backward 15 of 16 of
// 32; the others follow when places get free.  (With room for the sums of one CTA's warps alone, so that all but the last forward ones fit: 4 x 24108 x 85
// bf16 forward 54 -> 57 us, backward 170 -> 151; 65536 x 256 37 -> 39, 96 -> 92; 30000 x 500 fp32 60 -> 65, 104 -> 104; 32768 x 512 bf16 with 8-bit copies
// 50 -> 44, 72 -> 72.)
constexpr int kForwardThreads = 1024, kBackwardThreads = 512;
constexpr int kMostCluster = 8;
// Of the slots in shared memory, whatever lies before them: copies of 16 bytes whose neighbours in a warp start off a 128-byte line are far slower
// (16 bytes off: 16384 x 4096 bf16 backward 196 -> 220 us, 32768 x 1024 55 + 109 -> 151 + 192, 65536 x 256 36 + 95 -> 140 + 194).
constexpr int kLine = 128;
constexpr int kMostWarps = kMostThreads / 32 * kMostCluster;

// Set when a bounded wait gave up (rps_ops_check).
__device__ int g_norm_gave_up = 0;

// Room for the warps' sums of up to four values, double-buffered over successive exchanges, so that one barrier is enough.
struct Sums {
    float of[2][4][kMostWarps];
    uint64_t arrived[2];  // of a cluster: counts the bytes
};

// Of a cluster: before the first exchange.
__device__ __forceinline__ void start_exchanges(Sums& sums)
{
    if (threadIdx.x == 0) {
        for (int k = 0; k < 2; ++k) rps::mbar_init(rps::smem_addr(&sums.arrived[k]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    cluster_sync();
}

// Of a cluster: after the last one.  No CTA may end while another's sums may still be on their way to it.  Where all waits were met they have
// arrived; after one that ran out (its CTA may have had some of them sent just now) they are given time, once nobody sends any more.
__device__ __forceinline__ void end_exchanges(bool fine)
{
    if (!fine) {
        copies_arrived<0>();
        if (threadIdx.x % 32 == 0) atomicExch(&g_norm_gave_up, 1);
    }
    __syncwarp();
    cluster_sync();
    if (!fine) __nanosleep(200000);
}

// A warp's sum of each of `values` values to every CTA that shares the row, and the wait for all of them.  Some lanes (8 at least) have the sum of
// a value, and `index` numbers them.  In a cluster each of them sends it to one CTA, whose barrier counts the bytes: a barrier of the whole
// cluster would first see the stores of the row before through to memory (2200 rows of 4096 fp32: 52 + 70 us, 38 + 51 so).  A warp sends
// again only after it has read all sums of the exchange before, so nobody is more than one exchange ahead, and two rooms are enough.
// A warp whose wait runs out (fine = false, for all of its lanes) is done: it neither arrives nor sends again, as a barrier must not be
// arrived on twice in a phase, and so the others' waits run out one exchange later at most.
template <bool CLUSTER>
__device__ __forceinline__ void exchange(const NormParams& prm, Sums& sums, int turn, uint32_t parity, int value, int values, float v, int index, int cluster,
                                         uint32_t rank, bool& fine)
{
    const int warps = blockDim.x / 32, warp = threadIdx.x / 32;
    if constexpr (!CLUSTER) {
        if (index == 0) sums.of[turn][value][warp] = v;
        __syncthreads();
    } else {
        const uint32_t bar = rps::smem_addr(&sums.arrived[turn]);
        if (threadIdx.x == 0) rps::mbar_arrive_expect_tx(bar, (uint32_t)(warps * cluster * values) * 4);
        if (index < cluster && (prm.withhold_sums == 0 || rank + 1 < (uint32_t)cluster)) {
            uint32_t there, counter;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(rps::smem_addr(&sums.of[turn][value][rank * warps + warp])), "r"(index));
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(counter) : "r"(bar), "r"(index));
            asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(there), "r"(__float_as_uint(v)), "r"(counter)
                         : "memory");
        }
        __syncwarp();
        fine = __all_sync(0xFFFFFFFFu, wait_for(bar, parity, prm.wait_limit_ms > 0 ? (uint64_t)prm.wait_limit_ms * 1000000u : rps::kDefaultWaitLimitNs));
    }
}

// The sum of a value over the threads that share a row; every thread gets it, added in the same order.
template <bool CLUSTER>
__device__ __forceinline__ float row_sum(const NormParams& prm, float v, Sums& sums, int turn, uint32_t parity, int cluster, uint32_t rank, bool& fine)
{
    const int lane = threadIdx.x % 32, used = blockDim.x / 32 * cluster;
#pragma unroll
    for (int s = 16; s > 0; s /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, s);
    if (!CLUSTER && used == 1) return v;
    exchange<CLUSTER>(prm, sums, turn, parity, 0, 1, v, lane, cluster, rank, fine);
    if constexpr (!CLUSTER) {  // at most 16 warps
        v = lane % 16 < used ? sums.of[turn][0][lane % 16] : 0.0f;
    } else {
        v = 0.0f;
        for (int k = lane % 16; k < used; k += 16) v += sums.of[turn][0][k];
    }
#pragma unroll
    for (int s = 8; s > 0; s /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, s);
    return v;
}

// The same of three values at a time: the lanes share the values out while they add (8 lanes to a value), 6 exchanges between lanes
// instead of 15.
template <bool CLUSTER>
__device__ __forceinline__ void row_sums(const NormParams& prm, float (&v)[3], Sums& sums, int turn, uint32_t parity, int cluster, uint32_t rank, bool& fine)
{
    const int lane = threadIdx.x % 32, used = blockDim.x / 32 * cluster, value = lane / 8;
    const bool high = lane & 16, odd = lane & 8;
    float a = high ? v[2] : v[0], b = high ? 0.0f : v[1];  // values 0, 1 stay below, 2 (and an empty 3) above
    a += __shfl_xor_sync(0xFFFFFFFFu, high ? v[0] : v[2], 16);
    b += __shfl_xor_sync(0xFFFFFFFFu, high ? v[1] : 0.0f, 16);
    float s = odd ? b : a;
    s += __shfl_xor_sync(0xFFFFFFFFu, odd ? a : b, 8);
#pragma unroll
    for (int k = 4; k > 0; k /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, k);
    if (CLUSTER || used > 1) {
        exchange<CLUSTER>(prm, sums, turn, parity, value, 4, s, lane % 8, cluster, rank, fine);
        s = 0.0f;
        for (int k = lane % 8; k < used; k += 8) s += sums.of[turn][value][k];
#pragma unroll
        for (int k = 4; k > 0; k /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, k);
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, s, 8 * i);
}

// Rows of one CTA follow one another, so that their addresses, their worker and their gate are counted up instead of divided out.
// The arithmetic goes two columns at a time: at one column an instruction (447 of them for 8 columns of a row forward, 640 backward)
// the kernels were bound by instruction issue, at 4.3 TB/s.
template <typename T, int ALIGN, bool PACK, bool CLUSTER>
__global__ void __launch_bounds__(kMostThreads, kForwardThreads / kMostThreads) rps_norm_forward_kernel(const NormParams prm)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth, P = W / 2;
    extern __shared__ __align__(kLine) uint4 ring[];
    __shared__ Sums sums;
    const uint32_t copied = (uint32_t)__cvta_generic_to_shared(ring);
    const int cluster = CLUSTER ? prm.cluster : 1, D = (int)prm.cols;
    const uint32_t rank = CLUSTER ? cluster_rank() : 0;
    bool fine = true;
    if (CLUSTER) start_exchanges(sums);
    const int c = ((int)rank * blockDim.x + threadIdx.x) * W;
    const int64_t rows = prm.n * prm.tokens, first = rows * (blockIdx.x / cluster) / (gridDim.x / cluster);
    const int count = (int)(rows * (blockIdx.x / cluster + 1) / (gridDim.x / cluster) - first);
    const float inv = 1.0f / (float)D;
    const T* const x_rows = static_cast<const T*>(prm.x) + first * D;
    const T* const f_rows = static_cast<const T*>(prm.f) + first * D;
    T* const h_rows = static_cast<T*>(prm.h) + first * D;
    T* const y_rows = static_cast<T*>(prm.y) + first * D;
    const int64_t worker0 = first / prm.tokens, token0 = first - worker0 * prm.tokens;

    // of the next row to be copied
    const uint32_t array = blockDim.x * 16, slot = 3 * array, end_of_ring = copied + kSlots * slot + threadIdx.x * 16;
    uint32_t into = copied + threadIdx.x * 16;
    int to_send = count, rows_per_gate = (int)prm.rows_per_gate, tokens = (int)prm.tokens;
    int left_in_gate = rows_per_gate - (int)(token0 % rows_per_gate), left_in_worker = tokens - (int)token0;
    int64_t worker = worker0, ahead = 0;
    const T* gate_at = static_cast<const T*>(prm.gate) + worker0 * prm.gate_worker + token0 / prm.rows_per_gate * D;
    const auto send = [&] {
        if (to_send > 0) {
            --to_send;
            copy_slice<T, ALIGN>(into, x_rows + ahead, c, D);
            copy_slice<T, ALIGN>(into + array, f_rows + ahead, c, D);
            copy_slice<T, ALIGN>(into + 2 * array, gate_at, c, D);
            ahead += D;
            if (--left_in_gate == 0) left_in_gate = rows_per_gate, gate_at += D;
            if (--left_in_worker == 0) left_in_worker = tokens, gate_at = static_cast<const T*>(prm.gate) + ++worker * prm.gate_worker;
        }
        copies_sent();
        into += slot;
        if (into == end_of_ring) into -= kSlots * slot;
    };
    for (int i = 0; i < kAhead; ++i) send();

    // of the row that is worked on
    Pair post[P], pre[P];
    int rows_of_worker = tokens - (int)token0;
    const T* post_at = static_cast<const T*>(prm.post) + worker0 * prm.post_worker;
    const T* pre_at = static_cast<const T*>(prm.pre) + worker0 * prm.pre_worker;
    const auto parameters = [&] {
        widen(load_slice<T, ALIGN, false>(post_at, c, D), post);
        widen(load_slice<T, ALIGN, false>(pre_at, c, D), pre);
#pragma unroll
        for (int j = 0; j < P; ++j) post[j] = post[j] * Pair(prm.scale);
    };
    parameters();
    uint32_t from = copied + threadIdx.x * 16;
    int64_t at = 0;
    for (int i = 0; i < count; ++i, at += D) {
        if (rows_of_worker-- == 0) {
            rows_of_worker = tokens - 1;
            post_at += prm.post_worker, pre_at += prm.pre_worker;
            parameters();
        }
        Pair x[P], f[P], gate[P];
        send();
        copies_arrived<kAhead>();
        widen(read_slot(from), x);
        widen(read_slot(from + array), f);
        widen(read_slot(from + 2 * array), gate);
        from += slot;
        if (from == end_of_ring) from -= kSlots * slot;
        Pair s(0.0f);
#pragma unroll
        for (int j = 0; j < P; ++j) s = fma(f[j], f[j], s);
        const float r_f = rsqrtf(fmaf(row_sum<CLUSTER>(prm, s.sum(), sums, 0, i & 1, cluster, rank, fine), inv, prm.eps));
        if (CLUSTER && !fine) break;
        if constexpr (PACK) {
            const int64_t row = first + i;
            float v[W];
#pragma unroll
            for (int j = 0; j < P; ++j) f[j].get(v[2 * j], v[2 * j + 1]);
            pack_slice(v, c < prm.pitch ? prm.f_codes + row * prm.pitch + c : nullptr, c < D ? prm.f_scales + row * prm.groups + c / RPS_PACK_GROUP : nullptr);
        }
        s = Pair(0.0f);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            x[j] = fma(gate[j] * post[j] * f[j], Pair(r_f), x[j]);  // h
            s = fma(x[j], x[j], s);
        }
        const uint4 h = narrow(x);
        store_slice<T, ALIGN>(h_rows + at, c, D, h);
        const float r_h = rsqrtf(fmaf(row_sum<CLUSTER>(prm, s.sum(), sums, 1, i & 1, cluster, rank, fine), inv, prm.eps));
        if (CLUSTER && !fine) break;
        if constexpr (PACK) {
            const int64_t row = first + i;
            float stored[W];  // as a reader of h sees it
            widen(h, stored);
            if constexpr (ALIGN != 16) {
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (c + j >= D) stored[j] = 0.0f;
            }
            pack_slice(stored, c < prm.pitch ? prm.h_codes + row * prm.pitch + c : nullptr,
                       c < D ? prm.h_scales + row * prm.groups + c / RPS_PACK_GROUP : nullptr);
        }
#pragma unroll
        for (int j = 0; j < P; ++j) x[j] = x[j] * (pre[j] * Pair(r_h));
        store_slice<T, ALIGN>(y_rows + at, c, D, narrow(x));
        if (prm.r_f != nullptr && rank == 0 && threadIdx.x == 0) {
            prm.r_f[first + i] = r_f;
            prm.r_h[first + i] = r_h;
        }
    }
    if (CLUSTER) end_exchanges(fine);
}

template <typename T, int ALIGN, bool PACKED, bool CLUSTER>
__global__ void __launch_bounds__(kMostThreads, kBackwardThreads / kMostThreads) rps_norm_backward_kernel(const NormParams prm)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth, P = W / 2;
    extern __shared__ __align__(kLine) uint4 ring[];
    __shared__ Sums sums;
    const uint32_t copied = (uint32_t)__cvta_generic_to_shared(ring);
    const int cluster = CLUSTER ? prm.cluster : 1, D = (int)prm.cols;
    const uint32_t rank = CLUSTER ? cluster_rank() : 0;
    bool fine = true;
    if (CLUSTER) start_exchanges(sums);
    const int c = ((int)rank * blockDim.x + threadIdx.x) * W;
    const float inv = 1.0f / (float)D;
    const int64_t block = blockIdx.x / cluster, w = blockIdx.y;
    int64_t first, end;  // tokens of this block
    if (prm.chunks > 0) {
        const int64_t g = block / prm.chunks;
        first = g * prm.rows_per_gate + block % prm.chunks * prm.rows_per_block;
        end = min(first + prm.rows_per_block, (g + 1) * prm.rows_per_gate);
    } else {
        first = block * prm.rows_per_block;
        end = min(first + prm.rows_per_block, prm.tokens);
    }
    const int count = (int)max((int64_t)0, end - first);
    const int64_t row0 = w * prm.tokens + first;
    const T* const dy_rows = static_cast<const T*>(prm.dy) + row0 * D;
    const T* const dh_rows = prm.dh != nullptr ? static_cast<const T*>(prm.dh) + row0 * D : nullptr;
    T* const dx_rows = static_cast<T*>(prm.dx) + row0 * D;
    T* const df_rows = static_cast<T*>(prm.df) + row0 * D;
    Pair post[P], pre[P], dpost[P], dpre[P], dgate[P];
    widen(load_slice<T, ALIGN, false>(static_cast<const T*>(prm.post) + w * prm.post_worker, c, D), post);
    widen(load_slice<T, ALIGN, false>(static_cast<const T*>(prm.pre) + w * prm.pre_worker, c, D), pre);
#pragma unroll
    for (int j = 0; j < P; ++j) {
        post[j] = post[j] * Pair(prm.scale);
        dpost[j] = dpre[j] = dgate[j] = Pair(0.0f);
    }

    // of the next row to be copied
    const uint32_t array = blockDim.x * 16, slot = 5 * array, end_of_ring = copied + kSlots * slot + threadIdx.x * 16;
    uint32_t into = copied + threadIdx.x * 16;
    const int rows_per_gate = (int)prm.rows_per_gate;
    int to_send = count, left_in_gate = rows_per_gate - (int)(first % rows_per_gate);
    int rows_of_gate = left_in_gate;  // of the row that is worked on
    int64_t gate_row = w * prm.gates + first / rows_per_gate, ahead = 0;
    const T* gate_at = static_cast<const T*>(prm.gate) + w * prm.gate_worker + first / rows_per_gate * D;
    const T* const f_rows = PACKED ? nullptr : static_cast<const T*>(prm.f) + row0 * D;
    const T* const kept_rows = PACKED ? nullptr : static_cast<const T*>(prm.h_in) + row0 * D;
    int64_t code_at = c < D ? row0 * prm.pitch + c : 0, scale_at = c < D ? row0 * prm.groups + c / RPS_PACK_GROUP : 0;
    const auto send = [&] {
        if (to_send > 0) {
            --to_send;
            copy_slice<T, ALIGN>(into, dy_rows + ahead, c, D);
            if (dh_rows != nullptr) copy_slice<T, ALIGN>(into + array, dh_rows + ahead, c, D);
            copy_slice<T, ALIGN>(into + 2 * array, gate_at, c, D);
            if constexpr (PACKED) {  // the codes, and behind them the scale
                const bool in = c < D;
                copy_async<W>(into + 3 * array, static_cast<const int8_t*>(prm.f) + code_at, in);
                copy_async<4>(into + 3 * array + 8, prm.f_scales + scale_at, in);
                copy_async<W>(into + 4 * array, static_cast<const int8_t*>(prm.h_in) + code_at, in);
                copy_async<4>(into + 4 * array + 8, prm.h_scales + scale_at, in);
                if (in) code_at += prm.pitch, scale_at += prm.groups;
            } else {
                copy_slice<T, ALIGN>(into + 3 * array, f_rows + ahead, c, D);
                copy_slice<T, ALIGN>(into + 4 * array, kept_rows + ahead, c, D);
            }
            ahead += D;
            if (--left_in_gate == 0) left_in_gate = rows_per_gate, gate_at += D;
        }
        copies_sent();
        into += slot;
        if (into == end_of_ring) into -= kSlots * slot;
    };
    const auto kept = [&](const uint4& held, Pair (&v)[P]) {
        if constexpr (PACKED) {
            float e[W];
            Codes<W> codes;
            codes.w[0] = held.x;
            if constexpr (W == 8) codes.w[1] = held.y;
            codes.values(__uint_as_float(held.z), e);
#pragma unroll
            for (int j = 0; j < P; ++j) v[j] = Pair(e[2 * j], e[2 * j + 1]);
        } else {
            widen(held, v);
        }
    };
    float rf_next = 0.0f, rh_next = 0.0f;
    const auto statistics = [&](int i) {
        if (i < count) rf_next = __ldg(prm.r_f + row0 + i), rh_next = __ldg(prm.r_h + row0 + i);
    };
    for (int i = 0; i < kAhead; ++i) send();
    statistics(0);
    uint32_t from = copied + threadIdx.x * 16;
    int64_t at = 0;
    for (int i = 0; i < count; ++i, at += D) {
        Pair f[P], h[P], dx[P], sgp[P], gate[P];  // sgp: scale * gate * post
        float s[3];
        send();
        copies_arrived<kAhead>();
        const float r_f = rf_next, r_h = rh_next;
        statistics(i + 1);
        kept(read_slot(from + 3 * array), f), kept(read_slot(from + 4 * array), h);
        {
            Pair dy[P], s0(0.0f), s1(0.0f), s2(0.0f);
            widen(read_slot(from), dy);
            if (dh_rows != nullptr) {
                widen(read_slot(from + array), dx);
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) dx[j] = Pair(0.0f);
            }
            widen(read_slot(from + 2 * array), gate);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                dpre[j] = fma(dy[j], h[j] * Pair(r_h), dpre[j]);
                const Pair a = dy[j] * pre[j];
                sgp[j] = gate[j] * post[j];
                const Pair q = sgp[j] * f[j];
                dx[j] = fma(a, Pair(r_h), dx[j]);  // dh + r_h a
                s0 = fma(a, h[j], s0);
                s1 = fma(q, dx[j], s1);
                s2 = fma(q, h[j], s2);
            }
            s[0] = s0.sum(), s[1] = s1.sum(), s[2] = s2.sum();
        }
        from += slot;
        if (from == end_of_ring) from -= kSlots * slot;
        row_sums<CLUSTER>(prm, s, sums, i & 1, i >> 1 & 1, cluster, rank, fine);
        if (CLUSTER && !fine) break;
        const float mean_h = s[0] * inv * r_h * r_h * r_h;
        const float mean_f = (s[1] - mean_h * s[2]) * inv * r_f * r_f * r_f;
        Pair df[P];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            dx[j] = fma(h[j], Pair(-mean_h), dx[j]);
            const Pair e = dx[j] * f[j] * Pair(r_f);
            dgate[j] = fma(e, post[j], dgate[j]);
            dpost[j] = fma(e, gate[j], dpost[j]);
            df[j] = fma(dx[j] * sgp[j], Pair(r_f), f[j] * Pair(-mean_f));
        }
        store_slice<T, ALIGN>(dx_rows + at, c, D, narrow(dx));
        store_slice<T, ALIGN>(df_rows + at, c, D, narrow(df));
        if (--rows_of_gate == 0) {
            rows_of_gate = rows_per_gate;
            if (prm.chunks == 0) {  // the block held the whole gate group
                store_slice<T, ALIGN>(static_cast<T*>(prm.dgate) + gate_row * D, c, D, narrow(dgate));
                ++gate_row;
#pragma unroll
                for (int j = 0; j < P; ++j) dgate[j] = Pair(0.0f);
            }
        }
    }
    float* partial = prm.partial + (w * prm.blocks + block) * 3 * D;
#pragma unroll
    for (int j = 0; j < P; ++j) {
        float v[3][2];
        (dpost[j] * Pair(prm.scale)).get(v[0][0], v[0][1]), dpre[j].get(v[1][0], v[1][1]), dgate[j].get(v[2][0], v[2][1]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (c + 2 * j + k < D) {
                partial[c + 2 * j + k] = v[0][k];
                partial[D + c + 2 * j + k] = v[1][k];
                if (prm.chunks > 0) partial[2 * D + c + 2 * j + k] = v[2][k];
            }
        }
    }
    if (CLUSTER) end_exchanges(fine);
}

// Sums of the blocks' sums: 32 columns to a CTA, the blocks dealt to its 16 warps, whose sums are added in their order.
template <typename T>
__global__ void __launch_bounds__(512) rps_norm_reduce_kernel(const NormParams prm)
{
    after_the_kernel_before();
    __shared__ float slots[16][33];
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x % 32, w = blockIdx.z, D = prm.cols;
    const int warp = threadIdx.x / 32;
    for (int64_t job = blockIdx.y; job < 2 + (prm.chunks > 0 ? prm.gates : 0); job += gridDim.y) {
        const int64_t b0 = job < 2 ? 0 : (job - 2) * prm.chunks, b1 = job < 2 ? prm.blocks : b0 + prm.chunks;
        const float* partial = prm.partial + (w * prm.blocks * 3 + (job < 2 ? job : 2)) * D + c;
        float s = 0.0f;
        if (c < D) {
#pragma unroll 4
            for (int64_t b = b0 + warp; b < b1; b += 16) s += partial[b * 3 * D];
        }
        slots[warp][threadIdx.x % 32] = s;
        __syncthreads();
        if (warp == 0 && c < D) {
            for (int k = 1; k < 16; ++k) s += slots[k][threadIdx.x];
            T* out = static_cast<T*>(job == 0 ? prm.dpost : job == 1 ? prm.dpre : prm.dgate);
            out[(job < 2 ? w : w * prm.gates + job - 2) * D + c] = from_float<T>(s);
        }
        __syncthreads();
    }
}

// Threads of a CTA and CTAs of a cluster for a row of `slices` 16-byte slices: the fewest threads (a power of two of warps) that hold it, up
// to 512, then a cluster.  About `most` threads are resident on an SM at once, and a row of a cluster of 3 to 8 takes some 1.7 times as long as
// one of 2, whatever their number (its sums go from CTA to CTA twice, or backward once), so the cluster that has most rows through in a given
// time is taken.  2200 rows of fp32 in us, what is taken first:
//   4488 columns  forward 6 CTAs of 192 threads 64, 5 of 256 67, 4 of 288 69, 8 of 160 72, 3 of 384 78
//                 backward 5 of 256 103, 6 of 192 108, 8 of 160 108, 3 of 384 116, 4 of 288 130
//   6200 columns  backward 7 of 224 150, 8 of 224 167, 4 of 416 168, 5 of 320 180, 6 of 288 207
//   2100 columns  backward 2 of 288 39, 6 of 96 51
void shape_of_row(int64_t slices, int most, int* threads, int* cluster)
{
    *threads = 32, *cluster = 1;
    while (*threads < kMostThreads && *threads < slices) *threads *= 2;
    if (*threads >= slices) return;
    double best = 0.0;
    for (int c = 2; c <= 8; ++c) {
        const int64_t each = round_up(ceil_div(slices, c), 32);
        if (each > kMostThreads) continue;
        const double rate = (double)(kSms * (most / each) / c) / (c == 2 ? 1.0 : 1.7);
        if (rate > best) best = rate, *threads = (int)each, *cluster = c;
    }
}

// `arrays` slices of each of kSlots rows to a thread in shared memory.
template <typename Kernel>
cudaError_t launch_rows(rps::LaunchState& state, Kernel kernel, const NormParams& prm, dim3 grid, int threads, int arrays, cudaStream_t stream)
{
    const uint32_t bytes = (uint32_t)(threads * 16 * arrays * kSlots);
    cudaError_t err = rps::grant_smem(state, kernel, bytes);
    if (err != cudaSuccess) return err;
    return launch_after(kernel, grid, threads, bytes, stream, prm.cluster, prm);
}

template <typename T, int ALIGN, bool PACK>
cudaError_t run_forward(const NormParams& prm, dim3 grid, int threads, cudaStream_t stream)
{
    static rps::LaunchState state, shared_rows;
    return prm.cluster > 1 ? launch_rows(shared_rows, rps_norm_forward_kernel<T, ALIGN, PACK, true>, prm, grid, threads, 3, stream)
                           : launch_rows(state, rps_norm_forward_kernel<T, ALIGN, PACK, false>, prm, grid, threads, 3, stream);
}

template <typename T, int ALIGN, bool PACKED>
cudaError_t run_backward(const NormParams& prm, dim3 grid, int threads, cudaStream_t stream)
{
    static rps::LaunchState state, shared_rows;
    return prm.cluster > 1 ? launch_rows(shared_rows, rps_norm_backward_kernel<T, ALIGN, PACKED, true>, prm, grid, threads, 5, stream)
                           : launch_rows(state, rps_norm_backward_kernel<T, ALIGN, PACKED, false>, prm, grid, threads, 5, stream);
}

// What all arrays of a call can be moved in.
template <typename T>
int common_alignment(const NormParams& prm)
{
    int align = std::min({alignment<T>(prm.gate, prm.cols, prm.gate_worker), alignment<T>(prm.post, prm.cols, prm.post_worker),
                          alignment<T>(prm.pre, prm.cols, prm.pre_worker)});
    for (const void* p : {prm.x, prm.dh, prm.dy, (const void*)prm.h, (const void*)prm.y, (const void*)prm.dx, (const void*)prm.df, (const void*)prm.dgate,
                          prm.packed ? nullptr : prm.f, prm.packed ? nullptr : prm.h_in})
        align = std::min(align, alignment<T>(p, prm.cols, 0));
    return align;
}

template <typename T>
cudaError_t forward(NormParams prm, cudaStream_t stream)
{
    const bool pack = prm.f_codes != nullptr;
    int threads = 0, sms = 0;
    shape_of_row(ceil_div(pack ? prm.pitch : prm.cols, Slice<T>::kWidth), kForwardThreads, &threads, &prm.cluster);
    cudaError_t err = sm_count(&sms);
    if (err != cudaSuccess) return err;
    const int align = common_alignment<T>(prm);
    const int64_t rows = prm.n * prm.tokens, resident = (int64_t)sms * (kForwardThreads / threads) / prm.cluster;
    const dim3 grid((unsigned)((rows < resident ? rows : resident) * prm.cluster));
    constexpr int kLeast = sizeof(T);
    if (align == 16) return pack ? run_forward<T, 16, true>(prm, grid, threads, stream) : run_forward<T, 16, false>(prm, grid, threads, stream);
    if (align == 4) return pack ? run_forward<T, 4, true>(prm, grid, threads, stream) : run_forward<T, 4, false>(prm, grid, threads, stream);
    return pack ? run_forward<T, kLeast, true>(prm, grid, threads, stream) : run_forward<T, kLeast, false>(prm, grid, threads, stream);
}

template <typename T>
cudaError_t backward(NormParams prm, cudaStream_t stream)
{
    int threads = 0;
    shape_of_row(ceil_div(prm.cols, Slice<T>::kWidth), kBackwardThreads, &threads, &prm.cluster);
    const int align = common_alignment<T>(prm);
    const dim3 grid((unsigned)(prm.blocks * prm.cluster), (unsigned)prm.n);
    constexpr int kLeast = sizeof(T);
    cudaError_t err;
    if (align == 16)
        err = prm.packed ? run_backward<T, 16, true>(prm, grid, threads, stream) : run_backward<T, 16, false>(prm, grid, threads, stream);
    else if (align == 4)
        err = prm.packed ? run_backward<T, 4, true>(prm, grid, threads, stream) : run_backward<T, 4, false>(prm, grid, threads, stream);
    else
        err = prm.packed ? run_backward<T, kLeast, true>(prm, grid, threads, stream) : run_backward<T, kLeast, false>(prm, grid, threads, stream);
    if (err != cudaSuccess) return err;
    const int64_t jobs = 2 + (prm.chunks > 0 ? prm.gates : 0);
    return launch_after(rps_norm_reduce_kernel<T>, dim3((unsigned)ceil_div(prm.cols, 32), (unsigned)(jobs < 4096 ? jobs : 4096), (unsigned)prm.n), 512,
                        0, stream, 1, prm);
}

}  // namespace

cudaError_t read_norm_gave_up(int* value, cudaStream_t stream) { return read_and_clear(g_norm_gave_up, value, stream); }

void plan_norm_backward(NormParams* prm)
{
    int threads = 0, cluster = 0;
    shape_of_row(ceil_div(prm->cols, prm->f32 ? Slice<float>::kWidth : Slice<bf16>::kWidth), kBackwardThreads, &threads, &cluster);
    // as many blocks over all workers as are resident at once (512 threads of each SM); of the two nearest ways
    // to cut the rows the one whose longest SM has fewer of them
    int64_t want = (int64_t)kSms * (kBackwardThreads / threads) / cluster / prm->n;
    if (want < 1) want = 1;
    const int64_t rows = prm->rows_per_gate, target = ceil_div(prm->tokens, want);
    const bool whole = rows <= target;
    const auto cut = [&](int64_t k) {  // k gate groups a block, or k blocks a gate group
        prm->chunks = whole ? 0 : k;
        prm->rows_per_block = whole ? k * rows : ceil_div(rows, k);
        prm->blocks = whole ? ceil_div(prm->tokens, prm->rows_per_block) : prm->gates * k;
        return ceil_div(prm->blocks, want) * prm->rows_per_block;
    };
    const int64_t k = whole ? target / rows : rows / target;
    if (cut(k + 1) > cut(k)) return;
    cut(k + 1);
}

cudaError_t launch_norm_forward(const NormParams& prm, cudaStream_t stream)
{
    return prm.f32 ? forward<float>(prm, stream) : forward<bf16>(prm, stream);
}

cudaError_t launch_norm_backward(const NormParams& prm, cudaStream_t stream)
{
    return prm.f32 ? backward<float>(prm, stream) : backward<bf16>(prm, stream);
}

}  // namespace rps_ops
