// Rows of a table looked up by token, and the gradient of the table.
//
// Both are bound by memory.  The gradient's rows are sums over the tokens that name them.  Atomics would add them in another order every
// time and write fp32; here the tokens are sorted by row first (stably, so that a row's sum goes through its tokens in their order),
// then every run of equal tokens is summed in fp32 registers and its row written once, rounded once.
//
//   sort   least significant digit first, 8 bits or fewer a pass; up to kSortHere tokens of a worker stay in one CTA's shared memory, more
//          go through passes of counting, scanning and scattering
//   sum    the sorted tokens are cut into tiles of equal length, a warp to a tile and 32 slices of 16 bytes of the columns, so that a
//          word that every other token is does not make one warp's work; runs that cross tiles leave fp32 parts, which are joined in order
#include <algorithm>

#include "rps_kernels.h"
#include "rps_rows.cuh"

namespace rps_ops {
namespace {

constexpr int kRowThreads = 256, kRowsAtATime = 4;

// Rows of the table: a thread takes its slices of four tokens at a time, 2^log_across threads to a row.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(kRowThreads) rps_embed_lookup_kernel(const EmbedParams prm, int log_across)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth;
    const int across = 1 << log_across, down = kRowThreads >> log_across, D = (int)prm.cols, w = blockIdx.y;
    const int64_t* tokens = prm.tokens + w * prm.count;
    const T* table = static_cast<const T*>(prm.weight) + w * prm.weight_worker;
    T* out = static_cast<T*>(prm.out) + w * prm.count * prm.cols;
    const int64_t t0 = (int64_t)blockIdx.x * down * kRowsAtATime + (threadIdx.x >> log_across);
    int64_t token[kRowsAtATime];
#pragma unroll
    for (int i = 0; i < kRowsAtATime; ++i) {
        const int64_t t = t0 + i * down;
        token[i] = t < prm.count ? __ldg(tokens + t) : prm.ignore_index;
    }
    for (int c = (threadIdx.x & (across - 1)) * W; c < D; c += across * W) {
        uint4 slice[kRowsAtATime];
        bool there[kRowsAtATime];
#pragma unroll
        for (int i = 0; i < kRowsAtATime; ++i) {
            there[i] = token[i] != prm.ignore_index && token[i] >= 0 && token[i] < prm.vocab;
            slice[i] = load_slice<T, ALIGN, false>(table + (there[i] ? token[i] : 0) * prm.weight_row, c, there[i] ? D : 0);
        }
#pragma unroll
        for (int i = 0; i < kRowsAtATime; ++i) {
            const int64_t t = t0 + i * down;
            if (t >= prm.count) break;
            float v[W];
            widen(slice[i], v);
            // a token that names no row gives NaN
            const float factor = there[i] ? prm.scale : token[i] == prm.ignore_index ? 0.0f : __int_as_float(0x7FFFFFFF);
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] *= factor;
            store_slice<T, ALIGN>(out + t * prm.cols, c, D, narrow(v));
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------- sort
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kBins = 256;
constexpr int kBlockItems = 4;                               // of a thread where several CTAs sort
constexpr int kSortBlock = kSortThreads * kBlockItems;
constexpr int kMostItems = 16, kSortHere = kSortThreads * kMostItems;

struct SortShared {
    uint32_t of_warp[kSortWarps][kBins];  // items of each digit in each warp, then where they go
    uint32_t total[kBins], scan[kBins];
};

// What a token sorts by: the row that it names, or one past the last.
__device__ __forceinline__ uint32_t sort_key(const EmbedParams& prm, int64_t token)
{
    return token != prm.ignore_index && token >= 0 && token < prm.vocab ? (uint32_t)token : (uint32_t)prm.vocab;
}

// Place of each item among the CTA's, by one digit and stably; a warp's items follow one another, 32 at a time (kNone: no item).
// Leaves the number of items of each digit in sh.total and the first place of each in sh.scan.
constexpr uint32_t kNone = 0xFFFFFFFFu;

template <int ITEMS>
__device__ __forceinline__ void rank_items(SortShared& sh, const uint32_t (&key)[ITEMS], uint32_t (&place)[ITEMS], int shift, int bits)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const uint32_t mask = (1u << bits) - 1;
    for (int b = lane; b < kBins; b += 32) sh.of_warp[warp][b] = 0;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const bool item = key[i] != kNone;
        const uint32_t digit = key[i] >> shift & mask;
        uint32_t same = __ballot_sync(0xFFFFFFFFu, item);
        if (!item) same = ~same;
        for (int b = 0; b < bits; ++b) {
            const bool set = digit >> b & 1;
            const uint32_t with = __ballot_sync(0xFFFFFFFFu, set);
            same &= set ? with : ~with;
        }
        const uint32_t before = __popc(same & ((1u << lane) - 1));
        const uint32_t base = item ? sh.of_warp[warp][digit] : 0;
        __syncwarp();
        if (item && before == 0) sh.of_warp[warp][digit] = base + __popc(same);
        __syncwarp();
        place[i] = base + before;
    }
    __syncthreads();
    // over the warps of each digit, a thread to a digit, then over the digits
    if (threadIdx.x < kBins) {
        uint32_t sum = 0;
#pragma unroll 8
        for (int k = 0; k < kSortWarps; ++k) {
            const uint32_t n = sh.of_warp[k][threadIdx.x];
            sh.of_warp[k][threadIdx.x] = sum;
            sum += n;
        }
        sh.total[threadIdx.x] = sum;
    }
    __syncthreads();
    if (warp == 0) {
        uint32_t mine[kBins / 32], sum = 0;
#pragma unroll
        for (int j = 0; j < kBins / 32; ++j) mine[j] = sh.total[lane * (kBins / 32) + j], sum += mine[j];
        uint32_t upto = sum;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const uint32_t n = __shfl_up_sync(0xFFFFFFFFu, upto, s);
            if (lane >= s) upto += n;
        }
        upto -= sum;
#pragma unroll
        for (int j = 0; j < kBins / 32; ++j) sh.scan[lane * (kBins / 32) + j] = upto, upto += mine[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (key[i] != kNone) place[i] += sh.of_warp[warp][key[i] >> shift & mask];
}

// A worker's tokens in one CTA.
template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads) rps_embed_sort_kernel(const EmbedParams prm)
{
    after_the_kernel_before();
    extern __shared__ uint32_t raw[];
    SortShared& sh = *reinterpret_cast<SortShared*>(raw);
    uint32_t* keys = raw + sizeof(SortShared) / 4;
    uint32_t* from = keys + kSortThreads * ITEMS;
    const int w = blockIdx.x, count = (int)prm.count, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int first = warp * 32 * ITEMS + lane;
    uint32_t key[ITEMS], token[ITEMS], place[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int t = first + i * 32;
        token[i] = (uint32_t)t;
        key[i] = t < count ? sort_key(prm, __ldg(prm.tokens + w * prm.count + t)) : kNone;
    }
    for (int shift = 0; shift < prm.key_bits; shift += prm.digit_bits) {
        rank_items<ITEMS>(sh, key, place, shift, prm.digit_bits);
        const uint32_t mask = (1u << prm.digit_bits) - 1;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (key[i] == kNone) continue;
            const uint32_t to = place[i] + sh.scan[key[i] >> shift & mask];
            keys[to] = key[i], from[to] = token[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = first + i * 32;
            if (at < count) key[i] = keys[at], token[i] = from[at];
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int at = first + i * 32;
        if (at < count) prm.keys[0][w * prm.count + at] = key[i], prm.from[0][w * prm.count + at] = token[i];
    }
}

// Several CTAs to a worker: how many items of each digit every block has ([digit][block] of a worker) ...
__global__ void __launch_bounds__(kSortThreads) rps_embed_count_kernel(const EmbedParams prm, int pass)
{
    after_the_kernel_before();
    __shared__ uint32_t bins[kBins];
    const int w = blockIdx.y, shift = pass * prm.digit_bits;
    const uint32_t mask = (1u << prm.digit_bits) - 1;
    if (threadIdx.x < kBins) bins[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBlockItems; ++i) {
        const int64_t t = (int64_t)blockIdx.x * kSortBlock + i * kSortThreads + threadIdx.x;
        if (t >= prm.count) break;
        const uint32_t key = pass == 0 ? sort_key(prm, __ldg(prm.tokens + w * prm.count + t)) : prm.keys[(pass + 1) & 1][w * prm.count + t];
        atomicAdd(&bins[key >> shift & mask], 1u);
    }
    __syncthreads();
    if (threadIdx.x < kBins) prm.counts[((int64_t)w * kBins + threadIdx.x) * gridDim.x + blockIdx.x] = bins[threadIdx.x];
}

// ... where each block's items of each digit begin (a CTA to a worker) ...
__global__ void __launch_bounds__(kSortThreads) rps_embed_scan_kernel(const EmbedParams prm, int blocks)
{
    after_the_kernel_before();
    __shared__ uint32_t sums[kSortWarps];
    uint32_t* counts = prm.counts + (int64_t)blockIdx.x * kBins * blocks;
    const int total = kBins * blocks, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    uint32_t before = 0;
    for (int i0 = 0; i0 < total; i0 += kSortThreads * 8) {
        const int i = i0 + threadIdx.x * 8;
        uint32_t n[8], sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = i + j < total ? counts[i + j] : 0, sum += n[j];
        uint32_t upto = sum;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, upto, s);
            if (lane >= s) upto += x;
        }
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
        uint32_t warps = sums[lane];
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, warps, s);
            if (lane >= s) warps += x;
        }
        uint32_t at = before + upto - sum + (warp > 0 ? __shfl_sync(0xFFFFFFFFu, warps, warp - 1) : 0);
        before += __shfl_sync(0xFFFFFFFFu, warps, 31);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (i + j < total) counts[i + j] = at;
            at += n[j];
        }
        __syncthreads();
    }
}

// ... and the items moved there.
__global__ void __launch_bounds__(kSortThreads) rps_embed_scatter_kernel(const EmbedParams prm, int pass)
{
    after_the_kernel_before();
    __shared__ SortShared sh;
    const int w = blockIdx.y, shift = pass * prm.digit_bits, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const uint32_t mask = (1u << prm.digit_bits) - 1;
    const int64_t base = w * prm.count;
    uint32_t key[kBlockItems], token[kBlockItems], place[kBlockItems];
#pragma unroll
    for (int i = 0; i < kBlockItems; ++i) {
        const int64_t t = (int64_t)blockIdx.x * kSortBlock + warp * 32 * kBlockItems + i * 32 + lane;
        const bool there = t < prm.count;
        if (pass == 0)
            token[i] = (uint32_t)t, key[i] = there ? sort_key(prm, __ldg(prm.tokens + base + t)) : kNone;
        else
            token[i] = there ? prm.from[(pass + 1) & 1][base + t] : 0, key[i] = there ? prm.keys[(pass + 1) & 1][base + t] : kNone;
    }
    rank_items<kBlockItems>(sh, key, place, shift, prm.digit_bits);
#pragma unroll
    for (int i = 0; i < kBlockItems; ++i) {
        if (key[i] == kNone) continue;
        const uint32_t digit = key[i] >> shift & mask;
        const int64_t to = base + prm.counts[((int64_t)w * kBins + digit) * gridDim.x + blockIdx.x] + place[i];
        prm.keys[pass & 1][to] = key[i], prm.from[pass & 1][to] = token[i];
    }
}

// ----------------------------------------------------------------------------------------------------------------- sum
constexpr int kSumWarps = 8;

template <typename T, int ALIGN>
__device__ __forceinline__ void write_row(const EmbedParams& prm, int w, uint32_t row, int c, const float (&sum)[Slice<T>::kWidth])
{
    constexpr int W = Slice<T>::kWidth;
    T* out = static_cast<T*>(prm.dweight) + w * prm.dweight_worker + (int64_t)row * prm.dweight_row;
    float v[W];
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = 0.0f;
    if (prm.accumulate) widen(load_slice<T, ALIGN, false>(out, c, (int)prm.cols), v);
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = prm.accumulate ? fmaf(prm.scale, sum[j], v[j]) : prm.scale * sum[j];
    store_slice<T, ALIGN>(out, c, (int)prm.cols, narrow(v));
}

// A warp for 32 slices of the columns of a tile of sorted tokens.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(32 * kSumWarps) rps_embed_sum_kernel(const EmbedParams prm, int slabs)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth, kAtATime = 8;
    const int lane = threadIdx.x % 32, w = blockIdx.y, D = (int)prm.cols;
    const int64_t item = (int64_t)blockIdx.x * kSumWarps + threadIdx.x / 32;
    const int64_t tile = item / slabs;
    if (tile >= prm.tiles) return;
    const int c = ((int)(item - tile * slabs) * 32 + lane) * W;
    const uint32_t* keys = prm.keys[prm.sorted] + w * prm.count;
    const uint32_t* from = prm.from[prm.sorted] + w * prm.count;
    const T* dout = static_cast<const T*>(prm.dout) + w * prm.count * prm.cols;
    const int64_t p0 = tile * prm.tile, p1 = min(p0 + prm.tile, prm.count);
    float* parts = prm.parts + (w * prm.tiles + tile) * 2 * prm.part_row + c;
    uint32_t current = __ldg(keys + p0);
    if (current >= prm.vocab) return;
    bool head = p0 > 0 && __ldg(keys + p0 - 1) == current;  // the run goes on from the tile before
    float sum[W];
#pragma unroll
    for (int j = 0; j < W; ++j) sum[j] = 0.0f;
    const auto store_part = [&](int slot) {
        float* to = parts + slot * prm.part_row;
        if (c >= D) return;
#pragma unroll
        for (int j = 0; j < W; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
    };
    for (int64_t p = p0; p < p1; p += 32) {
        const bool mine = p + lane < p1;
        const uint32_t my_key = mine ? __ldg(keys + p + lane) : (uint32_t)prm.vocab, my_from = mine ? __ldg(from + p + lane) : 0;
        const int here = (int)min((int64_t)32, p1 - p);
        for (int q = 0; q < here; q += kAtATime) {
            uint4 slice[kAtATime];
            uint32_t key[kAtATime];
#pragma unroll
            for (int i = 0; i < kAtATime; ++i) {
                key[i] = __shfl_sync(0xFFFFFFFFu, my_key, q + i);
                const int64_t row = __shfl_sync(0xFFFFFFFFu, my_from, q + i);
                slice[i] = load_slice<T, ALIGN, true>(dout + row * prm.cols, c, key[i] < prm.vocab ? D : 0);
            }
#pragma unroll
            for (int i = 0; i < kAtATime; ++i) {
                if (key[i] != current) {
                    if (current < prm.vocab) {
                        if (head)
                            store_part(0);
                        else
                            write_row<T, ALIGN>(prm, w, current, c, sum);
                    }
                    head = false, current = key[i];
#pragma unroll
                    for (int j = 0; j < W; ++j) sum[j] = 0.0f;
                }
                float v[W];
                widen(slice[i], v);
#pragma unroll
                for (int j = 0; j < W; ++j) sum[j] += v[j];
            }
        }
    }
    if (current >= prm.vocab) return;
    const bool on = p1 < prm.count && __ldg(keys + p1) == current;  // it goes on in the next
    if (head || on)
        store_part(head ? 0 : 1);
    else
        write_row<T, ALIGN>(prm, w, current, c, sum);
}

// Runs that cross tiles: the warp of the tile that a run begins in adds its parts up.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(32 * kSumWarps) rps_embed_join_kernel(const EmbedParams prm, int slabs)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth;
    const int lane = threadIdx.x % 32, w = blockIdx.y, D = (int)prm.cols;
    const int64_t item = (int64_t)blockIdx.x * kSumWarps + threadIdx.x / 32;
    const int64_t tile = item / slabs;
    if (tile + 1 >= prm.tiles) return;
    const uint32_t* keys = prm.keys[prm.sorted] + w * prm.count;
    const int64_t p0 = tile * prm.tile, p1 = p0 + prm.tile;
    const uint32_t key = __ldg(keys + p1);
    if (key >= prm.vocab || __ldg(keys + p1 - 1) != key) return;                                   // none crosses
    if (__ldg(keys + p0) == key && p0 > 0 && __ldg(keys + p0 - 1) == key) return;                  // it began before
    const int c = ((int)(item - tile * slabs) * 32 + lane) * W;
    // the run's last tile
    int64_t last = tile + 1;
    while (last + 1 < prm.tiles) {
        const int64_t at = last + 1 + lane;
        const bool on = at < prm.tiles && __ldg(keys + at * prm.tile) == key;
        const uint32_t all = __ballot_sync(0xFFFFFFFFu, on);
        const int n = all == 0xFFFFFFFFu ? 32 : __ffs(~all) - 1;
        last += n;
        if (n < 32) break;
    }
    if (c >= D) return;
    float sum[W];
    const float* parts = prm.parts + w * prm.tiles * 2 * prm.part_row + c;
    const auto add = [&](int64_t t, int slot, bool first) {
        const float* at = parts + (t * 2 + slot) * prm.part_row;
#pragma unroll
        for (int j = 0; j < W; j += 4) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(at + j));
            sum[j] = first ? v.x : sum[j] + v.x, sum[j + 1] = first ? v.y : sum[j + 1] + v.y;
            sum[j + 2] = first ? v.z : sum[j + 2] + v.z, sum[j + 3] = first ? v.w : sum[j + 3] + v.w;
        }
    };
    add(tile, 1, true);
#pragma unroll 8
    for (int64_t t = tile + 1; t <= last; ++t) add(t, 0, false);
    write_row<T, ALIGN>(prm, w, key, c, sum);
}

// Zeros into the rows of the gradient.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(kRowThreads) rps_embed_clear_kernel(const EmbedParams prm, int log_across)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth;
    const int across = 1 << log_across, down = kRowThreads >> log_across, D = (int)prm.cols;
    T* out = static_cast<T*>(prm.dweight) + blockIdx.y * prm.dweight_worker;
    for (int64_t v = (int64_t)blockIdx.x * down + (threadIdx.x >> log_across); v < prm.vocab; v += (int64_t)gridDim.x * down)
        for (int c = (threadIdx.x & (across - 1)) * W; c < D; c += across * W) store_slice<T, ALIGN>(out + v * prm.dweight_row, c, D, make_uint4(0, 0, 0, 0));
}

// ---------------------------------------------------------------------------------------------------------------- host
int log_threads_across(int64_t cols, int width)
{
    int log = 0;
    while (log < 8 && (width << log) < cols) ++log;
    return log;
}

template <typename T>
cudaError_t lookup(const EmbedParams& prm, cudaStream_t stream)
{
    const int log = log_threads_across(prm.cols, Slice<T>::kWidth);
    const int align = std::min({alignment<T>(prm.weight, prm.cols, prm.weight_row), alignment<T>(prm.weight, prm.cols, prm.weight_worker),
                                alignment<T>(prm.out, prm.cols, prm.cols)});
    const dim3 grid((unsigned)ceil_div(prm.count, (kRowThreads >> log) * kRowsAtATime), (unsigned)prm.n);
    const auto kernel = align == 16 ? rps_embed_lookup_kernel<T, 16> : align == 4 ? rps_embed_lookup_kernel<T, 4> : rps_embed_lookup_kernel<T, sizeof(T)>;
    return launch_after(kernel, grid, kRowThreads, 0, stream, 1, prm, log);
}

template <int ITEMS>
cudaError_t sort_here(const EmbedParams& prm, cudaStream_t stream)
{
    static rps::LaunchState state;
    const uint32_t bytes = sizeof(SortShared) + kSortThreads * ITEMS * 8;
    const cudaError_t err = rps::grant_smem(state, rps_embed_sort_kernel<ITEMS>, bytes);
    if (err != cudaSuccess) return err;
    return launch_after(rps_embed_sort_kernel<ITEMS>, dim3((unsigned)prm.n), kSortThreads, bytes, stream, 1, prm);
}

cudaError_t sort(const EmbedParams& prm, cudaStream_t stream)
{
    if (prm.count <= kSortThreads) return sort_here<1>(prm, stream);
    if (prm.count <= kSortThreads * 4) return sort_here<4>(prm, stream);
    if (prm.count <= kSortHere) return sort_here<kMostItems>(prm, stream);
    const dim3 grid((unsigned)ceil_div(prm.count, kSortBlock), (unsigned)prm.n);
    cudaError_t err = cudaSuccess;
    for (int pass = 0; pass * prm.digit_bits < prm.key_bits && err == cudaSuccess; ++pass) {
        err = launch_after(rps_embed_count_kernel, grid, kSortThreads, 0, stream, 1, prm, pass);
        if (err == cudaSuccess) err = launch_after(rps_embed_scan_kernel, dim3((unsigned)prm.n), kSortThreads, 0, stream, 1, prm, (int)grid.x);
        if (err == cudaSuccess) err = launch_after(rps_embed_scatter_kernel, grid, kSortThreads, 0, stream, 1, prm, pass);
    }
    return err;
}

template <typename T>
cudaError_t gradient(const EmbedParams& prm, cudaStream_t stream)
{
    cudaError_t err = cudaSuccess;
    const int out_align = std::min(alignment<T>(prm.dweight, prm.cols, prm.dweight_row), alignment<T>(prm.dweight, prm.cols, prm.dweight_worker));
    if (!prm.accumulate) {
        const int log = log_threads_across(prm.cols, Slice<T>::kWidth);
        const dim3 grid((unsigned)std::min<int64_t>(ceil_div(prm.vocab, kRowThreads >> log), ceil_div((int64_t)kSms * 8, prm.n)), (unsigned)prm.n);
        const auto kernel = out_align == 16 ? rps_embed_clear_kernel<T, 16> : out_align == 4 ? rps_embed_clear_kernel<T, 4> : rps_embed_clear_kernel<T, sizeof(T)>;
        if ((err = launch_after(kernel, grid, kRowThreads, 0, stream, 1, prm, log)) != cudaSuccess) return err;
    }
    if (prm.count == 0) return cudaSuccess;
    if ((err = sort(prm, stream)) != cudaSuccess) return err;
    const int align = std::min(out_align, alignment<T>(prm.dout, prm.cols, prm.cols));
    const int slabs = (int)ceil_div(prm.cols, 32 * Slice<T>::kWidth);
    const dim3 grid((unsigned)ceil_div(prm.tiles * slabs, kSumWarps), (unsigned)prm.n);
    const auto kernel = align == 16 ? rps_embed_sum_kernel<T, 16> : align == 4 ? rps_embed_sum_kernel<T, 4> : rps_embed_sum_kernel<T, sizeof(T)>;
    if ((err = launch_after(kernel, grid, 32 * kSumWarps, 0, stream, 1, prm, slabs)) != cudaSuccess || prm.tiles == 1) return err;
    const auto join = align == 16 ? rps_embed_join_kernel<T, 16> : align == 4 ? rps_embed_join_kernel<T, 4> : rps_embed_join_kernel<T, sizeof(T)>;
    return launch_after(join, grid, 32 * kSumWarps, 0, stream, 1, prm, slabs);
}

}  // namespace

void plan_embed(EmbedParams* prm)
{
    EmbedParams& p = *prm;
    p.key_bits = 1;
    while (p.vocab >> p.key_bits) ++p.key_bits;  // keys are 0..vocab
    const int passes = (int)ceil_div(p.key_bits, 8);
    p.digit_bits = (int)ceil_div(p.key_bits, passes);
    p.sorted = p.count <= kSortHere ? 0 : (passes - 1) & 1;
    p.sort_blocks = p.count <= kSortHere ? 0 : ceil_div(p.count, kSortBlock);
    const int width = p.f32 ? Slice<float>::kWidth : Slice<bf16>::kWidth;
    const int64_t slabs = ceil_div(p.cols, 32 * width);
    // long tiles leave fewer parts, short ones more warps
    p.tile = 256;
    while (p.tile > 16 && p.n * ceil_div(p.count, p.tile) * slabs < kSms * 24) p.tile /= 2;
    p.tiles = ceil_div(p.count, p.tile);
    p.part_row = slabs * 32 * width;
}

cudaError_t launch_embed_lookup(const EmbedParams& prm, cudaStream_t stream) { return prm.f32 ? lookup<float>(prm, stream) : lookup<bf16>(prm, stream); }

cudaError_t launch_embed_gradient(const EmbedParams& prm, cudaStream_t stream) { return prm.f32 ? gradient<float>(prm, stream) : gradient<bf16>(prm, stream); }

}  // namespace rps_ops
