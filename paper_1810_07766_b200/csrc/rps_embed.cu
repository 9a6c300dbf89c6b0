// Rows of a table looked up by token, and the gradient of the table.
//
// Both are bound by memory.  The gradient's rows are sums over the tokens that name them.  Atomics would add them in another order every
// time and write fp32; here the tokens are sorted by row first (stably, so that a row's sum goes through its tokens in their order),
// then every run of equal tokens is summed in fp32 registers and its row written once, rounded once.
//
//   few    up to kFew tokens of a worker: one launch, whose CTAs each sort all of them and then write their own rows of the gradient, zeros or sums
//   sort   least significant digit first, 8 bits or fewer a pass; up to kSortHere tokens of a worker stay in the shared memory of a cluster of
//          eight CTAs, which write to each other's, more go through launches of counting, scanning and scattering.  Few SMs have work in
//          these; the others clear the gradient meanwhile.
//   sum    the sorted tokens are cut into tiles of equal length, a warp to a tile and 512 bytes of the columns, so that a
//          word that every other token is does not make one warp's work; runs that cross tiles leave fp32 parts, which are joined in order
#include <algorithm>
#include <type_traits>

#include "rps_cluster.cuh"
#include "rps_rows.cuh"

namespace rps_ops {
namespace {

// 16 bytes of a row are a thread's, in pieces of ALIGN bytes: what all rows' addresses are multiples of.  `across` threads side by side take the first
// pieces, then the second ones, so that any alignment is read and written in whole lines.
template <typename T, int ALIGN>
struct Piece {
    static constexpr int kWidth = 16 / sizeof(T), kEach = ALIGN / sizeof(T), kPieces = 16 / ALIGN;
    using Word = std::conditional_t<ALIGN == 16, uint4, std::conditional_t<ALIGN == 8, uint2, std::conditional_t<ALIGN == 4, uint32_t, unsigned short>>>;
    // column of piece j of thread x where the threads' columns begin at `first`
    static __device__ __forceinline__ int column(int first, int x, int across, int j) { return first + (j * across + x) * kEach; }
    static __device__ __forceinline__ uint4 load(const T* row, int first, int x, int across, int cols)
    {
        union {
            Word word[kPieces];
            uint4 all;
        } v;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int c = column(first, x, across, j);
            v.word[j] = c < cols ? __ldcs(reinterpret_cast<const Word*>(row + c)) : Word{};
        }
        return v.all;
    }
    static __device__ __forceinline__ void store(T* row, int first, int x, int across, int cols, const uint4& value)
    {
        union {
            Word word[kPieces];
            uint4 all;
        } v;
        v.all = value;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int c = column(first, x, across, j);
            if (c < cols) __stcs(reinterpret_cast<Word*>(row + c), v.word[j]);
        }
    }
};

constexpr int kRowThreads = 256, kRowsAtATime = 4;

// Rows of the table: a thread takes its pieces of four tokens at a time, 2^log_across threads to a row.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(kRowThreads) rps_embed_lookup_kernel(const EmbedParams prm, int log_across)
{
    after_the_kernel_before();
    using P = Piece<T, ALIGN>;
    const int across = 1 << log_across, down = kRowThreads >> log_across, D = (int)prm.cols, w = blockIdx.y, x = threadIdx.x & (across - 1);
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
    for (int c = 0; c < D; c += across * P::kWidth) {
        uint4 slice[kRowsAtATime];
        bool there[kRowsAtATime];
#pragma unroll
        for (int i = 0; i < kRowsAtATime; ++i) {
            there[i] = token[i] != prm.ignore_index && token[i] >= 0 && token[i] < prm.vocab;
            slice[i] = P::load(table + (there[i] ? token[i] : 0) * prm.weight_row, c, x, across, there[i] ? D : 0);
        }
#pragma unroll
        for (int i = 0; i < kRowsAtATime; ++i) {
            const int64_t t = t0 + i * down;
            if (t >= prm.count) break;
            float v[P::kWidth];
            widen(slice[i], v);
            // a token that names no row gives NaN
            const float factor = there[i] ? prm.scale : token[i] == prm.ignore_index ? 0.0f : __int_as_float(0x7FFFFFFF);
#pragma unroll
            for (int j = 0; j < P::kWidth; ++j) v[j] *= factor;
            P::store(out + t * prm.cols, c, x, across, D, narrow(v));
        }
    }
}

// Zeros into rows v0 .. v1 - 1 of each worker's gradient by some warps of a launch, of which this one is number `warp`: a row at a time.
template <typename T, int ALIGN>
__device__ __forceinline__ void clear_rows(const EmbedParams& prm, int64_t v0, int64_t v1, int64_t warp, int64_t warps)
{
    using P = Piece<T, ALIGN>;
    const int D = (int)prm.cols, lane = threadIdx.x % 32;
    for (int w = 0; w < prm.n; ++w) {
        T* out = static_cast<T*>(prm.dweight) + w * prm.dweight_worker;
        for (int64_t v = v0 + warp; v < v1; v += warps) {
#pragma unroll 4
            for (int c = 0; c < D; c += 32 * P::kWidth) P::store(out + v * prm.dweight_row, c, lane, 32, D, make_uint4(0, 0, 0, 0));
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------- sort
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kBins = 256;
// Items of a thread where several CTAs sort: one, so that many CTAs share them, but of very many tokens 8, as one CTA scans the CTAs' counts.
constexpr int kManyItems = 8, kMany = 1 << 18;
constexpr int kCluster = 8, kMostItems = 16, kSortHere = kCluster * kSortThreads * kMostItems;

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

// The first place of each digit out of their numbers, by one warp.
__device__ __forceinline__ void scan_bins(SortShared& sh)
{
    const int lane = threadIdx.x % 32;
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
    if (warp == 0) scan_bins(sh);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (key[i] != kNone) place[i] += sh.of_warp[warp][key[i] >> shift & mask];
}

// CTAs of a launch that have no sorting to do clear their share of the gradient: of `launches` launches this is number `launch`.  Rows that follow one
// another without gaps are one run of bytes, which goes out as copies of kZeros of shared memory (`zeros`), a few to a CTA at a time; others, element by element.
// (32768 of 131072 x 2048 bf16, 537 MB cleared and the tokens sorted: 100 us.)
constexpr int kZeros = 16384;

template <typename T, int ALIGN>
__device__ __forceinline__ void clear_meanwhile(const EmbedParams& prm, int sorting, int launch, int launches, void* zeros)
{
    if (prm.accumulate) return;
    const int64_t v0 = prm.vocab * launch / launches, v1 = prm.vocab * (launch + 1) / launches, cta = blockIdx.x - sorting, ctas = gridDim.x - sorting;
    if (prm.dweight_row != prm.cols) return clear_rows<T, ALIGN>(prm, v0, v1, cta * kSortWarps + threadIdx.x / 32, ctas * kSortWarps);
    for (int i = threadIdx.x; i < kZeros / 16; i += kSortThreads) static_cast<uint4*>(zeros)[i] = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    if (threadIdx.x >= 32) return;
    const uint32_t from = rps::smem_addr(zeros);
    for (int w = 0; w < prm.n; ++w) {
        unsigned char* const base = static_cast<unsigned char*>(prm.dweight) + w * prm.dweight_worker * (int64_t)sizeof(T);
        unsigned char *const begin = base + v0 * prm.cols * sizeof(T), *const end = base + v1 * prm.cols * sizeof(T);
        // what lies between boundaries of 16 bytes, and the elements around it
        unsigned char* const first = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(begin) + 15) / 16 * 16);
        unsigned char* const last = reinterpret_cast<unsigned char*>(reinterpret_cast<uintptr_t>(end) / 16 * 16);
        if (first > last) {  // less than 16 bytes, across no boundary
            if (cta == 0)
                for (T* p = reinterpret_cast<T*>(begin) + threadIdx.x; p < reinterpret_cast<T*>(end); p += 32) *p = from_float<T>(0.0f);
            continue;
        }
        if (cta == 0) {
            if (T* p = reinterpret_cast<T*>(begin) + threadIdx.x; p < reinterpret_cast<T*>(first)) *p = from_float<T>(0.0f);
            if (T* p = reinterpret_cast<T*>(last) + threadIdx.x; p < reinterpret_cast<T*>(end)) *p = from_float<T>(0.0f);
        }
        if (threadIdx.x < 4)
            for (unsigned char* to = first + (cta * 4 + threadIdx.x) * kZeros; to < last; to += ctas * 4 * kZeros)
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(from), "r"((uint32_t)min((int64_t)kZeros, (int64_t)(last - to)))
                             : "memory");
    }
    asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group 0;" ::: "memory");
}

__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

__device__ __forceinline__ uint32_t read_from(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void write_to(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }

// A worker's tokens sorted in shared memory: their rows, and their numbers.  CTAS of them share the tokens, ITEMS * kSortThreads each in their order.
template <int ITEMS, int CTAS>
__device__ __forceinline__ void sort_in_shared(const EmbedParams& prm, int w, SortShared& sh, uint32_t* keys, uint32_t* from)
{
    constexpr int kHere = ITEMS * kSortThreads;
    const int rank = CTAS > 1 ? (int)cluster_rank() : 0, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int count = (int)prm.count - rank * kHere;  // of this CTA and the ones behind it
    const int first = warp * 32 * ITEMS + lane;
    uint32_t key[ITEMS], token[ITEMS], place[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int t = first + i * 32;
        token[i] = (uint32_t)(rank * kHere + t);
        key[i] = t < count ? sort_key(prm, __ldg(prm.tokens + w * prm.count + rank * kHere + t)) : kNone;
    }
    for (int shift = 0; shift < prm.key_bits; shift += prm.digit_bits) {
        rank_items<ITEMS>(sh, key, place, shift, prm.digit_bits);
        const uint32_t mask = (1u << prm.digit_bits) - 1;
        if constexpr (CTAS > 1) {
            // where each digit's items begin among all CTAs', and this CTA's among those
            cluster_sync();
            uint32_t before = 0, all = 0;
            if (threadIdx.x < kBins) {
                const uint32_t mine = rps::smem_addr(&sh.total[threadIdx.x]);
#pragma unroll
                for (int c = 0; c < CTAS; ++c) {
                    const uint32_t n = read_from(in_cta(mine, c));
                    before += c < rank ? n : 0, all += n;
                }
            }
            cluster_sync();  // totals have been read, as have the keys of the pass before
            if (threadIdx.x < kBins) sh.total[threadIdx.x] = all;
            __syncthreads();
            if (warp == 0) scan_bins(sh);
            __syncthreads();
            if (threadIdx.x < kBins) sh.scan[threadIdx.x] += before;
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (key[i] == kNone) continue;
            const uint32_t to = place[i] + sh.scan[key[i] >> shift & mask];
            if constexpr (CTAS > 1) {
                const uint32_t cta = to / kHere, at = to % kHere;
                write_to(in_cta(rps::smem_addr(keys + at), cta), key[i]), write_to(in_cta(rps::smem_addr(from + at), cta), token[i]);
            } else {
                keys[to] = key[i], from[to] = token[i];
            }
        }
        if constexpr (CTAS > 1)
            cluster_sync();
        else
            __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = first + i * 32;
            if (at < count) key[i] = keys[at], token[i] = from[at];
        }
    }
}

// A worker's tokens in a cluster.
template <int ITEMS, typename T, int ALIGN>
__global__ void __launch_bounds__(kSortThreads) rps_embed_sort_kernel(const EmbedParams prm)
{
    after_the_kernel_before();
    const int w = blockIdx.x / kCluster;
    extern __shared__ __align__(16) uint32_t raw[];
    if (w >= prm.n) return clear_meanwhile<T, ALIGN>(prm, prm.n * kCluster, 0, 1, raw);
    SortShared& sh = *reinterpret_cast<SortShared*>(raw);
    constexpr int kHere = ITEMS * kSortThreads;
    uint32_t* keys = raw + sizeof(SortShared) / 4;
    uint32_t* from = keys + kHere;
    sort_in_shared<ITEMS, kCluster>(prm, w, sh, keys, from);
    const int64_t first = (int64_t)cluster_rank() * kHere, to = w * prm.count + first;
    for (int at = threadIdx.x; at < kHere && first + at < prm.count; at += kSortThreads) prm.keys[0][to + at] = keys[at], prm.from[0][to + at] = from[at];
}

// Several CTAs to a worker: how many items of each digit every block has ([digit][block] of a worker) ...
template <int ITEMS, typename T, int ALIGN>
__global__ void __launch_bounds__(kSortThreads) rps_embed_count_kernel(const EmbedParams prm, int pass, int launches)
{
    after_the_kernel_before();
    __shared__ uint32_t bins[kBins];
    __shared__ uint4 zeros[kZeros / 16];
    const int blocks = (int)prm.sort_blocks, w = blockIdx.x / blocks, block = blockIdx.x - w * blocks;
    if (w >= prm.n) return clear_meanwhile<T, ALIGN>(prm, prm.n * blocks, 3 * pass, launches, zeros);
    const int shift = pass * prm.digit_bits;
    const uint32_t mask = (1u << prm.digit_bits) - 1;
    if (threadIdx.x < kBins) bins[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t t = (int64_t)block * kSortThreads * ITEMS + i * kSortThreads + threadIdx.x;
        if (t >= prm.count) break;
        const uint32_t key = pass == 0 ? sort_key(prm, __ldg(prm.tokens + w * prm.count + t)) : prm.keys[(pass + 1) & 1][w * prm.count + t];
        atomicAdd(&bins[key >> shift & mask], 1u);
    }
    __syncthreads();
    if (threadIdx.x < kBins) prm.counts[((int64_t)w * kBins + threadIdx.x) * blocks + block] = bins[threadIdx.x];
}

// ... where each block's items of each digit begin (a CTA to a worker) ...
template <typename T, int ALIGN>
__global__ void __launch_bounds__(kSortThreads) rps_embed_scan_kernel(const EmbedParams prm, int pass, int launches)
{
    after_the_kernel_before();
    __shared__ uint4 zeros[kZeros / 16];
    if ((int)blockIdx.x >= prm.n) return clear_meanwhile<T, ALIGN>(prm, prm.n, 3 * pass + 1, launches, zeros);
    __shared__ uint32_t sums[kSortWarps];
    const int blocks = (int)prm.sort_blocks;
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
template <int ITEMS, typename T, int ALIGN>
__global__ void __launch_bounds__(kSortThreads) rps_embed_scatter_kernel(const EmbedParams prm, int pass, int launches)
{
    after_the_kernel_before();
    __shared__ __align__(16) SortShared sh;
    const int blocks = (int)prm.sort_blocks, w = blockIdx.x / blocks, block = blockIdx.x - w * blocks;
    if (w >= prm.n) return clear_meanwhile<T, ALIGN>(prm, prm.n * blocks, 3 * pass + 2, launches, &sh);
    const int shift = pass * prm.digit_bits, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const uint32_t mask = (1u << prm.digit_bits) - 1;
    const int64_t base = w * prm.count;
    uint32_t key[ITEMS], token[ITEMS], place[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t t = (int64_t)block * kSortThreads * ITEMS + warp * 32 * ITEMS + i * 32 + lane;
        const bool there = t < prm.count;
        if (pass == 0)
            token[i] = (uint32_t)t, key[i] = there ? sort_key(prm, __ldg(prm.tokens + base + t)) : kNone;
        else
            token[i] = there ? prm.from[(pass + 1) & 1][base + t] : 0, key[i] = there ? prm.keys[(pass + 1) & 1][base + t] : kNone;
    }
    rank_items<ITEMS>(sh, key, place, shift, prm.digit_bits);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (key[i] == kNone) continue;
        const uint32_t digit = key[i] >> shift & mask;
        const int64_t to = base + prm.counts[((int64_t)w * kBins + digit) * blocks + block] + place[i];
        prm.keys[pass & 1][to] = key[i], prm.from[pass & 1][to] = token[i];
    }
}

// ----------------------------------------------------------------------------------------------------------------- sum
constexpr int kSumWarps = 8;

// 512 bytes of a row of the gradient from column `first` on, a warp's.
template <typename T, int ALIGN>
__device__ __forceinline__ T* row_of(const EmbedParams& prm, int w, uint32_t row)
{
    return static_cast<T*>(prm.dweight) + w * prm.dweight_worker + (int64_t)row * prm.dweight_row;
}

// `old`: what is there, where it is added to.
template <typename T, int ALIGN>
__device__ __forceinline__ void write_row(const EmbedParams& prm, int w, uint32_t row, int first, const float (&sum)[Slice<T>::kWidth], const uint4& old)
{
    using P = Piece<T, ALIGN>;
    T* out = row_of<T, ALIGN>(prm, w, row);
    const int lane = threadIdx.x % 32;
    float v[P::kWidth];
    widen(old, v);
#pragma unroll
    for (int j = 0; j < P::kWidth; ++j) v[j] = prm.accumulate ? fmaf(prm.scale, sum[j], v[j]) : prm.scale * sum[j];
    P::store(out, first, lane, 32, (int)prm.cols, narrow(v));
}

template <typename T, int ALIGN>
__device__ __forceinline__ void write_row(const EmbedParams& prm, int w, uint32_t row, int first, const float (&sum)[Slice<T>::kWidth])
{
    using P = Piece<T, ALIGN>;
    write_row<T, ALIGN>(prm, w, row, first, sum, prm.accumulate ? P::load(row_of<T, ALIGN>(prm, w, row), first, threadIdx.x % 32, 32, (int)prm.cols) : make_uint4(0, 0, 0, 0));
}

// A warp for 512 bytes of the columns of a tile of sorted tokens.  ADD: to what is there, which is read with the tokens of a run's end.
template <typename T, int ALIGN, bool ADD>
__global__ void __launch_bounds__(32 * kSumWarps) rps_embed_sum_kernel(const EmbedParams prm, int slabs)
{
    after_the_kernel_before();
    using P = Piece<T, ALIGN>;
    constexpr int W = P::kWidth, kAtATime = 8;
    const int lane = threadIdx.x % 32, w = blockIdx.y, D = (int)prm.cols;
    const int64_t item = (int64_t)blockIdx.x * kSumWarps + threadIdx.x / 32;
    const int64_t tile = item / slabs;
    if (tile >= prm.tiles) return;
    const int first = (int)(item - tile * slabs) * 32 * W;
    const uint32_t* keys = prm.keys[prm.sorted] + w * prm.count;
    const uint32_t* from = prm.from[prm.sorted] + w * prm.count;
    const T* dout = static_cast<const T*>(prm.dout) + w * prm.count * prm.cols;
    const int64_t p0 = tile * prm.tile, p1 = min(p0 + prm.tile, prm.count);
    float* parts = prm.parts + (w * prm.tiles + tile) * 2 * prm.part_row + first + lane * W;  // (whatever columns they are)
    uint32_t current = __ldg(keys + p0);
    if (current >= prm.vocab) return;
    bool head = p0 > 0 && __ldg(keys + p0 - 1) == current;  // the run goes on from the tile before
    float sum[W];
#pragma unroll
    for (int j = 0; j < W; ++j) sum[j] = 0.0f;
    const auto store_part = [&](int slot) {
        float* to = parts + slot * prm.part_row;
#pragma unroll
        for (int j = 0; j < W; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
    };
    for (int64_t p = p0; p < p1; p += 32) {
        const bool mine = p + lane < p1;
        const uint32_t my_key = mine ? __ldg(keys + p + lane) : (uint32_t)prm.vocab, my_from = mine ? __ldg(from + p + lane) : 0;
        const int here = (int)min((int64_t)32, p1 - p);
        for (int q = 0; q < here; q += kAtATime) {
            uint4 slice[kAtATime], old[ADD ? kAtATime : 1];
            uint32_t key[kAtATime];
#pragma unroll
            for (int i = 0; i < kAtATime; ++i) {
                key[i] = __shfl_sync(0xFFFFFFFFu, my_key, q + i);
                const int64_t row = __shfl_sync(0xFFFFFFFFu, my_from, q + i);
                slice[i] = P::load(dout + row * prm.cols, first, lane, 32, key[i] < prm.vocab ? D : 0);
                if constexpr (ADD) {
                    const uint32_t ending = i > 0 ? key[i - 1] : current;
                    old[i] = P::load(row_of<T, ALIGN>(prm, w, ending < prm.vocab ? ending : 0), first, lane, 32, ending != key[i] && ending < prm.vocab ? D : 0);
                }
            }
#pragma unroll
            for (int i = 0; i < kAtATime; ++i) {
                if (key[i] != current) {
                    if (current < prm.vocab) {
                        if (head)
                            store_part(0);
                        else
                            write_row<T, ALIGN>(prm, w, current, first, sum, ADD ? old[i] : make_uint4(0, 0, 0, 0));
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
        write_row<T, ALIGN>(prm, w, current, first, sum);
}

// Runs that cross tiles: the warp of the tile that a run begins in adds its parts up.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(32 * kSumWarps) rps_embed_join_kernel(const EmbedParams prm, int slabs)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth;
    const int lane = threadIdx.x % 32, w = blockIdx.y;
    const int64_t item = (int64_t)blockIdx.x * kSumWarps + threadIdx.x / 32;
    const int64_t tile = item / slabs;
    if (tile + 1 >= prm.tiles) return;
    const uint32_t* keys = prm.keys[prm.sorted] + w * prm.count;
    const int64_t p0 = tile * prm.tile, p1 = p0 + prm.tile;
    const uint32_t key = __ldg(keys + p1);
    if (key >= prm.vocab || __ldg(keys + p1 - 1) != key) return;                                   // none crosses
    if (__ldg(keys + p0) == key && p0 > 0 && __ldg(keys + p0 - 1) == key) return;                  // it began before
    const int first = (int)(item - tile * slabs) * 32 * W;
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
    float sum[W];
    const float* parts = prm.parts + w * prm.tiles * 2 * prm.part_row + first + lane * W;
    const auto add = [&](int64_t t, int slot, bool start) {
        const float* at = parts + (t * 2 + slot) * prm.part_row;
#pragma unroll
        for (int j = 0; j < W; j += 4) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(at + j));
            sum[j] = start ? v.x : sum[j] + v.x, sum[j + 1] = start ? v.y : sum[j + 1] + v.y;
            sum[j + 2] = start ? v.z : sum[j + 2] + v.z, sum[j + 3] = start ? v.w : sum[j + 3] + v.w;
        }
    };
    add(tile, 1, true);
#pragma unroll 16
    for (int64_t t = tile + 1; t <= last; ++t) add(t, 0, false);
    write_row<T, ALIGN>(prm, w, key, first, sum);
}

// ----------------------------------------------------------------------------------------------------------------- few
// All in one launch: every CTA sorts its worker's tokens and takes rows v0 .. v1 - 1 of the gradient (or, where it is added to, a share of the
// runs), a warp to 512 bytes of a row.
constexpr int kFew = 512, kFewRows = 4096;

template <typename T, int ALIGN>
__global__ void __launch_bounds__(kSortThreads) rps_embed_few_kernel(const EmbedParams prm, int slabs)
{
    after_the_kernel_before();
    using P = Piece<T, ALIGN>;
    constexpr int W = P::kWidth, kAtATime = 8;
    __shared__ union {
        SortShared sort;
        unsigned short start[kFewRows];  // of a row's run, kFew: none
    } sh;
    __shared__ uint32_t keys[kSortThreads], from[kSortThreads];
    const int w = blockIdx.y, count = (int)prm.count, lane = threadIdx.x % 32, warp = threadIdx.x / 32, D = (int)prm.cols;
    sort_in_shared<1, 1>(prm, w, sh.sort, keys, from);
    const T* dout = static_cast<const T*>(prm.dout) + w * prm.count * prm.cols;
    const auto sum_run = [&](int p, int first) {
        const uint32_t row = keys[p];
        float sum[W];
#pragma unroll
        for (int j = 0; j < W; ++j) sum[j] = 0.0f;
        for (bool on = true; on;) {
            uint4 slice[kAtATime];
#pragma unroll
            for (int i = 0; i < kAtATime; ++i, ++p) {
                on = on && p < count && keys[p] == row;
                slice[i] = P::load(dout + (on ? (int64_t)from[p] : 0) * prm.cols, first, lane, 32, on ? D : 0);
            }
#pragma unroll
            for (int i = 0; i < kAtATime; ++i) {
                float v[W];
                widen(slice[i], v);
#pragma unroll
                for (int j = 0; j < W; ++j) sum[j] += v[j];
            }
        }
        write_row<T, ALIGN>(prm, w, row, first, sum);
    };
    if (prm.accumulate) {
        __syncthreads();
        for (int item = blockIdx.x * kSortWarps + warp; item < count * slabs; item += gridDim.x * kSortWarps) {
            const int p = item / slabs;
            if (keys[p] < prm.vocab && (p == 0 || keys[p - 1] != keys[p])) sum_run(p, (item - p * slabs) * 32 * W);
        }
        return;
    }
    const int64_t v0 = prm.vocab * blockIdx.x / gridDim.x, v1 = prm.vocab * (blockIdx.x + 1) / gridDim.x;
    for (int64_t v = v0; v < v1; v += kFewRows) {
        const int rows = (int)min((int64_t)kFewRows, v1 - v);
        __syncthreads();
        for (int i = threadIdx.x; i < rows; i += kSortThreads) sh.start[i] = kFew;
        __syncthreads();
        if ((int)threadIdx.x < count) {
            const int p = threadIdx.x;
            const int64_t row = (int64_t)keys[p] - v;
            if (row >= 0 && row < rows && (p == 0 || keys[p - 1] != keys[p])) sh.start[row] = (unsigned short)p;
        }
        __syncthreads();
        for (int64_t item = warp; item < (int64_t)rows * slabs; item += kSortWarps) {
            const int row = (int)(item / slabs), first = (int)(item - (int64_t)row * slabs) * 32 * W, p = sh.start[row];
            if (p < kFew)
                sum_run(p, first);
            else
                P::store(static_cast<T*>(prm.dweight) + w * prm.dweight_worker + (v + row) * prm.dweight_row, first, lane, 32, D, make_uint4(0, 0, 0, 0));
        }
    }
}

template <typename T, int ALIGN>
__global__ void __launch_bounds__(kSortThreads) rps_embed_clear_kernel(const EmbedParams prm)
{
    after_the_kernel_before();
    __shared__ uint4 zeros[kZeros / 16];
    clear_meanwhile<T, ALIGN>(prm, 0, 0, 1, zeros);
}

// ---------------------------------------------------------------------------------------------------------------- host
int log_threads_across(int64_t cols, int width)
{
    int log = 0;
    while (log < 8 && (width << log) < cols) ++log;
    return log;
}

// Bytes that every row's address is a multiple of, and its length.
template <typename T>
int row_alignment(const void* p, int64_t cols, int64_t row, int64_t worker)
{
    const uint64_t bits = reinterpret_cast<uintptr_t>(p) | (uint64_t)(cols | row | worker) * sizeof(T);
    return bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 2;
}

template <typename T, int ALIGN>
cudaError_t lookup(const EmbedParams& prm, cudaStream_t stream)
{
    const int log = log_threads_across(prm.cols, Slice<T>::kWidth);
    const dim3 grid((unsigned)ceil_div(prm.count, (kRowThreads >> log) * kRowsAtATime), (unsigned)prm.n);
    return launch_after(rps_embed_lookup_kernel<T, ALIGN>, grid, kRowThreads, 0, stream, 1, prm, log);
}

// CTAs that clear beside those that sort.  Clusters of eight are placed whole, two to a group of SMs that has room for them: 16 at a time; with three
// more the clearing took two rounds (126 us instead of 100).
unsigned clusters_with_clearing(const EmbedParams& prm) { return (unsigned)(kCluster * (prm.n + (prm.accumulate ? 0 : std::max(16 - prm.n, 4)))); }
unsigned with_clearing(const EmbedParams& prm, int64_t sorting) { return (unsigned)(sorting + (prm.accumulate ? 0 : std::max<int64_t>(kSms - sorting, kSms / 2))); }

template <int ITEMS, typename T, int ALIGN>
cudaError_t sort_here(const EmbedParams& prm, cudaStream_t stream)
{
    static rps::LaunchState state;
    const uint32_t bytes = sizeof(SortShared) + kSortThreads * ITEMS * 8;
    const cudaError_t err = rps::grant_smem(state, rps_embed_sort_kernel<ITEMS, T, ALIGN>, bytes);
    if (err != cudaSuccess) return err;
    return launch_after(rps_embed_sort_kernel<ITEMS, T, ALIGN>, dim3(clusters_with_clearing(prm)), kSortThreads, bytes, stream, kCluster, prm);
}

template <int ITEMS, typename T, int ALIGN>
cudaError_t sort_in_passes(const EmbedParams& prm, cudaStream_t stream)
{
    const int passes = (int)ceil_div(prm.key_bits, prm.digit_bits);
    const dim3 grid(with_clearing(prm, prm.n * prm.sort_blocks)), scan(with_clearing(prm, prm.n));
    cudaError_t err = cudaSuccess;
    for (int pass = 0; pass < passes && err == cudaSuccess; ++pass) {
        err = launch_after(rps_embed_count_kernel<ITEMS, T, ALIGN>, grid, kSortThreads, 0, stream, 1, prm, pass, 3 * passes);
        if (err == cudaSuccess) err = launch_after(rps_embed_scan_kernel<T, ALIGN>, scan, kSortThreads, 0, stream, 1, prm, pass, 3 * passes);
        if (err == cudaSuccess) err = launch_after(rps_embed_scatter_kernel<ITEMS, T, ALIGN>, grid, kSortThreads, 0, stream, 1, prm, pass, 3 * passes);
    }
    return err;
}

template <typename T, int ALIGN>
cudaError_t sort(const EmbedParams& prm, cudaStream_t stream)
{
    constexpr int kOnce = kCluster * kSortThreads;
    if (prm.count <= kOnce) return sort_here<1, T, ALIGN>(prm, stream);
    if (prm.count <= kOnce * 4) return sort_here<4, T, ALIGN>(prm, stream);
    if (prm.count <= kSortHere) return sort_here<kMostItems, T, ALIGN>(prm, stream);
    return prm.count <= kMany ? sort_in_passes<1, T, ALIGN>(prm, stream) : sort_in_passes<kManyItems, T, ALIGN>(prm, stream);
}

template <typename T, int ALIGN>
cudaError_t gradient(const EmbedParams& prm, cudaStream_t stream)
{
    const int slabs = (int)ceil_div(prm.cols, 32 * Slice<T>::kWidth);
    if (prm.count == 0) {
        if (prm.accumulate) return cudaSuccess;
        return launch_after(rps_embed_clear_kernel<T, ALIGN>, dim3(2 * kSms), kSortThreads, 0, stream, 1, prm);
    }
    if (prm.count <= kFew) {
        const int64_t items = prm.accumulate ? prm.count * slabs : prm.vocab * slabs;
        const int64_t ctas = std::max<int64_t>(1, std::min(ceil_div(items, kSortWarps), ceil_div((int64_t)2 * kSms, prm.n)));
        return launch_after(rps_embed_few_kernel<T, ALIGN>, dim3((unsigned)ctas, (unsigned)prm.n), kSortThreads, 0, stream, 1, prm, slabs);
    }
    cudaError_t err = sort<T, ALIGN>(prm, stream);
    if (err != cudaSuccess) return err;
    const dim3 grid((unsigned)ceil_div(prm.tiles * slabs, kSumWarps), (unsigned)prm.n);
    const auto sum = prm.accumulate ? rps_embed_sum_kernel<T, ALIGN, true> : rps_embed_sum_kernel<T, ALIGN, false>;
    if ((err = launch_after(sum, grid, 32 * kSumWarps, 0, stream, 1, prm, slabs)) != cudaSuccess || prm.tiles == 1) return err;
    return launch_after(rps_embed_join_kernel<T, ALIGN>, grid, 32 * kSumWarps, 0, stream, 1, prm, slabs);
}

// The kernels for rows of this alignment.
#define RPS_BY_ALIGNMENT(function, align)                                                                        \
    (prm.f32 ? ((align) == 16  ? function<float, 16>(prm, stream)                                                \
                : (align) == 8 ? function<float, 8>(prm, stream)                                                 \
                               : function<float, 4>(prm, stream))                                                \
             : ((align) == 16  ? function<bf16, 16>(prm, stream)                                                 \
                : (align) == 8 ? function<bf16, 8>(prm, stream)                                                  \
                : (align) == 4 ? function<bf16, 4>(prm, stream)                                                  \
                               : function<bf16, 2>(prm, stream)))

int alignment_of(const EmbedParams& prm, const void* dense, const void* rows, int64_t row, int64_t worker)
{
    return prm.f32 ? std::min(row_alignment<float>(dense, prm.cols, 0, 0), row_alignment<float>(rows, prm.cols, row, worker))
                   : std::min(row_alignment<bf16>(dense, prm.cols, 0, 0), row_alignment<bf16>(rows, prm.cols, row, worker));
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
    p.sort_blocks = p.count <= kSortHere ? 0 : ceil_div(p.count, kSortThreads * (p.count <= kMany ? 1 : kManyItems));
    const int width = p.f32 ? Slice<float>::kWidth : Slice<bf16>::kWidth;
    const int64_t slabs = ceil_div(p.cols, 32 * width);
    // long tiles leave fewer parts, short ones more warps
    p.tile = 256;
    while (p.tile > 16 && p.n * ceil_div(p.count, p.tile) * slabs < kSms * 24) p.tile /= 2;
    p.tiles = p.count <= kFew ? 1 : ceil_div(p.count, p.tile);
    p.part_row = slabs * 32 * width;
}

cudaError_t launch_embed_lookup(const EmbedParams& prm, cudaStream_t stream)
{
    const int align = alignment_of(prm, prm.out, prm.weight, prm.weight_row, prm.weight_worker);
    return RPS_BY_ALIGNMENT(lookup, align);
}

cudaError_t launch_embed_gradient(const EmbedParams& prm, cudaStream_t stream)
{
    const int align = alignment_of(prm, prm.dout, prm.dweight, prm.dweight_row, prm.dweight_worker);
    return RPS_BY_ALIGNMENT(gradient, align);
}

}  // namespace rps_ops
