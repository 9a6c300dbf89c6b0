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

#include "rps_kernels.h"
#include "rps_rows.cuh"

namespace rps_ops {
namespace {

constexpr int kMostThreads = 512;
constexpr int kSlots = 4, kAhead = kSlots - 1;      // rows in shared memory: this one and those ahead
constexpr int kForwardThreads = 1024, kBackwardThreads = 512;  // resident on an SM: 48 KB and 40 KB of slots for each row
constexpr int kMostCluster = 8;
constexpr int kMostWarps = kMostThreads / 32 * kMostCluster;

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// Sums of N values over the threads that share a row.  `slots` is double-buffered over successive calls (`turn`), so
// that one barrier a call is enough.  Every thread gets the sums, added in the same order.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*slots)[N][kMostWarps], int turn, int cluster, uint32_t rank)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int s = 16; s > 0; s /= 2) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], s);
    const int warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (warps * cluster == 1) return;
    if (cluster == 1) {
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) slots[turn][i][warp] = v[i];
        }
        __syncthreads();
    } else {
        if (lane < cluster) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t own = (uint32_t)__cvta_generic_to_shared(&slots[turn][i][rank * warps + warp]);
                uint32_t there;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(own), "r"(lane));
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v[i]) : "memory");
            }
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    }
    const int slots_used = warps * cluster;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float s = 0.0f;
        for (int k = lane; k < slots_used; k += 32) s += slots[turn][i][k];
#pragma unroll
        for (int k = 16; k > 0; k /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, k);
        v[i] = s;
    }
}

// This thread's slots: `arrays` of 16 bytes for each row of the ring.
template <int ARRAYS>
__device__ __forceinline__ uint32_t slot_of(uint32_t slots, int turn, int array)
{
    return slots + ((uint32_t)(turn * ARRAYS + array) * blockDim.x + threadIdx.x) * 16;
}

template <typename T, int ALIGN, bool PACK>
__global__ void __launch_bounds__(kMostThreads, kForwardThreads / kMostThreads) rps_norm_forward_kernel(const NormParams prm)
{
    constexpr int W = Slice<T>::kWidth;
    extern __shared__ uint4 ring[];
    __shared__ float slots[2][1][kMostWarps];
    const uint32_t copied = (uint32_t)__cvta_generic_to_shared(ring);
    const int cluster = prm.cluster, D = (int)prm.cols;
    const uint32_t rank = cluster > 1 ? cluster_rank() : 0;
    const int c = ((int)rank * blockDim.x + threadIdx.x) * W;
    const uint32_t rows = (uint32_t)(prm.n * prm.tokens), step = gridDim.x / cluster, tokens = (uint32_t)prm.tokens;
    const float inv = 1.0f / (float)D;
    int into = 0;
    const auto send = [&](uint32_t r) {
        if (r < rows) {
            const uint32_t w = r / tokens, g = (r - w * tokens) / (uint32_t)prm.rows_per_gate;
            copy_slice<T, ALIGN>(slot_of<3>(copied, into, 0), static_cast<const T*>(prm.x) + (int64_t)r * D, c, D);
            copy_slice<T, ALIGN>(slot_of<3>(copied, into, 1), static_cast<const T*>(prm.f) + (int64_t)r * D, c, D);
            copy_slice<T, ALIGN>(slot_of<3>(copied, into, 2), static_cast<const T*>(prm.gate) + w * prm.gate_worker + (int64_t)g * D, c, D);
        }
        copies_sent();
        into = into + 1 == kSlots ? 0 : into + 1;
    };
    uint32_t row = blockIdx.x / cluster;
    for (int i = 0; i < kAhead; ++i) send(row + i * step);
    int turn = 0, from = 0;
    for (; row < rows; row += step) {
        float x[W], f[W], gate[W], post[W], pre[W];
        const uint32_t w = row / tokens;
        const uint4 post_slice = load_slice<T, ALIGN, false>(static_cast<const T*>(prm.post) + w * prm.post_worker, c, D);
        const uint4 pre_slice = load_slice<T, ALIGN, false>(static_cast<const T*>(prm.pre) + w * prm.pre_worker, c, D);
        send(row + kAhead * step);
        copies_arrived<kAhead>();
        widen(read_slot(slot_of<3>(copied, from, 0)), x);
        widen(read_slot(slot_of<3>(copied, from, 1)), f);
        widen(read_slot(slot_of<3>(copied, from, 2)), gate);
        from = from + 1 == kSlots ? 0 : from + 1;
        widen(post_slice, post), widen(pre_slice, pre);
        float s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < W; ++j) s[0] = fmaf(f[j], f[j], s[0]);
        row_sums<1>(s, slots, turn, cluster, rank), turn ^= 1;
        const float r_f = rsqrtf(fmaf(s[0], inv, prm.eps));
        if constexpr (PACK) {
            const bool in = c < prm.pitch;
            pack_slice(f, in ? prm.f_codes + (int64_t)row * prm.pitch + c : nullptr, c < D ? prm.f_scales + (int64_t)row * prm.groups + c / RPS_PACK_GROUP : nullptr);
        }
        s[0] = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            x[j] = fmaf(prm.scale * gate[j], f[j] * r_f * post[j], x[j]);  // h
            s[0] = fmaf(x[j], x[j], s[0]);
        }
        const uint4 h = narrow(x);
        store_slice<T, ALIGN>(static_cast<T*>(prm.h) + (int64_t)row * D, c, D, h);
        row_sums<1>(s, slots, turn, cluster, rank), turn ^= 1;
        const float r_h = rsqrtf(fmaf(s[0], inv, prm.eps));
        if constexpr (PACK) {
            float stored[W];  // as a reader of h sees it
            widen(h, stored);
            if constexpr (ALIGN != 16) {
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (c + j >= D) stored[j] = 0.0f;
            }
            pack_slice(stored, c < prm.pitch ? prm.h_codes + (int64_t)row * prm.pitch + c : nullptr,
                       c < D ? prm.h_scales + (int64_t)row * prm.groups + c / RPS_PACK_GROUP : nullptr);
        }
#pragma unroll
        for (int j = 0; j < W; ++j) x[j] = x[j] * r_h * pre[j];
        store_slice<T, ALIGN>(static_cast<T*>(prm.y) + (int64_t)row * D, c, D, narrow(x));
        if (prm.r_f != nullptr && rank == 0 && threadIdx.x == 0) {
            prm.r_f[row] = r_f;
            prm.r_h[row] = r_h;
        }
    }
    // another CTA's sums may still be on their way here
    if (cluster > 1) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

template <typename T, int ALIGN, bool PACKED>
__global__ void __launch_bounds__(kMostThreads, kBackwardThreads / kMostThreads) rps_norm_backward_kernel(const NormParams prm)
{
    constexpr int W = Slice<T>::kWidth;
    extern __shared__ uint4 ring[];
    __shared__ float slots[2][3][kMostWarps];
    const uint32_t copied = (uint32_t)__cvta_generic_to_shared(ring);
    const int cluster = prm.cluster, D = (int)prm.cols;
    const uint32_t rank = cluster > 1 ? cluster_rank() : 0;
    const int c = ((int)rank * blockDim.x + threadIdx.x) * W;
    const float inv = 1.0f / (float)D;
    const int64_t block = blockIdx.x / cluster, w = blockIdx.y;
    int64_t first, end;
    if (prm.chunks > 0) {
        const int64_t g = block / prm.chunks;
        first = g * prm.rows_per_gate + block % prm.chunks * prm.rows_per_block;
        end = min(first + prm.rows_per_block, (g + 1) * prm.rows_per_gate);
    } else {
        first = block * prm.rows_per_block;
        end = min(first + prm.rows_per_block, prm.tokens);
    }
    const uint4 post_slice = load_slice<T, ALIGN, false>(static_cast<const T*>(prm.post) + w * prm.post_worker, c, D);
    const uint4 pre_slice = load_slice<T, ALIGN, false>(static_cast<const T*>(prm.pre) + w * prm.pre_worker, c, D);
    float dpost[W] = {}, dpre[W] = {}, dgate[W] = {};

    float rf_next = 0.0f, rh_next = 0.0f;
    int64_t gate_row = first / prm.rows_per_gate, in_gate = first - gate_row * prm.rows_per_gate;  // of the next row to be copied
    int64_t left_in_gate = prm.rows_per_gate - in_gate;
    int into = 0;
    const auto send = [&](int64_t t) {
        if (t < end) {
            const int64_t r = w * prm.tokens + t;
            copy_slice<T, ALIGN>(slot_of<5>(copied, into, 0), static_cast<const T*>(prm.dy) + r * D, c, D);
            if (prm.dh != nullptr) copy_slice<T, ALIGN>(slot_of<5>(copied, into, 1), static_cast<const T*>(prm.dh) + r * D, c, D);
            copy_slice<T, ALIGN>(slot_of<5>(copied, into, 2), static_cast<const T*>(prm.gate) + w * prm.gate_worker + gate_row * D, c, D);
            if constexpr (PACKED) {  // the codes, and behind them the scale
                const bool in = c < D;
                const int64_t at = in ? r * prm.pitch + c : 0, group = in ? r * prm.groups + c / RPS_PACK_GROUP : 0;
                copy_async<W>(slot_of<5>(copied, into, 3), static_cast<const int8_t*>(prm.f) + at, in);
                copy_async<4>(slot_of<5>(copied, into, 3) + 8, prm.f_scales + group, in);
                copy_async<W>(slot_of<5>(copied, into, 4), static_cast<const int8_t*>(prm.h_in) + at, in);
                copy_async<4>(slot_of<5>(copied, into, 4) + 8, prm.h_scales + group, in);
            } else {
                copy_slice<T, ALIGN>(slot_of<5>(copied, into, 3), static_cast<const T*>(prm.f) + r * D, c, D);
                copy_slice<T, ALIGN>(slot_of<5>(copied, into, 4), static_cast<const T*>(prm.h_in) + r * D, c, D);
            }
            if (++in_gate == prm.rows_per_gate) in_gate = 0, ++gate_row;
        }
        copies_sent();
        into = into + 1 == kSlots ? 0 : into + 1;
    };
    const auto kept = [&](int from, int array, float (&v)[W]) {
        const uint4 slot = read_slot(slot_of<5>(copied, from, array));
        if constexpr (PACKED) {
            Codes<W> codes;
            codes.w[0] = slot.x;
            if constexpr (W == 8) codes.w[1] = slot.y;
            codes.values(__uint_as_float(slot.z), v);
        } else {
            widen(slot, v);
        }
    };
    const auto statistics = [&](int64_t t) {
        if (t < end) rf_next = __ldg(prm.r_f + w * prm.tokens + t), rh_next = __ldg(prm.r_h + w * prm.tokens + t);
    };
    for (int i = 0; i < kAhead; ++i) send(first + i);
    statistics(first);
    int turn = 0, from = 0;
    for (int64_t t = first; t < end; ++t) {
        const int64_t row = w * prm.tokens + t;
        float f[W], h[W], dy[W], dx[W] = {}, gate[W], post[W];
        send(t + kAhead);
        copies_arrived<kAhead>();
        widen(read_slot(slot_of<5>(copied, from, 0)), dy);
        if (prm.dh != nullptr) widen(read_slot(slot_of<5>(copied, from, 1)), dx);
        widen(read_slot(slot_of<5>(copied, from, 2)), gate);
        kept(from, 3, f), kept(from, 4, h);
        from = from + 1 == kSlots ? 0 : from + 1;
        widen(post_slice, post);
        const float r_f = rf_next, r_h = rh_next;
        statistics(t + 1);
        float s[3] = {};
        {
            float pre[W];
            widen(pre_slice, pre);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                dpre[j] = fmaf(dy[j], h[j] * r_h, dpre[j]);
                const float a = dy[j] * pre[j], q = prm.scale * gate[j] * post[j] * f[j];
                dx[j] = fmaf(r_h, a, dx[j]);  // dh + r_h a
                s[0] = fmaf(a, h[j], s[0]);
                s[1] = fmaf(q, dx[j], s[1]);
                s[2] = fmaf(q, h[j], s[2]);
            }
        }
        row_sums<3>(s, slots, turn, cluster, rank), turn ^= 1;
        const float mean_h = s[0] * inv * r_h * r_h * r_h;
        const float mean_f = (s[1] - mean_h * s[2]) * inv * r_f * r_f;
        float df[W];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            dx[j] = fmaf(-h[j], mean_h, dx[j]);
            const float g = prm.scale * dx[j], n = f[j] * r_f;
            dgate[j] = fmaf(g, n * post[j], dgate[j]);
            dpost[j] = fmaf(g * gate[j], n, dpost[j]);
            df[j] = r_f * (g * gate[j] * post[j] - f[j] * mean_f);
        }
        store_slice<T, ALIGN>(static_cast<T*>(prm.dx) + row * D, c, D, narrow(dx));
        store_slice<T, ALIGN>(static_cast<T*>(prm.df) + row * D, c, D, narrow(df));
        if (--left_in_gate == 0) {
            left_in_gate = prm.rows_per_gate;
            if (prm.chunks == 0) {  // the block held the whole gate group
                store_slice<T, ALIGN>(static_cast<T*>(prm.dgate) + (w * prm.gates + t / prm.rows_per_gate) * D, c, D, narrow(dgate));
#pragma unroll
                for (int j = 0; j < W; ++j) dgate[j] = 0.0f;
            }
        }
    }
    float* partial = prm.partial + (w * prm.blocks + block) * 3 * D;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        if (c + j < D) {
            partial[c + j] = dpost[j];
            partial[D + c + j] = dpre[j];
            if (prm.chunks > 0) partial[2 * D + c + j] = dgate[j];
        }
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// Sums of the blocks' sums: 32 columns to a CTA, the blocks dealt to its 16 warps, whose sums are added in their order.
template <typename T>
__global__ void __launch_bounds__(512) rps_norm_reduce_kernel(const NormParams prm)
{
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

// Threads of a CTA and CTAs of a cluster for a row of `slices` 16-byte slices: the fewest threads (a power of two of
// warps) that hold it, up to 512, then a cluster.
void shape_of_row(int64_t slices, int* threads, int* cluster)
{
    *threads = 32, *cluster = 1;
    while (*threads < kMostThreads && *threads < slices) *threads *= 2;
    while (*threads * *cluster < slices) *cluster *= 2;
}

// `arrays` slices of each of kSlots rows to a thread in shared memory.
template <typename Kernel>
cudaError_t launch_rows(rps::LaunchState& state, Kernel kernel, const NormParams& prm, dim3 grid, int threads, int arrays, cudaStream_t stream)
{
    const uint32_t bytes = (uint32_t)(threads * 16 * arrays * kSlots);
    cudaError_t err = rps::grant_smem(state, kernel, bytes);
    if (err != cudaSuccess) return err;
    cudaLaunchConfig_t config{};
    config.gridDim = grid, config.blockDim = dim3((unsigned)threads), config.dynamicSmemBytes = bytes, config.stream = stream;
    cudaLaunchAttribute attribute{};
    attribute.id = cudaLaunchAttributeClusterDimension;
    attribute.val.clusterDim.x = (unsigned)prm.cluster, attribute.val.clusterDim.y = attribute.val.clusterDim.z = 1;
    config.attrs = &attribute, config.numAttrs = prm.cluster > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&config, kernel, prm);
}

template <typename T, int ALIGN, bool PACK>
cudaError_t run_forward(const NormParams& prm, dim3 grid, int threads, cudaStream_t stream)
{
    static rps::LaunchState state;
    return launch_rows(state, rps_norm_forward_kernel<T, ALIGN, PACK>, prm, grid, threads, 3, stream);
}

template <typename T, int ALIGN, bool PACKED>
cudaError_t run_backward(const NormParams& prm, dim3 grid, int threads, cudaStream_t stream)
{
    static rps::LaunchState state;
    return launch_rows(state, rps_norm_backward_kernel<T, ALIGN, PACKED>, prm, grid, threads, 5, stream);
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
    shape_of_row(ceil_div(pack ? prm.pitch : prm.cols, Slice<T>::kWidth), &threads, &prm.cluster);
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
    shape_of_row(ceil_div(prm.cols, Slice<T>::kWidth), &threads, &prm.cluster);
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
    rps_norm_reduce_kernel<T><<<dim3((unsigned)ceil_div(prm.cols, 32), (unsigned)(jobs < 4096 ? jobs : 4096), (unsigned)prm.n), 512, 0, stream>>>(prm);
    return cudaGetLastError();
}

}  // namespace

void plan_norm_backward(NormParams* prm)
{
    int threads = 0, cluster = 0;
    shape_of_row(ceil_div(prm->cols, prm->f32 ? Slice<float>::kWidth : Slice<bf16>::kWidth), &threads, &cluster);
    // as many blocks over all workers as are resident at once (512 threads of each of the 148 SMs); of the two nearest ways
    // to cut the rows the one whose longest SM has fewer of them
    int64_t want = (int64_t)148 * (kBackwardThreads / threads) / cluster / prm->n;
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
