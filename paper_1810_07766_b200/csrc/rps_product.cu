// Matrix products of the training operators with their epilogues.
#include "rps_ops_kernels.h"

namespace rps_ops {
namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;

__device__ __forceinline__ float element(const Operand& o, int worker, int planes, int64_t row, int64_t col)
{
    if (row >= o.rows || col >= o.cols) return 0.0f;
    const bf16* p = o.base + worker * o.worker + row * o.row + col;
    float v = 0.0f;
    for (int i = 0; i < planes; ++i) v += __bfloat162float(p[i * o.plane]);
    return v;
}

template <Product WHICH>
__global__ void __launch_bounds__(kThreads) rps_product_kernel(const ProductParams prm)
{
    __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1], sc[kTile][kTile + 1];
    const int w = blockIdx.z, m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
    const int count = prm.count != nullptr ? prm.count[w] : (WHICH == Product::kDweight ? prm.k : prm.m);
    const int m_end = WHICH == Product::kDweight ? prm.m : count;
    const int k_end = WHICH == Product::kDweight ? count : prm.k;
    // dl is cleared up to the end of the last token tile that holds a row
    const int m_tiles = WHICH == Product::kDlogits ? (m_end + kTokenTile - 1) / kTokenTile * kTokenTile : m_end;
    if (m0 >= m_tiles) return;
    float c[4][4] = {};
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (int k0 = 0; k0 < k_end; k0 += kDepth) {
        for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
            const int r = i / kDepth, k = i % kDepth;
            const bool in = k0 + k < k_end;
            sa[k][r] = !in || m0 + r >= m_end ? 0.0f
                       : WHICH == Product::kDweight ? element(prm.a, w, prm.planes, k0 + k, m0 + r)
                                                    : element(prm.a, w, prm.planes, m0 + r, k0 + k);
            sb[k][r] = !in ? 0.0f
                       : WHICH == Product::kDweight || WHICH == Product::kDhidden ? element(prm.b, w, prm.planes, k0 + k, n0 + r)
                                                                                  : element(prm.b, w, prm.planes, n0 + r, k0 + k);
        }
        __syncthreads();
        for (int k = 0; k < kDepth; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) c[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], c[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) sc[ty * 4 + i][tx * 4 + j] = c[i][j];
    __syncthreads();
    if (threadIdx.x >= kTile) return;
    const int row = m0 + threadIdx.x;
    const float* v = sc[threadIdx.x];
    const int cols = min(kTile, (WHICH == Product::kLse || WHICH == Product::kDlogits ? prm.vocab - prm.v0 : prm.n) - n0);
    if constexpr (WHICH == Product::kLse) {
        if (row >= count) return;
        float top = -INFINITY, sum = 0.0f;
        for (int j = 0; j < cols; ++j) top = fmaxf(top, v[j]);
        const float at = top == -INFINITY ? 0.0f : top;
        for (int j = 0; j < cols; ++j) sum += __expf(v[j] - at);
        prm.part[((int64_t)w * prm.vocab_tiles + (prm.v0 + n0) / kVocabTile) * prm.tokens_padded + row] = make_float2(top, sum);
        const int t = prm.target[w * prm.tokens_padded + row] - prm.v0 - n0;
        if (t >= 0 && t < cols) prm.hit[w * prm.tokens_padded + row] = v[t];
    } else if constexpr (WHICH == Product::kDlogits) {
        bf16* dl = prm.dl + ((int64_t)w * prm.planes * prm.tokens_padded + row) * prm.piece + n0;
        const float2 info = row < count ? prm.info[w * prm.tokens_padded + row] : make_float2(0.0f, 0.0f);
        const int t = row < count ? prm.target[w * prm.tokens_padded + row] - prm.v0 - n0 : -1;
        for (int j = 0; j < kTile && n0 + j < prm.piece; ++j) {
            const float d = row < count && j < cols ? info.y * (__expf(v[j] - info.x) - (j == t ? 1.0f : 0.0f)) : 0.0f;
            if (prm.planes == 1) {
                dl[j] = __float2bfloat16_rn(d);
            } else {
                bf16 p[3];
                split_planes(d, p);
                for (int q = 0; q < 3; ++q) dl[q * prm.tokens_padded * prm.piece + j] = p[q];
            }
        }
    } else if constexpr (WHICH == Product::kDhidden) {
        if (row >= count) return;
        float* acc = prm.acc + (w * prm.tokens_padded + row) * prm.n + n0;
        const int64_t at = w * prm.out_worker + (int64_t)prm.rows[w * prm.tokens + row] * prm.out_row + n0;
        for (int j = 0; j < cols; ++j) {
            const float s = prm.first ? v[j] : acc[j] + v[j];
            if (!prm.last)
                acc[j] = s;
            else if (prm.out_f32)
                static_cast<float*>(prm.out)[at + j] = s;
            else
                static_cast<bf16*>(prm.out)[at + j] = __float2bfloat16_rn(s);
        }
    } else {
        if (row >= prm.m) return;
        const int64_t at = w * prm.out_worker + (int64_t)(prm.v0 + row) * prm.out_row + n0;
        for (int j = 0; j < cols; ++j) {
            if (prm.out_f32)
                static_cast<float*>(prm.out)[at + j] = v[j];
            else
                static_cast<bf16*>(prm.out)[at + j] = __float2bfloat16_rn(v[j]);
        }
    }
}

}  // namespace

cudaError_t launch_product(Product which, const ProductParams& prm, cudaStream_t stream)
{
    const dim3 grid((unsigned)ceil_div(prm.n, kTile), (unsigned)ceil_div(prm.m, kTile), (unsigned)prm.workers);
    switch (which) {
        case Product::kLse: rps_product_kernel<Product::kLse><<<grid, kThreads, 0, stream>>>(prm); break;
        case Product::kDlogits: rps_product_kernel<Product::kDlogits><<<grid, kThreads, 0, stream>>>(prm); break;
        case Product::kDhidden: rps_product_kernel<Product::kDhidden><<<grid, kThreads, 0, stream>>>(prm); break;
        case Product::kDweight: rps_product_kernel<Product::kDweight><<<grid, kThreads, 0, stream>>>(prm); break;
    }
    return cudaGetLastError();
}

}  // namespace rps_ops
