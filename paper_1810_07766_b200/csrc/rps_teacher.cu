// Distillation's teacher: of each token's kept logits the probabilities, sorted by word, so that the products' epilogues meet those of their
// columns in order, and where those of each of kTopBuckets equal parts of the vocabulary begin, so that an epilogue need not search all of them
// for its first.  A warp to a token, its entries in registers (element e in lane e % 32), sorted by a bitonic network.  Bound by reading the
// entries and writing them back.
#include "rps_ops_kernels.h"

namespace rps_ops {
namespace {

constexpr int kThreads = 256;
constexpr int kNoWord = 0x7FFFFFFF;

__device__ __forceinline__ float load_logit(const void* logits, int f32, int64_t i)
{
    return f32 ? __ldcs(static_cast<const float*>(logits) + i) : __bfloat162float(static_cast<const bf16*>(logits)[i]);
}

// PER: 32 entries each.
template <int PER>
__global__ void __launch_bounds__(kThreads) rps_teacher_kernel(const TeacherParams prm)
{
    after_the_kernel_before();
    const int lane = threadIdx.x % 32;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (t >= prm.n * prm.tokens) return;
    const int64_t first = t * prm.top;
    int id[PER];
    float x[PER];
    bool wrong = false;
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int e = r * 32 + lane;
        id[r] = kNoWord, x[r] = -INFINITY;
        if (e >= prm.top) continue;
        const int64_t word = __ldcs(prm.ids + first + e);
        if (word == prm.ignore_index) continue;
        if (word < 0 || word >= prm.vocab) {
            wrong = true;
            continue;
        }
        x[r] = load_logit(prm.logits, prm.top_f32, first + e);
        wrong = wrong || !(x[r] < INFINITY);
        if (x[r] != -INFINITY) id[r] = (int)word;
        top = fmaxf(top, x[r]);
    }
    wrong = __any_sync(0xFFFFFFFFu, wrong);
#pragma unroll
    for (int s = 16; s > 0; s /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
    const bool none = top == -INFINITY;
    float e[PER], sum = 0.0f;
    // differences before the temperature: they may be exact where logits divided by it are not, or are infinite
#pragma unroll
    for (int r = 0; r < PER; ++r) x[r] = (x[r] - top) * prm.sharpness, e[r] = id[r] != kNoWord ? expf(x[r]) : 0.0f, sum += e[r];
#pragma unroll
    for (int s = 16; s > 0; s /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        e[r] = none || wrong ? 0.0f : e[r] / sum;
        if (e[r] == 0.0f) id[r] = kNoWord;  // takes no part
    }
    if (lane == 0) prm.targets[t] = wrong ? -1 : none ? kNoTeacher : 0;
#pragma unroll
    for (int size = 2; size <= 32 * PER; size *= 2)
#pragma unroll
        for (int stride = size / 2; stride > 0; stride /= 2) {
            if (stride >= 32) {
#pragma unroll
                for (int r = 0; r < PER; ++r) {
                    const int other = r ^ stride / 32;
                    if (other < r) continue;
                    const bool up = ((r * 32 + lane) & size) == 0;
                    if (up == (id[r] > id[other]) && id[r] != id[other]) {
                        const int i = id[r];
                        const float w = e[r];
                        id[r] = id[other], e[r] = e[other], id[other] = i, e[other] = w;
                    }
                }
            } else {
#pragma unroll
                for (int r = 0; r < PER; ++r) {
                    const int i = __shfl_xor_sync(0xFFFFFFFFu, id[r], stride);
                    const float w = __shfl_xor_sync(0xFFFFFFFFu, e[r], stride);
                    const bool up = ((r * 32 + lane) & size) == 0, lower = (lane & stride) == 0;
                    // the lower one of a pair takes the smaller word where the run rises
                    if (up == lower ? i < id[r] : i > id[r]) id[r] = i, e[r] = w;
                }
            }
        }
    // the buckets that begin with each entry: those behind its predecessor's up to its own
    unsigned short* bucket = prm.entry_bucket + t * kTopBuckets;
    int before = -1;  // of the last entry of the 32 before
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int at = r * 32 + lane, own = min(id[r] / prm.bucket_rows, kTopBuckets - 1);
        const int left = __shfl_up_sync(0xFFFFFFFFu, own, 1), previous = lane > 0 ? left : before;
        for (int b = previous + 1; b <= own; ++b) bucket[b] = (unsigned short)min(at, prm.top);
        before = __shfl_sync(0xFFFFFFFFu, own, 31);
        if (at < prm.top) prm.entry_id[first + at] = id[r], prm.entry_weight[first + at] = e[r];
    }
    // (what is no entry sorts behind all buckets but the last; where there is no such place all are entries)
    for (int b = before + 1 + lane; b < kTopBuckets; b += 32) bucket[b] = (unsigned short)prm.top;
}

}  // namespace

cudaError_t launch_teacher(const TeacherParams& prm, cudaStream_t stream)
{
    const dim3 grid((unsigned)ceil_div(prm.n * prm.tokens, kThreads / 32));
    const auto kernel = prm.top <= 32 ? rps_teacher_kernel<1> : prm.top <= 64 ? rps_teacher_kernel<2> : prm.top <= 128 ? rps_teacher_kernel<4> : rps_teacher_kernel<8>;
    return launch_after(kernel, grid, kThreads, 0, stream, 1, prm);
}

}  // namespace rps_ops
