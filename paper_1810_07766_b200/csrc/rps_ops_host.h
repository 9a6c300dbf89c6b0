// What the files with the C ABI of the training operators share: errors, argument checks and the layout of lent workspaces.
#pragma once

#include "rps_ops_kernels.h"

namespace rps_ops {

int fail(int code, const char* format, ...);  // keeps the reason (rps_ops_last_error) and gives the code back
int start();                                  // of every call: no reason yet

inline int cuda_status(cudaError_t err, const char* where)
{
    if (err == cudaSuccess) return RPS_OK;
    return fail(RPS_ECUDA, "%s: %s", where, cudaGetErrorString(err));
}

#define RPS_TRY(call)                                              \
    do {                                                           \
        const int status_ = cuda_status((call), __func__);         \
        if (status_ != RPS_OK) return status_;                     \
    } while (0)

// Hands out 256-byte aligned parts of a workspace; with base 0 it only counts.
struct Carver {
    unsigned char* base;
    size_t used = 0;
    template <typename T>
    T* take(int64_t count)
    {
        T* at = reinterpret_cast<T*>(base + used);
        used += (size_t)round_up(count * (int64_t)sizeof(T), 256);
        return at;
    }
};

inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

constexpr int64_t kMaxSize = (1ll << 24) - 1;

inline int check_output_strides(const char* name, int n, int64_t rows, int64_t cols, int64_t row, int64_t worker)
{
    if (row < cols) return fail(RPS_EINVAL, "%s: a row stride of %lld is less than the %lld columns", name, (long long)row, (long long)cols);
    if (row >= 1ll << 31) return fail(RPS_EINVAL, "%s: a row stride of %lld", name, (long long)row);
    if (n > 1 && worker < (rows - 1) * row + cols && (worker < cols || row < (n - 1) * worker + cols))
        return fail(RPS_EINVAL, "%s: the workers' parts overlap (worker stride %lld)", name, (long long)worker);
    return RPS_OK;
}

inline int check_common(int dtype, int n)
{
    if (dtype != RPS_F32 && dtype != RPS_BF16) return fail(RPS_EINVAL, "dtype %d is neither RPS_F32 nor RPS_BF16", dtype);
    if (n < 1 || n > RPS_MAX_WORKERS) return fail(RPS_EINVAL, "n = %d workers; 1..%d are possible", n, (int)RPS_MAX_WORKERS);
    return RPS_OK;
}

inline int check_workspace(const void* workspace, size_t have, size_t want)
{
    if (have < want) return fail(RPS_EINVAL, "a workspace of %zu bytes is needed, %zu were given", want, have);
    if (want > 0 && (workspace == nullptr || !aligned(workspace, 256))) return fail(RPS_EINVAL, "the workspace is NULL or not 256-byte aligned");
    return RPS_OK;
}

}  // namespace rps_ops
