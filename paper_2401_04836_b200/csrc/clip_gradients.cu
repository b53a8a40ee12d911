// The global norm of many gradients, and the gradients scaled so that it is at most a given one:
//     norm = sqrt(sum over all values of x^2),   y = x min(1, max_norm / norm).
// Bound by memory: every value is read for the norm, and read again and written for the scaling.  The scaling starts with the
// values that the norm read last, so that what still lies in L2 (126 MB) is not fetched again; in place and below the limit
// it is skipped.
// Squares are added in fp32 over the 16 bytes .. 64 bytes a thread loads at once and in fp64 from there on, every sum in an
// order that only the sizes decide: the same call gives the same bits.
#include <cuda_bf16.h>

#include <algorithm>

#include "common.cuh"

namespace cb {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 768;              // tensors a launch: their table is a kernel argument (32 KB at most)
constexpr int kUnroll = 4;               // 16-byte loads a thread has under way
constexpr int kBlocks = 148 * 8;         // also the number of partial sums

struct Table {
    const void *in[kBatch];
    void *out[kBatch];
    int64_t n[kBatch];
    int32_t chunk[kBatch + 1];           // first chunk of a tensor
    int count;
    int blocks;                          // of the sum: partial sums to add up (of earlier launches too)
    int first;                           // where this launch's partial sums begin
};

template <typename T>
__host__ __device__ constexpr int chunk_values() { return kThreads * kUnroll * (16 / (int)sizeof(T)); }

__device__ __forceinline__ int tensor_of(const Table &t, int c) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.chunk[mid] <= c) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <typename T> struct Wide { static constexpr int kN = 16 / (int)sizeof(T); T v[kN]; };

template <typename T>
__device__ __forceinline__ Wide<T> load_wide(const T *p) {
    const uint4 raw = __ldg(reinterpret_cast<const uint4 *>(p));
    Wide<T> w;
    memcpy(&w, &raw, 16);
    return w;
}
__device__ __forceinline__ float as_number(float x) { return x; }
__device__ __forceinline__ double as_number(double x) { return x; }
__device__ __forceinline__ float as_number(__nv_bfloat16 x) { return __bfloat162float(x); }

// Sum of squares of what a thread loaded, in fp32 where that neither overflows nor loses small values, else in fp64.
template <typename T, int N>
__device__ __forceinline__ double squares(const T (&v)[N]) {
    if constexpr (sizeof(T) == 8) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) s = fma((double)v[i], (double)v[i], s);
        return s;
    } else {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) s = fmaf(as_number(v[i]), as_number(v[i]), s);
        // below 1e-28 a term may have been rounded as a subnormal; above 1e37 a sum may overflow (NaN and infinities come here too)
        if (s > 1e-28f && s < 1e37f) return (double)s;
        double d = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) d = fma((double)as_number(v[i]), (double)as_number(v[i]), d);
        return d;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) clip_sum(const __grid_constant__ Table t, double *__restrict__ partial) {
    constexpr int kWide = Wide<T>::kN, kChunk = chunk_values<T>();
    after_last_kernel();
    __shared__ double warp_sums[kThreads / 32];
    double sum = 0.0;
    const int chunks = t.chunk[t.count];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int at = tensor_of(t, c);
        const int64_t first = (int64_t)(c - t.chunk[at]) * kChunk;
        const T *in = static_cast<const T *>(t.in[at]) + first;
        const int64_t n = min(t.n[at] - first, (int64_t)kChunk);
        if (n == kChunk && (reinterpret_cast<uintptr_t>(in) & 15u) == 0) {
            Wide<T> w[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) w[u] = load_wide(in + (u * kThreads + threadIdx.x) * kWide);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) sum += squares(w[u].v);
        } else {
            for (int64_t i = threadIdx.x; i < n; i += kThreads) {
                const T one[1] = {in[i]};
                sum += squares(one);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x % 32 == 0) warp_sums[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int w = 0; w < kThreads / 32; ++w) s += warp_sums[w];
        partial[t.first + blockIdx.x] = s;
    }
    start_next_kernel();
}

template <typename T>
__global__ void __launch_bounds__(kThreads) clip_scale(const __grid_constant__ Table t, const double *__restrict__ partial, double max_norm,
                                                       void *norm_out) {
    using Number = std::conditional_t<sizeof(T) == 8, double, float>;
    constexpr int kWide = Wide<T>::kN, kChunk = chunk_values<T>();
    after_last_kernel();
    start_next_kernel();
    __shared__ double warp_sums[kThreads / 32];
    double sum = 0.0;
    for (int i = threadIdx.x; i < t.blocks; i += kThreads) sum += partial[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x % 32 == 0) warp_sums[threadIdx.x / 32] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) sum += warp_sums[w];
    const double norm = sqrt(sum);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *static_cast<Number *>(norm_out) = (Number)norm;
    // a norm that is no finite number scales nothing: the caller sees it and drops the step
    const bool scales = norm > max_norm && isfinite(norm);
    const Number factor = scales ? (Number)(max_norm / norm) : (Number)1;
    const int chunks = t.chunk[t.count];
    for (int c = chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const int at = tensor_of(t, c);
        if (!scales && t.out[at] == t.in[at]) continue;
        const int64_t first = (int64_t)(c - t.chunk[at]) * kChunk;
        const T *in = static_cast<const T *>(t.in[at]) + first;
        T *out = static_cast<T *>(t.out[at]) + first;
        const int64_t n = min(t.n[at] - first, (int64_t)kChunk);
        if (n == kChunk && ((reinterpret_cast<uintptr_t>(in) | reinterpret_cast<uintptr_t>(out)) & 15u) == 0) {
            uint4 raw[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) raw[u] = *reinterpret_cast<const uint4 *>(in + (u * kThreads + threadIdx.x) * kWide);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                Wide<T> w;
                memcpy(&w, &raw[u], 16);
                if (scales)
#pragma unroll
                    for (int i = 0; i < kWide; ++i) w.v[i] = (T)(as_number(w.v[i]) * factor);
                memcpy(&raw[u], &w, 16);
                *reinterpret_cast<uint4 *>(out + (u * kThreads + threadIdx.x) * kWide) = raw[u];
            }
        } else {
            for (int64_t i = threadIdx.x; i < n; i += kThreads) out[i] = scales ? (T)(as_number(in[i]) * factor) : in[i];
        }
    }
}

template <typename T>
const_status_t run(int count, const void *const *in, void *const *out, const int64_t *sizes, double max_norm, void *norm, cudaStream_t stream) {
    const int batches = std::max(1, (count + kBatch - 1) / kBatch);
    double *partial = nullptr;
    if (scratch_alloc((void **)&partial, sizeof(double) * (size_t)kBlocks * batches, stream) != cudaSuccess) {
        (void)cudaGetLastError();                                      // the next launch must not find this error
        return CONST_ERR_CUDA;
    }
    cudaError_t e = cudaSuccess;
    int sums = 0;
    Table t;
    auto fill = [&](int b) {
        t.count = 0;
        int64_t chunks = 0;
        for (int i = b * kBatch; i < std::min(count, (b + 1) * kBatch); ++i) {
            if (sizes[i] == 0) continue;
            t.in[t.count] = in[i];
            t.out[t.count] = out[i];
            t.n[t.count] = sizes[i];
            t.chunk[t.count++] = (int32_t)chunks;
            chunks += (sizes[i] + chunk_values<T>() - 1) / chunk_values<T>();
        }
        t.chunk[t.count] = (int32_t)chunks;
        return (int)std::max<int64_t>(1, std::min<int64_t>(chunks, kBlocks));
    };
    for (int b = 0; b < batches && e == cudaSuccess; ++b) {
        const int blocks = fill(b);
        t.first = sums;
        sums += blocks;
        CB_LAUNCH("clip_sum", stream, e = launch_early(clip_sum<T>, blocks, kThreads, 0, stream, t, partial));
    }
    t.blocks = sums;
    for (int b = batches - 1; b >= 0 && e == cudaSuccess; --b) {       // the last batch is the one that L2 still holds
        const int blocks = fill(b);
        CB_LAUNCH("clip_scale", stream, e = launch_early(clip_scale<T>, blocks, kThreads, 0, stream, t, (const double *)partial, max_norm, b == 0 ? norm : nullptr));
    }
    if (cudaFreeAsync(partial, stream) != cudaSuccess || e != cudaSuccess) return CONST_ERR_CUDA;
    return CONST_OK;
}

}  // namespace

const_status_t run_clip_gradients(int count, const void *const *in, void *const *out, const int64_t *sizes, const_dtype_t dtype, double max_norm,
                                  void *norm, cudaStream_t stream) {
    // chunks of a launch are counted in 32 bits
    int64_t total = 0;
    for (int i = 0; i < count; ++i) total += sizes[i] / 1024 + 1;
    if (total >= 2147483647ll) return CONST_ERR_UNSUPPORTED;
    if (dtype == CONST_F32) return run<float>(count, in, out, sizes, max_norm, norm, stream);
    if (dtype == CONST_F64) return run<double>(count, in, out, sizes, max_norm, norm, stream);
    return run<__nv_bfloat16>(count, in, out, sizes, max_norm, norm, stream);
}

}  // namespace cb
