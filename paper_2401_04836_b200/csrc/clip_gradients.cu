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
constexpr int kMostTensors = 768;        // of a launch: their table is a kernel argument (32 KB at most)
constexpr int kUnroll = 4;               // 16-byte loads a thread has under way
constexpr int kBlocks = 148 * 8;         // also the number of partial sums

// The tensors of a launch; of three sizes, since an argument is copied at every launch.
template <int N>
struct Table {
    const void *in[N];
    void *out[N];
    int64_t n[N];
    int32_t chunk[N + 1];                // first chunk of a tensor
    int count;
    int blocks;                          // of the sum: partial sums to add up (of earlier launches too)
    int first;                           // where this launch's partial sums begin
};

template <typename T>
__host__ __device__ constexpr int chunk_values() { return kThreads * kUnroll * (16 / (int)sizeof(T)); }

template <int N>
__device__ __forceinline__ int tensor_of(const Table<N> &t, int c) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.chunk[mid] <= c) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <typename T> struct Wide { static constexpr int kN = 16 / (int)sizeof(T); T v[kN]; };

// Values [0, n) of a chunk that starts at `in`, as a thread holds them: kUnroll times 16 bytes, the loads all under way at once; zeros
// behind the end.
template <typename T>
__device__ __forceinline__ void load_chunk(const T *in, int n, Wide<T> (&w)[kUnroll]) {
    constexpr int kWide = Wide<T>::kN;
    if ((reinterpret_cast<uintptr_t>(in) & 15u) == 0) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int at = (u * kThreads + threadIdx.x) * kWide;
            if (at + kWide <= n) {
                const uint4 raw = *reinterpret_cast<const uint4 *>(in + at);
                memcpy(&w[u], &raw, 16);
            } else {
#pragma unroll
                for (int i = 0; i < kWide; ++i) w[u].v[i] = at + i < n ? in[at + i] : T(0.f);
            }
        }
    } else {                             // any address: neighbours read neighbours
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < kWide; ++i) {
                const int at = (u * kWide + i) * kThreads + threadIdx.x;
                w[u].v[i] = at < n ? in[at] : T(0.f);
            }
    }
}
// The same values to `out`, which the chunk was loaded for: the way back is the way of the load.
template <typename T>
__device__ __forceinline__ void store_chunk(T *out, int n, const Wide<T> (&w)[kUnroll], bool wide) {
    constexpr int kWide = Wide<T>::kN;
    const bool aligned = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int at = (u * kThreads + threadIdx.x) * kWide;
        if (wide && aligned && at + kWide <= n) {
            uint4 raw;
            memcpy(&raw, &w[u], 16);
            *reinterpret_cast<uint4 *>(out + at) = raw;
        } else {
#pragma unroll
            for (int i = 0; i < kWide; ++i) {
                const int one = wide ? at + i : (u * kWide + i) * kThreads + (int)threadIdx.x;
                if (one < n) out[one] = w[u].v[i];
            }
        }
    }
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

template <typename T, int N>
__global__ void __launch_bounds__(kThreads) clip_sum(const __grid_constant__ Table<N> t, double *__restrict__ partial) {
    constexpr int kChunk = chunk_values<T>();
    after_last_kernel();
    __shared__ double warp_sums[kThreads / 32];
    double sum = 0.0;
    const int chunks = t.chunk[t.count];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int at = tensor_of(t, c);
        const int64_t first = (int64_t)(c - t.chunk[at]) * kChunk;
        Wide<T> w[kUnroll];
        load_chunk(static_cast<const T *>(t.in[at]) + first, (int)min(t.n[at] - first, (int64_t)kChunk), w);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) sum += squares(w[u].v);
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

template <typename T, int N>
__global__ void __launch_bounds__(kThreads) clip_scale(const __grid_constant__ Table<N> t, const double *__restrict__ partial, double max_norm,
                                                       void *norm_out) {
    using Number = std::conditional_t<sizeof(T) == 8, double, float>;
    constexpr int kChunk = chunk_values<T>();
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
        const int n = (int)min(t.n[at] - first, (int64_t)kChunk);
        Wide<T> w[kUnroll];
        load_chunk(in, n, w);
        if (scales)
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
#pragma unroll
                for (int i = 0; i < Wide<T>::kN; ++i) w[u].v[i] = (T)(as_number(w[u].v[i]) * factor);
        store_chunk(static_cast<T *>(t.out[at]) + first, n, w, (reinterpret_cast<uintptr_t>(in) & 15u) == 0);
    }
}

template <typename T, int N>
const_status_t run(int count, const void *const *in, void *const *out, const int64_t *sizes, double max_norm, void *norm, cudaStream_t stream) {
    const int batches = std::max(1, (count + N - 1) / N);
    double *partial = nullptr;
    if (scratch_alloc((void **)&partial, sizeof(double) * (size_t)kBlocks * batches, stream) != cudaSuccess) {
        (void)cudaGetLastError();                                      // the next launch must not find this error
        return CONST_ERR_CUDA;
    }
    cudaError_t e = cudaSuccess;
    int sums = 0;
    Table<N> t;
    auto fill = [&](int b) {
        t.count = 0;
        int64_t chunks = 0;
        for (int i = b * N; i < std::min(count, (b + 1) * N); ++i) {
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
        CB_LAUNCH("clip_sum", stream, e = launch_early(clip_sum<T, N>, blocks, kThreads, 0, stream, t, partial));
    }
    t.blocks = sums;
    for (int b = batches - 1; b >= 0 && e == cudaSuccess; --b) {       // the last batch is the one that L2 still holds
        const int blocks = fill(b);
        CB_LAUNCH("clip_scale", stream, e = launch_early(clip_scale<T, N>, blocks, kThreads, 0, stream, t, (const double *)partial, max_norm, b == 0 ? norm : nullptr));
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
    auto sized = [&](auto one) {
        using T = decltype(one);
        if (count <= 16) return run<T, 16>(count, in, out, sizes, max_norm, norm, stream);
        if (count <= 128) return run<T, 128>(count, in, out, sizes, max_norm, norm, stream);
        return run<T, kMostTensors>(count, in, out, sizes, max_norm, norm, stream);
    };
    return dtype == CONST_F32 ? sized(float()) : dtype == CONST_F64 ? sized(double()) : sized(__nv_bfloat16());
}

}  // namespace cb
