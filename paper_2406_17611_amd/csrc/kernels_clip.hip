// The norm of all gradients together, and gradients limited to it: out = f g or w -= lr f g with f = min(1, limit / norm).
// Squares are summed in fp64 (a square of an fp32 number is exact there and neither overflows nor vanishes, and 300 million of them keep
// 1e-13): the multiprocessors have that to spare, the kernels are bound by reading the gradients.
// A launch per 284 tensors for the sums of squares per workgroup, then one per 180 that scales: with one of each, its workgroups add those few sums
// themselves, in one order, instead of a launch in between that does it once (six matrices of a small network: 10.1 us, 11.5 with it). The sums of
// several launches are added once (5,000 tensors of 60 million elements, clipped copies 567 us; every workgroup for itself, 128 tensors a launch: 1,008).
// 403 tensors of 300 million fp32 elements: norm 186 us (6.5 TB/s), clipped copies 661 us, step 867 us (5.5 TB/s; with loads and stores that the
// caches keep 219, 744, 978).
#include <algorithm>
#include <type_traits>

#include "codes_device.h"
#include "varco_scaled.h"

namespace {

constexpr int kThreads = 256;
// Tensors of one launch: their table is a kernel argument (4 KiB at most; 16 tensors, as a network of a few layers has, fill a smaller one).
constexpr int kRead = 284, kScaled = 180, kFewTensors = 16;
constexpr int kWorkgroups = 1024;    // that sum the squares of one launch
constexpr int kOwnSums = 1024;       // partial sums (one launch's) that every workgroup adds itself; more are added once, in a launch of its own

// Tensors are cut into chunks, numbered through the tensors of a launch.
template <int N>
struct Table {
    static constexpr int kMost = N;
    const void* src[N];
    int32_t first[N + 1];
    int32_t tensors, chunk;          // elements of a chunk: a multiple of 1024, 16,384 at most
    uint16_t missing[N];             // elements that a tensor's last chunk lacks

    __device__ __forceinline__ int32_t elements(int k, int32_t c) const { return chunk - (c + 1 == first[k + 1] ? missing[k] : 0); }
};
template <int N>
struct OutTable : Table<N> {
    void* dst[N];
};
static_assert(sizeof(Table<kRead>) + 64 <= 4096 && sizeof(OutTable<kScaled>) + 64 <= 4096, "a kernel's arguments");

// The tensor that chunk c belongs to.
template <typename TABLE>
__device__ __forceinline__ int tensor_of(const TABLE& t, int32_t c) {
    int lo = 0, hi = t.tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.first[mid] <= c)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// Sum over the workgroup, in one order, in all its threads.
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[kThreads];
    __syncthreads();
    part[threadIdx.x] = x;
    __syncthreads();
    for (int s = kThreads / 2; s > 0; s >>= 1) {
        if (int(threadIdx.x) < s) part[threadIdx.x] += part[threadIdx.x + s];
        __syncthreads();
    }
    return part[0];
}

template <typename T, typename TABLE>
__global__ __launch_bounds__(kThreads) void square_sums_kernel(TABLE t, double* partial) {
    using Row = RowPiece<T>;
    constexpr int P = Row::P;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    const int32_t chunks = t.first[t.tensors];
    for (int32_t c = blockIdx.x; c < chunks; c += int32_t(gridDim.x)) {
        const int k = tensor_of(t, c);
        const int64_t at = int64_t(c - t.first[k]) * t.chunk;
        const T* const p = static_cast<const T*>(t.src[k]) + at;
        const int32_t n = t.elements(k, c);
        auto add = [&](auto any) {
#pragma unroll 4
            for (int32_t i = threadIdx.x * P; i < n; i += kThreads * P) {
                float v[P];
                Row::template load<decltype(any)::value, true>(p, i, n, v);
#pragma unroll
                for (int j = 0; j < P; ++j) sum[j & 3] = fma(double(v[j]), double(v[j]), sum[j & 3]);
            }
        };
        if (n % P)
            add(std::true_type{});
        else
            add(std::false_type{});
    }
    const double total = block_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
    if (threadIdx.x == 0) partial[blockIdx.x] = total;
}

// Norm and factor from the sums of squares. A NaN or infinite norm is not below any limit: the factor becomes NaN or 0, and the
// elements at fault stay visible.
__device__ __forceinline__ float factor_of(const double* partial, int32_t n_partial, float max_norm, float* out) {
    double x = 0.0;
    for (int32_t i = threadIdx.x; i < n_partial; i += kThreads) x += partial[i];
    const double norm = sqrt(block_sum(x));
    const float f = norm <= double(max_norm) ? 1.f : float(double(max_norm) / norm);
    if (out && threadIdx.x == 0) out[0] = float(norm), out[1] = f;
    return f;
}
__global__ __launch_bounds__(kThreads) void norm_out_kernel(const double* partial, int32_t n_partial, float max_norm, float* out) {
    factor_of(partial, n_partial, max_norm, out);
}

// STEP: dst -= lr f src (fp32), else dst = f src. n_partial = 0: out holds norm and factor already.
template <typename T, bool STEP, typename TABLE>
__global__ __launch_bounds__(kThreads) void scale_kernel(TABLE t, const double* partial, int32_t n_partial, float max_norm, float lr, float* out) {
    using Row = RowPiece<T>;
    constexpr int P = Row::P;
    float f = n_partial ? factor_of(partial, n_partial, max_norm, blockIdx.x == 0 ? out : nullptr) : out[1];
    const bool same = f == 1.f;
    if (STEP) f *= lr;
    const int32_t chunks = t.first[t.tensors];
    for (int32_t c = blockIdx.x; c < chunks; c += int32_t(gridDim.x)) {
        const int k = tensor_of(t, c);
        const int64_t at = int64_t(c - t.first[k]) * t.chunk;
        const T* const p = static_cast<const T*>(t.src[k]) + at;
        T* const q = static_cast<T*>(t.dst[k]) + at;
        if (!STEP && same && p == q) continue;             // in place and within the limit: the elements stay as they are
        const int32_t n = t.elements(k, c);
        auto scale = [&](auto any) {
            constexpr bool ANY = decltype(any)::value;
#pragma unroll 4
            for (int32_t i = threadIdx.x * P; i < n; i += kThreads * P) {
                float v[P], w[P];
                Row::template load<ANY, true>(p, i, n, v);
                if (STEP) Row::template load<ANY, true>(q, i, n, w);
#pragma unroll
                for (int j = 0; j < P; ++j) v[j] = STEP ? fmaf(-f, v[j], w[j]) : f * v[j];
                Row::template store<ANY, true>(q, i, n, v);
            }
        };
        if (n % P)
            scale(std::true_type{});
        else
            scale(std::false_type{});
    }
}

int64_t total_of(int32_t n_tensors, const int64_t* sizes) {
    int64_t n = 0;
    for (int32_t i = 0; i < n_tensors; ++i) n += sizes[i];
    return n;
}
// 1024 elements, up to 16 times as many where that still makes 2,048 chunks.
int32_t chunk_of(int64_t total) { return int32_t(1024 * std::max<int64_t>(1, std::min<int64_t>(16, total / (1024 * 2048)))); }
int64_t chunks_of(int64_t n, int64_t chunk) { return (n + chunk - 1) / chunk; }

// Calls f(first tensor, tensors, chunks) for each launch of `most` tensors.
template <typename F>
void over_launches(int32_t most, int32_t n_tensors, const int64_t* sizes, int64_t chunk, F f) {
    for (int32_t i = 0; i < n_tensors; i += most) {
        const int32_t n = std::min(most, n_tensors - i);
        int64_t chunks = 0;
        for (int32_t k = 0; k < n; ++k) chunks += chunks_of(sizes[i + k], chunk);
        if (chunks) f(i, n, chunks);
    }
}
int64_t workgroups(int64_t chunks) { return std::min<int64_t>(chunks, kWorkgroups); }
template <typename TABLE>
void fill(TABLE& t, int32_t i, int32_t n, const void* const* src, const int64_t* sizes, int32_t chunk) {
    int64_t c = 0;
    for (int32_t k = 0; k < n; ++k) {
        const int64_t chunks = chunks_of(sizes[i + k], chunk);
        t.src[k] = src[i + k], t.first[k] = int32_t(c), t.missing[k] = uint16_t(chunks * chunk - sizes[i + k]);
        c += chunks;
    }
    t.first[n] = int32_t(c);
    t.tensors = n, t.chunk = chunk;
}

template <int MOST, typename F>
void with_table(int32_t tensors, F f) {
    if (tensors <= kFewTensors)
        f(std::integral_constant<int, kFewTensors>{});
    else
        f(std::integral_constant<int, MOST>{});
}

template <typename T, bool STEP>
hipError_t launch_scale(int32_t n_tensors, const void* const* src, void* const* dst, const int64_t* sizes, const double* partial, int32_t n_partial,
                        float max_norm, float lr, float* out, hipStream_t stream) {
    const int32_t chunk = chunk_of(total_of(n_tensors, sizes));
    hipError_t err = hipSuccess;
    if (n_partial > kOwnSums) err = varco_launch_norm_out(partial, n_partial, max_norm, out, stream), n_partial = 0;
    over_launches(kScaled, n_tensors, sizes, chunk, [&](int32_t i, int32_t n, int64_t chunks) {
        with_table<kScaled>(n, [&](auto most) {
            using TABLE = OutTable<decltype(most)::value>;
            TABLE t;
            fill(t, i, n, src, sizes, chunk);
            for (int32_t k = 0; k < n; ++k) t.dst[k] = dst[i + k];
            hipLaunchKernelGGL((scale_kernel<T, STEP, TABLE>), dim3(unsigned(std::min<int64_t>(chunks, 2048))), dim3(kThreads), 0, stream, t, partial,
                               n_partial, max_norm, lr, out);
        });
        if (err == hipSuccess) err = hipGetLastError();
        if (n_partial) out = nullptr;                    // (written by the first)
    });
    return err;
}

}  // namespace

int32_t varco_clip_partials(int32_t n_tensors, const int64_t* sizes) {
    const int32_t chunk = chunk_of(total_of(n_tensors, sizes));
    int64_t n = 0;
    over_launches(kRead, n_tensors, sizes, chunk, [&](int32_t, int32_t, int64_t chunks) { n += workgroups(chunks); });
    return int32_t(n);
}

hipError_t varco_launch_square_sums(int dtype, int32_t n_tensors, const void* const* grads, const int64_t* sizes, double* partial,
                                    hipStream_t stream) {
    const int32_t chunk = chunk_of(total_of(n_tensors, sizes));
    hipError_t err = hipSuccess;
    over_launches(kRead, n_tensors, sizes, chunk, [&](int32_t i, int32_t n, int64_t chunks) {
        const int64_t blocks = workgroups(chunks);
        with_table<kRead>(n, [&](auto most) {
            using TABLE = Table<decltype(most)::value>;
            TABLE t;
            fill(t, i, n, grads, sizes, chunk);
            if (dtype == VARCO_BF16)
                hipLaunchKernelGGL((square_sums_kernel<bf16_t, TABLE>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, t, partial);
            else
                hipLaunchKernelGGL((square_sums_kernel<float, TABLE>), dim3(unsigned(blocks)), dim3(kThreads), 0, stream, t, partial);
        });
        if (err == hipSuccess) err = hipGetLastError();
        partial += blocks;
    });
    return err;
}

hipError_t varco_launch_norm_out(const double* partial, int32_t n_partial, float max_norm, float* out, hipStream_t stream) {
    hipLaunchKernelGGL(norm_out_kernel, dim3(1), dim3(kThreads), 0, stream, partial, n_partial, max_norm, out);
    return hipGetLastError();
}

hipError_t varco_launch_clip(int dtype, int32_t n_tensors, const void* const* grads, void* const* into, const int64_t* sizes,
                             const double* partial, int32_t n_partial, float max_norm, float* out, hipStream_t stream) {
    if (dtype == VARCO_BF16) return launch_scale<bf16_t, false>(n_tensors, grads, into, sizes, partial, n_partial, max_norm, 0.f, out, stream);
    return launch_scale<float, false>(n_tensors, grads, into, sizes, partial, n_partial, max_norm, 0.f, out, stream);
}

hipError_t varco_launch_sgd_clipped(int32_t n_tensors, void* const* w, const void* const* dw, const int64_t* sizes, float lr,
                                    const double* partial, int32_t n_partial, float max_norm, float* out, hipStream_t stream) {
    return launch_scale<float, true>(n_tensors, dw, w, sizes, partial, n_partial, max_norm, lr, out, stream);
}
