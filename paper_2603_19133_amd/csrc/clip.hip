// The norm over many tensors, and the tensors scaled to at most a given one:
//   norm = sqrt(sum of g^2 over all of them),  out = g min(1, max_norm / (norm + 1e-6))
// What bounds it: every tensor read once for the norm, read again and written where it is scaled.  Squares are summed in 64 bits (the square of any fp32 value is in range there, and
// millions of them lose nothing), one partial sum a workgroup in an order that the sizes decide.  Every workgroup of the second pass adds the
// partial sums up by itself, so nothing stands between the passes but the launch.  In place, tensors whose norm is below the limit are not read again.
#include "kernels.hpp"
#include "vectors.hpp"

namespace picospec {

namespace {

constexpr int kCT = 256, kCW = kCT / kWave, kUnroll = 4;

template <int N>
__device__ __forceinline__ double squares(const float (&f)[N])
{
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < N; ++e) { const double v = f[e]; s = __builtin_fma(v, v, s); }
    return s;
}

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double sh[kCW];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    v = wave_sum(v);
    if (lane == 0) sh[wave] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kCW; ++w) s += sh[w];
    return s;
}

// The tensor that block `k` of the launch lies in (kClipBlock elements each, a tensor's last one shorter)
__device__ __forceinline__ int tensor_of(const ClipTensors& c, int64_t k)
{
    int lo = 0, hi = c.n;                                         // c.first[lo] <= k < c.first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((int64_t)c.first[mid] <= k) lo = mid; else hi = mid;
    }
    return lo;
}

// f(tensor, first element, end) for the blocks of this workgroup, ascending or descending
template <class F>
__device__ __forceinline__ void each_block(const ClipTensors& c, bool down, F f)
{
    const int64_t blocks = c.first[c.n];
    const int64_t trips = blocks > (int64_t)blockIdx.x ? (blocks - blockIdx.x + gridDim.x - 1) / gridDim.x : 0;
    for (int64_t i = 0; i < trips; ++i) {
        const int64_t k = (int64_t)blockIdx.x + (down ? trips - 1 - i : i) * gridDim.x;
        const int t = tensor_of(c, k);
        const int64_t begin = (k - (int64_t)c.first[t]) * kClipBlock;
        f(t, begin, min(begin + (int64_t)kClipBlock, c.numel[t]));
    }
}

template <bool BF16>
__device__ __forceinline__ double block_squares(const char* g, int64_t begin, int64_t end)
{
    constexpr int N = Vec<BF16>::N, STEP = kCT * N;
    double s = 0.0;
    for (int64_t x = begin + (int64_t)threadIdx.x * N; x < end; x += kUnroll * STEP) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
            raw[j] = make_uint4(0, 0, 0, 0);
            if (x + j * STEP < end) raw[j] = load_row_vec<BF16>(g, x + j * STEP, end);
        }
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
            float f[N];
            unpack<BF16>(raw[j], f);
            s += squares(f);
        }
    }
    return s;
}

__global__ __launch_bounds__(kCT) void clip_norm_kernel(const ClipTensors c, double* partial)
{
    double s = 0.0;
    each_block(c, false, [&](int t, int64_t begin, int64_t end) {
        const char* const g = (const char*)c.grad[t];
        s += c.bf16[t] ? block_squares<true>(g, begin, end) : block_squares<false>(g, begin, end);
    });
    s = block_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

template <bool BF16>
__device__ __forceinline__ void block_scale(const char* g, char* out, int64_t begin, int64_t end, double by)
{
    constexpr int N = Vec<BF16>::N, STEP = kCT * N;
    for (int64_t x = begin + (int64_t)threadIdx.x * N; x < end; x += kUnroll * STEP) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j)
            if (x + j * STEP < end) raw[j] = load_row_vec<BF16>(g, x + j * STEP, end);
#pragma unroll
        for (int j = 0; j < kUnroll; ++j)
            if (x + j * STEP < end) {
                if (by != 1.0) {
                    float f[N];
                    unpack<BF16>(raw[j], f);
#pragma unroll
                    for (int e = 0; e < N; ++e) f[e] = (float)((double)f[e] * by);
                    raw[j] = pack_vec<BF16>(f);
                }
                store_row_vec<BF16>(out, x + j * STEP, end, raw[j]);
            }
    }
}

__global__ __launch_bounds__(kCT) void clip_scale_kernel(const ClipTensors c, const double* partial, int partials, float max_norm, float* norm_out)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < partials; i += kCT) s += partial[i];
    const double norm = sqrt(block_sum(s)), by64 = (double)max_norm / (norm + 1e-6);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const double by = by64 >= 1.0 ? 1.0 : by64;                   // (a norm of NaN: NaN; in 64 bits: the factor of a norm beyond fp32's range is below its normal numbers)
    each_block(c, true, [&](int t, int64_t begin, int64_t end) {
        const char* const g = (const char*)c.grad[t];
        char* const out = (char*)c.out[t];
        if (by == 1.0 && out == g) return;
        if (c.bf16[t]) block_scale<true>(g, out, begin, end, by);
        else block_scale<false>(g, out, begin, end, by);
    });
}

}  // namespace

hipError_t launch_clip_norm(const ClipTensors& c, double* partial, int groups, hipStream_t stream)
{
    hipLaunchKernelGGL(clip_norm_kernel, dim3((unsigned)groups), dim3(kCT), 0, stream, c, partial);
    return hipGetLastError();
}

hipError_t launch_clip_scale(const ClipTensors& c, const double* partial, int partials, float max_norm, float* norm, int groups, hipStream_t stream)
{
    hipLaunchKernelGGL(clip_scale_kernel, dim3((unsigned)groups), dim3(kCT), 0, stream, c, partial, partials, max_norm, norm);
    return hipGetLastError();
}

}  // namespace picospec
