// The norm over many tensors, and the tensors scaled to at most a given one:
//   norm = sqrt(sum of g^2 over all of them),  out = g min(1, max_norm / (norm + 1e-6))
// What bounds it: every tensor read once for the norm, read again and written where it is scaled.  Squares are summed in 64 bits (the square of any fp32 value is in range there, and
// millions of them lose nothing), one partial sum a workgroup in an order that the sizes decide.  Every workgroup of the second pass adds the
// partial sums up by itself, so nothing stands between the passes but the launch.  In place, tensors whose norm is below the limit are not read again.
#include "kernels.hpp"
#include "vectors.hpp"

namespace picospec {

namespace {

constexpr int kCT = 256, kCW = kCT / kWave;

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

// f(tensor, first element, end, block) for the blocks blockIdx.x, blockIdx.x + gridDim.x, .. of the launch's tensors (c.block elements each, a tensor's last one shorter), ascending or descending
template <int MOST, class F>
__device__ __forceinline__ void each_block(const ClipList<MOST>& c, bool down, F f)
{
    const int64_t blocks = c.first[c.n], here = blockIdx.x, step = gridDim.x;
    if (here >= blocks) return;
    const int64_t trips = (blocks - here + step - 1) / step;
    int lo = 0, hi = c.n;                                         // c.first[lo] <= k < c.first[hi]
    for (int64_t i = 0; i < trips; ++i) {
        const int64_t k = here + (down ? trips - 1 - i : i) * step;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if ((int64_t)c.first[mid] <= k) lo = mid; else hi = mid;
        }
        while ((int64_t)c.first[lo + 1] <= k) ++lo;               // (from the block before on: a step or none, mostly)
        while ((int64_t)c.first[lo] > k) --lo;
        hi = lo + 1;
        const int64_t begin = (k - (int64_t)c.first[lo]) * c.block;
        f(lo, begin, min(begin + (int64_t)c.block, c.numel[lo]), k);
    }
}

template <bool BF16, bool STREAM>
__device__ __forceinline__ double block_squares(const char* g, int64_t begin, int64_t end)
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4, STEP = kCT * N, AHEAD = 4;
    double s = 0.0;
    int64_t x = begin + (int64_t)threadIdx.x * N;
    for (int64_t whole = begin + AHEAD * STEP; whole <= end; whole += AHEAD * STEP, x += AHEAD * STEP) {
        uint4 raw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const loose_t* const p = reinterpret_cast<const loose_t*>(g + (x + j * STEP) * ESZ);
            const u32x4_t v = STREAM ? __builtin_nontemporal_load(p) : *p;
            raw[j] = make_uint4(v.x, v.y, v.z, v.w);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float f[N];
            unpack<BF16>(raw[j], f);
            s += squares(f);
        }
    }
    // (what is left together, too: 203 million bf16, 7 vectors a thread and block, 87 us with 3 of them behind each other, 81)
    if (x >= end) return s;
    uint4 raw[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        raw[j] = make_uint4(0, 0, 0, 0);
        if (x + j * STEP < end) raw[j] = load_row_vec<BF16>(g, x + j * STEP, end);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        float f[N];
        unpack<BF16>(raw[j], f);
        s += squares(f);
    }
    return s;
}

template <int MOST>
__global__ __launch_bounds__(kCT) void clip_norm_kernel(const ClipList<MOST> c, double* partial)
{
    double s = 0.0;
    each_block(c, false, [&](int t, int64_t begin, int64_t end, int64_t k) {
        const char* const g = (const char*)c.grad[t];
        if (k < (int64_t)c.stream) s += c.bf16[t] ? block_squares<true, true>(g, begin, end) : block_squares<false, true>(g, begin, end);
        else s += c.bf16[t] ? block_squares<true, false>(g, begin, end) : block_squares<false, false>(g, begin, end);
    });
    s = block_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

template <bool BF16>
__device__ __forceinline__ uint4 scaled(const uint4& raw, double by)
{
    if (by == 1.0) return raw;                                    // (the tensor's bits)
    float f[Vec<BF16>::N];
    unpack<BF16>(raw, f);
#pragma unroll
    for (int e = 0; e < Vec<BF16>::N; ++e) f[e] = (float)((double)f[e] * by);
    return pack_vec<BF16>(f);
}

template <bool BF16>
__device__ __forceinline__ void block_scale(const char* g, char* out, int64_t begin, int64_t end, double by)
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4, STEP = kCT * N, AHEAD = 4;
    int64_t x = begin + (int64_t)threadIdx.x * N;
    for (int64_t whole = begin + AHEAD * STEP; whole <= end; whole += AHEAD * STEP, x += AHEAD * STEP) {
        uint4 raw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const u32x4_t v = *reinterpret_cast<const loose_t*>(g + (x + j * STEP) * ESZ);
            raw[j] = make_uint4(v.x, v.y, v.z, v.w);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const uint4 r = scaled<BF16>(raw[j], by);
            __builtin_nontemporal_store(u32x4_t{r.x, r.y, r.z, r.w}, reinterpret_cast<loose_t*>(out + (x + j * STEP) * ESZ));
        }
    }
    if (x >= end) return;
    uint4 raw[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
        if (x + j * STEP < end) raw[j] = load_row_vec<BF16>(g, x + j * STEP, end);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
        if (x + j * STEP < end) store_row_vec<BF16, true>(out, x + j * STEP, end, scaled<BF16>(raw[j], by));
}

template <int MOST>
__global__ __launch_bounds__(kCT) void clip_scale_kernel(const ClipList<MOST> c, const double* partial, int partials, float max_norm, float* norm_out)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < partials; i += kCT) s += partial[i];
    const double norm = sqrt(block_sum(s)), by64 = (double)max_norm / (norm + 1e-6);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const double by = by64 >= 1.0 || max_norm == __builtin_huge_valf() ? 1.0 : by64;        // (a norm of NaN: NaN; in 64 bits: the factor of a norm beyond fp32's range is below its normal numbers)
    if (by == 1.0 && c.in_place) return;
    each_block(c, true, [&](int t, int64_t begin, int64_t end, int64_t) {
        const char* const g = (const char*)c.grad[t];
        char* const out = (char*)c.out[t];
        if (c.bf16[t]) block_scale<true>(g, out, begin, end, by);
        else block_scale<false>(g, out, begin, end, by);
    });
}

// f(list) with a short list where that holds the tensors: the host pays half a microsecond for a kilobyte of arguments (two tensors 12.7 us a call with the long one, 9.1 so; lists of 64 gained nothing)
template <class F>
hipError_t with_list(const ClipTensors& c, F f)
{
    if (c.n <= kClipFew) {
        ClipList<kClipFew> few;                                   // (read as far as it is filled)
        std::copy_n(c.grad, c.n, few.grad);
        std::copy_n(c.out, c.n, few.out);
        std::copy_n(c.numel, c.n, few.numel);
        std::copy_n(c.first, c.n + 1, few.first);
        std::copy_n(c.bf16, c.n, few.bf16);
        few.n = c.n; few.block = c.block; few.stream = c.stream; few.in_place = c.in_place;
        f(few);
    } else {
        f(c);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_clip_norm(const ClipTensors& c, double* partial, int groups, hipStream_t stream)
{
    return with_list(c, [&](const auto& list) { clip_norm_kernel<<<dim3((unsigned)groups), dim3(kCT), 0, stream>>>(list, partial); });
}

hipError_t launch_clip_scale(const ClipTensors& c, const double* partial, int partials, float max_norm, float* norm, int groups, hipStream_t stream)
{
    return with_list(c, [&](const auto& list) { clip_scale_kernel<<<dim3((unsigned)groups), dim3(kCT), 0, stream>>>(list, partial, partials, max_norm, norm); });
}

}  // namespace picospec
