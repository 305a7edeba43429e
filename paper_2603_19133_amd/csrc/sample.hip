// One token per row of logits with temperature, top-k, top-p and min-p from a given uniform.  For a row z (NaN as -inf, +inf as the largest finite
// number), M = max z, c = log2(e) / T: w = 2^((z - M) c); the order is (logit descending, id ascending); kept are the first top_k of it, of
// these the shortest prefix whose mass reaches top_p of theirs, of these the ones with w >= min_p; the token is the first id, ascending, at
// which the kept mass up to and with it exceeds u times all of it.
//
// What top-k and top-p keep is a prefix of the order, so it is one pair (t, i): z > t, or z = t and id <= i.  The row is streamed as segments of 256
// vectors; the kept mass of every segment, added up in id order, names the segment in which the draw falls, and that one segment is read again.
//
// Weights and their sums are fp64: where a prefix ends and which token is drawn are comparisons of sums over the whole vocabulary with tokens
// of 10^-6 of it and less between their steps.  With fp32 weights (bf16 logits take few values, so their errors do not average out) sums are off by 10^-8 and
// more of the row's mass, and one row in a hundred would end its prefix, or draw, an id off.  At 10^-12, the error of weight(), it is one in a million.
#include "common.hpp"
#include "kernels.hpp"

namespace picospec {

namespace {

constexpr int kST = 512;                          // threads: one row
constexpr int kSW = kST / kWave;
constexpr int kSegs = kMaxV / 1024 + 2;           // segments of the longest row (fp32, off the boundary)
constexpr int kBins = 2048;                       // of a histogram: four a thread
constexpr int kBinsPer = kBins / kST;
constexpr int kSegsPer = (kSegs + kST - 1) / kST;
constexpr double kLog2e = 1.4426950408889634;
constexpr float kFloatMax = 3.4028234663852886e38f;

struct SampleArgs {
    const void* logits; int64_t ld; int V;
    float T; int top_k; float top_p, min_p;
    const float* T_rows; const int32_t* k_rows; const float *p_rows, *minp_rows; const float* u;
    int32_t* tok; float* prob; int32_t* count; float* lse;
};

// 2^(d c), d = z - ref in fp64 (exact unless the two lie 2^29 apart).  The exponent is split at the nearest integer by adding 1.5 * 2^52, whose sum's low word
// is that integer; 2^f = 1 + f P(f), |f| <= 1/2, P of degree 7 fitted for the smallest largest relative error, 1.1e-12, and exact at 0.
struct Weights {
    double ref, c, d_min;                         // d_min = -1000 / c: what lies below, -inf and NaN too, weighs 2^-1000
    __device__ __forceinline__ void set(float ref_, float T) { ref = (double)ref_; c = kLog2e / (double)T; d_min = -1000.0 / c; }
    __device__ __forceinline__ double exponent(float z) const { return ((double)z - ref) * c; }
    __device__ __forceinline__ double weight(float z) const {
        const double d = fmax((double)z - ref, d_min);
        const double t = fma(d, c, 6755399441055744.0), f = fma(d, c, -(t - 6755399441055744.0));
        double p = 0x1.663487d8abc81p-20;
        p = fma(p, f, 0x1.00ee071c7c030p-16);
        p = fma(p, f, 0x1.4306c1165a375p-13);
        p = fma(p, f, 0x1.5d872975c4ed2p-10);
        p = fma(p, f, 0x1.3b2ab7f3b3217p-7);
        p = fma(p, f, 0x1.c6b08defc25fdp-5);
        p = fma(p, f, 0x1.ebfbdff7c5a79p-3);
        p = fma(p, f, 0x1.62e42fef7a78bp-1);
        return ldexp(fma(p, f, 1.0), (int)__double2loint(t));
    }
};

// NaN: -inf; +inf: the largest finite number
__device__ __forceinline__ float cleaned(float z) { return fminf(fmaxf(z, kNegInf), kFloatMax); }

// What a row keeps: the prefix of the order that ends with (t, id), and of it the exponents from a_min on
struct Cut {
    float t; int id; double a_min;
    __device__ __forceinline__ bool keeps(float z, int x, const Weights& w) const {
        return (z > t || (z == t && x <= id)) && w.exponent(z) >= a_min;
    }
};

struct RowShared {
    double seg[kSegs];                            // kept mass of the segments
    unsigned long long mass[kBins];
    uint32_t count[kBins];
    double red[2 * kSW];
    unsigned long long redu[kSW + 2];
    int at, last;
    float f[kSW + 1];
};

template <bool BF16>
struct RowStream {
    RowView rv;
    int nq, n_seg;
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ RowStream(const void* logits, int64_t ld, int64_t row, int V) : rv(row_view<BF16>(logits, ld, row, V)) {
        nq = (rv.L + Vec<BF16>::N - 1) / Vec<BF16>::N;
        n_seg = stats_segments(nq);
        rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)rv.base, 0, nq * 16, 0x00020000);
    }
    __device__ __forceinline__ uint4 vec(int q) const {                      // (a vector behind the row reads as zero and touches no memory)
        const u32x4_t t = __builtin_amdgcn_raw_buffer_load_b128(rsrc, q * 16, 0, 0);
        return make_uint4(t.x, t.y, t.z, t.w);
    }
    __device__ __forceinline__ void load(int s, uint4 (&raw)[kSplitStatsNV]) const {
        const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
        for (int j = 0; j < kSplitStatsNV; ++j) {
            const u32x4_t t = __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane * 16, stats_group_first(s, j) * 16, 0);
            raw[j] = make_uint4(t.x, t.y, t.z, t.w);
        }
    }
    // the values of vector q, -inf outside the row, and the id of the first of them
    __device__ __forceinline__ void values(const uint4& raw, int q, float (&v)[Vec<BF16>::N]) const {
        unpack<BF16>(raw, v);
        if (q == 0 || q >= nq - 1) {
            const unsigned vm = vec_valid_mask<BF16>(rv, q);
#pragma unroll
            for (int e = 0; e < Vec<BF16>::N; ++e) v[e] = (vm >> e) & 1u ? v[e] : kNegInf;
        }
    }
    __device__ __forceinline__ int first_id(int q) const { return q * Vec<BF16>::N - rv.o; }
    // f(s, raw) for every segment, a wave each, the next one's loads in flight
    template <class F>
    __device__ __forceinline__ void each(const F& f) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        uint4 cur[kSplitStatsNV], next[kSplitStatsNV];
        load(wave, cur);
        for (int s = wave; s < n_seg; s += kSW) {
            load(s + kSW, next);
            f(s, cur);
#pragma unroll
            for (int j = 0; j < kSplitStatsNV; ++j) cur[j] = next[j];
        }
    }
    // f(z, x) for every element z (cleaned) with id x above -inf
    template <class F>
    __device__ __forceinline__ void each_value(const F& f) const {
        const int lane = threadIdx.x & (kWave - 1);
        each([&](int s, const uint4 (&raw)[kSplitStatsNV]) {
#pragma unroll
            for (int j = 0; j < kSplitStatsNV; ++j) {
                const int q = stats_group_first(s, j) + lane;
                float v[Vec<BF16>::N];
                values(raw[j], q, v);
#pragma unroll
                for (int e = 0; e < Vec<BF16>::N; ++e) {
                    const float z = cleaned(v[e]);
                    if (z > kNegInf) f(z, first_id(q) + e, s);
                }
            }
        });
    }
};

// ---------------------------------------------------------------- workgroup reductions and scans (fixed order: the same bits every time)

__device__ __forceinline__ float block_max(float v, RowShared& sh)
{
    const float w = wave_max(v);
    if ((threadIdx.x & (kWave - 1)) == 0) sh.f[threadIdx.x / kWave] = w;
    __syncthreads();
    float m = kNegInf;
#pragma unroll
    for (int i = 0; i < kSW; ++i) m = fmaxf(m, sh.f[i]);
    __syncthreads();
    return m;
}

// sum over the threads in front of this one, and over all of them in `total`
template <typename T>
__device__ __forceinline__ T block_scan_excl(T v, T* red, T& total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const T incl = wave_scan_incl(v);
    if (lane == kWave - 1) red[wave] = incl;
    __syncthreads();
    T before = T(0);
    total = T(0);
#pragma unroll
    for (int w = 0; w < kSW; ++w) {
        if (w < wave) before += red[w];
        total += red[w];
    }
    __syncthreads();
    return before + (incl - v);
}

// ---------------------------------------------------------------- the draw

// The segments' kept masses are in sh.seg: their sum, the token and its probability.
template <bool BF16>
__device__ __forceinline__ void draw(const RowStream<BF16>& rs, const Weights& w, const Cut& cut, float u, RowShared& sh, int& tok, double& total)
{
    constexpr int N = Vec<BF16>::N;
    const int tid = threadIdx.x;
    double mine[kSegsPer], sum = 0.0;
#pragma unroll
    for (int i = 0; i < kSegsPer; ++i) {
        const int s = tid * kSegsPer + i;
        mine[i] = s < rs.n_seg ? sh.seg[s] : 0.0;
        sum += mine[i];
    }
    if (tid == 0) { sh.at = INT32_MAX; sh.last = -1; }
    double before = block_scan_excl(sum, sh.red, total);
    const double target = (u >= 0.f ? (double)u : 0.0) * total;
    // the first segment whose end exceeds the target; where rounding leaves none, the last with any mass
    {
        double b = before, b_hit = 0.0;
        int hit = INT32_MAX;
#pragma unroll
        for (int i = 0; i < kSegsPer; ++i) {
            if (mine[i] > 0.0) {
                if (b + mine[i] > target && hit == INT32_MAX) { hit = tid * kSegsPer + i; b_hit = b; atomicMin(&sh.at, hit); }
                atomicMax(&sh.last, tid * kSegsPer + i);
            }
            b += mine[i];
        }
        __syncthreads();
        if (hit != INT32_MAX && hit == sh.at) sh.red[kSW] = b_hit;
    }
    __syncthreads();
    const bool found = sh.at != INT32_MAX;
    const int s = found ? sh.at : sh.last;
    const double rest = found ? target - sh.red[kSW] : (double)INFINITY;
    __syncthreads();
    if (tid == 0) { sh.at = INT32_MAX; sh.last = -1; }
    // that segment again, a vector a thread
    double kept[N], in_vec = 0.0;
    const int q = s * (64 * kSplitStatsNV) + tid;
    const bool have = s >= 0 && tid < 64 * kSplitStatsNV;
    float v[N];
    rs.values(have ? rs.vec(q) : make_uint4(0, 0, 0, 0), q, v);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float z = cleaned(v[e]);
        kept[e] = have && z > kNegInf && cut.keeps(z, rs.first_id(q) + e, w) ? w.weight(z) : 0.0;
        in_vec += kept[e];
    }
    double all;
    double b = block_scan_excl(in_vec, sh.red, all);
    int hit = INT32_MAX, last = -1;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        b += kept[e];
        if (kept[e] > 0.0) {
            if (b > rest && hit == INT32_MAX) hit = rs.first_id(q) + e;
            last = rs.first_id(q) + e;
        }
    }
    if (hit != INT32_MAX) atomicMin(&sh.at, hit);
    if (last >= 0) atomicMax(&sh.last, last);
    __syncthreads();
    tok = sh.at != INT32_MAX ? sh.at : sh.last;
    __syncthreads();
}

// ---------------------------------------------------------------- the careful way: any row, by passes over its keys

// The bin, descending, in which `above` + the sums up to and with it reach the target; `above` becomes what lies in front of it.  -1: none does.
template <typename T>
__device__ __forceinline__ int crossing(const T* bins, unsigned long long& above, double target, RowShared& sh, unsigned long long* total = nullptr)
{
    const int tid = threadIdx.x;
    unsigned long long mine[kBinsPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kBinsPer; ++i) { mine[i] = bins[tid * kBinsPer + i]; sum += mine[i]; }
    if (tid == 0) sh.at = -1;
    unsigned long long all, b = above + block_scan_excl(sum, sh.redu, all);
    if (total) { *total = all; target *= (double)all; }
#pragma unroll
    for (int i = 0; i < kBinsPer; ++i) {
        if ((double)b < target && (double)(b + mine[i]) >= target) { sh.at = tid * kBinsPer + i; sh.redu[kSW] = b; }
        b += mine[i];
    }
    __syncthreads();
    const int at = sh.at;
    if (at >= 0) above = sh.redu[kSW];
    __syncthreads();
    return at;
}

template <bool BF16>
__device__ __forceinline__ void sample_careful(const RowStream<BF16>& rs, float T, int k, float p, float min_p, int V,
                                               RowShared& sh, Weights& w, Cut& cut, int& kept, float& M)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    float mx = kNegInf, mn = __builtin_huge_valf();
    unsigned n = 0;
    rs.each_value([&](float z, int, int) { mx = fmaxf(mx, z); mn = fminf(mn, z); ++n; });
    M = block_max(mx, sh);
    const float least = -block_max(-mn, sh);
    unsigned long long finite;
    block_scan_excl((unsigned long long)n, sh.redu, finite);
    kept = 0;
    cut = Cut{kNegInf, -1, -__builtin_huge_val()};
    if (M == kNegInf) return;                                                    // (uniform)
    w.set(M, T);
    if (min_p > 0.f) cut.a_min = log2((double)fminf(min_p, 1.f));
    const uint32_t key_max = key_of_bits(__float_as_uint(M));
    uint32_t key_min = key_of_bits(__float_as_uint(least));
    // (a mass is an integer of 2^-shift: sums are exact, whatever their order; of 2^62 at most)
    const int shift = 62 - (32 - __builtin_clz((unsigned)V));
    uint32_t t_key = 0;                                                          // the cut's key; `ties` of its elements are kept
    unsigned long long ties = 0;
    bool has_cut = false;
    auto clear = [&] {
        for (int i = tid; i < kBins; i += kST) { sh.mass[i] = 0; sh.count[i] = 0; }
        __syncthreads();
    };
    auto fixed = [&](float z) { return (unsigned long long)(ldexp(w.weight(z), shift) + 0.5); };
    if (k > 0 && (unsigned long long)k < finite) {
        uint32_t lo = key_min, hi = key_max;
        unsigned long long above = 0;
        for (;;) {
            const uint32_t span = hi - lo;
            const int sft = max(0, 32 - 11 - (span ? __builtin_clz(span) : 32));
            clear();
            rs.each_value([&](float z, int, int) {
                const uint32_t key = key_of_bits(__float_as_uint(z));
                if (key >= lo && key <= hi) atomicAdd(&sh.count[(hi - key) >> sft], 1u);
            });
            __syncthreads();
            const int bin = max(0, crossing(sh.count, above, (double)k, sh));
            hi -= (uint32_t)bin << sft;
            if (sft == 0) break;
            const uint32_t next = hi - ((1u << sft) - 1u);
            lo = next > hi || next < lo ? lo : next;
        }
        t_key = hi;
        ties = (unsigned long long)k - above;
        has_cut = true;
    }
    if (p > 0.f && p < 1.f) {
        uint32_t lo = has_cut ? t_key : key_min, hi = key_max;
        const bool top = has_cut;
        const uint32_t k_key = t_key;
        const unsigned long long k_ties = ties, k_one = has_cut ? fixed(__uint_as_float(bits_of_key(t_key))) : 0;
        unsigned long long above = 0, total = 0;
        double target = (double)p;
        for (bool first = true;; first = false) {
            const uint32_t span = hi - lo;
            const int sft = max(0, 32 - 11 - (span ? __builtin_clz(span) : 32));
            clear();
            rs.each_value([&](float z, int, int) {
                const uint32_t key = key_of_bits(__float_as_uint(z));
                if (key >= lo && key <= hi && !(top && key == k_key)) {
                    atomicAdd(&sh.mass[(hi - key) >> sft], fixed(z));
                    atomicAdd(&sh.count[(hi - key) >> sft], 1u);
                }
            });
            if (top && tid == 0 && k_key >= lo && k_key <= hi) {                 // (of the ties at the end of the first top_k, those that are among them)
                atomicAdd(&sh.mass[(hi - k_key) >> sft], k_one * k_ties);
                atomicAdd(&sh.count[(hi - k_key) >> sft], (unsigned)k_ties);
            }
            __syncthreads();
            const int bin = max(0, crossing(sh.mass, above, target, sh, first ? &total : nullptr));
            if (first) target *= (double)total;
            hi -= (uint32_t)bin << sft;
            if (sft == 0) {
                // The integers' roundings, equal for equal logits, name the value; how many of its elements are kept is decided in fp64.
                const unsigned long long have = sh.count[bin];
                const float z_t = __uint_as_float(bits_of_key(hi)), z_k = top ? __uint_as_float(bits_of_key(k_key)) : kNegInf;
                double over = 0.0, all = 0.0;
                rs.each_value([&](float z, int, int) {
                    const double x = z > z_k ? w.weight(z) : 0.0;
                    all += x;
                    over += z > z_t ? x : 0.0;
                });
                double over_all, all_all;
                block_scan_excl(over, sh.red, over_all);
                block_scan_excl(all, sh.red, all_all);
                if (top) all_all += (double)k_ties * w.weight(z_k);
                const double need = ceil(((double)p * all_all - over_all) / w.weight(z_t));
                ties = need >= (double)have ? have : need < 1.0 ? 1 : (unsigned long long)need;
                break;
            }
            const uint32_t next = hi - ((1u << sft) - 1u);
            lo = next > hi || next < lo ? lo : next;
        }
        t_key = hi;
        has_cut = true;
    }
    if (has_cut) {
        // of the elements that tie with the last one kept, those of the lowest ids: the id of the `ties`-th
        cut.t = __uint_as_float(bits_of_key(t_key));
        static_assert(kSegs <= kBins, "a count for every segment");
        clear();
        rs.each_value([&](float z, int, int s) { if (z == cut.t) atomicAdd(&sh.count[s], 1u); });
        __syncthreads();
        unsigned long long above = 0;
        const int s = crossing(sh.count, above, (double)ties, sh);
        if (tid == 0) sh.at = INT32_MAX;
        __syncthreads();
        if (s >= 0) {
            constexpr int N = Vec<BF16>::N;
            const int q = s * (64 * kSplitStatsNV) + tid;
            const bool have = tid < 64 * kSplitStatsNV;
            float v[N];
            rs.values(have ? rs.vec(q) : make_uint4(0, 0, 0, 0), q, v);
            unsigned long long mine = 0, all;
#pragma unroll
            for (int e = 0; e < N; ++e) mine += have && cleaned(v[e]) == cut.t;
            unsigned long long b = above + block_scan_excl(mine, sh.redu, all);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (have && cleaned(v[e]) == cut.t && ++b == ties) sh.at = rs.first_id(q) + e;
        }
        __syncthreads();
        cut.id = sh.at;
        __syncthreads();
    }
    // the segments' kept masses
    unsigned mine = 0;
    rs.each([&](int s, const uint4 (&raw)[kSplitStatsNV]) {
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < kSplitStatsNV; ++j) {
            const int q = stats_group_first(s, j) + lane;
            float v[Vec<BF16>::N];
            rs.values(raw[j], q, v);
#pragma unroll
            for (int e = 0; e < Vec<BF16>::N; ++e) {
                const float z = cleaned(v[e]);
                const bool keep = z > kNegInf && cut.keeps(z, rs.first_id(q) + e, w);
                sum += keep ? w.weight(z) : 0.0;
                mine += keep;
            }
        }
        sum = wave_sum(sum);
        if (lane == 0) sh.seg[s] = sum;
    });
    unsigned long long n_kept;
    block_scan_excl((unsigned long long)mine, sh.redu, n_kept);
    kept = (int)n_kept;
}

template <bool BF16>
__global__ __launch_bounds__(kST, 4) void sample_kernel(const SampleArgs a)
{
    __shared__ RowShared sh;
    const int64_t row = blockIdx.x;
    const RowStream<BF16> rs(a.logits, a.ld, row, a.V);
    float T = a.T_rows ? a.T_rows[row] : a.T;
    int k = a.k_rows ? a.k_rows[row] : a.top_k;
    const float p = a.p_rows ? a.p_rows[row] : a.top_p, min_p = a.minp_rows ? a.minp_rows[row] : a.min_p;
    if (!(T > 0.f)) { T = 1.f; k = 1; }                                          // (greedy)
    T = fminf(T, kFloatMax);
    Weights w;
    Cut cut;
    int kept, tok = -1;
    float M;
    double total = 0.0;
    sample_careful<BF16>(rs, T, k, p, min_p, a.V, sh, w, cut, kept, M);
    if (M > kNegInf) draw<BF16>(rs, w, cut, a.u[row], sh, tok, total);
    if (threadIdx.x == 0) {
        a.tok[row] = tok;
        a.prob[row] = tok < 0 ? 0.f : (float)(w.weight(cleaned(logit_at<BF16>(a.logits, a.ld, row, tok))) / total);
        a.count[row] = kept;
        a.lse[row] = tok < 0 ? kNegInf : (float)(w.ref / (double)T + log(total));
    }
}

}  // namespace

hipError_t launch_sample(const void* logits, int dtype, int64_t ld, int n_rows, int V, float temperature, int top_k, float top_p, float min_p,
                         const float* temperature_rows, const int32_t* top_k_rows, const float* top_p_rows, const float* min_p_rows,
                         const float* uniforms, int32_t* tok, float* prob, int32_t* count, float* lse, hipStream_t stream)
{
    if (n_rows == 0) return hipSuccess;
    const SampleArgs a{logits, ld, V, temperature, top_k, top_p, min_p, temperature_rows, top_k_rows, top_p_rows, min_p_rows, uniforms, tok, prob, count, lse};
    if (dtype == 1) hipLaunchKernelGGL((sample_kernel<true>), dim3((unsigned)n_rows), dim3(kST), 0, stream, a);
    else hipLaunchKernelGGL((sample_kernel<false>), dim3((unsigned)n_rows), dim3(kST), 0, stream, a);
    return hipGetLastError();
}

}  // namespace picospec
