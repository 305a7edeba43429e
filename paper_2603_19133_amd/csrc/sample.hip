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
//
// What bounds it.  A row is read once (top-p alone: twice, the second time partly from the caches).  Plain draws, and top-p's second pass over fp32, are bound by a workgroup's own arithmetic,
// a dozen fp64 operations an element, and its waits: 256 rows of 151,936 fp32, 156 MB, one workgroup per CU, 38 to 41 us = 4.0 TB/s (a bare read 23), 129 of them 35, 512, two per CU, 71 = 4.4 TB/s.
// Lists take a comparison an element and come near the memory (512 rows of 100,000 fp32, top-k 50, 47 us = 4.4 TB/s), short ones are a chain of peek, pass, the list's logits, ordering and draw (min-p
// on rows of 50,001 bf16: 16 us for 129 to 256 rows, 20 to 21 for 300 to 512); top-p alone is bound by the counting in LDS and the ALU (64 to 256 rows of 152,064 bf16 57 to 59 us, 512, two per CU, 86).
// Few rows are bound by latency: one of 32,000 with top-k and top-p 15 us, peek, pass, hand-over, ordering and draw behind each other.
#include "common.hpp"
#include "kernels.hpp"

namespace picospec {

namespace {

constexpr int kST = kSampleThreads;
constexpr int kSW = kST / kWave;
constexpr int kSegs = kMaxV / 1024 + 2;           // segments of the longest row (fp32, off the boundary)
constexpr int kSegsPer = (kSegs + kST - 1) / kST;
constexpr int kBins = 2048;                       // of a histogram over the row
constexpr int kListBins = 1024;                   // ... over a list
constexpr int kPeek = kSamplePeek;                // elements that are looked at before the row is streamed
constexpr double kLog2e = 1.4426950408889634;
constexpr float kFloatMax = 3.4028234663852886e38f;

struct SampleArgs {
    const void* logits; int64_t ld; int V;
    float T; int top_k; float top_p, min_p;
    const float* T_rows; const int32_t* k_rows; const float *p_rows, *minp_rows; const float* u;
    int32_t* tok; float* prob; int32_t* count; float* lse;
    char* scratch; int parts;                     // workgroups of a row; scratch of sample_scratch(...) where there are several
};

// 2^(d c), d = z - ref in fp64 (exact unless the two lie 2^29 apart).  The exponent is split at the nearest integer by adding 1.5 * 2^52, whose sum's low word
// is that integer; 2^f = 1 + f P(f), |f| <= 1/2, P of degree 7 fitted for the smallest largest relative error, 1.1e-12, and exact at 0.
struct Weights {
    double ref, c, d_min;                         // d_min = -1000 / c: what lies below, -inf and NaN too, weighs 2^-1000
    __device__ __forceinline__ void set(float ref_, float T) { ref = (double)ref_; c = kLog2e / (double)T; d_min = (double)T * (-1000.0 / kLog2e); }
    __device__ __forceinline__ void move(float ref_) { ref = (double)ref_; }
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
        p = fma(p, f, 1.0);
        return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));     // (from 2^-1000 to 2^1000: no subnormal)
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
    union {
        unsigned long long list[kSampleList];     // composites: (logit descending, id ascending) == descending
        unsigned long long hist[2][kBins];        // (how many, in 2^40; the sum of their places in the bin, in 2^-20); a copy for odd and one for even lanes
        struct { unsigned long long mass[kBins]; uint32_t count[kBins]; } row;
    };
    unsigned long long mass[kListBins];
    uint32_t count[kListBins];
    double red[2 * kSW];
    unsigned long long redu[kSW + 2];
    unsigned long long entry, ends[2][kSW];
    int at, last, n;
    float f[kSW + 1];
    uint32_t votes[2][3][kSW];
    int part_at[kWave];                           // ends of the parts' lists
};
static_assert(sizeof(RowShared) <= 80 * 1024, "two workgroups per CU");

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
    // (a vector behind the row reads as zero and touches no memory)
    __device__ __forceinline__ uint4 peeked(int i, int n_blocks, int blocks) const {
        const u32x4_t t = __builtin_amdgcn_raw_buffer_load_b128(rsrc, (peek_group_first(i, n_blocks, blocks) + (int)(threadIdx.x & (kWave - 1))) * 16, 0, 0);
        return make_uint4(t.x, t.y, t.z, t.w);
    }
    __device__ __forceinline__ uint4 of_segment(int s) const {               // vector tid of a segment
        const u32x4_t t = __builtin_amdgcn_raw_buffer_load_b128(rsrc, (stats_group_first(s, 0) + (int)threadIdx.x) * 16, 0, 0);
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
    __device__ __forceinline__ void values(const uint4& raw, int q, int s, float (&v)[Vec<BF16>::N]) const {       // (of segment s)
        unpack<BF16>(raw, v);
        if (s == 0 || s >= n_seg - 1) {
            const unsigned vm = vec_valid_mask<BF16>(rv, q);
#pragma unroll
            for (int e = 0; e < Vec<BF16>::N; ++e) v[e] = (vm >> e) & 1u ? v[e] : kNegInf;
        }
    }
    __device__ __forceinline__ int first_id(int q) const { return q * Vec<BF16>::N - rv.o; }
    // f(s, raw) for every segment of workgroup `part` of `parts`, a wave each, the next one's loads in flight; `cur` holds the first one's vectors (first_of)
    __device__ __forceinline__ int segment(int part, int trip, int parts) const { return shared_segment(part, (int)__builtin_amdgcn_readfirstlane(threadIdx.x / kWave), trip, parts, kSW); }
    __device__ __forceinline__ void first_of(int part, uint4 (&cur)[kSplitStatsNV]) const { load(segment(part, 0, 1), cur); }
    template <class F>
    __device__ __forceinline__ void each_from(uint4 (&cur)[kSplitStatsNV], const F& f, int part, int parts) const {
        uint4 next[kSplitStatsNV];
        for (int trip = 0, s = segment(part, 0, parts); s < n_seg; s = segment(part, ++trip, parts)) {
            load(segment(part, trip + 1, parts), next);
            f(s, cur);
#pragma unroll
            for (int j = 0; j < kSplitStatsNV; ++j) cur[j] = next[j];
        }
    }
    template <class F>
    __device__ __forceinline__ void each(const F& f, int part = 0, int parts = 1) const {
        uint4 cur[kSplitStatsNV];
        first_of(part, cur);
        each_from(cur, f, part, parts);
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
                values(raw[j], q, s, v);
#pragma unroll
                for (int e = 0; e < Vec<BF16>::N; ++e) {
                    const float z = cleaned(v[e]);
                    if (z > kNegInf) f(z, first_id(q) + e, s);
                }
                __builtin_amdgcn_sched_barrier(0);
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
//
// What weighs 2^-1000 (weight()) may lie below that by any distance, masked ids above all: no uniform, 0 included, may draw it. So a segment of less than
// 2^-978 of the kept mass counts as empty, and so does an id of less than 2^-990 of it. The kept mass is 1 at least: a segment's 2^11 ids of 2^-1000 stay below
// the one, and a segment that does not count as empty has an id that does not.
constexpr double kNoSegment = 0x1p-978, kNoId = 0x1p-990;

// The segments' kept masses are in sh.seg: their sum, the token and its probability.
template <bool BF16>
__device__ __forceinline__ void draw(const RowStream<BF16>& rs, const Weights& w, const Cut& cut, float u, RowShared& sh, int& tok, float& z_tok, double& total)
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
    const double target = (u >= 0.f ? (double)u : 0.0) * total, no_segment = total * kNoSegment, no_id = total * kNoId;
    // the first segment whose end exceeds the target; where rounding leaves none, the last with any mass
    {
        double b = before, b_hit = 0.0;
        int hit = INT32_MAX;
#pragma unroll
        for (int i = 0; i < kSegsPer; ++i) {
            if (mine[i] > no_segment) {
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
    const int q = stats_group_first(s, 0) + tid;
    const bool have = s >= 0 && tid < 64 * kSplitStatsNV;
    float v[N];
    rs.values(have ? rs.of_segment(s) : make_uint4(0, 0, 0, 0), q, s, v);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float z = cleaned(v[e]);
        kept[e] = have && z > kNegInf && cut.keeps(z, rs.first_id(q) + e, w) ? w.weight(z) : 0.0;
        kept[e] = kept[e] > no_id ? kept[e] : 0.0;
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
#pragma unroll
    for (int e = 0; e < N; ++e) if (have && rs.first_id(q) + e == tok) sh.f[0] = cleaned(v[e]);
    __syncthreads();
    z_tok = sh.f[0];
    __syncthreads();
}

// ---------------------------------------------------------------- the careful way: any row, by passes over its keys

// The bin, descending, in which `above` + the sums up to and with it reach the target; `above` becomes what lies in front of it.  -1: none does.
template <int BINS, typename T>
__device__ __forceinline__ int crossing(const T* bins, unsigned long long& above, double target, RowShared& sh, unsigned long long* total = nullptr)
{
    constexpr int PER = BINS / kST;
    const int tid = threadIdx.x;
    unsigned long long mine[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) { mine[i] = bins[tid * PER + i]; sum += mine[i]; }
    if (tid == 0) sh.at = -1;
    unsigned long long all, b = above + block_scan_excl(sum, sh.redu, all);
    if (total) { *total = all; target *= (double)all; }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if ((double)b < target && (double)(b + mine[i]) >= target) { sh.at = tid * PER + i; sh.redu[kSW] = b; }
        b += mine[i];
    }
    __syncthreads();
    const int at = sh.at;
    if (at >= 0) above = sh.redu[kSW];
    __syncthreads();
    return at;
}

// The id of the `ties`-th element that equals t, from how many the segments have of it (kBins counts, cleared behind the row).
template <bool BF16>
__device__ __forceinline__ int id_of_tie(const RowStream<BF16>& rs, const uint32_t* per_segment, float t, unsigned long long ties, RowShared& sh)
{
    constexpr int N = Vec<BF16>::N;
    static_assert(kSegs <= kBins, "a count for every segment");
    const int tid = threadIdx.x;
    unsigned long long above = 0;
    const int s = crossing<kBins>(per_segment, above, (double)ties, sh);
    if (tid == 0) sh.at = INT32_MAX;
    __syncthreads();
    if (s >= 0) {
        const int q = stats_group_first(s, 0) + tid;
        const bool have = tid < 64 * kSplitStatsNV;
        float v[N];
        rs.values(have ? rs.of_segment(s) : make_uint4(0, 0, 0, 0), q, s, v);
        unsigned long long mine = 0, all;
#pragma unroll
        for (int e = 0; e < N; ++e) mine += have && cleaned(v[e]) == t;
        unsigned long long b = above + block_scan_excl(mine, sh.redu, all);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (have && cleaned(v[e]) == t && ++b == ties) sh.at = rs.first_id(q) + e;
    }
    __syncthreads();
    const int id = sh.at;
    __syncthreads();
    return id;
}

template <bool BF16>
__device__ __attribute__((noinline)) void sample_careful(const void* logits, int64_t ld, int64_t row, float T, int k, float p, float min_p, int V,
                                               RowShared& sh, Weights& w, Cut& cut, int& kept, float& M)
{
    const RowStream<BF16> rs(logits, ld, row, V);
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
        for (int i = tid; i < kBins; i += kST) { sh.row.mass[i] = 0; sh.row.count[i] = 0; }
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
                if (key >= lo && key <= hi) atomicAdd(&sh.row.count[(hi - key) >> sft], 1u);
            });
            __syncthreads();
            const int bin = max(0, crossing<kBins>(sh.row.count, above, (double)k, sh));
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
                    atomicAdd(&sh.row.mass[(hi - key) >> sft], fixed(z));
                    atomicAdd(&sh.row.count[(hi - key) >> sft], 1u);
                }
            });
            if (top && tid == 0 && k_key >= lo && k_key <= hi) {                 // (of the ties at the end of the first top_k, those that are among them)
                atomicAdd(&sh.row.mass[(hi - k_key) >> sft], k_one * k_ties);
                atomicAdd(&sh.row.count[(hi - k_key) >> sft], (unsigned)k_ties);
            }
            __syncthreads();
            const int bin = max(0, crossing<kBins>(sh.row.mass, above, target, sh, first ? &total : nullptr));
            if (first) target *= (double)total;
            hi -= (uint32_t)bin << sft;
            if (sft == 0) {
                // The integers' roundings, equal for equal logits, name the value; how many of its elements are kept is decided in fp64.
                const unsigned long long have = sh.row.count[bin];
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
        rs.each_value([&](float z, int, int s) { if (z == cut.t) atomicAdd(&sh.row.count[s], 1u); });
        __syncthreads();
        cut.id = id_of_tie<BF16>(rs, sh.row.count, cut.t, ties, sh);
    }
    // the segments' kept masses
    unsigned mine = 0;
    rs.each([&](int s, const uint4 (&raw)[kSplitStatsNV]) {
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < kSplitStatsNV; ++j) {
            const int q = stats_group_first(s, j) + lane;
            float v[Vec<BF16>::N];
            rs.values(raw[j], q, s, v);
#pragma unroll
            for (int e = 0; e < Vec<BF16>::N; ++e) {
                const float z = cleaned(v[e]);
                const bool keep = z > kNegInf && cut.keeps(z, rs.first_id(q) + e, w);
                sum += keep ? w.weight(z) : 0.0;
                mine += keep;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        sum = wave_sum(sum);
        if (lane == 0) sh.seg[s] = sum;
    });
    unsigned long long n_kept;
    block_scan_excl((unsigned long long)mine, sh.redu, n_kept);
    kept = (int)n_kept;
}

// ---------------------------------------------------------------- the quick ways
//
// kPeek elements of the row, taken evenly from it, say beforehand how the row can be served in one pass over it, or in two:
//   sum      nothing is cut off: the segments' masses, against the largest element of the peek.
//   list     what may be kept is short (min-p alone that keeps more than the list holds takes a second pass, which sums): the elements at or above a threshold go to a list in LDS.  top-k: the value of rank optimistic_rank(..) of
//            the peek.  min-p alone: what min-p leaves against the peek's largest, which is no larger than the row's.  top-p alone: about kTopPList elements, with the mass
//            of the whole row beside, where the peek has its mass there.
//   values  top-p alone on bf16 rows (count_values below).
//   histogram  top-p alone on fp32 rows whose mass is spread: a first pass counts by logit (2048 bins of 1/64 nat below the peek's largest, with the mean place
//            of a bin's elements, of whose mass it gives 10^-5), which names the bin, or the few, in which the prefix ends; a second one sums the segments'
//            masses above them and lists what lies in them.  (Counts, not masses: LDS adds a wave's 64 integers in 10 to 20 cycles, 64 floats in 195.)
//            Elements that are likely behind the prefix are left out of the counts; a prefix that ends among them after all takes a third pass.
// Whatever the peek promised is checked against the row (lists that are short or overflow, a prefix that does not end in its bins, +inf): such
// rows, and a top_k beyond the list, take the careful way: up to ten passes of one workgroup (top_k = 9000, 151,936 fp32: one row 303 us, 256 rows 355).  Rows that are masked whole take it too, and
// leave it after its first pass.
enum Way : int { kCareful, kSum, kList, kHist };
constexpr int kTopPList = 1024;                   // (64 rows of 128,256 fp32 of that kind 41 us, spread ones, by the histogram, 58)
constexpr double kHistFar = 3e-5;                 // relative error allowed for the histogram's sums (checked in fp64 behind it)
constexpr float kHistPerNat = 64.f;

// ref: the peek's largest; least: what goes to the list; total: the row's mass as well; far: the bins that are counted
struct Plan { Way way; float ref, least; bool total; float far; };

template <bool BF16>
__device__ __forceinline__ Plan peek(const RowStream<BF16>& rs, int V, float T, int k, float p, float min_p, RowShared& sh)
{
    constexpr int N = Vec<BF16>::N, PER = kPeek / (kST * N);                    // vectors a thread
    constexpr int BLOCKS = PER * kSW;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int n_blocks = (rs.nq + kWave - 1) / kWave;
    float v[PER][N];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        // (rows of fewer blocks than that: each once)
        const int i = j * kSW + wave;
        rs.values(rs.peeked(i, n_blocks, BLOCKS), peek_group_first(i, n_blocks, BLOCKS) + lane, 0, v[j]);
    }
    float mx = kNegInf;
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            v[j][e] = fmaxf(v[j][e], kNegInf);                                  // (NaN)
            mx = fmaxf(mx, v[j][e]);
        }
    const float ref = block_max(mx, sh);
    Plan pl{kCareful, ref, kNegInf, false, (float)(kBins - 1)};
    if (!(ref > kNegInf) || !(ref <= kFloatMax)) return pl;
    const bool cut_p = p > 0.f && p < 1.f, all = V <= kSampleList;
    if (k <= 0 && !cut_p && !(min_p > 0.f)) { pl.way = kSum; return pl; }
    if (all) { pl.way = kList; pl.total = k <= 0 && cut_p; return pl; }
    if (k <= 0 && !cut_p) {                                                     // min-p alone
        pl.way = kList;
        pl.least = float_below(float_below((float)((double)ref + (double)T * log((double)fminf(min_p, 1.f)))));
        return pl;
    }
    if (BF16 && k <= 0) { pl.way = kHist; return pl; }                           // (values are counted whether the mass is spread or not)
    const int want = k > 0 ? k : kTopPList;
    const int rank = want <= kSampleList ? optimistic_rank(want, V, min(kPeek, V), kSampleList) : 0;
    if (rank == 0) {
        if (k <= 0) pl.way = kHist;
        return pl;
    }
    // the peek's element of a rank, or one a little behind: `rank` to 1.25 `rank` elements lie at or above it
    const float least_max = -block_max(-mx, sh);                                // (every thread has one at or above the least of their largest)
    auto of_rank = [&](int rank) {
        uint32_t lo = key_of_bits(__float_as_uint(rank <= kST ? least_max : kNegInf)), hi = key_of_bits(__float_as_uint(ref));
        for (int i = 0; lo < hi; ++i) {                                         // (count at or above lo >= rank, above hi: none; a quarter is left every time)
            const uint32_t span = hi - lo, key[3] = {lo + span / 4 + 1, lo + span / 2 + 1, lo + span / 2 + span / 4 + 1};
            uint32_t n[3] = {0, 0, 0};
#pragma unroll
            for (int m = 0; m < 3; ++m) {
                const float t = __uint_as_float(bits_of_key(key[m]));
#pragma unroll
                for (int j = 0; j < PER; ++j)
#pragma unroll
                    for (int e = 0; e < N; ++e) n[m] += (uint32_t)__builtin_popcountll(__ballot(v[j][e] >= t));
                if (lane == 0) sh.votes[i & 1][m][wave] = n[m];
            }
            __syncthreads();
            uint32_t best = 0;
#pragma unroll
            for (int m = 0; m < 3; ++m) {
                n[m] = 0;
#pragma unroll
                for (int w = 0; w < kSW; ++w) n[m] += sh.votes[i & 1][m][w];
            }
            // (the highest threshold that still has `rank`)
            if (n[2] >= (uint32_t)rank) { lo = key[2]; best = n[2]; }
            else if (n[1] >= (uint32_t)rank) { lo = key[1]; hi = key[2] - 1; best = n[1]; }
            else if (n[0] >= (uint32_t)rank) { lo = key[0]; hi = key[1] - 1; best = n[0]; }
            else hi = key[0] - 1;
            if (best && best <= (uint32_t)(rank + rank / 4)) break;
        }
        __syncthreads();
        return __uint_as_float(bits_of_key(lo));
    };
    pl.least = of_rank(rank);
    pl.way = kList;
    if (BF16 || k > 0) return pl;
    pl.total = true;
    const float c = (float)(kLog2e / (double)T);
    // (without the peek's eight largest: what is by chance among the row's few that hold much of it says nothing of the rest)
    const float few = of_rank(8);
    float above = 0.f, total = 0.f;
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float x = v[j][e] < few ? exp_stream(v[j][e], ref, c) : 0.f;
            total += x;
            above += v[j][e] >= pl.least ? x : 0.f;
        }
    double a_all, t_all;
    block_scan_excl((double)above, sh.red, a_all);
    block_scan_excl((double)total, sh.red, t_all);
    if (a_all >= ((double)p + 0.3 * (1.0 - (double)p)) * t_all) return pl;
    pl.way = kHist;
    // bins behind which the peek has less than 1 / 1.15 of what top-p leaves out
    float near = 0.f, far = (float)(kBins - 1);
    for (int i = 0; i < 7; ++i) {
        const float mid = 0.5f * (near + far);
        float behind = 0.f;
#pragma unroll
        for (int j = 0; j < PER; ++j)
#pragma unroll
            for (int e = 0; e < N; ++e) behind += (ref - v[j][e]) * (kHistPerNat / T) > mid ? exp_stream(v[j][e], ref, c) : 0.f;
        double all_behind;
        block_scan_excl((double)behind, sh.red, all_behind);
        if (all_behind * 1.15 <= (1.0 - (double)p) * t_all) far = mid;
        else near = mid;
    }
    pl.far = far;
    return pl;
}

// Appends the ids of the elements of a segment whose bit is set (bit j * N + e) to the list; sh.n counts on behind the list's end.  fill_list reads their logits
// again, from the caches, all at once: with the values at hand here a segment takes 340 instructions, a test for every element in registers.
template <bool BF16>
__device__ __forceinline__ void append(const RowStream<BF16>& rs, int s, unsigned mask, RowShared& sh, int cap = kSampleList)
{
    constexpr int N = Vec<BF16>::N;
    if (!__ballot(mask != 0u)) return;
    const int lane = threadIdx.x & (kWave - 1);
    const int mine = __builtin_popcount(mask), incl = wave_scan_incl(mine), total = read_lane(incl, kWave - 1);
    int base = 0;
    if (lane == 0) base = atomicAdd(&sh.n, total);
    int at = read_lane(base, 0) + incl - mine;
    for (unsigned left = mask; left; left &= left - 1u, ++at) {
        const int bit = __builtin_ctz(left);
        if (at < cap) sh.list[at] = (unsigned)rs.first_id(stats_group_first(s, bit / N) + lane) + (unsigned)(bit % N);
    }
}

// The list's first n entries, ids so far, with their logits.  Called behind a barrier; ends with one.
template <bool BF16>
__device__ __forceinline__ void fill_list(const RowStream<BF16>& rs, int n, RowShared& sh)
{
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kST) {
        const int x = (int)sh.list[i], v = rs.rv.o + x;                        // (ids of elements inside the row)
        const uint32_t bits = BF16 ? (uint32_t)reinterpret_cast<const uint16_t*>(rs.rv.base)[v] << 16 : reinterpret_cast<const uint32_t*>(rs.rv.base)[v];
        sh.list[i] = composite_of(bits, (uint32_t)x);
    }
    __syncthreads();
}

__device__ __forceinline__ unsigned long long pack2(uint32_t a, uint32_t b) { return (unsigned long long)a | (unsigned long long)b << 32; }

__device__ __forceinline__ float composite_value(unsigned long long c) { return __uint_as_float(bits_of_key((uint32_t)(c >> 32))); }
__device__ __forceinline__ int composite_id(unsigned long long c) { return (int)(0xFFFFFFFFu - (uint32_t)c); }

// one pass of a workgroup over its part of the row
template <bool BF16, Way WAY, bool TOTAL>
__device__ __forceinline__ void first_pass(const RowStream<BF16>& rs, uint4 (&ahead)[kSplitStatsNV], int part, int parts, const Plan& pl, const Weights& w, float T, RowShared& sh,
                                           float& M, int& n_finite, double& total, double& above_ref)
{
    constexpr int N = Vec<BF16>::N;
    const int lane = threadIdx.x & (kWave - 1);
    const float c = (float)w.c, per = kHistPerNat / T;
    float mx = kNegInf;
    int n = 0;                                                                   // (of the wave)
    double sum_all = 0.0, sum_over = 0.0;
    rs.each_from(ahead, [&](int s, const uint4 (&raw)[kSplitStatsNV]) {
        unsigned mask = 0u;
        double sum = 0.0;
        float mass = 0.f, over = 0.f;
#pragma unroll
        for (int j = 0; j < kSplitStatsNV; ++j) {
            float v[N];
            rs.values(raw[j], stats_group_first(s, j) + lane, s, v);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                mx = fmaxf(mx, v[e]);
                if constexpr (WAY == kSum || TOTAL) sum += w.weight(v[e]);
                if constexpr (WAY == kSum) n += __builtin_popcountll(__ballot(v[e] >= -kFloatMax));
                if constexpr (WAY == kList) mask |= (v[e] >= pl.least && v[e] > kNegInf) ? 1u << (j * N + e) : 0u;
                if constexpr (WAY == kHist) {
                    const float z = fmaxf(v[e], kNegInf), x = fminf(fmaxf((pl.ref - z) * per, 0.f), (float)(kBins - 1));
                    const float one = exp_stream(z, pl.ref, c);
                    mass += one;
                    over += fmaxf(one, 1.f);                                    // (what lies above the reference is counted as lying at it)
                    if (x <= pl.far) {
                        const unsigned bin = (unsigned)x;
                        atomicAdd(&sh.hist[lane & 1][bin], pack2((unsigned)((x - (float)bin) * 0x1p20f), 1u << 8));
                    }
                }
                if ((WAY == kSum || TOTAL) && (e & 3) == 3) __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_sched_barrier(0);                                  // (a vector's exponentials side by side, not the segment's: registers)
        }
        if constexpr (WAY == kList) append<BF16>(rs, s, mask, sh);
        if constexpr (WAY == kSum) {
            sum = wave_sum(sum);
            if (lane == 0) sh.seg[s] = sum;
        }
        if constexpr (TOTAL) sum_all += sum;
        if constexpr (WAY == kHist) { sum_all += (double)mass; sum_over += (double)(over - (float)(N * kSplitStatsNV)); }
    }, part, parts);
    M = block_max(mx, sh);
    n_finite = 0;
    total = 0.0;
    if constexpr (WAY == kSum) { unsigned long long t; block_scan_excl((unsigned long long)(lane == 0 ? n : 0), sh.redu, t); n_finite = (int)t; }
    if constexpr (TOTAL || WAY == kHist) block_scan_excl(sum_all, sh.red, total);
    if constexpr (WAY == kHist) block_scan_excl(sum_over, sh.red, above_ref);
    __syncthreads();
    if constexpr (WAY == kList) fill_list<BF16>(rs, min(sh.n, kSampleList), sh);
}

// The entry of the list's first n, from composite `from` on, with which the sum over the entries at or above it reaches the target: counts, or masses of 2^-kListShift.
// 0: none.
constexpr int kListShift = 49;
static_assert(kSampleList <= 1 << 13, "sums of masses stay below 2^62");
__device__ __forceinline__ unsigned long long list_mass(unsigned long long comp, const Weights& w)
{
    return (unsigned long long)(ldexp(w.weight(composite_value(comp)), kListShift) + 0.5);
}

template <bool MASS>
__device__ __forceinline__ unsigned long long select(int n, unsigned long long from, double target, const Weights& w, RowShared& sh)
{
    const int tid = threadIdx.x;
    unsigned long long lo = ~0ull, hi = 0ull, above = 0;
    for (int i = tid; i < n; i += kST) {
        const unsigned long long c = sh.list[i];
        if (c >= from) { lo = min(lo, c); hi = max(hi, c); }
    }
    lo = wave_min_u64(lo);
    hi = wave_max_u64(hi);
    if ((tid & (kWave - 1)) == 0) { sh.ends[0][tid / kWave] = lo; sh.ends[1][tid / kWave] = hi; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSW; ++i) { lo = min(lo, sh.ends[0][i]); hi = max(hi, sh.ends[1][i]); }
    if (lo > hi) return 0ull;
    for (;;) {
        const unsigned long long span = hi - lo;
        const int sft = span ? max(0, 64 - 10 - __builtin_clzll(span)) : 0;
        for (int i = tid; i < kListBins; i += kST) { sh.mass[i] = 0; sh.count[i] = 0; }
        __syncthreads();
        for (int i = tid; i < n; i += kST) {
            const unsigned long long c = sh.list[i];
            if (c >= lo && c <= hi) {
                const int bin = (int)((hi - c) >> sft);
                atomicAdd(&sh.count[bin], 1u);
                if constexpr (MASS) atomicAdd(&sh.mass[bin], list_mass(c, w));
            }
        }
        __syncthreads();
        int bin;
        if constexpr (MASS) bin = crossing<kListBins>(sh.mass, above, target, sh);
        else bin = crossing<kListBins>(sh.count, above, target, sh);
        if (bin < 0) return 0ull;
        hi -= (unsigned long long)bin << sft;
        if (sft == 0) return hi;
        const unsigned long long next = hi - ((1ull << sft) - 1ull);
        lo = next > hi || next < lo ? lo : next;
        if (sh.count[bin] == 1u) {
            for (int i = tid; i < n; i += kST) {
                const unsigned long long c = sh.list[i];
                if (c >= lo && c <= hi) sh.entry = c;
            }
            __syncthreads();
            return sh.entry;
        }
        __syncthreads();
    }
}

// sum of the masses of the list's entries at or above `from`
__device__ __forceinline__ unsigned long long list_sum(int n, unsigned long long from, const Weights& w, RowShared& sh)
{
    unsigned long long mine = 0, all;
    for (int i = threadIdx.x; i < n; i += kST) { const unsigned long long c = sh.list[i]; if (c >= from) mine += list_mass(c, w); }
    block_scan_excl(mine, sh.redu, all);
    return all;
}

// Adds the masses of the kept entries to their segments' (as integers of 2^-kListShift: exact, whatever the order) and counts them. A segment that keeps nothing but
// what rounds to no unit, and more than draw() calls empty, is marked with 2^-60: a uniform of 0 draws its first kept id.
template <bool BF16>
__device__ __forceinline__ int list_to_segments(const RowStream<BF16>& rs, int n, const Cut& cut, const Weights& w, bool add, RowShared& sh)
{
    unsigned long long* const extra = sh.mass;                                  // (segments in blocks of kListBins: one, but for fp32 rows of a million)
    unsigned long long mine = 0, all;
    for (int first = 0; first < rs.n_seg; first += kListBins) {
        for (int i = threadIdx.x; i < kListBins; i += kST) { extra[i] = 0; sh.count[i] = 0u; }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kST) {
            const unsigned long long c = sh.list[i];
            const int x = composite_id(c), s = (rs.rv.o + x) / (64 * kSplitStatsNV * Vec<BF16>::N) - first;
            if (s >= 0 && s < kListBins && cut.keeps(composite_value(c), x, w)) {
                const unsigned long long m = list_mass(c, w);
                ++mine;
                if (m) atomicAdd(&extra[s], m);
                else if (w.weight(composite_value(c)) > kNoSegment * kSampleList) sh.count[s] = 1u;
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < kListBins && first + i < rs.n_seg; i += kST) {
            const double m = extra[i] || !sh.count[i] ? ldexp((double)extra[i], -kListShift) : 0x1p-60;
            sh.seg[first + i] = add ? sh.seg[first + i] + m : m;
        }
        __syncthreads();
    }
    block_scan_excl(mine, sh.redu, all);
    return (int)all;
}

// what hand-over between the workgroups of a row, and between the two launches of a histogram, goes through
template <bool BF16>
struct RowScratch {
    unsigned long long *word, *head, *seg, *hist, *lists;
    int cap;
    __device__ __forceinline__ RowScratch(const SampleArgs& a, int64_t row) {
        const SampleScratch l = sample_scratch(BF16, a.V, a.parts);
        char* const base = a.scratch + row * (int64_t)l.row_bytes;
        word = (unsigned long long*)base;
        head = (unsigned long long*)(base + kArrivalStride);
        seg = (unsigned long long*)(base + l.seg_at);
        hist = (unsigned long long*)(base + l.hist_at);
        lists = (unsigned long long*)(base + l.list_at);
        cap = l.list_cap;
    }
};

// The parts' shares together in the last of a row's workgroups to arrive: segments, lists, and M, count and total.  False in the others.
template <bool BF16>
__device__ __forceinline__ bool gather(const RowStream<BF16>& rs, const RowScratch<BF16>& rx, int part, int parts, bool segs, bool lists,
                                       float& M, int& count, double& total, RowShared& sh)
{
    const int tid = threadIdx.x;
    const int n = lists ? sh.n : 0;
    if (segs)
        for (int i = tid; i < rs.n_seg; i += kST)
            if (i / kSW % parts == part) put_shared(&rx.seg[i], (unsigned long long)__double_as_longlong(sh.seg[i]));
    for (int i = tid; i < min(n, rx.cap); i += kST) put_shared(&rx.lists[(int64_t)part * rx.cap + i], sh.list[i]);
    if (tid == 0) {
        put_shared(&rx.head[part * 3], pack2((uint32_t)n, __float_as_uint(M)));
        put_shared(&rx.head[part * 3 + 1], (unsigned long long)(unsigned)count);
        put_shared(&rx.head[part * 3 + 2], (unsigned long long)__double_as_longlong(total));
    }
    if (!arrive_last(rx.word, (unsigned)parts, tid == 0)) return false;
    // (loads that pass by the L2 take a microsecond: all heads at once, then everything else at once)
    static_assert(kSampleMostParts <= kWave, "a lane for each part");
    {
        const int lane = tid & (kWave - 1);
        const bool mine = lane < parts;
        const unsigned long long h0 = mine ? get_shared(&rx.head[lane * 3]) : pack2(0u, __float_as_uint(kNegInf));
        const unsigned long long h1 = mine ? get_shared(&rx.head[lane * 3 + 1]) : 0ull, h2 = mine ? get_shared(&rx.head[lane * 3 + 2]) : 0ull;
        const int m = (int)(uint32_t)h0, incl = wave_scan_incl(m);
        M = wave_max(__uint_as_float((uint32_t)(h0 >> 32)));
        count = read_lane(wave_scan_incl((int)h1), kWave - 1);
        total = wave_sum(__longlong_as_double((long long)h2));
        const bool over = __ballot(m > rx.cap) != 0ull;                         // (a part's list overflowed: so does the row's)
        const int all = read_lane(incl, kWave - 1);
        if (tid < kWave) { sh.part_at[tid] = incl; if (tid == 0) sh.n = over ? kSampleList + 1 : all; }
        __syncthreads();
        if (!over) {
            const int listed = min(all, kSampleList);
            for (int e0 = 0; e0 < listed; e0 += 4 * kST) {
                unsigned long long got[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = e0 + i * kST + tid;
                    if (e < listed) {
                        int pt = 0;
                        while (sh.part_at[pt] <= e) ++pt;
                        got[i] = get_shared(&rx.lists[(int64_t)pt * rx.cap + (e - (pt ? sh.part_at[pt - 1] : 0))]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) { const int e = e0 + i * kST + tid; if (e < listed) sh.list[e] = got[i]; }
            }
        }
    }
    if (segs)
        for (int i = tid; i < rs.n_seg; i += kST) sh.seg[i] = __longlong_as_double((long long)get_shared(&rx.seg[i]));
    __syncthreads();
    return true;
}

// What the counts say: the bins in which the prefix ends, [from, to) down from the reference; by_min_p: min-p cuts above them.  1: found; 0: the prefix ends
// behind what was counted; -1: nothing that the second pass could use.
struct Bracket { bool by_min_p; float from, to; };
__device__ __forceinline__ int bracket(float p, double total, double above_ref, float far, RowShared& sh, Bracket& br)
{
    constexpr int PER = kBins / kST;
    const int tid = threadIdx.x;
    double mine[PER], sum = 0.0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned long long h = sh.hist[0][tid * PER + i] + sh.hist[1][tid * PER + i];
        const double n = (double)(h >> 40), place = (double)(h & ((1ull << 40) - 1)) * 0x1p-20;
        mine[i] = n > 0.0 ? n * exp2_split(((double)(tid * PER + i) + place / n) * (-kLog2e / (double)kHistPerNat)) : 0.0;
        if (i == 0 && tid == 0) mine[0] += above_ref;
        sum += mine[i];
    }
    if (tid == 0) { sh.at = INT32_MAX; sh.last = INT32_MAX; }
    double b = block_scan_excl(sum, sh.red, all);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        b += mine[i];
        if (b >= (double)p * total * (1.0 - kHistFar)) atomicMin(&sh.at, tid * PER + i);
        if (b >= (double)p * total * (1.0 + kHistFar)) atomicMin(&sh.last, tid * PER + i);
    }
    __syncthreads();
    const int first = sh.at, last = sh.last;
    __syncthreads();
    if (!(total < __builtin_huge_val())) return -1;
    if ((float)(last + 1) > far || last == INT32_MAX) return far < (float)(kBins - 1) ? 0 : -1;    // (the last bin holds all that is far)
    br = Bracket{false, (float)first, (float)(last + 1)};
    return 1;
}

// The segments' masses of what lies above the bracket, and what lies in it to the list; MIN_P: of what min-p leaves, and no list.
template <bool BF16, bool MIN_P>
__device__ __forceinline__ void second_pass(const RowStream<BF16>& rs, int part, int parts, const Bracket& br, float ref, float per, const Weights& w, double a_min, RowShared& sh,
                                            int& n_above, double& total)
{
    constexpr int N = Vec<BF16>::N;
    const int lane = threadIdx.x & (kWave - 1);
    const float from = br.from > 0.f ? br.from : kNegInf, to = br.to;
    int n = 0;
    double sum_all = 0.0;
    rs.each([&](int s, const uint4 (&raw)[kSplitStatsNV]) {
        unsigned mask = 0u;
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < kSplitStatsNV; ++j) {
            float v[N];
            rs.values(raw[j], stats_group_first(s, j) + lane, s, v);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const double x = w.weight(v[e]);
                bool above;
                if constexpr (MIN_P) {
                    above = w.exponent(v[e]) >= a_min;
                } else {
                    // (the place of the first pass, but for its ends, which lie outside the bracket; what is not a number lies nowhere)
                    const float at = (ref - v[e]) * per;
                    above = at < from;
                    mask |= at >= from && at < to ? 1u << (j * N + e) : 0u;
                    sum_all += x;
                }
                sum += above ? x : 0.0;
                n += above;
                if ((e & 3) == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (!MIN_P) append<BF16>(rs, s, mask, sh);
        sum = wave_sum(sum);
        if (lane == 0) sh.seg[s] = sum;
    }, part, parts);
    unsigned long long t;
    block_scan_excl((unsigned long long)n, sh.redu, t);
    n_above = (int)t;
    block_scan_excl(sum_all, sh.red, total);
    __syncthreads();
    if constexpr (!MIN_P) fill_list<BF16>(rs, min(sh.n, kSampleList), sh);
}

// bf16 rows with top-p alone, by one workgroup: the values themselves are counted.  A window of 16 octaves of magnitude less eight values, up to the end of the one that
// holds a quarter more than the peek's largest and what lies 50 T off it (the row's largest is seldom in the peek), has kWindow values of either sign; what is smaller lies between the two signs' and goes to the list; what lies
// below weighs less than e^-50 and is passed over.  Counts times weights are the row's exact masses, so the prefix's end is known after one pass without an
// exponential, and the second one looks weights up.  Elements are taken two at a time, as 16-bit integers.
constexpr int kWindow = 16 * 128 - 8, kValues = 2 * kWindow + 1, kValuesPer = (kValues + kST - 1) / kST;
static_assert(kValuesPer == 8, "all but a few of the threads' places hold a value");
constexpr int kSmallList = kSampleList - kValues;                               // (the counts, two copies, and then the weights, lie behind the list)
typedef short short2_t __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));

// 16-bit magnitude in front of the window's first: -1: no such window
__device__ __forceinline__ int window_base(float ref, float T)
{
    const float x = fmaxf(1.25f * fabsf(ref), fabsf(ref) + 50.f * T);
    const int e = (int)(__float_as_uint(x) >> 23);
    return e <= 252 ? max(((e + 1) << 7) - kWindow, 128) - 1 : -1;
}
// Where values lie in the order: -kWindow .. kWindow from the largest down, 0: the small ones; kWindow + 1 of either sign: outside
__device__ __forceinline__ void value_places(const RowStream<true>& rs, const uint4& raw, int q, int s, int base, short2_t (&at)[4])
{
    uint32_t word[4] = {raw.x, raw.y, raw.z, raw.w};
    if (s == 0 || s >= rs.n_seg - 1) {                                           // (outside the row: -inf)
        const unsigned vm = vec_valid_mask<true>(rs.rv, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!((vm >> (2 * i)) & 1u)) word[i] = (word[i] & 0xFFFF0000u) | 0xFF80u;
            if (!((vm >> (2 * i + 1)) & 1u)) word[i] = (word[i] & 0xFFFFu) | 0xFF800000u;
        }
    }
    const ushort2_t base2 = {(unsigned short)base, (unsigned short)base}, far = {kWindow + 1, kWindow + 1};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t mag = word[i] & 0x7FFF7FFFu;
        ushort2_t d, w;
        __builtin_memcpy(&d, &mag, 4);
        __builtin_memcpy(&w, &word[i], 4);
        d = __builtin_elementwise_min(__builtin_elementwise_sub_sat(d, base2), far);
        const short2_t positive = ~((short2_t)w >> 15);                          // -1 or 0
        at[i] = ((short2_t)d ^ positive) - positive;
    }
}
__device__ __forceinline__ float value_at(int place, int base)
{
    return __uint_as_float(place < 0 ? (unsigned)(base - place) << 16 : ((unsigned)(base + place) << 16) | 0x80000000u);
}

__device__ __forceinline__ bool count_values(const RowStream<true>& rs, const Plan& pl, float T, float p, double a_min, Weights& w, Cut& cut, int& kept, float& M, RowShared& sh)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), base = window_base(pl.ref, T);
    if (base < 0) return false;
    double* const weight = reinterpret_cast<double*>(&sh.list[kSmallList]);
    uint32_t* const counts = reinterpret_cast<uint32_t*>(weight);
    for (int i = tid; i < 2 * kValues; i += kST) counts[i] = 0u;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    uint32_t* const mine = counts + (lane & 1) * kValues;
    short2_t first = {kWindow + 1, kWindow + 1};
    rs.each([&](int s, const uint4 (&raw)[kSplitStatsNV]) {
        unsigned mask = 0u;
#pragma unroll
        for (int j = 0; j < kSplitStatsNV; ++j) {
            short2_t at[4];
            value_places(rs, raw[j], stats_group_first(s, j) + lane, s, base, at);
            ushort2_t least = {0xFFFF, 0xFFFF};                                  // (of the magnitudes: 0 where one is small)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                first = __builtin_elementwise_min(first, at[i]);
                least = __builtin_elementwise_min(least, (ushort2_t)__builtin_elementwise_abs(at[i]));
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int place = at[i][h];
                    if ((unsigned)(place + kWindow) <= (unsigned)(2 * kWindow)) atomicAdd(&mine[kWindow + place], 1u);
                }
            }
            if (__ballot(least[0] == 0 || least[1] == 0)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) mask |= at[e / 2][e % 2] == 0 ? 1u << (j * 8 + e) : 0u;
            }
        }
        append<true>(rs, s, mask, sh, kSmallList);
    });
    const int n_first = (int)-block_max(-(float)min((int)first[0], (int)first[1]), sh);
    const int n_small = sh.n;
    if (n_first < -kWindow || n_first > kWindow || n_small > kSmallList) return false;
    fill_list<true>(rs, n_small, sh);
    M = value_at(n_first, base);
    if (n_first == 0) {
        float mx = kNegInf;
        for (int i = tid; i < n_small; i += kST) mx = fmaxf(mx, composite_value(sh.list[i]));
        M = block_max(mx, sh);
    }
    w.move(M);
    const double small = ldexp((double)list_sum(n_small, 0ull, w, sh), -kListShift);
    // masses in order; the first bin with which they reach the target
    uint32_t n[kValuesPer];
    double one[kValuesPer], sum = 0.0, total;
#pragma unroll
    for (int i = 0; i < kValuesPer; ++i) {
        const int bin = tid * kValuesPer + i;
        n[i] = bin < kValues ? counts[bin] + counts[kValues + bin] : 0u;
        one[i] = n[i] && bin != kWindow ? w.weight(value_at(bin - kWindow, base)) : 0.0;
        sum += bin == kWindow ? small : (double)n[i] * one[i];
    }
    if (tid == 0) sh.at = INT32_MAX;
    double b = block_scan_excl(sum, sh.red, total), b_hit = 0.0;
    const double target = (double)p * total;
    int hit = INT32_MAX, n_hit = 0;
#pragma unroll
    for (int i = 0; i < kValuesPer; ++i) {
        const int bin = tid * kValuesPer + i;
        const double next = b + (bin == kWindow ? small : (double)n[i] * one[i]);
        if (n[i] && next >= target && hit == INT32_MAX) { hit = bin; b_hit = b; n_hit = (int)n[i]; atomicMin(&sh.at, bin); }
        b = next;
    }
    __syncthreads();
    const int last = sh.at;
    if (last == INT32_MAX) return false;                                         // (uniform)
    if (hit == last) { sh.red[kSW] = b_hit; sh.last = n_hit; }
    __syncthreads();
    const double rest = target - sh.red[kSW];
    const float t = value_at(last - kWindow, base);
    const double w_t = w.weight(t);
    int ties = 0;
    cut = Cut{t, INT32_MAX, a_min};
    if (last != kWindow) {
        const double need = ceil(rest / w_t);
        ties = need >= (double)sh.last ? sh.last : need < 1.0 ? 1 : (int)need;
        if (w.exponent(t) < a_min) ties = 0;
    }
    __syncthreads();
    if (last == kWindow) {
        const unsigned long long c = select<true>(n_small, 0ull, ldexp(rest, kListShift), w, sh);
        if (!c) return false;
        cut.t = composite_value(c);
        cut.id = composite_id(c);
    }
    unsigned long long mine_kept = 0, all_kept;
#pragma unroll
    for (int i = 0; i < kValuesPer; ++i) {
        const int bin = tid * kValuesPer + i;
        const bool keep = bin < last && bin != kWindow && n[i] && w.exponent(value_at(bin - kWindow, base)) >= a_min;
        if (keep) mine_kept += n[i];
        if (bin < kValues) weight[bin] = keep ? one[i] : 0.0;                    // (the counts are in registers: list_sum and the scan lie between)
    }
    uint32_t* const tied = reinterpret_cast<uint32_t*>(sh.mass);                 // per segment
    static_assert(sizeof(sh.mass) >= kBins * sizeof(uint32_t), "counts for id_of_tie");
    for (int i = tid; i < kBins; i += kST) tied[i] = 0u;
    block_scan_excl(mine_kept, sh.redu, all_kept);
    kept = (int)all_kept + ties;
    rs.each([&](int s, const uint4 (&raw)[kSplitStatsNV]) {
        double seg = 0.0;
        int eq = 0;
#pragma unroll
        for (int j = 0; j < kSplitStatsNV; ++j) {
            short2_t at[4];
            value_places(rs, raw[j], stats_group_first(s, j) + lane, s, base, at);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int place = at[e / 2][e % 2];
                if (place < last - kWindow) seg += weight[kWindow + place];      // (none lies in front of the window: M would)
                eq += __builtin_popcountll(__ballot(place == last - kWindow));
            }
        }
        seg = wave_sum(seg);
        if (lane == 0) { sh.seg[s] = seg; tied[s] = (uint32_t)eq; }
    });
    __syncthreads();
    if (ties > 0) {
        // the first `ties` of them by id
        unsigned long long c[kSegsPer], own = 0, all;
#pragma unroll
        for (int i = 0; i < kSegsPer; ++i) { const int s = tid * kSegsPer + i; c[i] = s < rs.n_seg ? tied[s] : 0u; own += c[i]; }
        unsigned long long before = block_scan_excl(own, sh.redu, all);
#pragma unroll
        for (int i = 0; i < kSegsPer; ++i) {
            const int s = tid * kSegsPer + i;
            if (s < rs.n_seg && before < (unsigned long long)ties) sh.seg[s] += w_t * (double)min(c[i], (unsigned long long)ties - before);
            before += c[i];
        }
        cut.id = id_of_tie<true>(rs, tied, t, (unsigned long long)ties, sh);
    }
    if (n_small > 0 && last >= kWindow) kept += list_to_segments<true>(rs, n_small, cut, w, true, sh);
    return true;
}

// The list in its order, by one histogram: every entry's place is its bin's start and the number of entries of the bin in front of it.  False: a list of more than half the room, or
// with a bin of more than kDeep entries (many equal logits).
constexpr int kSortMost = kSampleList / 2 - 4, kDeep = 192;
__device__ __forceinline__ bool sort_list(int n, RowShared& sh)
{
    constexpr int PER = (kSortMost + kST - 1) / kST;
    const int tid = threadIdx.x;
    if (n > kSortMost) return false;                                             // (uniform)
    float hi_z = kNegInf, lo_z = kNegInf;
    unsigned long long c[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int i = e * kST + tid;
        c[e] = i < n ? sh.list[i] : 0ull;
        if (i < n) { const float z = composite_value(c[e]); hi_z = fmaxf(hi_z, z); lo_z = fmaxf(lo_z, -z); }
    }
    for (int i = tid; i < kListBins; i += kST) sh.count[i] = 0u;
    if (tid == 0) sh.at = 0;
    const float top = block_max(hi_z, sh), bottom = -block_max(lo_z, sh);
    // (bins even in the logit: of the keys, most lie near 0)
    const float scale = (float)(kListBins - 1) / (top - bottom);                 // (0 or infinite where the two are far apart or equal)
    int bin[PER], pos[PER], deep = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e)
        if (e * kST + tid < n) {
            bin[e] = (int)fminf(fmaxf((top - composite_value(c[e])) * scale, 0.f), (float)(kListBins - 1));
            pos[e] = (int)atomicAdd(&sh.count[bin[e]], 1u);
            deep = max(deep, pos[e]);
        }
    if (__ballot(deep >= kDeep) && (tid & (kWave - 1)) == 0) sh.at = 1;
    __syncthreads();
    if (sh.at) return false;
    const uint32_t n0 = sh.count[2 * tid], n1 = sh.count[2 * tid + 1];
    static_assert(kListBins == 2 * kST, "two bins a thread");
    unsigned long long all;
    const int start = (int)block_scan_excl((unsigned long long)(n0 + n1), sh.redu, all);
    int* const starts = reinterpret_cast<int*>(sh.mass);
    starts[2 * tid] = start;
    starts[2 * tid + 1] = start + (int)n0;
    __syncthreads();
    unsigned long long* const by_bin = &sh.list[kSortMost];                      // (and four words behind its end)
#pragma unroll
    for (int e = 0; e < PER; ++e) if (e * kST + tid < n) by_bin[starts[bin[e]] + pos[e]] = c[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        if (e * kST >= n) break;                                                 // (uniform)
        if (e * kST + tid < n) {
            const int s0 = starts[bin[e]], m = (int)sh.count[bin[e]];
            int rank = s0;
            for (int i = 0; i < m; i += 4) {                                     // (entries behind the bin's, or the list's, are smaller or not counted)
#pragma unroll
                for (int j = 0; j < 4; ++j) rank += i + j < m && by_bin[s0 + i + j] > c[e];
            }
            sh.list[rank] = c[e];
        }
    }
    __syncthreads();
    return true;
}

// Of the ordered list's first n_k entries: how many top-p (a prefix that reaches the target mass; infinite: all) and min-p leave.  `listed`: the mass of the n_k.
__device__ __forceinline__ int kept_of_list(int n_k, double p, double target, double a_min, const Weights& w, RowShared& sh, double& listed)
{
    constexpr int PER = (kSortMost + kST - 1) / kST;
    const int tid = threadIdx.x, each = (n_k + kST - 1) / kST, first = tid * each;
    double one[PER], sum = 0.0;
    int fails = INT32_MAX;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        one[e] = 0.0;
        if (e < each && first + e < n_k) {
            const float z = composite_value(sh.list[first + e]);
            one[e] = w.weight(z);
            if (w.exponent(z) < a_min) fails = min(fails, first + e);
        }
        sum += one[e];
    }
    if (tid == 0) sh.at = n_k;
    double before = block_scan_excl(sum, sh.red, listed);
    if (!(target < (double)INFINITY)) target = p * listed;                       // (of theirs)
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        if (e < each && first + e < n_k && !(before < target)) fails = min(fails, first + e);
        before += one[e];
    }
    if (fails < n_k) atomicMin(&sh.at, fails);
    __syncthreads();
    const int kept = sh.at;
    __syncthreads();
    return kept;
}

// The draw from the ordered list's first `kept` <= kST entries, one a thread: their order by id is found by counting the ids in front of each.
__device__ __forceinline__ void draw_short(int kept, float u, const Weights& w, RowShared& sh, int& tok, float& z_tok, double& total)
{
    const int tid = threadIdx.x;
    const unsigned long long c = tid < kept ? sh.list[tid] : 0ull;
    const uint32_t x = (uint32_t)composite_id(c);
    static_assert(kST + 16 <= kListBins && kST <= kSegs, "the arrays that lend their room");
    if (tid < kept) sh.count[tid] = x;
    if (tid < 16) sh.count[kept + tid] = 0xFFFFFFFFu;
    if (tid == 0) { sh.at = INT32_MAX; sh.last = -1; }
    __syncthreads();
    if ((tid & ~(kWave - 1)) < kept) {
        int rank = 0;
        for (int j = 0; j < kept; j += 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) rank += sh.count[j + i] < x;
        }
        if (tid < kept) {
            const float z = composite_value(c);
            sh.mass[rank] = pack2(x, __float_as_uint(z));
            const double one = w.weight(z);
            sh.seg[rank] = one > kNoId * kST ? one : 0.0;                        // (of a kept mass of kST at most)
        }
    }
    __syncthreads();
    const double mine = tid < kept ? sh.seg[tid] : 0.0, before = block_scan_excl(mine, sh.red, total);
    if (mine > 0.0) {
        if (before + mine > (u >= 0.f ? (double)u : 0.0) * total) atomicMin(&sh.at, tid);
        atomicMax(&sh.last, tid);
    }
    __syncthreads();
    const unsigned long long drawn = sh.mass[sh.at != INT32_MAX ? sh.at : sh.last];
    tok = (int)(uint32_t)drawn;
    z_tok = __uint_as_float((uint32_t)(drawn >> 32));
}

// PHASE 0: everything but the second pass of histograms whose rows have several workgroups; 1: those.
// (128 registers, so that two workgroups share a CU with their LDS.  What they do not hold, 8 to 16 values a thread, is written to scratch between the passes, once a row, and in none of their loops;
// only sample_careful has a few such accesses in its loops.)
template <bool BF16, int PHASE>
__global__ __launch_bounds__(kST, 4) void sample_kernel(const SampleArgs a)
{
    __shared__ RowShared sh;
    const int tid = threadIdx.x, parts = a.parts, part = blockIdx.x % parts;
    const int64_t row = blockIdx.x / parts;
    const RowStream<BF16> rs(a.logits, a.ld, row, a.V);
    float T = a.T_rows ? a.T_rows[row] : a.T;
    int k = a.k_rows ? a.k_rows[row] : a.top_k;
    const float p = a.p_rows ? a.p_rows[row] : a.top_p, min_p = a.minp_rows ? a.minp_rows[row] : a.min_p;
    if (!(T > 0.f && T <= kFloatMax)) { T = 1.f; k = 1; }                        // (greedy)
    const bool cut_p = p > 0.f && p < 1.f;
    if (PHASE == 1 && (k > 0 || !cut_p)) return;
    const float per = kHistPerNat / T;
    const double a_min = min_p > 0.f ? log2((double)fminf(min_p, 1.f)) : -__builtin_huge_val();

    Weights w;
    w.set(0.f, T);
    Cut cut{kNegInf, -1, a_min};
    Plan pl;
    Bracket br{false, 0.f, 0.f};
    uint4 ahead[kSplitStatsNV];
    int kept = 0;
    float M = kNegInf;
    double total = 0.0, above_ref = 0.0;
    bool done = false, drawn = false;
    int tok = -1;
    float z_tok = 0.f;
    const float u = a.u[row];
    if (tid == 0) sh.n = 0;
    if constexpr (PHASE == 0) {
        if (parts > 1 && tid == 0) open_arrival(RowScratch<BF16>(a, row).word);
        rs.first_of(part, ahead);                                                // (under way while the peek is looked at)
        pl = peek<BF16>(rs, a.V, T, k, p, min_p, sh);
        w.move(pl.ref);
        if (!BF16 && parts > 1 && cut_p && k <= 0 && pl.way != kHist && part == 0 && tid == 0) RowScratch<BF16>(a, row).head[parts * 3] = 0ull;   // (nothing for the second launch)
        __syncthreads();
    } else {
        const RowScratch<BF16> rx(a, row);
        const unsigned long long h = rx.head[parts * 3], ends = rx.head[parts * 3 + 1];
        if ((uint32_t)h == 0u) return;
        pl = Plan{kHist, __uint_as_float((uint32_t)(h >> 32)), kNegInf, false, 0.f};
        br = Bracket{(uint32_t)h == 2u, __uint_as_float((uint32_t)ends), __uint_as_float((uint32_t)(ends >> 32))};
        M = __uint_as_float((uint32_t)(rx.head[parts * 3 + 2] >> 32));
        if (tid == 0) open_arrival(rx.word);
        __syncthreads();
    }
    if (pl.way == kCareful && part != 0) return;
    bool alone = parts == 1;
    if (BF16 && pl.way == kHist && part != 0) return;                            // (counted by one)
    if (pl.way == kSum || pl.way == kList) {
        if constexpr (PHASE == 0) {
            if (pl.way == kSum) first_pass<BF16, kSum, false>(rs, ahead, part, parts, pl, w, T, sh, M, kept, total, above_ref);
            else if (pl.total) first_pass<BF16, kList, true>(rs, ahead, part, parts, pl, w, T, sh, M, kept, total, above_ref);
            else first_pass<BF16, kList, false>(rs, ahead, part, parts, pl, w, T, sh, M, kept, total, above_ref);
            if (parts > 1 && !gather<BF16>(rs, RowScratch<BF16>(a, row), part, parts, pl.way == kSum, pl.way == kList, M, kept, total, sh)) return;
            const bool near = fabs(((double)M - (double)pl.ref) * w.c) < 500.0;   // (+inf: not)
            if (pl.way == kSum) {
                done = near;
            } else if (near && sh.n <= kSampleList) {
                const int n = sh.n;
                w.move(M);
                const double row_total = pl.total ? total * w.weight(pl.ref) : 0.0;  // (it was summed against the peek's largest)
                unsigned long long last = 0;
                done = k <= 0 || n >= k || !(pl.least > kNegInf);
                if (done && sort_list(n, sh)) {
                    double listed;
                    const int n_k = k > 0 ? min(n, k) : n;
                    const int m = kept_of_list(n_k, cut_p ? (double)p : 2.0, pl.total ? (double)p * row_total : (double)INFINITY, a_min, w, sh, listed);
                    done = !pl.total || listed >= (double)p * row_total;
                    if (done && m <= kST) {
                        drawn = true;
                        kept = m;
                        draw_short(m, u, w, sh, tok, z_tok, total);
                    } else if (done) {
                        cut.t = composite_value(sh.list[m - 1]);
                        cut.id = composite_id(sh.list[m - 1]);
                        kept = list_to_segments<BF16>(rs, m, cut, w, false, sh);
                    }
                } else if (done) {
                    __syncthreads();
                    if (k > 0 && k < n) last = select<false>(n, 0ull, (double)k, w, sh);
                    if (cut_p) {
                        const unsigned long long listed = list_sum(n, last, w, sh);
                        const double target = k > 0 ? (double)p * (double)listed : ldexp((double)p * row_total, kListShift);
                        done = target <= (double)listed;
                        if (done) last = max(last, select<true>(n, last, target, w, sh));
                    }
                    if (done) {
                        if (last) { cut.t = composite_value(last); cut.id = composite_id(last); }
                        kept = list_to_segments<BF16>(rs, n, cut, w, false, sh);
                    }
                }
            }
            if (!done && near && pl.total) { pl.way = kHist; alone = true; }     // (the peek took a spread row for a peaked one)
            if (!done && near && pl.way == kList && k <= 0 && !cut_p) {          // (min-p alone, and a list too short for it: a pass that sums)
                w.move(M);
                second_pass<BF16, true>(rs, 0, 1, br, pl.ref, per, w, a_min, sh, kept, total);
                done = true;
            }
        }
    }
    if constexpr (BF16) {
        __syncthreads();
        if (pl.way == kHist) done = count_values(rs, pl, T, p, a_min, w, cut, kept, M, sh);
    } else if (pl.way == kHist) {
        const int at = alone ? 0 : part, of = alone ? 1 : parts;
        bool good = PHASE == 1;
        if constexpr (PHASE == 0) {
            w.move(pl.ref);
            __syncthreads();
            if (!alone) pl.far = (float)(kBins - 1);                             // (there is no third pass)
            for (int i = tid; i < 2 * kBins; i += kST) sh.hist[0][i] = 0ull;
            __syncthreads();
            rs.first_of(at, ahead);
            first_pass<BF16, kHist, false>(rs, ahead, at, of, pl, w, T, sh, M, kept, total, above_ref);
            bool last = true;
            if (!alone) {
                const RowScratch<BF16> rx(a, row);
                for (int i = tid; i < kBins; i += kST) put_shared(&rx.hist[(int64_t)part * kBins + i], sh.hist[0][i] + sh.hist[1][i]);
                if (tid == 0) {
                    put_shared(&rx.head[part * 3], pack2(0u, __float_as_uint(M)));
                    put_shared(&rx.head[part * 3 + 1], (unsigned long long)__double_as_longlong(total));
                    put_shared(&rx.head[part * 3 + 2], (unsigned long long)__double_as_longlong(above_ref));
                }
                last = arrive_last(rx.word, (unsigned)parts, tid == 0);
                if (!last) return;                                               // (the second launch goes on)
                unsigned long long sums[kBins / kST] = {};
#pragma unroll 4
                for (int j = 0; j < parts; ++j)
#pragma unroll
                    for (int i = 0; i < kBins / kST; ++i) sums[i] += get_shared(&rx.hist[(int64_t)j * kBins + i * kST + tid]);
                const int lane = tid & (kWave - 1), mine = min(lane, parts - 1);
                const unsigned long long h0 = get_shared(&rx.head[mine * 3]), h1 = get_shared(&rx.head[mine * 3 + 1]), h2 = get_shared(&rx.head[mine * 3 + 2]);
                M = wave_max(__uint_as_float((uint32_t)(h0 >> 32)));
                total = wave_sum(lane < parts ? __longlong_as_double((long long)h1) : 0.0);
                above_ref = wave_sum(lane < parts ? __longlong_as_double((long long)h2) : 0.0);
#pragma unroll
                for (int i = 0; i < kBins / kST; ++i) { sh.hist[0][i * kST + tid] = sums[i]; sh.hist[1][i * kST + tid] = 0ull; }
                __syncthreads();
            }
            int found = M <= kFloatMax ? bracket(p, total, above_ref, pl.far, sh, br) : -1;
            if (found == 0) {
                pl.far = (float)(kBins - 1);
                for (int i = tid; i < 2 * kBins; i += kST) sh.hist[0][i] = 0ull;
                __syncthreads();
                rs.first_of(0, ahead);
                first_pass<BF16, kHist, false>(rs, ahead, 0, 1, pl, w, T, sh, M, kept, total, above_ref);
                found = bracket(p, total, above_ref, pl.far, sh, br);
            }
            good = found > 0;
            if (good && a_min > -__builtin_huge_val()) {
                // min-p against where top-p ends, in bins: clearly above, then it alone decides (the first bin reaches up without end: nothing lies clearly above
                // that); or else the list begins two bins earlier, so that whatever fails min-p is in it
                const double x = ((double)pl.ref - ((double)M + a_min / kLog2e * (double)T)) * (double)per;
                br.by_min_p = br.from >= 1.f && x < (double)br.from - 1.0;
                if (!br.by_min_p && x < (double)br.to + 1.0) br.from = fmaxf(br.from - 2.f, 0.f);
            }
            if (!alone) {
                if (tid == 0) {
                    const RowScratch<BF16> rx(a, row);
                    put_shared(&rx.head[parts * 3], pack2(good ? (br.by_min_p ? 2u : 1u) : 0u, __float_as_uint(pl.ref)));
                    put_shared(&rx.head[parts * 3 + 1], pack2(__float_as_uint(br.from), __float_as_uint(br.to)));
                    put_shared(&rx.head[parts * 3 + 2], pack2(0u, __float_as_uint(M)));
                }
                if (good) return;
            }
        }
        if (good) {
            w.move(M);
            if (tid == 0) sh.n = 0;
            __syncthreads();
            if (br.by_min_p) second_pass<BF16, true>(rs, at, of, br, pl.ref, per, w, a_min, sh, kept, total);
            else second_pass<BF16, false>(rs, at, of, br, pl.ref, per, w, a_min, sh, kept, total);
            if (!alone && !gather<BF16>(rs, RowScratch<BF16>(a, row), part, parts, true, true, M, kept, total, sh)) return;
            if (br.by_min_p) {
                done = true;
            } else if (sh.n <= kSampleList) {
                const int n = sh.n;
                double above = 0.0, mine = 0.0;
                for (int i = tid * kSegsPer; i < min((tid + 1) * kSegsPer, rs.n_seg); ++i) mine += sh.seg[i];
                block_scan_excl(mine, sh.red, above);
                const double target = (double)p * total - above;
                unsigned long long last = 0;
                int m = n;                                                   // (0: min-p leaves nothing of the list)
                if (!(target > 0.0)) {
                } else if (sort_list(n, sh)) {
                    double listed;
                    m = kept_of_list(n, 1.0, target, a_min, w, sh, listed);
                    done = target <= listed;
                    if (done && m > 0) last = sh.list[m - 1];
                } else {
                    __syncthreads();
                    const unsigned long long listed = list_sum(n, 0ull, w, sh);
                    done = ldexp(target, kListShift) <= (double)listed;
                    if (done) last = select<true>(n, 0ull, ldexp(target, kListShift), w, sh);
                }
                if (done && m > 0) {
                    cut = Cut{composite_value(last), composite_id(last), a_min};
                    kept += list_to_segments<BF16>(rs, n, cut, w, true, sh);
                }
            }
        }
    }
    if (!done) {
        __syncthreads();
        Weights w2;                                                              // (what a call takes by reference lives in memory)
        Cut cut2;
        int kept2;
        float M2;
        sample_careful<BF16>(a.logits, a.ld, row, T, k, p, min_p, a.V, sh, w2, cut2, kept2, M2);
        w = w2;
        cut = cut2;
        kept = kept2;
        M = M2;
    }
    if (!drawn && M > kNegInf) draw<BF16>(rs, w, cut, u, sh, tok, z_tok, total);
    if (tid == 0) {
        a.tok[row] = tok;
        a.prob[row] = tok < 0 ? 0.f : (float)(w.weight(z_tok) / total);
        a.count[row] = kept;
        a.lse[row] = tok < 0 ? kNegInf : (float)(w.ref / (double)T + log(total));
    }
}

template <bool BF16>
hipError_t launch(const SampleArgs& a, int64_t rows, bool hist, hipStream_t stream)
{
    hipLaunchKernelGGL((sample_kernel<BF16, 0>), dim3((unsigned)(rows * a.parts)), dim3(kST), 0, stream, a);
    if constexpr (!BF16)
        if (a.parts > 1 && hist) hipLaunchKernelGGL((sample_kernel<BF16, 1>), dim3((unsigned)(rows * a.parts)), dim3(kST), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const void* logits, int dtype, int64_t ld, int n_rows, int V, float temperature, int top_k, float top_p, float min_p,
                         const float* temperature_rows, const int32_t* top_k_rows, const float* top_p_rows, const float* min_p_rows,
                         const float* uniforms, int32_t* tok, float* prob, int32_t* count, float* lse, void* scratch, size_t scratch_bytes, hipStream_t stream)
{
    if (n_rows == 0) return hipSuccess;
    const int parts = scratch && scratch_bytes >= sample_scratch_bytes(dtype, n_rows, V) ? sample_parts(dtype, n_rows, V) : 1;
    const SampleArgs a{logits, ld, V, temperature, top_k, top_p, min_p, temperature_rows, top_k_rows, top_p_rows, min_p_rows, uniforms, tok, prob, count, lse,
                       (char*)scratch, parts};
    const bool greedy = !temperature_rows && temperature == 0.f;
    const bool hist = !greedy && (top_p_rows || (top_p > 0.f && top_p < 1.f)) && (top_k_rows || top_k <= 0);   // (may a row take two passes?)
    return dtype == 1 ? launch<true>(a, n_rows, hist, stream) : launch<false>(a, n_rows, hist, stream);
}

}  // namespace picospec
