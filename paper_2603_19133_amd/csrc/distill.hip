// Distillation of a drafter on the target's Top-K records: Kullback-Leibler divergence of q = softmax(z / T) from a record
// (id_j, p_j), j < count, with its gradient, and the expected acceptance sum_j min(p_j, q_j).  With y = (z - M) / T, w = e^y,
// S = sum w, q = w / S:
//   tail 0   L = sum_j ph_j (ln ph_j - ln q_j), ph = p / sum p
//            T dL/dz_v = q_v - ph_v
//   tail 1   L = sum_j p_j (ln p_j - ln q_j) + pt (ln pt - ln qt),  pt = max(0, 1 - sum p), qt = q's mass off the record
//            T dL/dz_v = W q_v - p_v on the record, (W - pt / qt) q_v off it,  W = sum p + pt
// What bounds it: the row is read once (forward) and the gradient written once, at the rate of a copy where both are in one call (2048 rows of 128,256 fp32 with records of
// 1024 450 us = 4.7 TB/s, 4096 of 151,936 bf16 500 us = 5.0 TB/s); the forward alone is at 5.5 TB/s with short records.  With the gradient in the same call a row is
// read twice by its workgroup, but for what a thread holds of it, and the second time from the caches.
// qt is summed directly: 1 - sum_j q_j loses it where the record holds nearly all of q, and the gradient off the record has pt / qt in it. What is off the record is summed and, in
// the gradient, formed against its own largest logit R, not M: 87 T below M fp32 weights are 0, where pt q_v / qt still is of the size of pt. Against M stands one factor,
// 2^((R - M) c), in 64 bits; where they do not hold it either (745 T) nothing is off the record.
// The maxima pass NaN by; the sums carry it: S of a row with NaN or +inf in it is NaN, M of it may be anything, -inf as of a row that is masked whole.
#include "common.hpp"
#include "kernels.hpp"

namespace picospec {

namespace {

// two (bf16) or one (fp32) values of -inf
template <bool BF16> constexpr uint32_t kMaskedPair = BF16 ? 0xFF80FF80u : 0xFF800000u;

// What the roundings of a record's entries may leave of 1: half a step of fp32 each, 2^-24 of their sum, and what they share of the error of their
// row's sum (records of picospec_compress: a few 10^-7)
constexpr double kRounding = 0x1p-20;

constexpr float kNoReference = -67108864.f;      // -2^26: above it r is no more than 2 below the largest exponent

// 2^a, -1200 <= a <= 0 (common.hpp's without its branch, behind which the compiler takes 40 registers more here)
__device__ __forceinline__ double exp2_down(double a)
{
    const double n = rint(a);
    return ldexp((double)__builtin_amdgcn_exp2f((float)(a - n)), (int)n);
}

// two floats as one word, of a hand-over or of the statistics
__device__ __forceinline__ unsigned long long two_floats(float a, float b) { return (unsigned long long)__float_as_uint(a) | (unsigned long long)__float_as_uint(b) << 32; }
__device__ __forceinline__ float first_float(unsigned long long w) { return __uint_as_float((uint32_t)w); }
__device__ __forceinline__ float second_float(unsigned long long w) { return __uint_as_float((uint32_t)(w >> 32)); }

enum Slots : int { kNone, kEntries, kHalves };  // of a long record, in LDS

struct DistillArgs {
    const void* logits; int64_t ld; int V; float T;
    const int32_t* idx; const float* prob; const int32_t* count; int k, tail;
    float *loss, *accept; double4* stats; const float* weight; void* grad; int64_t ld_grad;
    char* scratch; int parts;                     // workgroups of a row, 1 but for SPLIT
};

// sums of N doubles over the workgroup, the same bits in every thread (fixed order)
template <int kDW, int N>
__device__ __forceinline__ void block_sums(double (&v)[N], double* sh)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const double s = wave_sum(v[i]);
        if (lane == 0) sh[i * kDW + wave] = s;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < kDW; ++w) s += sh[i * kDW + w];
        v[i] = s;
    }
    __syncthreads();
}

// log2 p, p > 0 and finite, to 2^-24 or so whatever its size: the exponent apart, the mantissa's logarithm in fp32 (a 64-bit logarithm per entry of a long record costs as
// much as the row)
__device__ __forceinline__ double log2_of(float p)
{
    return (double)__builtin_amdgcn_frexp_expf(p) + (double)__builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(p));
}

// 16 bytes to an address that is element-aligned only: the output rows need not lie like the input's (global stores take any alignment).  Non-temporal: the
// gradient is not read here again, and the rows that are read twice keep their place in the caches (2048 rows of 128,256 fp32: 671 -> 544 us).
template <bool BF16>
__device__ __forceinline__ void store_vec(char* grad_row, const RowView& rv, int q, const float (&g)[Vec<BF16>::N])
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4;
    const int x = q * N - rv.o;
    if (x >= 0 && x + N <= rv.L - rv.o) {
        u32x4_t t;
        if constexpr (BF16) { t.x = pack_bf16(g[0], g[1]); t.y = pack_bf16(g[2], g[3]); t.z = pack_bf16(g[4], g[5]); t.w = pack_bf16(g[6], g[7]); }
        else { t.x = __float_as_uint(g[0]); t.y = __float_as_uint(g[1]); t.z = __float_as_uint(g[2]); t.w = __float_as_uint(g[3]); }
        __builtin_nontemporal_store(t, reinterpret_cast<loose_t*>(grad_row + (int64_t)x * ESZ));
        return;
    }
    const unsigned vm = vec_valid_mask<BF16>(rv, q);
#pragma unroll
    for (int e = 0; e < N; ++e)
        if ((vm >> e) & 1u) {
            if constexpr (BF16) reinterpret_cast<uint16_t*>(grad_row)[x + e] = (uint16_t)pack_bf16(g[e], 0.f);
            else reinterpret_cast<float*>(grad_row)[x + e] = g[e];
        }
}

template <bool BF16>
__device__ __forceinline__ void store_one(char* grad_row, int x, float g)
{
    if constexpr (BF16) reinterpret_cast<uint16_t*>(grad_row)[x] = (uint16_t)pack_bf16(g, 0.f);
    else reinterpret_cast<float*>(grad_row)[x] = g;
}

// One row per workgroup.  FWD: loss, acceptance and the row's statistics; GRAD: the gradient, from the statistics of this or of an earlier call.
// HELD: vectors that a thread keeps from the sum to the gradient; its registers are bound to what lets two workgroups share a CU (with the tail the compiler took two more: 2000 rows
// of 32,000 bf16, 300 entries, gradient in the call 107 us, so 78).
//
// Weights are 2^(z c - r), c = log2(e) / T in fp32 and r an integer that is the same for a wave, near its largest exponent: one fused multiply-add and one
// exponential per element (the product inside is exact, so the error is that of (z - M) c).  r moves up, and the lanes' sums are rescaled, only when an element
// lies more than 2^64 above it.  What a wave has seen so far may be ids masked with a finite value, of which r would have no more than fp32's 24 bits and the exponents
// be what its rounding leaves, 2^439 for -1e10: below kNoReference r is not taken and the weights are 0 (a row of no more than that has |R c| >= 2^24).  Rows with |R c| >= 2^24, where r is no integer near R c any more, take (z - R) c and read the row once more.
//
// What the record's entries need of the row, and the row of them (SLOTS):
//   entries The record lies in LDS in the order of its ids: a bit per element, the number of bits in front of every 32, and the entries' p.  The streaming finds the
//           entry of a marked element by counting bits; it leaves the element's logit there (FWD) and writes its gradient in place (GRAD).
//   halves  The same without gradient, for bf16 records with the tail: a marked element's half of its vector goes to the slot of the half's first mark, as it came from
//           memory (two writes a vector instead of one for each of its elements that some lane has marked), and the entries find their logits in them behind the stream.
//   none    The logits are gathered, and the entries' gradients written over what the streaming left in their places: less to prepare, but every entry touches a line
//           of the row each way.  For short records, and for vocabularies whose marks do not fit (kDistillLds).
// Forward kernels but for halves are held to 64 registers, eight waves per SIMD (with the tail the compiler took 66 to 68 of its own accord).
// SPLIT: a row's workgroups take consecutive trips of it; forward, the last of them to arrive adds their sums up and goes on with the record.
template <bool BF16, bool FWD, bool GRAD, bool TAIL, int SLOTS, bool SPLIT, int kDT, int HELD>
__global__ __launch_bounds__(kDT, HELD ? 4 : FWD && !GRAD && SLOTS != kHalves ? 8 : kDT / 256) void distill_kernel(const DistillArgs a)
{
    constexpr int N = Vec<BF16>::N, G = 2, kDW = kDT / kWave;    // G: vectors per step
    static_assert(HELD % G == 0 && HELD <= kDistillMostHeld && G + 1 <= kDistillAhead && (!SPLIT || (HELD == 0 && !SLOTS && FWD != GRAD)), "whole steps; split rows in the plainest form");
    constexpr bool HALVES = SLOTS == kHalves;
    static_assert(!HALVES || (FWD && !GRAD), "halves of vectors serve what only reads");
    __shared__ double sh[5 * kDW];
    extern __shared__ __attribute__((aligned(8))) uint32_t on_record[];   // (TAIL && FWD) || SLOTS: bit o + id
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int parts = SPLIT ? a.parts : 1, part = SPLIT ? (int)(blockIdx.x % (unsigned)parts) : 0;
    const int64_t row = SPLIT ? blockIdx.x / (unsigned)parts : blockIdx.x;
    const RowView rv = row_view<BF16>(a.logits, a.ld, row, a.V);
    const int nq = (rv.L + N - 1) / N, all_trips = (nq + kDT - 1) / kDT, share = SPLIT ? (all_trips + parts - 1) / parts : all_trips;
    const int begin = SPLIT ? min(part * share, all_trips) : 0, trips = SPLIT ? min(begin + share, all_trips) : all_trips;
    const float c = 1.4426950408889634f / a.T;
    const double c64 = 1.4426950408889634 / (double)a.T;
    const int count = min(max(a.count[row], 0), a.k);
    char* const grad_row = (char*)a.grad + row * a.ld_grad * (BF16 ? 2 : 4);
    if (count == 0) {                                            // (a position that is not trained on)
        if (FWD && tid == 0 && part == 0) {
            a.loss[row] = 0.f;
            if (a.accept) a.accept[row] = 0.f;
            if (a.stats) a.stats[row] = make_double4(0.0, 1.0, 0.0, 0.0);
        }
        if constexpr (GRAD) {
            const float zero[N] = {};
            for (int i = begin; i < trips; ++i) if (i * kDT + tid < nq) store_vec<BF16>(grad_row, rv, i * kDT + tid, zero);
        }
        return;
    }

    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)rv.base, 0, nq * 16, 0x00020000);
    auto load = [&](int i, auto aux) {                           // vector i * kDT + tid; behind the row: zero
        const u32x4_t t = __builtin_amdgcn_raw_buffer_load_b128(rsrc, tid * 16, trip_group_first(i, kDT) * 16, decltype(aux)::value);
        return make_uint4(t.x, t.y, t.z, t.w);
    };
    using Stream = std::integral_constant<int, 2>;               // (read once: non-temporal)
    using Keep = std::integral_constant<int, 0>;
    using First = std::conditional_t<GRAD, Keep, Stream>;        // (what is not held is read again by the gradient)

    if constexpr (SPLIT && FWD) {
        if (tid == 0) open_arrival(reinterpret_cast<unsigned long long*>(a.scratch + row * (int64_t)distill_scratch_row(parts)));
    }
    uint4 held[HELD ? HELD : 1];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) held[i] = i < trips ? load(i, Stream{}) : make_uint4(0, 0, 0, 0);
    }

    // the record: entries tid, tid + kDT, .. (ids outside the vocabulary: no entry)
    struct Entry { int id; float p, z; };
    auto id_of = [&](int s) {
        const int id = s < count ? a.idx[row * a.k + s] : -1;
        if ((unsigned)id >= (unsigned)a.V) return -1;
        if (SPLIT && GRAD && ((rv.o + id) / (N * kDT) < begin || (rv.o + id) / (N * kDT) >= trips)) return -1;       // (another part's)
        return id;
    };
    const int words = (rv.L + 31) / 32;
    constexpr bool MARKS = SLOTS || (TAIL && FWD);
    uint16_t* const in_front = reinterpret_cast<uint16_t*>(on_record + words);
    float* const slot_p = reinterpret_cast<float*>(on_record + words + (words + 1) / 2);
    float* const slot_z = slot_p + a.k;
    uint2* const slot_half = reinterpret_cast<uint2*>(on_record + (words + (words + 1) / 2 + 1) / 2 * 2);
    int n_slots = 0;
    Entry own{-1, 0.f, 0.f};
    if constexpr (!SLOTS) {
        own.id = id_of(tid);
        if (own.id >= 0) own.p = a.prob[row * a.k + tid];
        if (!(SPLIT && FWD) && own.id >= 0) own.z = logit_at<BF16>(a.logits, a.ld, row, own.id);      // (where the row is split, the one that needs it is not known yet)
    }
    if constexpr (MARKS) {
        constexpr int PER = kMaxK / kDT;
        int id[PER];
        float p[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            id[j] = id_of(j * kDT + tid);
            p[j] = SLOTS == kEntries && id[j] >= 0 ? a.prob[row * a.k + j * kDT + tid] : 0.f;
        }
        for (int w = tid; w < words; w += kDT) on_record[w] = 0u;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (id[j] >= 0) atomicOr(&on_record[(rv.o + id[j]) >> 5], 1u << ((rv.o + id[j]) & 31));
        __syncthreads();
        if constexpr (SLOTS) {
            const int each = (words + kDT - 1) / kDT, first = tid * each, end = min(first + each, words);
            int mine = 0;
            for (int w = first; w < end; ++w) mine += __builtin_popcount(on_record[w]);
            const int incl = wave_scan_incl(mine);
            int* const wave_sums = reinterpret_cast<int*>(sh);
            if (lane == kWave - 1) wave_sums[wave] = incl;
            __syncthreads();
            int before = incl - mine;
#pragma unroll
            for (int w = 0; w < kDW; ++w) { if (w < wave) before += wave_sums[w]; n_slots += wave_sums[w]; }
            for (int w = first; w < end; ++w) { in_front[w] = (uint16_t)before; before += __builtin_popcount(on_record[w]); }
            __syncthreads();
            if constexpr (SLOTS == kEntries) {
#pragma unroll
                for (int j = 0; j < PER; ++j)
                    if (id[j] >= 0) {
                        const int v = rv.o + id[j];
                        slot_p[in_front[v >> 5] + __builtin_popcount(on_record[v >> 5] & ((1u << (v & 31)) - 1u))] = p[j];
                    }
                __syncthreads();
            }
        }
    }
    // marks of vector q, and the slot of the first of them
    auto marks = [&](int q, int& slot) {
        const int v = min(q, nq - 1) * N, at = v & 31;
        const uint32_t word = on_record[v >> 5];
        if constexpr (SLOTS) slot = in_front[v >> 5] + __builtin_popcount(word & ((1u << at) - 1u));
        return (word >> at) & ((1u << N) - 1u);
    };
    Entry mine[HALVES ? kMaxK / kDT : 1];                          // HALVES: entries tid, tid + kDT, ..
    auto each_entry = [&](auto f) {
        if constexpr (HALVES) {
#pragma unroll
            for (int j = 0; j < kMaxK / kDT; ++j) if (mine[j].id >= 0) f(mine[j]);
        } else if constexpr (SLOTS) {
            for (int s = tid; s < n_slots; s += kDT) f(Entry{0, slot_p[s], slot_z[s]});
        } else {
            if (own.id >= 0) f(own);
#pragma unroll 1
            for (int s = tid + kDT; s < count; s += 4 * kDT) {                  // (four gathers under way at a time)
                Entry e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[i].id = id_of(s + i * kDT);
                    e[i].p = e[i].id >= 0 ? a.prob[row * a.k + s + i * kDT] : 0.f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i].z = e[i].id >= 0 ? logit_at<BF16>(a.logits, a.ld, row, e[i].id) : 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) if (e[i].id >= 0) f(e[i]);
            }
        }
    };

    float M, R;                                                     // largest logits: of the row, and of what is off the record (without TAIL: of the row)
    double S, b, mass, whole;                                       // sum of weights against M; of what is off the record: T dL/dz per weight against R; sum p; W
    if constexpr (FWD) {
        // the row's maximum and the sum: over all elements, TAIL over those off the record, whose maximum is mo
        float mx = kNegInf, mo = kNegInf, r = kNegInf, s = 0.f;
        auto values = [&](int q, const uint4& raw, float (&t)[N]) {           // -inf: not in the sum
            unpack<BF16>(raw, t);
            unsigned out = 0u;
            int slot = 0;
            if constexpr (MARKS) out = marks(q, slot);
            if (q == 0 || q >= nq - 1) {
                const unsigned vm = vec_valid_mask<BF16>(rv, q);
#pragma unroll
                for (int e = 0; e < N; ++e) t[e] = (vm >> e) & 1u ? t[e] : kNegInf;
            }
            if constexpr (TAIL && !SLOTS) {
#pragma unroll
                for (int e = 0; e < N; ++e) mx = fmaxf(mx, t[e]);
            }
            if constexpr (HALVES) {
                const unsigned in = q < nq ? out : 0u, low = in & ((1u << (N / 2)) - 1u);
                if (low != 0u) slot_half[slot] = make_uint2(raw.x, raw.y);
                if (in != low) slot_half[slot + __builtin_popcount(low)] = make_uint2(raw.z, raw.w);
            } else if constexpr (SLOTS) {
                const unsigned in = q < nq ? out : 0u;
                if (__ballot(in != 0u)) {
#pragma unroll
                    for (int e = 0; e < N; ++e) if ((in >> e) & 1u) slot_z[slot++] = t[e];
                }
            }
            if constexpr (TAIL) {
#pragma unroll
                for (int e = 0; e < N; ++e) {                                  // (the bit as a mask over the value)
                    const uint32_t on = (uint32_t)((int)(out << (31 - e)) >> 31);
                    t[e] = __uint_as_float((on & 0xFF800000u) | (~on & __float_as_uint(t[e])));
                }
            }
        };
        auto add = [&](int i0, const uint4 (&raw)[G]) {
            float v[G * N];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float t[N];
                values((i0 + g) * kDT + tid, raw[g], t);
#pragma unroll
                for (int e = 0; e < N; ++e) v[g * N + e] = t[e];
            }
            float bm = v[0];
#pragma unroll
            for (int e = 1; e < G * N; ++e) bm = fmaxf(bm, v[e]);
            if constexpr (TAIL) mo = fmaxf(mo, bm);
            else mx = fmaxf(mx, bm);
            if (__ballot(bm * c > r + 64.f)) {                                // (uniform; the first step, and outliers)
                const float rn = ceilf(wave_max(bm) * c);
                if (rn > r && rn > kNoReference) { s *= __builtin_amdgcn_exp2f(r - rn); r = rn; }   // (r = -inf: s is 0 and stays 0)
            }
            const float nr = r == kNegInf ? 0.f : -r;
            s += tree_sum<0, G * N>([&](int e) { return __builtin_amdgcn_exp2f(fmaf(v[e], c, nr)); });
        };
        if constexpr (HELD > 0) {
#pragma unroll
            for (int i = 0; i < HELD; i += G)
                if (i < trips) { const uint4 raw[G] = {held[i], held[i + 1]}; add(i, raw); }
        }
        if (HELD == 0 || HELD < trips) {
            const int from = SPLIT ? begin : HELD;
            uint4 cur[G], nxt[G];
#pragma unroll
            for (int g = 0; g < G; ++g) cur[g] = load(from + g, First{});
            for (int i = from; i < trips; i += G) {
                if (SPLIT && i + 1 == trips) cur[1] = make_uint4(kMaskedPair<BF16>, kMaskedPair<BF16>, kMaskedPair<BF16>, kMaskedPair<BF16>);   // (the next part's)
#pragma unroll
                for (int g = 0; g < G; ++g) nxt[g] = load(i + G + g, First{});
                add(i, cur);
#pragma unroll
                for (int g = 0; g < G; ++g) cur[g] = nxt[g];
            }
        }
        if constexpr (SLOTS) __syncthreads();                     // (the logits are in their slots)
        if constexpr (HALVES) {
#pragma unroll
            for (int j = 0; j < kMaxK / kDT; ++j) {
                mine[j].id = id_of(j * kDT + tid);
                mine[j].p = mine[j].id >= 0 ? a.prob[row * a.k + j * kDT + tid] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < kMaxK / kDT; ++j) {
                if (mine[j].id < 0) continue;
                const int v = rv.o + mine[j].id, first = v & 31 & ~(N / 2 - 1);
                const int slot = in_front[v >> 5] + __builtin_popcount(on_record[v >> 5] & ((1u << first) - 1u));
                const uint32_t bits = BF16 ? (uint32_t)reinterpret_cast<const uint16_t*>(&slot_half[slot])[v % (N / 2)] << 16 : reinterpret_cast<const uint32_t*>(&slot_half[slot])[v % (N / 2)];
                mine[j].z = __uint_as_float(bits);
            }
        }
        if constexpr (TAIL && SLOTS) {                            // (the record's come behind the stream)
            mx = mo;
            each_entry([&](const Entry& e) { mx = fmaxf(mx, e.z); });
        }
        const float wm = wave_max(mx), wo = TAIL ? wave_max(mo) : wm;
        unsigned long long* const maxima = reinterpret_cast<unsigned long long*>(sh);
        if (lane == 0) maxima[wave] = two_floats(wm, wo);
        __syncthreads();
        M = R = kNegInf;
#pragma unroll
        for (int w = 0; w < kDW; ++w) { M = fmaxf(M, first_float(maxima[w])); R = TAIL ? fmaxf(R, second_float(maxima[w])) : M; }
        __syncthreads();
        double sums[5] = {0.0, 0.0, 0.0, 0.0, 0.0};               // the weights against R; p, p log2 p, p log2(e) y and (TAIL) w of the record, against M
        if (fabsf(R * c) < 16777216.f || R == kNegInf) {         // (nothing but masked ids: s is 0, or NaN)
            sums[0] = r == kNegInf ? (double)s : (double)s * exp2_split((double)r - (double)R * (double)c);
        } else {
            for (int i = begin; i < trips; ++i) {
                float t[N];
                values(i * kDT + tid, load(i, Keep{}), t);
#pragma unroll
                for (int e = 0; e < N; ++e) sums[0] += (double)exp_stream(t[e], R, c);
            }
        }
        if constexpr (SPLIT) {
            // (the maxima and the sum of this part; together in the last of the row's workgroups to arrive)
            unsigned long long* const word = reinterpret_cast<unsigned long long*>(a.scratch + row * (int64_t)distill_scratch_row(parts));
            unsigned long long* const shares = word + kArrivalStride / 8;
            double mine[1] = {sums[0]};
            block_sums<kDW>(mine, sh);
            if (tid == 0) {
                put_shared(&shares[2 * part], two_floats(M, R));
                put_shared(&shares[2 * part + 1], (unsigned long long)__double_as_longlong(mine[0]));
            }
            if (!arrive_last(word, (unsigned)parts, tid == 0)) return;
            if (own.id >= 0) own.z = logit_at<BF16>(a.logits, a.ld, row, own.id);
            static_assert(kDistillMostParts <= kWave, "a lane for each part");
            const unsigned long long of_part = lane < parts ? get_shared(&shares[2 * lane]) : two_floats(kNegInf, kNegInf);
            const double s_part = lane < parts ? __longlong_as_double((long long)get_shared(&shares[2 * lane + 1])) : 0.0;
            const float ref = second_float(of_part);
            M = wave_max(first_float(of_part));
            R = wave_max(ref);
            sums[0] = wave_sum(ref == R ? s_part : s_part * exp2_split(((double)ref - (double)R) * (double)c));
            if (tid != 0) sums[0] = 0.0;
        }
        each_entry([&](const Entry& e) {
            if constexpr (TAIL) sums[4] += e.z < __builtin_huge_valf() ? exp_emit(e.z, M, c64) : (double)NAN;
            if (e.p > 0.f) {
                sums[1] += (double)e.p;
                sums[2] += (double)e.p * log2_of(e.p);
                sums[3] += (double)e.p * (((double)e.z - (double)M) * c64);
            }
        });
        block_sums<kDW>(sums, sh);
        mass = sums[1];
        const double gap = TAIL ? fmax(((double)R - (double)M) * c64, -1200.0) : 0.0, to_M = TAIL ? exp2_down(gap) : 1.0, off_mass = sums[0] * to_M;
        S = off_mass + sums[4];
        double pt = 0.0;
        if constexpr (TAIL) {
            pt = mass < 1.0 ? 1.0 - mass : 0.0;
            if (off_mass == 0.0 && pt <= kRounding) pt = 0.0;                  // (a record of all that the row allows)
            whole = mass + pt;
            b = off_mass > 0.0 ? whole * to_M / S - pt / sums[0] : S - S;     // (nothing off the record: every q there is 0; or NaN)
        } else {
            whole = mass > 0.0 ? 1.0 : 0.0;
            b = S == 0.0 ? 0.0 : whole / S;
        }
        if (tid == 0) {
            const double lnS = log(S);
            double loss = S - S;                                              // (0, or NaN)
            const double plain = (sums[2] - sums[3]) * 0.69314718055994531;    // sum of p (ln p - y)
            if (mass > 0.0) loss += TAIL ? plain + mass * lnS : plain / mass - log(mass) + lnS;
            if (pt > 0.0) loss += off_mass > 0.0 ? pt * (log(pt) - (log(sums[0]) + gap * 0.69314718055994531) + lnS) : (double)INFINITY;
            // (a row that is masked whole: there is no q, and nothing is learnt from it)
            a.loss[row] = S == 0.0 ? 0.f : (float)loss;
            if (a.stats) a.stats[row] = make_double4(__longlong_as_double((long long)two_floats(M, R)), S, b, TAIL ? whole : mass);
        }
    } else {
        const double4 st = a.stats[row];
        const unsigned long long maxima = (unsigned long long)__double_as_longlong(st.x);
        M = first_float(maxima); R = second_float(maxima); S = st.y; b = st.z; mass = st.w;
        whole = TAIL ? st.w : mass > 0.0 ? 1.0 : 0.0;
    }

    if constexpr (GRAD) {
        const double scale = (a.weight ? (double)a.weight[row] : 1.0) / (double)a.T;
        const bool masked = S == 0.0;
        const bool near = fabsf(R * c) < 16777216.f, far = !near && R > kNegInf;
        const float nr = near ? -(R * c) : 0.f;
        // (what the rounding of R c puts into every exponent is taken out of the factor)
        const double fix = near ? exp2_split((double)R * -(double)c - (double)nr) : 1.0;
        const float off = masked ? 0.f : (float)(scale * b * fix);
        // of a marked element: on_w w - on_p p, w against M (with TAIL as (z - M) c), in 64 bits (the two are often near each other)
        const double on_w = masked ? 0.0 : scale * whole / S * (TAIL ? 1.0 : fix);
        const double on_p = masked ? 0.0 : TAIL ? scale : mass > 0.0 ? scale / mass : 0.0;
        auto put = [&](int i, const uint4& raw, auto far_tag) {
            const int q = i * kDT + tid;
            if (q >= nq) return;
            float z[N], t[N], w[N];
            unpack<BF16>(raw, z);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                w[e] = decltype(far_tag)::value ? exp_stream(z[e], R, c) : __builtin_amdgcn_exp2f(fmaf(z[e], c, nr));
                t[e] = off * w[e];
            }
            if constexpr (SLOTS) {
                int slot;
                const unsigned in = marks(q, slot);
                if (__ballot(in != 0u)) {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if ((in >> e) & 1u) {
                            if constexpr (TAIL) w[e] = exp_stream(z[e], masked ? 0.f : M, c);
                            t[e] = (float)((double)w[e] * on_w - (double)slot_p[slot++] * on_p);
                        }
                }
            }
            store_vec<BF16>(grad_row, rv, q, t);
        };
        if (far) {
            for (int i = begin; i < trips; ++i) put(i, load(i, Keep{}), std::true_type{});
        } else {
            // (what is not held, last first: it was read last)
            const int from = SPLIT ? begin : HELD;
            for (int i = from + (trips - 1 - from) / 4 * 4; i >= from; i -= 4) {
                uint4 raw[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) raw[g] = load(i + g, Stream{});
#pragma unroll
                for (int g = 0; g < 4; ++g) if (!SPLIT || i + g < trips) put(i + g, raw[g], std::false_type{});
            }
            if constexpr (HELD > 0) {
#pragma unroll
                for (int i = 0; i < HELD; ++i) if (i < trips) put(i, held[i], std::false_type{});
            }
        }
    }
    if constexpr (FWD) {
        if (a.accept) {
            double acc[1] = {0.0};
            const double per_S = 1.0 / S;
            each_entry([&](const Entry& e) { acc[0] += fmin((double)e.p, exp_emit(e.z, M, c64) * per_S); });
            block_sums<kDW>(acc, sh);
            if (tid == 0) a.accept[row] = S == 0.0 ? 0.f : (float)(acc[0] + (S - S));
        }
    }
    if constexpr (GRAD && !SLOTS) {
        // the record's own entries over what the streaming wrote in their places
        const double scale = (a.weight ? (double)a.weight[row] : 1.0) / (double)a.T;
        const bool masked = S == 0.0;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const double on = TAIL ? 1.0 : mass > 0.0 ? 1.0 / mass : 0.0, per_S = whole / S;
        each_entry([&](const Entry& e) {
            store_one<BF16>(grad_row, e.id, masked ? 0.f : (float)(scale * (exp_emit(e.z, M, c64) * per_S - (e.p > 0.f ? (double)e.p * on : 0.0))));
        });
    }
}

constexpr int kDistillLds = 80 * 1024;            // a bound: slots of 4096 entries for vocabularies of up to 262,000, of 512 up to 408,000 (shorter ones leave room: 2048 entries of 152,064 ids, 45 KB, for three workgroups per CU)
constexpr size_t kDistillMostLds = 144 * 1024;    // the marks of the longest row alone
inline size_t mark_words(const DistillArgs& a) { return ((size_t)a.V + 8 + 31) / 32; }
inline size_t marks_lds(const DistillArgs& a) { return mark_words(a) * 4; }
inline size_t slots_lds(const DistillArgs& a, bool forward) { return ((mark_words(a) + (mark_words(a) + 1) / 2 + 1) / 2 * 2 + (size_t)a.k * (forward ? 2 : 1)) * 4; }

template <bool BF16, bool FWD, bool GRAD, bool TAIL, int SLOTS, bool SPLIT, int THREADS, int HELD>
hipError_t launch_one(const DistillArgs& a, int64_t rows, size_t lds, hipStream_t stream)
{
    const auto kernel = distill_kernel<BF16, FWD, GRAD, TAIL, SLOTS, SPLIT, THREADS, HELD>;
    static DeviceFlags done;
    int dev;
    if (lds > 32 * 1024)
        if (hipError_t e = raise_lds_limit_once((const void*)kernel, kDistillMostLds, done, dev)) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * a.parts)), dim3(THREADS), lds, stream, a);
    return hipGetLastError();
}

template <bool BF16, bool FWD, bool GRAD, int SLOTS, int THREADS, int HELD, bool SPLIT = false>
hipError_t launch(const DistillArgs& a, int64_t rows, hipStream_t stream)
{
    const size_t lds = SLOTS ? slots_lds(a, FWD) : FWD && a.tail ? marks_lds(a) : 0;
    return a.tail ? launch_one<BF16, FWD, GRAD, true, SLOTS, SPLIT, THREADS, HELD>(a, rows, lds, stream) : launch_one<BF16, FWD, GRAD, false, SLOTS, SPLIT, THREADS, HELD>(a, rows, lds, stream);
}

// Which way, by rows, type and record length (us, 1500 rows of 128,256 unless said):
//   loss      gathered up to 768 entries (fp32 and with the tail) or 1536 (bf16 without, where the marks cost the vector ALU more than the memory takes), slots beyond: 300 entries
//             134 / 135 fp32, 75 / 94 bf16; 1000 147 / 137, 91 / 101; 2500 184 / 149, 126 / 107.  Slots of halves, bf16 with the tail, gathered or by entries / so: 1088 rows of
//             152,064, 700 entries 78.6 / 76.8, 1024 82.5 / 78, 2048 97 / 82, 2000 rows of 32,000, 700 46.7 / 47.4, 1024 53.6 / 48.5, 2048 58 / 54; without the tail (2048 entries 47.5 / 55)
//             and in fp32 (1500 rows of 100,000 114 / 117) they lose.  512 threads; gathered calls of 1024 rows and more with up to 256 entries 256: 4096 rows of
//             32,000 bf16 50 against 57, 1024 of 128,256 fp32 86 against 93; of 256 rows of 151,936 fp32 50 against 33.
//   gradient  slots beyond 256 entries: 300 297 / 292, 147 / 144; 2500 418 / 294, 239 / 148.  1024 threads: 3000 rows of 100,000 450 against 469 with 512 (fp32), 233 against 250.
//   both      slots beyond 256 entries (fp32: 300 352 / 331, 2500 538 / 348), beyond 512 (bf16: 300 169 / 177, 1000 211 / 183, 2500 315 / 196), where there are fewer than 512
//             rows beyond 2048 (256 of 151,936: 1000 47 / 58, 2500 63 / 63).  512 threads that hold 12 vectors each, a third to two thirds of a row (4096 rows of 151,936 bf16: 500;
//             with none held 560, with 40, all of the row and one workgroup per CU, 575); none with bf16 slots (1000 entries 183 against 210).
template <bool BF16>
hipError_t launch_backward(const DistillArgs& a, int64_t rows, hipStream_t stream)
{
    DistillArgs b = a;
    b.parts = distill_parts(BF16, rows, a.V, kDistillBackward, true);
    if (b.parts > 1) return launch<BF16, false, true, kNone, kDistillBackward, 0, true>(b, rows, stream);
    return a.k > 256 && slots_lds(a, false) <= (size_t)kDistillLds ? launch<BF16, false, true, kEntries, kDistillBackward, 0>(b, rows, stream) : launch<BF16, false, true, kNone, kDistillBackward, 0>(b, rows, stream);
}

template <bool BF16>
hipError_t launch_forward(const DistillArgs& a, int64_t rows, hipStream_t stream)
{
    if (a.parts > 1) {
        DistillArgs f = a;
        if (!f.stats) f.stats = reinterpret_cast<double4*>(a.scratch + rows * (int64_t)distill_scratch_row(a.parts));
        if (hipError_t e = launch<BF16, true, false, kNone, kDistillForward, 0, true>(f, rows, stream)) return e;
        return a.grad ? launch_backward<BF16>(f, rows, stream) : hipSuccess;
    }
    if (a.grad) {
        const bool slots = a.k > (BF16 ? (rows >= 512 ? 512 : 2048) : 256) && slots_lds(a, true) <= (size_t)kDistillLds;
        return slots ? launch<BF16, true, true, kEntries, 512, BF16 ? 0 : 12>(a, rows, stream) : launch<BF16, true, true, kNone, 512, 12>(a, rows, stream);
    }
    if constexpr (BF16)
        if (a.tail && a.k > 768 && slots_lds(a, true) <= (size_t)kDistillLds)
            return launch_one<BF16, true, false, true, kHalves, false, kDistillForward, 0>(a, rows, slots_lds(a, true), stream);
    if (a.k > (BF16 ? 1536 : 768) && slots_lds(a, true) <= (size_t)kDistillLds) return launch<BF16, true, false, kEntries, kDistillForward, 0>(a, rows, stream);
    return rows >= 1024 && a.k <= 256 ? launch<BF16, true, false, kNone, 256, 0>(a, rows, stream) : launch<BF16, true, false, kNone, kDistillForward, 0>(a, rows, stream);
}

}  // namespace

hipError_t launch_distill(const void* logits, int dtype, int64_t ld, int n_rows, int V, float temperature,
                          const int32_t* idx, const float* prob, const int32_t* count, int k, int tail,
                          float* loss, float* accept, double* stats, const float* weight, void* grad, int64_t ld_grad, void* scratch, size_t scratch_bytes, hipStream_t stream)
{
    const size_t need = distill_scratch_bytes(dtype, n_rows, V);
    const int parts = need && scratch && scratch_bytes >= need && (!grad || distill_splits(dtype == 1, n_rows, V, true)) ? distill_parts(dtype == 1, n_rows, V, kDistillForward, false) : 1;
    const DistillArgs a{logits, ld, V, temperature, idx, prob, count, k, tail, loss, accept, reinterpret_cast<double4*>(stats), weight, grad, ld_grad, (char*)scratch, parts};
    if (n_rows == 0) return hipSuccess;
    return dtype == 1 ? launch_forward<true>(a, n_rows, stream) : launch_forward<false>(a, n_rows, stream);
}

hipError_t launch_distill_grad(const void* logits, int dtype, int64_t ld, int n_rows, int V, float temperature,
                               const int32_t* idx, const float* prob, const int32_t* count, int k, int tail,
                               const double* stats, const float* weight, void* grad, int64_t ld_grad, hipStream_t stream)
{
    const DistillArgs a{logits, ld, V, temperature, idx, prob, count, k, tail, nullptr, nullptr,
                        reinterpret_cast<double4*>(const_cast<double*>(stats)), weight, grad, ld_grad, nullptr, 1};
    if (n_rows == 0) return hipSuccess;
    return dtype == 1 ? launch_backward<true>(a, n_rows, stream) : launch_backward<false>(a, n_rows, stream);
}

}  // namespace picospec
