// Distillation of a drafter on the target's Top-K records: Kullback-Leibler divergence of q = softmax(z / T) from a record
// (id_j, p_j), j < count, with its gradient, and the expected acceptance sum_j min(p_j, q_j).  With y = (z - M) / T, w = e^y,
// S = sum w, q = w / S:
//   tail 0   L = sum_j ph_j (ln ph_j - ln q_j), ph = p / sum p
//            T dL/dz_v = q_v - ph_v
//   tail 1   L = sum_j p_j (ln p_j - ln q_j) + pt (ln pt - ln qt),  pt = max(0, 1 - sum p), qt = q's mass off the record
//            T dL/dz_v = W q_v - p_v on the record, (W - pt / qt) q_v off it,  W = sum p + pt
// What bounds it: the row is read once (forward) and the gradient written once.  With the gradient in the same call a thread can keep kDistillHeld
// vectors of its row in registers between the two (0: the gradient reads the row again).
// qt is summed directly: 1 - sum_j q_j loses it where the record holds nearly all of q, and the gradient off the record has pt / qt in it.
// The ids of the record are a bitmap in LDS, one bit per element (a byte per vector of eight bf16 values), which the streaming sum masks with.
#include "common.hpp"
#include "kernels.hpp"

namespace picospec {

namespace {

constexpr int kDT = kDistillThreads;
constexpr int kDW = kDT / kWave;

struct DistillArgs {
    const void* logits; int64_t ld; int V; float T;
    const int32_t* idx; const float* prob; const int32_t* count; int k, tail;
    float *loss, *accept; double4* stats; const float* weight; void* grad; int64_t ld_grad;
};

// sums of N doubles over the workgroup, the same bits in every thread (fixed order)
template <int N>
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

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    // (round to nearest, ties to even)
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    uint32_t r;
    __builtin_memcpy(&r, &v, 4);
    return r;
}

// 16 bytes to an address that is element-aligned only: the output rows need not lie like the input's (global stores take any alignment)
struct __attribute__((packed, aligned(2))) Loose16 { u32x4_t v; };

template <bool BF16>
__device__ __forceinline__ void store_vec(char* grad_row, const RowView& rv, int q, const float (&g)[Vec<BF16>::N])
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4;
    const int x = q * N - rv.o;
    if (x >= 0 && x + N <= rv.L - rv.o) {
        u32x4_t t;
        if constexpr (BF16) { t.x = pack_bf16(g[0], g[1]); t.y = pack_bf16(g[2], g[3]); t.z = pack_bf16(g[4], g[5]); t.w = pack_bf16(g[6], g[7]); }
        else { t.x = __float_as_uint(g[0]); t.y = __float_as_uint(g[1]); t.z = __float_as_uint(g[2]); t.w = __float_as_uint(g[3]); }
        reinterpret_cast<Loose16*>(grad_row + (int64_t)x * ESZ)->v = t;
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
template <bool BF16, bool FWD, bool GRAD, bool TAIL>
__global__ __launch_bounds__(kDT) void distill_kernel(const DistillArgs a)
{
    constexpr int N = Vec<BF16>::N, G = 2;                       // vectors per step
    constexpr int HELD = FWD && GRAD ? kDistillHeld : 0;         // vectors a thread keeps from the sum to the gradient
    static_assert(HELD % G == 0, "whole steps");
    __shared__ double sh[4 * kDW];
    extern __shared__ uint32_t on_record[];                      // TAIL && FWD: bit o + id
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const RowView rv = row_view<BF16>(a.logits, a.ld, row, a.V);
    const int nq = (rv.L + N - 1) / N, trips = (nq + kDT - 1) / kDT;
    const float c = 1.4426950408889634f / a.T;
    const int count = min(max(a.count[row], 0), a.k);
    char* const grad_row = (char*)a.grad + row * a.ld_grad * (BF16 ? 2 : 4);
    if (count == 0) {                                            // (a position that is not trained on)
        if (FWD && tid == 0) {
            a.loss[row] = 0.f;
            if (a.accept) a.accept[row] = 0.f;
            if (a.stats) a.stats[row] = make_double4(0.0, 1.0, 0.0, 0.0);
        }
        if constexpr (GRAD) {
            const float zero[N] = {};
            for (int q = tid; q < nq; q += kDT) store_vec<BF16>(grad_row, rv, q, zero);
        }
        return;
    }

    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)rv.base, 0, nq * 16, 0x00020000);
    auto load = [&](int i, auto aux) {                           // vector i * kDT + tid; behind the row: zero
        const u32x4_t t = __builtin_amdgcn_raw_buffer_load_b128(rsrc, tid * 16, i * (kDT * 16), decltype(aux)::value);
        return make_uint4(t.x, t.y, t.z, t.w);
    };
    using Stream = std::integral_constant<int, 2>;               // (read once: non-temporal)
    using Keep = std::integral_constant<int, 0>;
    using First = std::conditional_t<GRAD, Keep, Stream>;        // (what is not held is read again by the gradient)

    uint4 held[HELD ? HELD : 1];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) if (i < trips) held[i] = load(i, Stream{});
    }

    // the record: entries tid, tid + kDT, ..; a thread keeps its first one (ids outside the vocabulary: no entry)
    struct Entry { int id; float p, z; };
    auto entry = [&](int s) {
        Entry e{-1, 0.f, 0.f};
        if (s < count) {
            e.id = a.idx[row * a.k + s];
            if ((unsigned)e.id < (unsigned)a.V) { e.p = a.prob[row * a.k + s]; e.z = logit_at<BF16>(a.logits, a.ld, row, e.id); }
            else e.id = -1;
        }
        return e;
    };
    const Entry own = entry(tid);
    auto each_entry = [&](auto f) {
        if (own.id >= 0) f(own);
#pragma unroll 1
        for (int s = tid + kDT; s < count; s += kDT) { const Entry e = entry(s); if (e.id >= 0) f(e); }
    };

    float M;
    double S, b, mass, whole;
    if constexpr (FWD) {
        if constexpr (TAIL) {
            for (int w = tid; w < (rv.L + 31) / 32; w += kDT) on_record[w] = 0u;
            __syncthreads();
            each_entry([&](const Entry& e) { atomicOr(&on_record[(rv.o + e.id) >> 5], 1u << ((rv.o + e.id) & 31)); });
            __syncthreads();
        }
        // the maximum of the row and, TAIL, the sum off the record, else over all
        OnlineSum os;
        float mx = kNegInf;
        auto add = [&](int i0, const uint4 (&raw)[G]) {
            float v[G * N], bm = kNegInf;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float t[N];
                unpack<BF16>(raw[g], t);
                const int q = (i0 + g) * kDT + tid;
                unsigned out = 0u;                                // elements that do not count
                if constexpr (TAIL) {
                    const int qq = min(q, nq - 1);
                    const unsigned byte = reinterpret_cast<const uint8_t*>(on_record)[BF16 ? qq : qq >> 1];
                    out = BF16 ? byte : byte >> (4 * (qq & 1));
                }
                if (q == 0 || q >= nq - 1) {
                    const unsigned vm = vec_valid_mask<BF16>(rv, q);
                    out |= ~vm;
#pragma unroll
                    for (int e = 0; e < N; ++e) t[e] = (vm >> e) & 1u ? t[e] : kNegInf;
                }
                if constexpr (TAIL) {
#pragma unroll
                    for (int e = 0; e < N; ++e) mx = fmaxf(mx, t[e]);
#pragma unroll
                    for (int e = 0; e < N; ++e) t[e] = (out >> e) & 1u ? kNegInf : t[e];
                }
#pragma unroll
                for (int e = 0; e < N; ++e) { v[g * N + e] = t[e]; bm = fmaxf(bm, t[e]); }
            }
            const float ref = os.rebase(bm, c);
            os.s += tree_sum<0, G * N>([&](int e) { return exp_stream(v[e], ref, c); });
        };
        if constexpr (HELD > 0) {
#pragma unroll
            for (int i = 0; i < HELD; i += G)
                if (i < trips) { const uint4 raw[G] = {held[i], held[i + 1]}; add(i, raw); }
        }
        uint4 cur[G], nxt[G];
#pragma unroll
        for (int g = 0; g < G; ++g) cur[g] = load(HELD + g, First{});
        for (int i = HELD; i < trips; i += G) {
#pragma unroll
            for (int g = 0; g < G; ++g) nxt[g] = load(i + G + g, First{});
            add(i, cur);
#pragma unroll
            for (int g = 0; g < G; ++g) cur[g] = nxt[g];
        }
        double sum;
        block_softmax_stats<kDW>(os.m, os.s, c, sh, M, sum);
        if constexpr (TAIL) {                                     // (the sum is relative to the largest element off the record)
            const float m_off = M;
            const int lane = tid & (kWave - 1), wave = tid / kWave;
            const float wm = wave_max(mx);
            if (lane == 0) sh[wave] = (double)wm;
            __syncthreads();
            M = kNegInf;
#pragma unroll
            for (int w = 0; w < kDW; ++w) M = fmaxf(M, (float)sh[w]);
            __syncthreads();
            if (m_off != M) sum = m_off == kNegInf ? (sum == sum ? 0.0 : sum) : sum * exp2_split(((double)m_off - (double)M) * 1.4426950408889634 / (double)a.T);
        }
        // the record's sums
        const double c64 = 1.4426950408889634 / (double)a.T;
        double s4[4] = {0.0, 0.0, 0.0, 0.0};                      // p, p ln p, p y, w (TAIL)
        each_entry([&](const Entry& e) {
            if constexpr (TAIL) s4[3] += exp_emit(e.z, M, c64);
            if (e.p > 0.f) {
                s4[0] += (double)e.p;
                s4[1] += (double)e.p * log((double)e.p);
                s4[2] += (double)e.p * (((double)e.z - (double)M) / (double)a.T);
            }
        });
        block_sums(s4, sh);
        mass = s4[0];
        S = TAIL ? sum + s4[3] : sum;
        const double lnS = log(S);
        double loss, acc[1] = {0.0};
        if constexpr (TAIL) {
            const double pt = mass < 1.0 ? 1.0 - mass : 0.0;
            whole = mass + pt;
            b = whole;
            loss = mass > 0.0 ? s4[1] - s4[2] + mass * lnS : 0.0;
            if (pt > 0.0) {
                const double qt = sum / S;
                loss += pt * (log(pt) - log(qt));
                b = qt > 0.0 ? whole - pt / qt : 0.0;             // (nothing left off the record: every q there is 0)
            }
        } else {
            whole = b = mass > 0.0 ? 1.0 : 0.0;
            loss = mass > 0.0 ? (s4[1] - s4[2]) / mass - log(mass) + lnS : 0.0;
        }
        each_entry([&](const Entry& e) { acc[0] += fmin((double)e.p, exp_emit(e.z, M, c64) / S); });
        block_sums(acc, sh);
        if (M == kNegInf) { loss = 0.0; acc[0] = 0.0; b = 0.0; whole = 0.0; mass = 0.0; S = 1.0; }   // (a row that is masked whole: there is no q, and nothing is learnt from it)
        if (tid == 0) {
            a.loss[row] = (float)loss;
            if (a.accept) a.accept[row] = (float)acc[0];
            if (a.stats) a.stats[row] = make_double4((double)M, S, b, mass);
        }
    } else {
        const double4 st = a.stats[row];
        M = (float)st.x; S = st.y; b = st.z; mass = st.w;
        whole = M == kNegInf ? 0.0 : TAIL ? mass + (mass < 1.0 ? 1.0 - mass : 0.0) : b;
    }

    if constexpr (GRAD) {
        const double scale = (a.weight ? (double)a.weight[row] : 1.0) / (double)a.T;
        const float off = M == kNegInf ? 0.f : (float)(scale * b / S);
        const float ref = M == kNegInf ? 0.f : M;
        auto put = [&](int i, const uint4& raw) {
            const int q = i * kDT + tid;
            if (q >= nq) return;
            float t[N];
            unpack<BF16>(raw, t);
#pragma unroll
            for (int e = 0; e < N; ++e) t[e] = off * exp_stream(t[e], ref, c);
            store_vec<BF16>(grad_row, rv, q, t);
        };
        // (what is not held, last first: it was read last)
        for (int i = HELD + (trips - 1 - HELD) / 4 * 4; i >= HELD; i -= 4) {
            uint4 raw[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) raw[g] = load(i + g, Stream{});
#pragma unroll
            for (int g = 0; g < 4; ++g) put(i + g, raw[g]);
        }
        if constexpr (HELD > 0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) if (i < trips) put(i, held[i]);
        }
        // the record's own entries over what the streaming wrote in their places
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const double on = TAIL ? (M == kNegInf ? 0.0 : 1.0) : (mass > 0.0 ? 1.0 / mass : 0.0), c64 = 1.4426950408889634 / (double)a.T;
        each_entry([&](const Entry& e) {
            store_one<BF16>(grad_row, e.id, M == kNegInf ? 0.f : (float)(scale * (whole * (exp_emit(e.z, M, c64) / S) - (e.p > 0.f ? (double)e.p * on : 0.0))));
        });
    }
}

template <bool BF16, bool FWD, bool GRAD>
hipError_t launch(const DistillArgs& a, int64_t rows, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    if (a.tail) {
        const size_t lds = FWD ? ((size_t)a.V + 8 + 31) / 32 * 4 : 0;
        static DeviceFlags done;
        int dev;
        if (lds > 32 * 1024)
            if (hipError_t e = raise_lds_limit_once((const void*)distill_kernel<BF16, FWD, GRAD, true>, ((size_t)kMaxV + 8 + 31) / 32 * 4, done, dev)) return e;
        hipLaunchKernelGGL((distill_kernel<BF16, FWD, GRAD, true>), dim3((unsigned)rows), dim3(kDT), lds, stream, a);
    } else {
        hipLaunchKernelGGL((distill_kernel<BF16, FWD, GRAD, false>), dim3((unsigned)rows), dim3(kDT), 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_distill(const void* logits, int dtype, int64_t ld, int n_rows, int V, float temperature,
                          const int32_t* idx, const float* prob, const int32_t* count, int k, int tail,
                          float* loss, float* accept, double* stats, const float* weight, void* grad, int64_t ld_grad, hipStream_t stream)
{
    const DistillArgs a{logits, ld, V, temperature, idx, prob, count, k, tail, loss, accept, reinterpret_cast<double4*>(stats), weight, grad, ld_grad};
    if (grad) return dtype == 1 ? launch<true, true, true>(a, n_rows, stream) : launch<false, true, true>(a, n_rows, stream);
    return dtype == 1 ? launch<true, true, false>(a, n_rows, stream) : launch<false, true, false>(a, n_rows, stream);
}

hipError_t launch_distill_grad(const void* logits, int dtype, int64_t ld, int n_rows, int V, float temperature,
                               const int32_t* idx, const float* prob, const int32_t* count, int k, int tail,
                               const double* stats, const float* weight, void* grad, int64_t ld_grad, hipStream_t stream)
{
    const DistillArgs a{logits, ld, V, temperature, idx, prob, count, k, tail, nullptr, nullptr,
                        reinterpret_cast<double4*>(const_cast<double*>(stats)), weight, grad, ld_grad};
    return dtype == 1 ? launch<true, false, true>(a, n_rows, stream) : launch<false, false, true>(a, n_rows, stream);
}

}  // namespace picospec
