// Rows of logits adjusted for what a request asks: penalties for tokens that its text holds already, biases of single tokens, a grammar's mask; and the gradient.
// With n the number of times that a token is in the sequence's history behind its prompt or among the drafted tokens in front of the row, and seen where it is in
// the history at all or among those:
//   z1 = seen ? (z > 0 ? z / repetition : z * repetition) : z
//   z2 = z1 - frequency n - [n > 0] presence + bias,   out = allowed ? z2 : -inf
//   d out / d z = allowed ? (seen ? (z > 0 ? 1 / repetition : repetition) : 1) : 0
// A workgroup has one sequence and one chunk of the vocabulary.  It counts the history's tokens of its chunk in LDS once, then takes the sequence's rows one by one; a thread has the same ids
// in every row and keeps a bit for each that is touched.
// What bounds it: the rows, read once and written once (2432 rows of 151,936 bf16, 1.48 GB: 272 us with nothing to adjust,
// 5.4 TB/s, where a copy on this card gets 4.9; 290 with histories of up to 16,384 tokens and masks).
#include "kernels.hpp"
#include "vectors.hpp"

namespace picospec {

namespace {

// A count: bit 0, a token of the prompt; from bit 1 on how often the token was generated
constexpr uint32_t kSeenBit = 1u, kOnce = 2u;

// -inf, as stored
template <bool BF16> constexpr uint32_t kMaskedBits = BF16 ? 0xFF80u : 0xFF800000u;

// A word that the kernel does not write and that a whole wave reads, by a scalar load (behind stores that may lie in front of it the compiler takes a vector load, and a sequence has ten such words:
// 5 to 10 % of a call)
template <class T>
__device__ __forceinline__ T input(const T* p) { return *(const __attribute__((address_space(4))) T*)p; }

__device__ __forceinline__ float setting(const float* rows, int b, float all) { return rows ? input(rows + b) : all; }

// T threads with VPT vectors of a row each
template <bool BF16, bool GRAD, int T, int VPT>
__device__ __forceinline__ void adjust_rows(const AdjustArgs& a)
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4, IDS = T * VPT * N;
    constexpr unsigned WHOLE = (1u << N) - 1u;
    extern __shared__ __attribute__((aligned(16))) uint32_t counts[];        // [IDS], the vectors that are being adjusted [IDS], the biases [IDS] where there are any
    char* const stage = reinterpret_cast<char*>(counts + IDS);
    float* const bias = reinterpret_cast<float*>(stage + IDS * ESZ);
    const int tid = threadIdx.x;
    const int chunk = (int)(blockIdx.x % (unsigned)a.chunks), rest = (int)(blockIdx.x / (unsigned)a.chunks), part = rest % a.parts, b = rest / a.parts;
    const int lo = chunk * IDS, ids = min(IDS, a.V - lo);

    // the sequence's rows of this part, and the drafted tokens in front of them (what the offsets say beyond the arrays is not followed)
    int off = 0, gamma = 0;
    if (a.seq_off) {
        off = min(max(input(a.seq_off + b), 0), a.n_draft);
        gamma = min(max(input(a.seq_off + b + 1), off), a.n_draft) - off;
    }
    const int n = a.seq_off ? gamma + a.bonus : 1, each = (n + a.parts - 1) / a.parts, t0 = part * each, t1 = min(t0 + each, n);
    const int64_t row0 = a.seq_off ? (int64_t)off + (a.bonus ? b : 0) : b;
    if (t0 >= t1) return;

    float rep = setting(a.repetition_rows, b, a.repetition), pres = GRAD ? 0.f : setting(a.presence_rows, b, a.presence), freq = GRAD ? 0.f : setting(a.frequency_rows, b, a.frequency);
    if (!(rep > 0.f && rep < __builtin_huge_valf())) rep = 1.f;
    if (!(fabsf(pres) < __builtin_huge_valf())) pres = 0.f;
    if (!(fabsf(freq) < __builtin_huge_valf())) freq = 0.f;
    const bool counted = rep != 1.f || pres != 0.f || freq != 0.f;
    int bias0 = 0, bias1 = 0;
    if (!GRAD && a.bias_off) {
        bias0 = min(max(input(a.bias_off + b), 0), a.n_bias);
        bias1 = min(max(input(a.bias_off + b + 1), bias0), a.n_bias);
    }
    const bool biased = bias1 > bias0;
    int length = 0, prompt = 0;
    if (a.hist_tok) {
        length = min(max(input(a.hist_len + b), 0), a.hist_cap);
        prompt = a.prompt_len ? input(a.prompt_len + b) : 0;
    }
    if (!counted) length = 0;

    // The first of the history, as vectors of four tokens: everything that the workgroup waits for is under way before it waits for any of it
    constexpr int AHEAD = 4;
    typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
    typedef i32x4_t loose_tok_t __attribute__((aligned(4)));
    const int32_t* const tok = a.hist_tok + (int64_t)b * a.ld_hist;
    const int tok_vecs = length / 4;
    i32x4_t toks[AHEAD];
    auto read_tokens = [&](int64_t i) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            toks[j] = i32x4_t{-1, -1, -1, -1};
            if (i + j * T < tok_vecs) toks[j] = *reinterpret_cast<const loose_tok_t*>(tok + (i + j * T) * 4);
        }
    };
    read_tokens(tid);

    // vectors tid, tid + T, .. of row t: the bits that its mask allows, and what is needed of the row
    uint32_t tm[VPT];                                             // touched: seen or biased
#pragma unroll
    for (int j = 0; j < VPT; ++j) tm[j] = 0u;
    auto allow = [&](int t, unsigned (&allowed)[VPT]) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) allowed[j] = WHOLE;
        if (!a.mask || t >= t1) return;
        const int m = a.mask_row ? input(a.mask_row + row0 + t) : (int)(row0 + t);
        if ((unsigned)m >= (unsigned)a.n_masks) return;
        const unsigned char* const mask = reinterpret_cast<const unsigned char*>(a.mask + (int64_t)m * a.ld_mask) + lo / 8;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int x = (tid + j * T) * N;
            if (x < ids) allowed[j] = (unsigned)mask[x / 8] >> (x & 7) & WHOLE;
        }
    };
    auto fetch_one = [&](const void* base, int64_t ld, int t, int j) { return load_row_vec<BF16>((const char*)base + ((row0 + t) * ld + lo) * ESZ, (tid + j * T) * N, ids); };
    auto fetch = [&](int t, const unsigned (&allowed)[VPT], uint4 (&raw)[VPT], uint4 (&z)[VPT]) {
        if (t >= t1) return;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if ((tid + j * T) * N >= ids || allowed[j] == 0u) continue;
            if (!a.in_place || allowed[j] != WHOLE || tm[j]) raw[j] = fetch_one(a.src, a.ld_src, t, j);
            if (GRAD && tm[j]) z[j] = fetch_one(a.logits, a.ld, t, j);
        }
    };
    unsigned allowed[VPT], allowed_next[VPT];
    uint4 raw[VPT], z[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) raw[j] = z[j] = make_uint4(0, 0, 0, 0);
    allow(t0, allowed);
    allow(t0 + 1, allowed_next);
    const bool early = !GRAD && !a.in_place;                      // (before the counting, where what is needed does not depend on it)
    if (early) fetch(t0, allowed, raw, z);

    auto clear = [&] {
        for (int i = tid * 4; i < IDS; i += T * 4) *reinterpret_cast<uint4*>(counts + i) = make_uint4(0, 0, 0, 0);
    };
    if (counted || biased) clear();
    if (biased) {
        // of entries for the same token the last one counts: every entry bids with its place, the one that holds the token writes
        for (int i = tid * 4; i < IDS; i += T * 4) *reinterpret_cast<float4*>(bias + i) = make_float4(0.f, 0.f, 0.f, 0.f);
        __syncthreads();
        for (int i = bias0 + tid; i < bias1; i += T) {
            const unsigned x = (unsigned)a.bias_id[i] - (unsigned)lo;
            if (x < (unsigned)ids) atomicMax(&counts[x], (uint32_t)(i - bias0) + 1u);
        }
        __syncthreads();
        for (int i = bias0 + tid; i < bias1; i += T) {
            const unsigned x = (unsigned)a.bias_id[i] - (unsigned)lo;
            if (x < (unsigned)ids && counts[x] == (uint32_t)(i - bias0) + 1u) bias[x] = a.bias_value[i];
        }
        __syncthreads();
        clear();
    }
    if (counted || biased) __syncthreads();
    if (counted) {
        auto count = [&](int tok, uint32_t as) {
            const unsigned x = (unsigned)tok - (unsigned)lo;
            if (x < (unsigned)ids) {
                if (as == kSeenBit) atomicOr(&counts[x], kSeenBit);
                else atomicAdd(&counts[x], kOnce);
            }
        };
        for (int64_t i = tid; i < tok_vecs;) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) count(toks[j][e], (i + j * T) * 4 + e < prompt ? kSeenBit : kOnce);
            i += AHEAD * T;
            read_tokens(i);
        }
        if (tid < length - tok_vecs * 4) count(tok[tok_vecs * 4 + tid], tok_vecs * 4 + tid < prompt ? kSeenBit : kOnce);
        for (int i = tid; i < t0; i += T) count(a.draft_tok[off + i], kOnce);
        __syncthreads();
    }
    // (from here on a thread looks at the counts of its own ids alone)
    if (counted || biased) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int x = (tid + j * T) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) tm[j] |= (unsigned)(counts[x + e] != 0u || (biased && bias[x + e] != 0.f)) << e;
        }
    }
    if (!early) fetch(t0, allowed, raw, z);

    const double by = (double)rep, inv = 1.0 / (double)rep, pres64 = pres, freq64 = freq;
    for (int t = t0; t < t1; ++t) {
        uint4 raw_next[VPT], z_next[VPT];
        unsigned allowed_after[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) raw_next[j] = z_next[j] = make_uint4(0, 0, 0, 0);
        fetch(t + 1, allowed_next, raw_next, z_next);
        allow(t + 2, allowed_after);

        // touched ids one by one, in LDS: a wave goes on until the thread with the most of them is done, which is much sooner than all elements in turn (the rows above with
        // every element looked at in fp64 where any of a vector's is touched, vectors loaded when they are needed: 547 us)
        unsigned left = 0u, positive = 0u;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const unsigned m = tm[j] & allowed[j];
            left |= m << (j * N);
            if (m) *reinterpret_cast<uint4*>(stage + (tid + j * T) * 16) = raw[j];
            if constexpr (GRAD) {
                float f[N];
                unpack<BF16>(z[j], f);
#pragma unroll
                for (int e = 0; e < N; ++e) positive |= (unsigned)(f[e] > 0.f) << (j * N + e);
            }
        }
        auto id_of = [&](int bit) { return (tid + bit / N * T) * N + bit % N; };
        auto staged = [&](int x) {
            if constexpr (BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(stage)[x] << 16);
            else return reinterpret_cast<const float*>(stage)[x];
        };
        auto put = [&](int x, float v) {
            if constexpr (BF16) reinterpret_cast<uint16_t*>(stage)[x] = (uint16_t)pack_bf16(v, 0.f);
            else reinterpret_cast<float*>(stage)[x] = v;
        };
        auto adjusted = [&](int bit, int x, float v, uint32_t c) {
            double y = (double)v;
            if constexpr (GRAD) {
                y *= positive >> bit & 1u ? inv : by;
            } else {
                y *= c ? (v > 0.f ? inv : by) : 1.0;
                y -= freq64 * (double)(c >> 1) + (c >> 1 ? pres64 : 0.0);
                if (biased) y += (double)bias[x];
            }
            return (float)y;
        };
        // (two at a time, from both ends, which may meet: each is a wait for LDS and a chain of fp64 instructions, and in the chunk of the frequent ids most are touched; the rows above 312 -> 307 us)
        for (unsigned m = left; m;) {
            const int bit0 = __builtin_ctz(m), bit1 = 31 - __builtin_clz(m), x0 = id_of(bit0), x1 = id_of(bit1);
            const float v0 = staged(x0), v1 = staged(x1);
            const uint32_t c0 = counts[x0], c1 = counts[x1];
            const float y0 = adjusted(bit0, x0, v0, c0), y1 = adjusted(bit1, x1, v1, c1);
            put(x0, y0);
            put(x1, y1);
            m &= ~(1u << bit0) & ~(1u << bit1);
        }
        char* const out = (char*)a.out + ((row0 + t) * a.ld_out + lo) * ESZ;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int x = (tid + j * T) * N;
            if (x >= ids || (a.in_place && !tm[j] && allowed[j] == WHOLE)) continue;
            uint4 r = raw[j];
            if (left >> (j * N) & WHOLE) r = *reinterpret_cast<const uint4*>(stage + (tid + j * T) * 16);
            if (allowed[j] != WHOLE) {
                uint32_t w[4] = {r.x, r.y, r.z, r.w};
                constexpr uint32_t away = GRAD ? 0u : kMaskedBits<BF16>;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (!(allowed[j] >> e & 1u)) {
                        if constexpr (BF16) w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | away << 16 : (w[e / 2] & 0xFFFF0000u) | away;
                        else w[e] = away;
                    }
                r = make_uint4(w[0], w[1], w[2], w[3]);
            }
            store_row_vec<BF16>(out, x, ids, r);
        }
        if (counted && t + 1 < t1) {
            // the drafted token between this row and the next, by the thread that has it
            const unsigned x = (unsigned)a.draft_tok[off + t] - (unsigned)lo;
            if (x < (unsigned)ids) {
#pragma unroll
                for (int j = 0; j < VPT; ++j)
                    if ((int)(x / N) == tid + j * T) {
                        counts[x] += kOnce;
                        const bool first = tm[j] == 0u;
                        tm[j] |= 1u << (x % N);
                        // (what the row ahead did not need of it)
                        if (first && allowed_next[j]) {
                            if (a.in_place && allowed_next[j] == WHOLE) raw_next[j] = fetch_one(a.src, a.ld_src, t + 1, j);
                            if (GRAD) z_next[j] = fetch_one(a.logits, a.ld, t + 1, j);
                        }
                    }
            }
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j) { raw[j] = raw_next[j]; z[j] = z_next[j]; allowed[j] = allowed_next[j]; allowed_next[j] = allowed_after[j]; }
    }
}

// Zeros in the rows that no sequence has, in front of the first one and behind the last, by workgroup `at` of a.idle: a few for every chunk of the vocabulary
template <bool BF16, int T, int IDS>
__device__ __forceinline__ void zero_rest(const AdjustArgs& a, int at)
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4;
    const int lo = at % a.chunks * IDS, ids = min(IDS, a.V - lo);
    const int64_t front = min(max(a.seq_off[0], 0), a.n_draft), back = (int64_t)min(max(a.seq_off[a.B], 0), a.n_draft) + (a.bonus ? a.B : 0), outside = front + a.n_rows - back;
    for (int64_t i = at / a.chunks; i < outside; i += a.idle / a.chunks) {
        char* const row = (char*)a.out + ((i < front ? i : back + i - front) * a.ld_out + lo) * ESZ;
        for (int x = (int)threadIdx.x * N; x < ids; x += T * N) store_row_vec<BF16>(row, x, ids, make_uint4(0, 0, 0, 0));
    }
}

// The workgroups behind those of the sequences are for the rows of none (there are none, mostly, and a workgroup that finds that out costs nothing there)
template <bool BF16, bool GRAD, int T, int VPT>
__global__ __launch_bounds__(T) void adjust_kernel(const AdjustArgs a)
{
    if (blockIdx.x < a.busy) adjust_rows<BF16, GRAD, T, VPT>(a);
    else zero_rest<BF16, T, T * VPT * Vec<BF16>::N>(a, (int)(blockIdx.x - a.busy));
}

template <bool BF16, bool GRAD, int T, int VPT>
hipError_t launch_one(const AdjustArgs& a, hipStream_t stream)
{
    constexpr int IDS = T * VPT * Vec<BF16>::N;
    const size_t lds = (size_t)IDS * (4 + (BF16 ? 2 : 4) + (!GRAD && a.bias_off ? 4 : 0));
    static DeviceFlags done;
    int dev;
    if (lds > 64 * 1024)
        if (hipError_t e = raise_lds_limit_once((const void*)adjust_kernel<BF16, GRAD, T, VPT>, 160 * 1024, done, dev)) return e;
    hipLaunchKernelGGL((adjust_kernel<BF16, GRAD, T, VPT>), dim3(a.busy + (unsigned)a.idle), dim3(T), lds, stream, a);
    return hipGetLastError();
}

template <bool BF16, bool GRAD>
hipError_t launch(const AdjustArgs& a, const AdjustPlan& plan, hipStream_t stream)
{
    constexpr int MOST = 8192 / (512 * Vec<BF16>::N);
    if (plan.T == 512) return plan.vectors == MOST ? launch_one<BF16, GRAD, 512, MOST>(a, stream) : launch_one<BF16, GRAD, 512, 1>(a, stream);
    if constexpr (!GRAD)
        if (plan.vectors == 2) return launch_one<BF16, GRAD, 256, 2>(a, stream);
    return launch_one<BF16, GRAD, 256, 1>(a, stream);
}

}  // namespace

// Which way, us:
//   512 threads             histories that are longer than what a sequence has of rows in a chunk (each chunk reads the history).  8192 ids where these are workgroups enough: 512 single rows of
//                           151,936 fp32, up to 32,768 tokens 193, with 2048 ids 252; 64 of bf16 23 (26, with one vector 28).  Else one vector: a row of 151,936 bf16 with 32,768 tokens 8.8 (8192 ids 10.6, 256
//                           threads 11.8), 9 rows of it with 100,000 20 (23, 30)
//   256 threads, 2 vectors  512 single rows of 151,936 bf16 87 (with one vector 124, 8192 ids 92), 64 of 128,256 fp32 17.6 (20, 19)
//   256 threads, 1 vector   gradients (128 sequences of 5.5 rows of 128,256 bf16 82, with two vectors 95) and what would leave compute units without work (64 of 6.5 rows of 50,001 bf16 27.7 / 30.1)
AdjustPlan adjust_plan(const AdjustArgs& a, int dtype, int B, int64_t n_rows, bool gradient)
{
    const int N = dtype == 1 ? Vec<true>::N : Vec<false>::N;
    const int64_t mean = (n_rows + B - 1) / B;
    auto chunks = [&](int ids) { return (a.V + ids - 1) / ids; };
    AdjustPlan p{256, 1};
    if (a.hist_tok && a.hist_cap > mean * (256 * 2 * N)) {
        p.T = 512;
        if ((int64_t)B * chunks(8192) >= 1024) p.vectors = 8192 / (512 * N);
    } else if (!gradient && (int64_t)B * chunks(256 * 2 * N) >= 1024) {
        p.vectors = 2;
    }
    p.chunks = chunks(p.T * p.vectors * N);
    // A sequence's rows shared out, each share counting the history again: where there are fewer than kAdjustGroups workgroups of 256 threads (us, one share / two / four: 8 sequences of 9 rows of 128,256 fp32
    // 14.2 / 12.5 / 14.2, gradients of 32 sequences of 9.5 rows of 32,000 fp32 27 / 20.5 / 20.4).  Two shares of what one makes 1000 to 1800 workgroups of are more than run at once, and take less all the
    // same, mostly (one / two: 1000 workgroups, 40 sequences of 5.5 rows of 50,001 bf16, 23.8 / 22.7; 1600, 64 of them, 28.2 / 27.8; 1470, 30 of 9.5 rows of 50,001 fp32, 28.8 / 25.8; but 1280, 40 of 5.5 rows
    // of 32,000 fp32, 16.3 / 17.5).  And where rows are so many that the sequences' ends are far apart (256 of 9.5 rows of 151,936 bf16 309 / 300 / 323;
    // of 5 rows of 75,000 fp32 177 / 182 / 208)
    const int64_t groups = (int64_t)B * p.chunks;
    p.parts = (int)std::min<int64_t>(mean, std::max<int64_t>((kAdjustGroups * 256 / p.T + groups - 1) / groups, mean >= 8 ? 2 : 1));
    p.busy = groups * p.parts;
    // (one workgroup for every chunk and 32 rows, up to 256: a batch that is mostly padding has a share of the chip to write it, and a small one not more of them than it has others)
    p.idle = a.whole && a.seq_off ? p.chunks * (int)std::min<int64_t>(std::max(256 / p.chunks, 1), (n_rows + 31) / 32) : 0;
    p.fits = (p.busy + p.idle) * p.T <= (int64_t)UINT32_MAX;
    return p;
}

hipError_t launch_adjust(AdjustArgs a, const AdjustPlan& plan, int dtype, int B, int64_t n_rows, bool gradient, hipStream_t stream)
{
    a.chunks = plan.chunks; a.parts = plan.parts; a.idle = plan.idle; a.busy = (uint32_t)plan.busy; a.B = B; a.n_rows = (int)n_rows;
    if (gradient) return dtype == 1 ? launch<true, true>(a, plan, stream) : launch<false, true>(a, plan, stream);
    return dtype == 1 ? launch<true, false>(a, plan, stream) : launch<false, false>(a, plan, stream);
}

}  // namespace picospec
