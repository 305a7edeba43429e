// Rows of logits adjusted for what a request asks: penalties for tokens that its text holds already, biases of single tokens, a grammar's mask; and the gradient.
// With n the number of times that a token is in the sequence's history behind its prompt or among the drafted tokens in front of the row, and seen where it is in
// the history at all or among those:
//   z1 = seen ? (z > 0 ? z / repetition : z * repetition) : z
//   z2 = z1 - frequency n - [n > 0] presence + bias,   out = allowed ? z2 : -inf
//   d out / d z = allowed ? (seen ? (z > 0 ? 1 / repetition : repetition) : 1) : 0
// A workgroup has one sequence and one chunk of the vocabulary.  It counts the history's tokens of its chunk in LDS once, then takes the sequence's rows one by one, and
// counts the drafted token between a row and the next.
// What bounds it: the rows, read once and written once.
#include "kernels.hpp"
#include "vectors.hpp"

namespace picospec {

namespace {

constexpr int kAT = kAdjustThreads;

// A count: bit 0, a token of the prompt; from bit 1 on how often the token was generated
constexpr uint32_t kSeenBit = 1u, kOnce = 2u;

// -inf, as stored
template <bool BF16> constexpr uint32_t kMaskedBits = BF16 ? 0xFF80u : 0xFF800000u;

__device__ __forceinline__ float setting(const float* rows, int b, float all) { return rows ? rows[b] : all; }

template <bool BF16, bool GRAD>
__global__ __launch_bounds__(kAT) void adjust_kernel(const AdjustArgs a)
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4;
    extern __shared__ __attribute__((aligned(16))) uint32_t counts[];        // [chunk], and behind it the biases [chunk] where there are any
    const int tid = threadIdx.x;
    const int chunk = (int)(blockIdx.x % (unsigned)a.chunks), rest = (int)(blockIdx.x / (unsigned)a.chunks), part = rest % a.parts, b = rest / a.parts;
    const int lo = chunk * a.chunk, ids = min(a.chunk, a.V - lo);

    // the sequence's rows of this part, and the drafted tokens in front of them (what the offsets say beyond the arrays is not followed)
    int off = 0, gamma = 0;
    if (a.seq_off) {
        off = min(max(a.seq_off[b], 0), a.n_draft);
        gamma = min(max(a.seq_off[b + 1], off), a.n_draft) - off;
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
        bias0 = min(max(a.bias_off[b], 0), a.n_bias);
        bias1 = min(max(a.bias_off[b + 1], bias0), a.n_bias);
    }
    float* const bias = reinterpret_cast<float*>(counts + a.chunk);
    auto clear = [&] {
        for (int i = tid * 4; i < a.chunk; i += kAT * 4) *reinterpret_cast<uint4*>(counts + i) = make_uint4(0, 0, 0, 0);
    };
    clear();
    if (bias1 > bias0) {
        // of entries for the same token the last one counts: every entry bids with its place, the one that holds the token writes
        for (int i = tid * 4; i < a.chunk; i += kAT * 4) *reinterpret_cast<float4*>(bias + i) = make_float4(0.f, 0.f, 0.f, 0.f);
        __syncthreads();
        for (int i = bias0 + tid; i < bias1; i += kAT) {
            const unsigned x = (unsigned)a.bias_id[i] - (unsigned)lo;
            if (x < (unsigned)ids) atomicMax(&counts[x], (uint32_t)(i - bias0) + 1u);
        }
        __syncthreads();
        for (int i = bias0 + tid; i < bias1; i += kAT) {
            const unsigned x = (unsigned)a.bias_id[i] - (unsigned)lo;
            if (x < (unsigned)ids && counts[x] == (uint32_t)(i - bias0) + 1u) bias[x] = a.bias_value[i];
        }
        __syncthreads();
        clear();
    }
    __syncthreads();
    if (counted) {
        auto count = [&](int tok, uint32_t as) {
            const unsigned x = (unsigned)tok - (unsigned)lo;
            if (x < (unsigned)ids) {
                if (as == kSeenBit) atomicOr(&counts[x], kSeenBit);
                else atomicAdd(&counts[x], kOnce);
            }
        };
        if (a.hist_tok) {
            const int length = min(max(a.hist_len[b], 0), a.hist_cap), prompt = a.prompt_len ? a.prompt_len[b] : 0;
            const int32_t* const tok = a.hist_tok + (int64_t)b * a.ld_hist;
            int i = tid;
            for (; i + 3 * kAT < length; i += 4 * kAT) {
                int t[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) t[j] = tok[i + j * kAT];
#pragma unroll
                for (int j = 0; j < 4; ++j) count(t[j], i + j * kAT < prompt ? kSeenBit : kOnce);
            }
            for (; i < length; i += kAT) count(tok[i], i < prompt ? kSeenBit : kOnce);
        }
        for (int i = tid; i < t0; i += kAT) count(a.draft_tok[off + i], kOnce);
        __syncthreads();
    }

    const double by = (double)rep, inv = 1.0 / (double)rep, pres64 = pres, freq64 = freq;
    const int vecs = (ids + N - 1) / N;
    for (int t = t0; t < t1; ++t) {
        if (counted && t > t0) {
            const unsigned x = (unsigned)a.draft_tok[off + t - 1] - (unsigned)lo;
            if (x < (unsigned)ids) {                                          // (the same token for the whole workgroup)
                __syncthreads();
                if (tid == 0) counts[x] += kOnce;
                __syncthreads();
            }
        }
        const int64_t row = row0 + t;
        const char* const src = (const char*)a.src + (row * a.ld_src + lo) * ESZ;
        const char* const z_row = (const char*)a.logits + (row * a.ld + lo) * ESZ;
        char* const out = (char*)a.out + (row * a.ld_out + lo) * ESZ;
        const int m = !a.mask ? -1 : a.mask_row ? a.mask_row[row] : (int)row;
        const unsigned char* const mask = (unsigned)m < (unsigned)a.n_masks ? reinterpret_cast<const unsigned char*>(a.mask + (int64_t)m * a.ld_mask) + lo / 8 : nullptr;
        for (int v = tid; v < vecs; v += kAT) {
            const int x = v * N;
            unsigned allowed = (1u << N) - 1u;
            if (mask) allowed = (unsigned)mask[x / 8] >> (x & 7) & ((1u << N) - 1u);
            uint32_t c[N];
            float bs[N];
            uint32_t any = 0u;
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const uint4 w = *reinterpret_cast<const uint4*>(counts + x + e);
                c[e] = w.x; c[e + 1] = w.y; c[e + 2] = w.z; c[e + 3] = w.w;
                any |= w.x | w.y | w.z | w.w;
                if (bias1 > bias0) {
                    const float4 f = *reinterpret_cast<const float4*>(bias + x + e);
                    bs[e] = f.x; bs[e + 1] = f.y; bs[e + 2] = f.z; bs[e + 3] = f.w;
                    any |= __float_as_uint(f.x) | __float_as_uint(f.y) | __float_as_uint(f.z) | __float_as_uint(f.w);
                } else {
                    bs[e] = bs[e + 1] = bs[e + 2] = bs[e + 3] = 0.f;
                }
            }
            const bool whole = allowed == (1u << N) - 1u;
            if (a.in_place && !any && whole) continue;
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (allowed) raw = load_row_vec<BF16>(src, x, ids);
            if (allowed && any) {
                float z[N], g[N];
                unpack<BF16>(raw, g);
                if constexpr (GRAD) unpack<BF16>(load_row_vec<BF16>(z_row, x, ids), z);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if constexpr (GRAD) {
                        g[e] = c[e] ? (float)((double)g[e] * (z[e] > 0.f ? inv : by)) : g[e];
                    } else {
                        double y = (double)g[e];
                        y = c[e] ? y * (g[e] > 0.f ? inv : by) : y;
                        y = y - freq64 * (double)(c[e] >> 1) - (c[e] >> 1 ? pres64 : 0.0) + (double)bs[e];
                        g[e] = c[e] || bs[e] != 0.f ? (float)y : g[e];
                    }
                }
                raw = pack_vec<BF16>(g);
            }
            if (!whole) {
                uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
                constexpr uint32_t put = GRAD ? 0u : kMaskedBits<BF16>;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (!(allowed >> e & 1u)) {
                        if constexpr (BF16) w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | put << 16 : (w[e / 2] & 0xFFFF0000u) | put;
                        else w[e] = put;
                    }
                raw = make_uint4(w[0], w[1], w[2], w[3]);
            }
            store_row_vec<BF16>(out, x, ids, raw);
        }
    }
}

template <bool BF16, bool GRAD>
hipError_t launch(const AdjustArgs& a, int B, hipStream_t stream)
{
    const size_t lds = (size_t)a.chunk * (!GRAD && a.bias_off ? 8 : 4);
    hipLaunchKernelGGL((adjust_kernel<BF16, GRAD>), dim3((unsigned)((int64_t)B * a.parts * a.chunks)), dim3(kAT), lds, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adjust(AdjustArgs a, int dtype, int B, int64_t n_rows, bool gradient, hipStream_t stream)
{
    if (n_rows == 0) return hipSuccess;
    a.chunk = a.bias_off ? kAdjustChunk / 2 : kAdjustChunk;
    while (a.chunk > 1024 && (int64_t)B * ((a.V + a.chunk - 1) / a.chunk) < 1024) a.chunk /= 2;
    a.chunks = (a.V + a.chunk - 1) / a.chunk;
    const int64_t groups = (int64_t)B * a.chunks, mean = (n_rows + B - 1) / B;
    a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(mean, 1024 / groups));
    if (gradient) return dtype == 1 ? launch<true, true>(a, B, stream) : launch<false, true>(a, B, stream);
    return dtype == 1 ? launch<true, false>(a, B, stream) : launch<false, false>(a, B, stream);
}

}  // namespace picospec
