// Token embeddings and their gradient.
//   out[i] = scale table[tok[i]], 0 where tok[i] is outside [0, V)
//   grad[v] = scale * sum of g[i] over the positions i with tok[i] = v, in the order of the positions, in fp32
// What bounds them: rows read and written once; of the gradient the whole table, zeros of tokens that do not occur among them.
//
// The gradient's sums have a fixed order without atomics on values: embed_sort_kernel lists the positions by token, positions of one token in ascending order;
// embed_sum_kernel adds up a token's rows and writes the table.  A token with 2 kPiece positions and more is shared out in pieces of kPiece to 2 kPiece - 1, whose sums
// embed_join_kernel adds up, so that no workgroup's work depends on how often a token occurs.
#include "kernels.hpp"
#include "vectors.hpp"

namespace picospec {

namespace {

constexpr int kRowThreads = 256;                                  // of a workgroup that moves rows

// Threads that share a row: the smallest power of two with a vector for each, 8 to 256
template <bool BF16> int row_threads_log2(int64_t d)
{
    int l = 3;
    while (l < 8 && ((int64_t)Vec<BF16>::N << l) < d) ++l;
    return l;
}

template <bool BF16>
__global__ __launch_bounds__(kRowThreads) void embed_kernel(const void* table, int64_t ld, int V, int64_t d, const int32_t* tok, int64_t n, float scale, void* out, int64_t ld_out, int share)
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4;
    for (int64_t i = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> share; i < n; i += (int64_t)gridDim.x * kRowThreads >> share) {
        const int t = tok[i];
        const bool there = (unsigned)t < (unsigned)V;
        const char* const src = (const char*)table + (there ? (int64_t)t * ld * ESZ : 0);
        char* const dst = (char*)out + i * ld_out * ESZ;
        for (int64_t x = (int64_t)(threadIdx.x & ((1 << share) - 1)) * N; x < d; x += (int64_t)N << share) {
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (there) raw = load_row_vec<BF16>(src, x, d);
            if (there && scale != 1.f) {
                float f[N];
                unpack<BF16>(raw, f);
#pragma unroll
                for (int e = 0; e < N; ++e) f[e] *= scale;
                raw = pack_vec<BF16>(f);
            }
            store_row_vec<BF16>(dst, x, d, raw);
        }
    }
}

// Positions by token.  A workgroup has a range of tokens and reads all positions twice: its waves take consecutive stretches of them, count, for every wave and token
// apart, and after a scan over (token, wave) each wave knows where its positions of a token go.  How many positions lie in front of the range it counts itself, so no workgroup waits for
// another.  first[v] .. first[v + 1] are token v's places in `order`; slot_tok names the token of each piece (embed_pieces).
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int32_t* tok, int n, int V, int range, int32_t* first, int32_t* order, int32_t* slot_tok)
{
    constexpr int W = kSortThreads / kWave;
    extern __shared__ int32_t counts[];                           // [W][range]
    __shared__ int sums[W], below[W];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int lo = blockIdx.x * range, ids = min(range, V - lo);
    int32_t* const mine = counts + wave * range;
    for (int i = tid; i < W * range; i += kSortThreads) counts[i] = 0;
    const int stretch = ((n + W - 1) / W + kWave - 1) / kWave * kWave, begin = min(wave * stretch, n), end = min(begin + stretch, n);
    __syncthreads();

    // f(x, lanes): once for every token lo + x of a step's 64 positions, with the lanes that have it (one lane writes, all read: the wave's LDS accesses are in order)
    auto each_token = [&](int t, auto f) {
        const int x = t - lo;
        const bool in = (unsigned)x < (unsigned)ids;
        unsigned long long left = __ballot(in);
        while (left) {
            const int xl = __builtin_amdgcn_readlane(x, __builtin_ctzll(left));
            const unsigned long long same = __ballot(in && x == xl);
            f(xl, same);
            left &= ~same;
        }
    };
    constexpr int AHEAD = 8;
    auto stream = [&](auto f) {
        for (int i = begin; i < end; i += AHEAD * kWave) {
            int t[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) t[j] = i + j * kWave + lane < end ? tok[i + j * kWave + lane] : -1;
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) f(i + j * kWave, t[j]);
        }
    };
    int front = 0;
    stream([&](int, int t) {
        front += t >= 0 && t < lo;
        each_token(t, [&](int x, unsigned long long same) {
            if (lane == 0) __hip_atomic_fetch_add(&mine[x], __builtin_popcountll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        });
    });
    front = wave_sum(front);
    if (lane == 0) below[wave] = front;
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) base += below[w];
    // thread x: token lo + x (range <= kSortThreads)
    int total = 0;
    if (tid < ids)
        for (int w = 0; w < W; ++w) total += counts[w * range + tid];
    const int incl = wave_scan_incl(total);
    if (lane == kWave - 1) sums[wave] = incl;
    __syncthreads();
    int at = base + incl - total;
#pragma unroll
    for (int w = 0; w < W; ++w) if (w < wave) at += sums[w];
    if (tid < ids) {
        first[lo + tid] = at;
        if (lo + tid == V - 1) first[V] = at + total;
        const EmbedPieces p = embed_pieces(at, total);
        for (int s = 0; s < p.count; ++s) slot_tok[p.slot + s] = lo + tid;
        for (int w = 0; w < W; ++w) {
            const int c = counts[w * range + tid];
            counts[w * range + tid] = at;
            at += c;
        }
    }
    __syncthreads();
    stream([&](int i, int t) {
        each_token(t, [&](int x, unsigned long long same) {
            int place = 0;
            if (lane == 0) place = __hip_atomic_fetch_add(&mine[x], __builtin_popcountll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            place = __builtin_amdgcn_readfirstlane(place);
            if (same >> lane & 1ull) order[place + __builtin_popcountll(same & ((1ull << lane) - 1ull))] = i + lane;
        });
    });
}

// sum += rows order[p0] .. order[p1 - 1], elements x .. x + N - 1
template <bool BF16>
__device__ __forceinline__ void add_rows(const char* g, int64_t ld, int64_t d, const int32_t* order, int p0, int p1, int64_t x, float (&sum)[Vec<BF16>::N])
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4, AHEAD = 4;
    int p = p0;
    for (; p + AHEAD <= p1; p += AHEAD) {
        uint4 raw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) raw[j] = load_row_vec<BF16>(g + (int64_t)order[p + j] * ld * ESZ, x, d);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float f[N];
            unpack<BF16>(raw[j], f);
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += f[e];
        }
    }
    for (; p < p1; ++p) {
        float f[N];
        unpack<BF16>(load_row_vec<BF16>(g + (int64_t)order[p] * ld * ESZ, x, d), f);
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += f[e];
    }
}

// a token's elements x .. x + N - 1 of the table (N of the gradient's type), N sums of them
template <bool OUT16, int N>
__device__ __forceinline__ void write_sums(char* row, int64_t x, int64_t d, float (&sum)[N], float scale, bool add)
{
    constexpr int M = Vec<OUT16>::N;
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] *= scale;
    if constexpr (N >= M) {
#pragma unroll
        for (int k = 0; k < N; k += M) {
            if (k && x + k >= d) break;
            float f[M];
            if (add) {
                unpack<OUT16>(load_row_vec<OUT16>(row, x + k, d), f);
#pragma unroll
                for (int e = 0; e < M; ++e) f[e] += sum[k + e];
            } else {
#pragma unroll
                for (int e = 0; e < M; ++e) f[e] = sum[k + e];
            }
            store_row_vec<OUT16>(row, x + k, d, pack_vec<OUT16>(f));
        }
    } else {                                                      // (fp32 rows into a bf16 table: half a vector, element by element)
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (x + e < d) {
                uint16_t* const p = reinterpret_cast<uint16_t*>(row) + x + e;
                const float old = add ? __uint_as_float((uint32_t)*p << 16) : 0.f;
                *p = (uint16_t)pack_bf16(add ? old + sum[e] : sum[e], 0.f);
            }
    }
}

template <bool BF16, bool OUT16>
__global__ __launch_bounds__(kRowThreads) void embed_sum_kernel(const EmbedGradArgs a)
{
    constexpr int N = Vec<BF16>::N;
    const int share = a.share, per = kRowThreads >> share, sub = threadIdx.x >> share;
    const int64_t x0 = (int64_t)(threadIdx.x & ((1 << share) - 1)) * N, step = (int64_t)N << share;
    const char* const g = (const char*)a.g;
    if ((int)blockIdx.x < a.slot_groups) {                        // pieces of the tokens that occur most, in front: they take longest
        const int s = (int)blockIdx.x * per + sub;
        if (s >= a.slots) return;
        const int v = a.slot_tok[s];                              // (what the sort has not written is not a token's that has this slot)
        if ((unsigned)v >= (unsigned)a.V) return;
        const int p0 = a.first[v], len = a.first[v + 1] - p0;
        const EmbedPieces p = embed_pieces(p0, len);
        if (s < p.slot || s >= p.slot + p.count) return;
        const int begin = p0 + (s - p.slot) * kPiece, end = s == p.slot + p.count - 1 ? p0 + len : begin + kPiece;
        for (int64_t x = x0; x < a.d; x += step) {
            float sum[N] = {};
            add_rows<BF16>(g, a.ld, a.d, a.order, begin, end, x, sum);
            float* const to = a.partial + (int64_t)s * a.d_pad + x;
#pragma unroll
            for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(to + e) = make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]);
        }
        return;
    }
    // tokens, those of a workgroup far apart: neighbours occur about as often
    const int groups = (int)gridDim.x - a.slot_groups;
    for (int v = ((int)blockIdx.x - a.slot_groups) * per + sub; v < a.V; v += groups * per) {
        const int p0 = a.first[v], p1 = a.first[v + 1];
        if (embed_pieces(p0, p1 - p0).count || (a.accumulate && p0 == p1)) continue;
        char* const row = (char*)a.out + (int64_t)v * a.ld_out * (OUT16 ? 2 : 4);
        for (int64_t x = x0; x < a.d; x += step) {
            float sum[N] = {};
            add_rows<BF16>(g, a.ld, a.d, a.order, p0, p1, x, sum);
            write_sums<OUT16, N>(row, x, a.d, sum, a.scale, a.accumulate);
        }
    }
}

// The sums of a token's pieces, by the workgroup of the first of them
template <bool BF16, bool OUT16>
__global__ __launch_bounds__(kRowThreads) void embed_join_kernel(const EmbedGradArgs a)
{
    constexpr int N = Vec<BF16>::N;
    const int s = (int)blockIdx.x;
    const int v = a.slot_tok[s];
    if ((unsigned)v >= (unsigned)a.V) return;
    const int p0 = a.first[v];
    const EmbedPieces p = embed_pieces(p0, a.first[v + 1] - p0);
    if (p.count == 0 || s != p.slot) return;
    char* const row = (char*)a.out + (int64_t)v * a.ld_out * (OUT16 ? 2 : 4);
    for (int64_t x = (int64_t)(blockIdx.y * kRowThreads + threadIdx.x) * N; x < a.d; x += (int64_t)gridDim.y * kRowThreads * N) {
        float sum[N] = {};
        for (int i = 0; i < p.count; ++i) {
            const float* const from = a.partial + (int64_t)(s + i) * a.d_pad + x;
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const float4 f = *reinterpret_cast<const float4*>(from + e);
                sum[e] += f.x; sum[e + 1] += f.y; sum[e + 2] += f.z; sum[e + 3] += f.w;
            }
        }
        write_sums<OUT16, N>(row, x, a.d, sum, a.scale, a.accumulate);
    }
}

template <bool BF16, bool OUT16>
hipError_t launch_sums(EmbedGradArgs a, hipStream_t stream)
{
    a.share = row_threads_log2<BF16>(a.d);
    const int per = kRowThreads >> a.share;
    a.slot_groups = (a.slots + per - 1) / per;
    const int groups = (int)std::min<int64_t>((a.V + per - 1) / per, 8192);
    hipLaunchKernelGGL((embed_sum_kernel<BF16, OUT16>), dim3((unsigned)(a.slot_groups + groups)), dim3(kRowThreads), 0, stream, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.slots < 2) return hipSuccess;                            // (no token has two pieces)
    const int64_t tiles = (a.d + kRowThreads * Vec<BF16>::N - 1) / (kRowThreads * Vec<BF16>::N);
    hipLaunchKernelGGL((embed_join_kernel<BF16, OUT16>), dim3((unsigned)a.slots, (unsigned)std::min<int64_t>(tiles, 64)), dim3(kRowThreads), 0, stream, a);
    return hipGetLastError();
}

template <bool BF16>
hipError_t launch_rows(const void* table, int64_t ld, int V, int64_t d, const int32_t* tok, int64_t n, float scale, void* out, int64_t ld_out, hipStream_t stream)
{
    const int share = row_threads_log2<BF16>(d);
    const int64_t blocks = std::min<int64_t>(((n << share) + kRowThreads - 1) / kRowThreads, 1 << 22);
    hipLaunchKernelGGL(embed_kernel<BF16>, dim3((unsigned)blocks), dim3(kRowThreads), 0, stream, table, ld, V, d, tok, n, scale, out, ld_out, share);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const void* table, int dtype, int64_t ld, int V, int64_t d, const int32_t* tok, int64_t n, float scale, void* out, int64_t ld_out, hipStream_t stream)
{
    if (n == 0) return hipSuccess;
    return dtype == 1 ? launch_rows<true>(table, ld, V, d, tok, n, scale, out, ld_out, stream) : launch_rows<false>(table, ld, V, d, tok, n, scale, out, ld_out, stream);
}

hipError_t launch_embed_grad(EmbedGradArgs a, int dtype, int out_dtype, const int32_t* tok, int n, void* workspace, hipStream_t stream)
{
    const EmbedScratch l = embed_scratch(n, a.V, a.d);
    char* const ws = (char*)workspace;
    int32_t* const first = reinterpret_cast<int32_t*>(ws);
    int32_t* const order = reinterpret_cast<int32_t*>(ws + l.order_at);
    int32_t* const slot_tok = reinterpret_cast<int32_t*>(ws + l.slot_at);
    a.first = first;
    a.order = order;
    a.slot_tok = slot_tok;
    a.partial = reinterpret_cast<float*>(ws + l.partial_at);
    a.slots = l.slots;
    a.d_pad = l.d_pad;
    const int range = embed_range(a.V);
    static DeviceFlags done;
    int dev;
    if (hipError_t e = raise_lds_limit_once((const void*)embed_sort_kernel, kSortLds, done, dev)) return e;
    hipLaunchKernelGGL(embed_sort_kernel, dim3((unsigned)((a.V + range - 1) / range)), dim3(kSortThreads), (size_t)range * (kSortThreads / kWave) * 4, stream, tok, n, a.V, range, first, order, slot_tok);
    if (hipError_t e = hipGetLastError()) return e;
    if (dtype == 1) return out_dtype == 1 ? launch_sums<true, true>(a, stream) : launch_sums<true, false>(a, stream);
    return out_dtype == 1 ? launch_sums<false, true>(a, stream) : launch_sums<false, false>(a, stream);
}

}  // namespace picospec
