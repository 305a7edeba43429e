// Token embeddings and their gradient.
//   out[i] = scale table[tok[i]], 0 where tok[i] is outside [0, V)
//   grad[v] = scale * sum of g[i] over the positions i with tok[i] = v, in the order of the positions, in fp32
// What bounds them: rows read and written once; of the gradient the whole table, zeros of tokens that do not occur among them.
//
// The gradient's sums have a fixed order without atomics on values: embed_sort_kernel lists the positions by token, positions of one token in ascending order;
// embed_sum_kernel adds up a token's rows and writes the table.  A token with 2 kPiece positions and more is shared out in up to kPiecesMost pieces.
#include "kernels.hpp"
#include "vectors.hpp"

namespace picospec {

namespace {

constexpr int kRowThreads = 256;                                  // of a workgroup that moves rows
constexpr int kFewRows = 8;                                       // of a token, that one group of threads adds up
constexpr int kChain = 32;                                        // rows of a token in a chain of additions, where all of them may be one thread's

// true in the last of `total` workgroups that arrive at a word that was 0 at the kernel's start.  What they hand over went by put_shared (see there).
__device__ __forceinline__ bool arrived_last(uint32_t* word, unsigned total)
{
    __shared__ int last;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");              // (every wave: its stores are where all can see them)
    __syncthreads();
    if (threadIdx.x == 0) last = __hip_atomic_fetch_add(word, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == total;
    __syncthreads();
    return last != 0;
}

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

// Positions by token, in the order of the positions.  A workgroup has every W-th token (W a power of two: tokens that occur often stand together in most vocabularies) and reads all
// positions once: its waves take consecutive stretches of them and keep a list of those that are its own, a few of 64 in each step.  After a scan over (token, wave) each wave knows where its
// positions of a token go, and puts them there 64 at a time: the lanes with the same token find each other by ten ballots over its bits.  How many positions lie in front of the workgroup's it
// counts itself, so no workgroup waits for another.  A wave whose list is full reads its stretch again instead.
// One pass over the tokens instead of two, and every W-th token instead of a range: 32,768 positions by a Zipf law 191 -> 15 us (the range of the frequent tokens took them).
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int32_t* tok, int n, int V, int own_log2, int range, int2* info, int2* order, int32_t* slot_tok, uint32_t* arrived)
{
    constexpr int W = kSortThreads / kWave, AHEAD = 16, LIST = kSortList;
    extern __shared__ int32_t counts[];                           // [W][range]
    __shared__ uint32_t lists[W][LIST];                           // place in the stretch << 10 | token
    __shared__ int sums[W], below[W];
    static_assert(kEmbedMostTokens / W <= 1 << 22 && kSortThreads <= 1 << 10, "an entry of a list is a word");
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int owner = blockIdx.x, step = 1 << own_log2;
    int32_t* const mine = counts + wave * range;
    uint32_t* const list = lists[wave];
    for (int i = tid; i < W * range; i += kSortThreads) counts[i] = 0;
    const int stretch = ((n + W - 1) / W + kWave - 1) / kWave * kWave, begin = min(wave * stretch, n), end = min(begin + stretch, n);
    __syncthreads();

    auto stream = [&](auto f) {
        for (int i = begin; i < end; i += AHEAD * kWave) {
            int t[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) t[j] = i + j * kWave + lane < end ? tok[i + j * kWave + lane] : -1;
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) f(i + j * kWave, t[j]);
        }
    };
    const unsigned long long lanes_below = (1ull << lane) - 1ull;
    auto own = [&](int t) { return (unsigned)t < (unsigned)V && (t & (step - 1)) == owner; };
    int front = 0, listed = 0;
    stream([&](int i, int t) {
        front += (unsigned)t < (unsigned)V && (t & (step - 1)) < owner;
        const bool in = own(t);
        const unsigned long long lanes = __ballot(in);
        if (lanes) {
            const int at = listed + __builtin_popcountll(lanes & lanes_below);
            if (in) {
                atomicAdd(&mine[t >> own_log2], 1);
                if (at < LIST) list[at] = (uint32_t)(i + lane - begin) << 10 | (uint32_t)(t >> own_log2);
            }
            listed += __builtin_popcountll(lanes);
        }
    });
    front = wave_sum(front);
    if (lane == 0) below[wave] = front;
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) base += below[w];
    // thread x: token x * step + owner (range <= kSortThreads)
    const int v = tid * step + owner;
    const bool there = tid < range && v < V;
    int total = 0;
    if (there)
        for (int w = 0; w < W; ++w) total += counts[w * range + tid];
    const int incl = wave_scan_incl(total);
    if (lane == kWave - 1) sums[wave] = incl;
    __syncthreads();
    int at = base + incl - total;
#pragma unroll
    for (int w = 0; w < W; ++w) if (w < wave) at += sums[w];
    if (tid == 0 && blockIdx.x == gridDim.x - 1) {                // (the last one's end is all that are in the table)
        int all = base;
        for (int w = 0; w < W; ++w) all += sums[w];
        info[V] = make_int2(all, 0);
    }
    if (there) {
        info[v] = make_int2(at, total);
        const EmbedPieces p = embed_pieces(at, total);
        for (int s = 0; s < p.count; ++s) slot_tok[p.slot + s] = v;
        if (p.count)
            for (int k = 0; k < kTilesMost; ++k) arrived[p.slot * kTilesMost + k] = 0u;
        for (int w = 0; w < W; ++w) {
            const int c = counts[w * range + tid];
            counts[w * range + tid] = at;
            at += c;
        }
    }
    __syncthreads();
    // 64 positions i of tokens x, in ascending order of the lanes
    auto place = [&](bool in, int x, int i) {
        unsigned long long same = __ballot(in);
#pragma unroll
        for (int k = 0; k < 10; ++k) {
            const bool bit = x >> k & 1;
            const unsigned long long set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        const int first = same ? __builtin_ctzll(same) : 0;
        int to = 0;
        if (in && lane == first) to = atomicAdd(&mine[x], (int)__builtin_popcountll(same));
        to = __shfl(to, first, kWave);
        if (in) order[to + __builtin_popcountll(same & lanes_below)] = make_int2(i, x * step + owner);
    };
    if (listed <= LIST) {
        for (int k = 0; k < listed; k += kWave) {
            const bool in = k + lane < listed;
            const uint32_t e = in ? list[k + lane] : 0u;
            place(in, (int)(e & 1023u), begin + (int)(e >> 10));
        }
    } else {
        stream([&](int i, int t) {
            const bool in = own(t);
            if (__ballot(in)) place(in, in ? t >> own_log2 : 0, i + lane);
        });
    }
}

// sum = rows at(p0) .. at(p1 - 1), elements x .. x + N - 1, added up, eight rows under way at a time (sum: zeros).  FAR: the places lie in memory, and the next eight are read beside the rows (32,768 rows for one token
// 196 -> 156 us; where they lie in LDS the registers cost more).  Where they lie in LDS the rows may be all of a token's, up to kFewTokens: every kChain of them are added up
// apart, so that no element goes through more than 2 kChain additions (rows behind each other in one chain were off by as many roundings as there are rows).
template <bool BF16, bool FAR, class At>
__device__ __forceinline__ void add_rows(const char* g, int64_t ld, int64_t d, At at, int p0, int p1, int64_t x, float (&sum)[Vec<BF16>::N])
{
    constexpr int N = Vec<BF16>::N, ESZ = BF16 ? 2 : 4, AHEAD = 8;
    static_assert(kChain % AHEAD == 0 && kChain * kChain >= kFewTokens, "a chain of chains");
    int i[AHEAD];
    float chains[N] = {};
    auto places = [&](int p) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) i[j] = p + j < p1 ? at(p + j) : 0;
    };
    if (FAR) places(p0);
    for (int p = p0; p < p1; p += AHEAD) {
        if (!FAR) places(p);
        uint4 raw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            raw[j] = make_uint4(0, 0, 0, 0);
            if (p + j < p1) raw[j] = load_row_vec<BF16>(g + (int64_t)i[j] * ld * ESZ, x, d);
        }
        if (FAR) places(p + AHEAD);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float f[N];
            unpack<BF16>(raw[j], f);
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += f[e];
        }
        if (!FAR && (p - p0) % kChain == kChain - AHEAD) {
#pragma unroll
            for (int e = 0; e < N; ++e) { chains[e] += sum[e]; sum[e] = 0.f; }
        }
    }
    if (!FAR && p1 - p0 > kChain - AHEAD) {
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += chains[e];
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

// Zeros for the rows row0 .. row0 + rows - 1 (up to 64) of the table but those with a bit in `kept`, by the workgroup; rows that lie without gaps as one stretch
template <bool OUT16>
__device__ __forceinline__ void zero_rows(const EmbedGradArgs& a, int64_t row0, int rows, unsigned long long kept)
{
    constexpr int M = Vec<OUT16>::N, ESZ = OUT16 ? 2 : 4;
    const int tid = threadIdx.x;
    for (int r = 0; r < rows;) {
        if (kept >> r & 1ull) { ++r; continue; }
        const unsigned long long next = kept >> r;
        const int end = a.ld_out != a.d ? r + 1 : min(rows, next ? r + (int)__builtin_ctzll(next) : rows);
        char* const to = (char*)a.out + (row0 + r) * a.ld_out * ESZ;
        const int64_t total = (end - r) * a.d;
        const int head = (int)min<int64_t>((16 - ((uintptr_t)to & 15)) % 16 / ESZ, total);
        if (tid < head) {
            if constexpr (OUT16) reinterpret_cast<uint16_t*>(to)[tid] = 0;
            else reinterpret_cast<float*>(to)[tid] = 0.f;
        }
        for (int64_t x = head + (int64_t)tid * M; x < total; x += (int64_t)kRowThreads * M) store_row_vec<OUT16>(to, x, total, make_uint4(0, 0, 0, 0));
        r = end;
    }
}

// The table's rows.  The workgroups in front take the pieces of the tokens that occur most, one each, and the last piece of a token to be done adds its pieces up; those behind them the
// other tokens that occur, by their positions; the rest writes zeros.  In this order: rows that are read beside a stream of writes come at the rate of a copy, the zeros alone
// at that of a fill.
template <bool BF16, bool OUT16>
__global__ __launch_bounds__(kRowThreads) void embed_sum_kernel(const EmbedGradArgs a)
{
    constexpr int N = Vec<BF16>::N, AHEAD = 8;
    __shared__ int2 info[kTokensMost];
    const int tid = threadIdx.x, per = kRowThreads >> a.share, sub = tid >> a.share;
    const char* const g = (const char*)a.g;
    if ((int)blockIdx.x < a.slots * a.tiles) {
        const int s = (int)blockIdx.x / a.tiles, tile = (int)blockIdx.x % a.tiles;
        const int v = a.slot_tok[s];                              // (what the sort has not written is not a token's that has this slot)
        if ((unsigned)v >= (unsigned)a.V) return;
        const int2 seg = a.info[v];
        const EmbedPieces p = embed_pieces(seg.x, seg.y);
        if (s < p.slot || s >= p.slot + p.count) return;
        const int len = (seg.y + p.count - 1) / p.count, begin = min(seg.x + (s - p.slot) * len, seg.x + seg.y), end = min(begin + len, seg.x + seg.y);
        const int64_t x0 = ((int64_t)tile * kRowThreads + tid) * N, step = (int64_t)a.tiles * kRowThreads * N;
        auto at = [&](int q) { return a.order[q].x; };
        for (int64_t x = x0; x < a.d; x += step) {
            float sum[N] = {};
            add_rows<BF16, true>(g, a.ld, a.d, at, begin, end, x, sum);
            float2* const to = reinterpret_cast<float2*>(a.partial + (int64_t)s * a.d_pad + x);
#pragma unroll
            for (int e = 0; e < N; e += 2) put_shared(to + e / 2, make_float2(sum[e], sum[e + 1]));
        }
        if (!arrived_last(&a.arrived[p.slot * kTilesMost + tile], (unsigned)p.count)) return;
        char* const row = (char*)a.out + (int64_t)v * a.ld_out * (OUT16 ? 2 : 4);
        for (int64_t x = x0; x < a.d; x += step) {
            float sum[N] = {};
            const float2* from = reinterpret_cast<const float2*>(a.partial + (int64_t)p.slot * a.d_pad + x);
            for (int i = 0; i < p.count; i += AHEAD / 2) {
                float2 f[AHEAD / 2][N / 2];
#pragma unroll
                for (int j = 0; j < AHEAD / 2; ++j)
#pragma unroll
                    for (int e = 0; e < N / 2; ++e) f[j][e] = i + j < p.count ? get_shared(from + (i + j) * (a.d_pad / 2) + e) : make_float2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < AHEAD / 2; ++j)
#pragma unroll
                    for (int e = 0; e < N / 2; ++e) { sum[2 * e] += f[j][e].x; sum[2 * e + 1] += f[j][e].y; }
            }
            write_sums<OUT16, N>(row, x, a.d, sum, a.scale, a.accumulate);
        }
        return;
    }
    const int behind = (int)blockIdx.x - a.slots * a.tiles;
    if (behind < a.windows * a.tiles) {
        // the tokens whose positions begin in kPiece of them (but those in pieces), so that every workgroup has about as many rows: batches of rows, which the tokens share
        const int w0 = (behind / a.tiles * per + sub) * kPiece, all = a.info[a.V].x;
        if (w0 >= all) return;
        const int w1 = min(w0 + kPiece, all);
        const int2 front = a.info[a.order[w0].y], back = a.info[a.order[w1 - 1].y];
        const int begin = front.x == w0 ? w0 : front.x + front.y, end = embed_pieces(back.x, back.y).count ? back.x : back.x + back.y;
        if (begin >= w1 || begin >= end) return;
        const int64_t x0 = (int64_t)(((behind % a.tiles) << a.share) + (tid & ((1 << a.share) - 1))) * N, step = ((int64_t)a.tiles * N) << a.share;
        for (int64_t x = x0; x < a.d; x += step) {
            float sum[N] = {};
            int2 o[AHEAD + 1];
            auto places = [&](int p) {
#pragma unroll
                for (int j = 0; j <= AHEAD; ++j) o[j] = p + j < end ? a.order[p + j] : make_int2(0, -1);
            };
            places(begin);
            for (int p = begin; p < end; p += AHEAD) {
                uint4 raw[AHEAD];
                int of[AHEAD];
                unsigned last = 0u;                               // bit j: row j is its token's last
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    last |= (unsigned)(o[j].y != o[j + 1].y) << j;
                    of[j] = o[j].y;
                    raw[j] = make_uint4(0, 0, 0, 0);
                    if (p + j < end) raw[j] = load_row_vec<BF16>(g + (int64_t)o[j].x * a.ld * (BF16 ? 2 : 4), x, a.d);
                }
                places(p + AHEAD);
                for (int j0 = 0; j0 < AHEAD && p + j0 < end;) {
                    const unsigned rest = last >> j0;
                    const int j1 = rest ? j0 + __builtin_ctz(rest) + 1 : AHEAD;
                    int v = 0;
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j)
                        if (j >= j0 && j < j1) {
                            v = of[j];
                            float f[N];
                            unpack<BF16>(raw[j], f);
#pragma unroll
                            for (int e = 0; e < N; ++e) sum[e] += f[e];
                        }
                    if (rest) {
                        write_sums<OUT16, N>((char*)a.out + (int64_t)v * a.ld_out * (OUT16 ? 2 : 4), x, a.d, sum, a.scale, a.accumulate);
#pragma unroll
                        for (int e = 0; e < N; ++e) sum[e] = 0.f;
                    }
                    j0 = j1;
                }
            }
        }
        return;
    }
    // zeros for the tokens that do not occur
    const int before = (a.slots + a.windows) * a.tiles, groups = (int)gridDim.x - before, group = (int)blockIdx.x - before;
    if (a.together) {
        const int rows = (a.V + groups - 1) / groups, row0 = group * rows, here = min(rows, a.V - row0);
        __shared__ unsigned long long kept;
        if (tid < kWave) {
            const unsigned long long some = __ballot(tid < here && a.info[row0 + tid].y != 0);
            if (tid == 0) kept = some;
        }
        __syncthreads();
        zero_rows<OUT16>(a, row0, here, kept);
        return;
    }
    const int tokens = (a.V - group + groups - 1) / groups;
    if (tid < tokens) info[tid] = a.info[group + tid * groups];
    __syncthreads();
    for (int k = sub; k < tokens; k += per) {
        if (info[k].y != 0) continue;
        char* const row = (char*)a.out + (int64_t)(group + k * groups) * a.ld_out * (OUT16 ? 2 : 4);
        constexpr int M = Vec<OUT16>::N;
        for (int64_t x = (int64_t)(tid & ((1 << a.share) - 1)) * M; x < a.d; x += (int64_t)M << a.share) store_row_vec<OUT16>(row, x, a.d, make_uint4(0, 0, 0, 0));
    }
}

// Few positions, in one launch: every workgroup looks its tokens' positions up itself.  777 positions, 50,001 x 501 fp32: 23 us, zeros alone 21; sorted and
// summed in launches of their own 46.  1024 positions of a Zipf law so / 1025 of it sorted, written and added: 32,000 x 200 fp32 12.5 / 26.4 and 9.7 / 26, 32,000 x 1024 fp32 39.5 / 42.4 and 13.3 / 26.4,
// 128,256 x 4096 bf16 195.5 / 197.2 and 30.7 / 35.  The other side: half of the 1024 positions one token's, whose rows are added up in one workgroup here: 46.4 / 27.4 and 40.1 / 27.2, 117 / 43.3
// and 95.8 / 27.2, 342 / 198 and 183 / 34.8.  How tokens spread is not known in front of the launch.
template <bool BF16, bool OUT16>
__global__ __launch_bounds__(kRowThreads) void embed_few_kernel(const EmbedGradArgs a, const int32_t* tok, int n, int groups_log2)
{
    constexpr int N = Vec<BF16>::N;
    __shared__ uint32_t found[kFewTokens], sorted[kFewTokens];    // token << 16 | position
    __shared__ int how_many, first[kTokensMost + 1];
    const int tid = threadIdx.x, per = kRowThreads >> a.share, sub = tid >> a.share;
    const int64_t x0 = (int64_t)(tid & ((1 << a.share) - 1)) * N, step = (int64_t)N << a.share;
    const int group = blockIdx.x, groups = 1 << groups_log2, tokens = (a.V - group + groups - 1) >> groups_log2;
    const int rows_here = (a.V + (int)gridDim.x - 1) / (int)gridDim.x, row0 = group * rows_here;      // a.together: the rows that it zeroes
    __shared__ unsigned long long kept;
    if (tid == 0) { how_many = 0; kept = 0ull; }
    __syncthreads();
    for (int i = tid; i < n; i += kRowThreads) {
        const int t = tok[i];
        if (a.together && (unsigned)t - (unsigned)row0 < (unsigned)rows_here) atomicOr(&kept, 1ull << (t - row0));
        if ((unsigned)t < (unsigned)a.V && (t & (groups - 1)) == group) found[atomicAdd(&how_many, 1)] = (uint32_t)(t >> groups_log2) << 16 | (uint32_t)i;
    }
    __syncthreads();
    const int m = how_many;
    for (int i = tid; i < m; i += kRowThreads) {                  // (every key is another: its place is the number of smaller ones)
        const uint32_t key = found[i];
        int at = 0;
        for (int j = 0; j < m; ++j) at += found[j] < key;
        sorted[at] = key;
    }
    __syncthreads();
    if (tid <= tokens && tid <= kTokensMost) {
        int lo = 0, hi = m;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (sorted[mid] >> 16 < (uint32_t)tid) lo = mid + 1; else hi = mid;
        }
        first[tid] = lo;
    }
    __syncthreads();
    auto at = [&](int p) { return (int)(sorted[p] & 0xFFFFu); };
    // tokens of many rows: the rows shared out among the threads that could have a row each, so that fewer batches stand behind each other (a batch that is read while the chip
    // writes zeros takes 4 us: the case above 28.6 -> 21.4 us).  Where a row takes all threads there is nothing to share out.
    if (per > 1) {
        __shared__ float part[kRowThreads][N];
        for (int k = 0; k < tokens; ++k) {
            const int p0 = first[k], rows = first[k + 1] - p0, each = (rows + per - 1) / per;
            if (rows <= kFewRows) continue;
            float sum[N] = {};
            if (x0 < a.d) add_rows<BF16, false>((const char*)a.g, a.ld, a.d, at, min(p0 + sub * each, p0 + rows), min(p0 + (sub + 1) * each, p0 + rows), x0, sum);
#pragma unroll
            for (int e = 0; e < N; ++e) part[tid][e] = sum[e];
            __syncthreads();
            if (sub == 0 && x0 < a.d) {
                for (int i = 1; i < per; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) sum[e] += part[(i << a.share) + tid][e];
                write_sums<OUT16, N>((char*)a.out + (int64_t)(group + (k << groups_log2)) * a.ld_out * (OUT16 ? 2 : 4), x0, a.d, sum, a.scale, a.accumulate);
            }
            __syncthreads();
        }
    }
    for (int k = sub; k < tokens; k += per) {
        const int p0 = first[k], p1 = first[k + 1];
        if (((a.accumulate || a.together) && p0 == p1) || (per > 1 && p1 - p0 > kFewRows)) continue;
        char* const row = (char*)a.out + (int64_t)(group + (k << groups_log2)) * a.ld_out * (OUT16 ? 2 : 4);
        for (int64_t x = x0; x < a.d; x += step) {
            float sum[N] = {};
            add_rows<BF16, false>((const char*)a.g, a.ld, a.d, at, p0, p1, x, sum);
            write_sums<OUT16, N>(row, x, a.d, sum, a.scale, a.accumulate);
        }
    }
    if (a.together && !a.accumulate) zero_rows<OUT16>(a, row0, min(rows_here, a.V - row0), kept);
}

// Workgroups that write the table's rows: 20 KB each, but 8 to kTokensMost rows, and no fewer than 2048 of them (116,340 rows of 320 fp32, 149 MB, 8 rows each 32 us, 16 27.8; of 512 33.8, 34.3, of 4 KB
// 22.8, 23.7: 7 TB/s)
template <bool OUT16> int row_groups(const EmbedGradArgs& a)
{
    const int rows = (int)std::min<int64_t>(std::max<int64_t>(20480 / (a.d * (OUT16 ? 2 : 4)), 8), kTokensMost);
    return std::max((a.V + rows - 1) / rows, std::min(a.V, 2048));
}

// Whether a workgroup zeroes rows that stand together, as one stretch where they lie without gaps, rather than every so many-th row.  us, apart / together: rows whose ends share a line with the
// next one's, which another workgroup writes (126,730 x 1124 fp32 135 / 108, 120,000 x 333 bf16 31 / 22), or leave lanes without work (116,340 x 320 fp32 30 / 25); but stretches that
// begin whole pages apart meet in the same channels of the memory (100,000 x 4096 bf16 146 / 157, x 2048 72 / 79).
template <bool OUT16> int together(const EmbedGradArgs& a) { return a.ld_out * (OUT16 ? 2 : 4) % 4096 != 0; }

template <bool BF16, bool OUT16>
hipError_t launch_sums(EmbedGradArgs a, int n, hipStream_t stream)
{
    a.share = row_threads_log2<BF16>(a.d);
    const int per = kRowThreads >> a.share;
    a.windows = ((n + kPiece - 1) / kPiece + per - 1) / per;
    a.tiles = (int)std::min<int64_t>((a.d + kRowThreads * Vec<BF16>::N - 1) / (kRowThreads * Vec<BF16>::N), kTilesMost);
    const int groups = a.accumulate ? 0 : row_groups<OUT16>(a);
    a.together = together<OUT16>(a);
    hipLaunchKernelGGL((embed_sum_kernel<BF16, OUT16>), dim3((unsigned)((a.slots + a.windows) * a.tiles + groups)), dim3(kRowThreads), 0, stream, a);
    return hipGetLastError();
}

template <bool BF16, bool OUT16>
hipError_t launch_few(EmbedGradArgs a, const int32_t* tok, int n, hipStream_t stream)
{
    a.share = row_threads_log2<BF16>(a.d);
    a.together = together<OUT16>(a);
    int log2 = 0;
    while ((1 << log2) < row_groups<OUT16>(a)) ++log2;
    const dim3 grid((unsigned)std::min(1 << log2, a.V));
    hipLaunchKernelGGL((embed_few_kernel<BF16, OUT16>), grid, dim3(kRowThreads), 0, stream, a, tok, n, log2);
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
    if (n <= kFewTokens) {
        if (dtype == 1) return out_dtype == 1 ? launch_few<true, true>(a, tok, n, stream) : launch_few<true, false>(a, tok, n, stream);
        return out_dtype == 1 ? launch_few<false, true>(a, tok, n, stream) : launch_few<false, false>(a, tok, n, stream);
    }
    const EmbedScratch l = embed_scratch(n, a.V, a.d);
    char* const ws = (char*)workspace;
    int2* const info = reinterpret_cast<int2*>(ws);
    int2* const order = reinterpret_cast<int2*>(ws + l.order_at);
    int32_t* const slot_tok = reinterpret_cast<int32_t*>(ws + l.slot_at);
    a.arrived = reinterpret_cast<uint32_t*>(ws + l.arrived_at);
    a.info = info;
    a.order = order;
    a.slot_tok = slot_tok;
    a.partial = reinterpret_cast<float*>(ws + l.partial_at);
    a.slots = l.slots;
    a.d_pad = l.d_pad;
    const int own_log2 = embed_owners_log2(a.V), owners = 1 << own_log2, range = (a.V + owners - 1) >> own_log2;
    static DeviceFlags done;
    int dev;
    if (hipError_t e = raise_lds_limit_once((const void*)embed_sort_kernel, kSortLds, done, dev)) return e;
    hipLaunchKernelGGL(embed_sort_kernel, dim3((unsigned)std::min(owners, a.V)), dim3(kSortThreads), (size_t)range * (kSortThreads / kWave) * 4, stream,
                       tok, n, a.V, own_log2, range, info, order, slot_tok, a.arrived);
    if (hipError_t e = hipGetLastError()) return e;
    if (dtype == 1) return out_dtype == 1 ? launch_sums<true, true>(a, n, stream) : launch_sums<true, false>(a, n, stream);
    return out_dtype == 1 ? launch_sums<false, true>(a, n, stream) : launch_sums<false, false>(a, n, stream);
}

}  // namespace picospec
