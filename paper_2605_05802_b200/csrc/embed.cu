// Embedding of tokens and the gradient of its table (sr_tokens.h).
//
// Both move rows: the forward call reads the rows that are taken and writes one a token, bound by HBM (65536 tokens of 2048 bf16: 64 us, 5.5 TB/s).
// The gradient adds up, for every row of the table, the rows of the tokens that took it.  Tokens are sorted first, so that a row's terms
// stand together in ascending order and nothing depends on the order of atomics; the sorted tokens are cut into pieces of equal length, each
// summed by one group of threads with the columns spread over them, and runs that cross pieces leave fp32 partial sums, which are added in
// order.  Rows that no token took are zeroed beside the sums, and some of them while the tokens are sorted.  65536 tokens of 2048 bf16 into 151936
// rows: 183 us of 136 (each from cold caches: sorting, with a part of the zeros, 35; sums and the other zeros 138 at 5.8 TB/s; the runs across pieces 18); added to
// a table that stands there, without zeros that hide the sort, 160.  Before: a CTA instead of a warp to a zeroed row, 206; zeros, sorting, sums and
// partial sums one after the other, 262; partial sums loaded one at a time, 38 instead of 14.
#include <cooperative_groups.h>

#include <math.h>

#include <algorithm>

#include "tokens.cuh"

namespace sr {
namespace {

namespace cg = cooperative_groups;

// kCols consecutive elements, as wide as their bytes allow (at most 16 at a time).
template <int kBytes>
struct Words;
template <> struct Words<16> { using Type = uint4; };
template <> struct Words<8> { using Type = uint2; };
template <> struct Words<4> { using Type = uint32_t; };
template <> struct Words<2> { using Type = uint16_t; };
template <typename T, int kCols>
struct Cols {
    static constexpr int kBytes = kCols * (int)sizeof(T), kPart = kBytes < 16 ? kBytes : 16, kParts = kBytes / kPart;
    using Part = typename Words<kPart>::Type;
    Part part[kParts];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) part[i] = reinterpret_cast<const Part*>(p)[i];
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < kParts; ++i) __stcs(reinterpret_cast<Part*>(p) + i, part[i]);
    }
    __device__ __forceinline__ void zero() { memset(part, 0, sizeof(part)); }
    __device__ __forceinline__ float at(int c) const {
        T v[kCols];
        memcpy(v, part, sizeof(part));
        return to_float(v[c]);
    }
    __device__ __forceinline__ void set(const float (&x)[kCols]) {
        T v[kCols];
#pragma unroll
        for (int c = 0; c < kCols; ++c) v[c] = from_float<T>(x[c]);
        memcpy(part, v, sizeof(part));
    }
};

constexpr int kThreads = 256;

// Zeros to a row of `bytes`, by a warp.  kWide: all rows are whole vectors of 16 bytes.  Otherwise they are vectors wherever
// the row begins, and two bytes at a time before and behind.
template <bool kWide>
__device__ __forceinline__ void zero_row(char* row, int bytes, int lane) {
    const int head = kWide ? 0 : min(bytes, (int)(-reinterpret_cast<intptr_t>(row) & 15)), body = kWide ? bytes : (bytes - head) & ~15;
#pragma unroll 4
    for (int c = lane * 16; c < body; c += 512) __stcs(reinterpret_cast<uint4*>(row + head + c), make_uint4(0u, 0u, 0u, 0u));
    if (!kWide)
        for (int c = lane * 2; c < bytes - body; c += 64) *reinterpret_cast<uint16_t*>(row + (c < head ? c : c + body)) = 0;
}

// How threads are spread over rows of `width` elements: `across` of them (a power of two) next to one another.
struct Spread {
    int across, tiles;
};
Spread spread(int width, int cols, int most) {
    const int vecs = (width - 1) / cols + 1;
    int across = 1;
    while (across < most && across < vecs) across *= 2;
    return Spread{across, (vecs - 1) / across + 1};
}

// ------------------------------------------------------------------------------------------------- forward
// A group of `across` threads takes kRows tokens at a time: their ids first, then their rows, so that as many loads are in flight.
template <typename Table, typename Out, int kCols, int kRows>
__global__ void __launch_bounds__(kThreads)
embed_kernel(const __grid_constant__ EmbedArgs a, int across, int tiles) {
    grid_begin();
    const int groups = kThreads / across, tile = blockIdx.x % tiles;
    const int c = (tile * across + (threadIdx.x & (across - 1))) * kCols;
    const int64_t t0 = ((int64_t)(blockIdx.x / tiles) * groups + threadIdx.x / across) * kRows;
    if (c >= a.width) return;
    int id[kRows];
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        id[k] = t0 + k < a.n_tokens ? a.tokens[t0 + k] : -1;
        bad |= id[k] >= a.vocab;
        if (id[k] >= a.vocab) id[k] = -1;
    }
    Cols<Table, kCols> v[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        if (id[k] >= 0) v[k].load(static_cast<const Table*>(a.table) + (int64_t)id[k] * a.table_pitch + c);
        else v[k].zero();
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        if (t0 + k >= a.n_tokens) break;
        float x[kCols];
#pragma unroll
        for (int e = 0; e < kCols; ++e) x[e] = id[k] >= 0 ? a.scale * v[k].at(e) : 0.0f;
        Cols<Out, kCols> o;
        o.set(x);
        o.store(static_cast<Out*>(a.out) + (t0 + k) * a.pitch + c);
    }
    if (bad && c == 0 && a.status) atomicOr(a.status, SR_STATUS_BAD_TARGET);
}

// Rows that do not lie on 16 bytes: a thread makes one aligned vector of the output from the aligned vectors that hold its elements in the
// table, moved against each other by what the two rows differ.  Vectors that reach out of the table go element by element.  65536 tokens of 2047
// bf16: 123 us, with single elements 227.
constexpr int kShiftRows = 4;
template <typename Table, typename Out>
__global__ void __launch_bounds__(kThreads)
embed_shift_kernel(const __grid_constant__ EmbedArgs a, int across, int tiles) {
    constexpr int E = 16 / (int)sizeof(Out);             // elements of an output vector
    constexpr int kParts = E * (int)sizeof(Table) / 16 + 1, kEach = 16 / (int)sizeof(Table);
    grid_begin();
    const int groups = kThreads / across, tile = blockIdx.x % tiles, lane = threadIdx.x & (across - 1);
    const int64_t t0 = ((int64_t)(blockIdx.x / tiles) * groups + threadIdx.x / across) * kShiftRows;
    const Table* const table = static_cast<const Table*>(a.table);
    const uintptr_t begin = reinterpret_cast<uintptr_t>(table), end = begin + ((uintptr_t)(a.vocab - 1) * a.table_pitch + a.width) * sizeof(Table);
    int id[kShiftRows];
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kShiftRows; ++k) {
        id[k] = t0 + k < a.n_tokens ? a.tokens[t0 + k] : -1;
        bad |= id[k] >= a.vocab;
        if (id[k] >= a.vocab) id[k] = -1;
    }
    // where the thread's vector of a row lies: elements before it, and how many of it are the row's
    const auto place = [&](int k, int& c) {
        const int off = (int)(reinterpret_cast<uintptr_t>(static_cast<Out*>(a.out) + (t0 + k) * a.pitch) & 15) / (int)sizeof(Out);
        c = (tile * across + lane) * E - off;
        return t0 + k < a.n_tokens && c < a.width;
    };
    uint4 part[kShiftRows][kParts];
#pragma unroll
    for (int k = 0; k < kShiftRows; ++k) {
        int c;
        const bool real = place(k, c) && id[k] >= 0;
        const uintptr_t from = (begin + ((uintptr_t)(real ? id[k] : 0) * a.table_pitch) * sizeof(Table) + (intptr_t)c * (int)sizeof(Table)) & ~(uintptr_t)15;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            part[k][i] = make_uint4(0u, 0u, 0u, 0u);
            if (real && from + 16 * i >= begin && from + 16 * i + 16 <= end) part[k][i] = *reinterpret_cast<const uint4*>(from + 16 * i);
        }
    }
#pragma unroll
    for (int k = 0; k < kShiftRows; ++k) {
        int c;
        if (!place(k, c)) continue;
        Out* const out = static_cast<Out*>(a.out) + (t0 + k) * a.pitch + c;
        const Table* const row = table + (int64_t)(id[k] >= 0 ? id[k] : 0) * a.table_pitch + c;
        const uintptr_t at = reinterpret_cast<uintptr_t>(row);
        const int shift = (int)(at & 15) / (int)sizeof(Table);
        float x[E];
        if (id[k] >= 0 && ((at & ~(uintptr_t)15) < begin || (at & ~(uintptr_t)15) + 16 * kParts > end)) {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = c + e >= 0 && c + e < a.width ? a.scale * to_float(row[e]) : 0.0f;
        } else {
            uint32_t w[4 * kParts];
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                w[4 * i] = part[k][i].x;
                w[4 * i + 1] = part[k][i].y;
                w[4 * i + 2] = part[k][i].z;
                w[4 * i + 3] = part[k][i].w;
            }
            const int words = shift * (int)sizeof(Table) / 4;
#pragma unroll
            for (int i = 0; i + 2 < 4 * kParts; ++i) w[i] = words & 2 ? w[i + 2] : w[i];
#pragma unroll
            for (int i = 0; i + 1 < 4 * kParts; ++i) w[i] = words & 1 ? w[i + 1] : w[i];
            if (sizeof(Table) == 2) {
#pragma unroll
                for (int i = 0; i + 1 < 4 * kParts; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (shift & 1) * 16);
            }
#pragma unroll
            for (int i = 0; i < E / kEach; ++i) {
                float y[kEach];
                unpack(make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]), y, Table());
#pragma unroll
                for (int e = 0; e < kEach; ++e) x[i * kEach + e] = id[k] >= 0 ? a.scale * y[e] : 0.0f;
            }
        }
        if (c >= 0 && c + E <= a.width) {
            store_once(reinterpret_cast<uint4*>(out), pack(x, Out()));
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (c + e >= 0 && c + e < a.width) out[e] = from_float<Out>(x[e]);
        }
    }
    if (bad && tile == 0 && lane == 0 && a.status) atomicOr(a.status, SR_STATUS_BAD_TARGET);
}

// ------------------------------------------------------------------------------------------------- sorting
// A stable radix sort of (token, position) by one cluster of 16 CTAs (8, with tokens and positions apart: 47 us for 65536 instead of 28): digits of up to 10 bits, two passes for vocabularies of up to a million.
// A warp has consecutive tokens and counts them in a histogram of its own, so that ranks follow the order of the tokens;
// the CTAs' histograms meet in global memory, with the cluster's barrier (release, acquire) around them.
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMostBits = 10;
constexpr int kSortCtas = 16;      // more than every GPU has to run together, but not more than a B200 does

struct SortScratch {
    int2* sorted[2];        // (token, position)
    uint32_t* count;        // [kSortCtas][1 << kMostBits]
};

// What other CTAs of the cluster have written, from L2; not moved over a barrier.
__device__ __forceinline__ int32_t load_l2(const void* p) {
    int32_t v;
    asm volatile("ld.global.cg.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ int2 load_l2(const int2* p) {
    int2 v;
    asm volatile("ld.global.cg.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t below(uint32_t peers) { return __popc(peers & ((1u << (threadIdx.x & 31)) - 1u)); }

// Rows of the table that are zeroed while the tokens are sorted: the first `rows`.
struct ZeroRows {
    char* table;
    int64_t pitch;                  // bytes
    int width, rows;
    bool wide;
};
constexpr int kZeroCtas = 112;      // with those that sort eight clusters: what the GPU's eight parts run at once

// The CTA's share, without those that a token took; bits of them in shared memory.
__device__ __forceinline__ void zero_share(const ZeroRows& z, const int32_t* tokens, int n, int share, uint32_t* taken, int most) {
    const int each = (z.rows - 1) / kZeroCtas + 1;
    for (int64_t begin = (int64_t)share * each; begin < min((int64_t)z.rows, (int64_t)(share + 1) * each); begin += most) {
        const int rows = (int)min(min((int64_t)z.rows, (int64_t)(share + 1) * each) - begin, (int64_t)most);
        __syncthreads();
        for (int i = threadIdx.x; i < (rows + 31) / 32; i += blockDim.x) taken[i] = 0u;
        __syncthreads();
        for (int64_t i0 = threadIdx.x; i0 < n; i0 += 8 * (int64_t)blockDim.x) {
            int32_t t[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) t[u] = i0 + u * (int64_t)blockDim.x < n ? tokens[i0 + u * (int64_t)blockDim.x] : -1;
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (t[u] >= begin && t[u] < begin + rows) atomicOr(&taken[(t[u] - (int)begin) >> 5], 1u << ((t[u] - (int)begin) & 31));
        }
        __syncthreads();
        for (int r = threadIdx.x >> 5; r < rows; r += blockDim.x >> 5) {
            if ((taken[r >> 5] >> (r & 31)) & 1u) continue;
            char* const row = z.table + (begin + r) * z.pitch;
            if (z.wide) zero_row<true>(row, z.width, threadIdx.x & 31);
            else zero_row<false>(row, z.width, threadIdx.x & 31);
        }
    }
}

constexpr int kHeld = 8;            // tokens a lane loads at a time; as many are held from counting to placing
__global__ void __launch_bounds__(kSortThreads)
sort_tokens_kernel(const int32_t* tokens, int n, int vocab, int passes, int bits, SortScratch ws, ZeroRows zero, int32_t* status) {
    extern __shared__ __align__(16) uint32_t s_hist[];  // [kSortWarps][bins]
    __shared__ uint32_t s_base[1 << kMostBits], s_warp[kSortWarps];
    grid_begin();
    if (blockIdx.x >= kSortCtas) {                       // other clusters
        zero_share(zero, tokens, n, blockIdx.x - kSortCtas, s_hist, kSortWarps << bits);
        return;
    }
    const int ctas = kSortCtas, cta = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bins = 1 << bits;
    const int64_t a_warp = (((int64_t)n - 1) / (ctas * kSortThreads) + 1) * 32;       // tokens, a multiple of 32
    const int64_t begin = ((int64_t)cta * kSortWarps + warp) * a_warp, end = min((int64_t)n, begin + a_warp);
    uint32_t* const hist = s_hist + warp * bins;
    bool bad = false;
    for (int p = 0; p < passes; ++p) {
        const int2* const from = ws.sorted[(p - 1) & 1];
        int2* const to = ws.sorted[p & 1];
        const int shift = p * bits;
        int32_t k[kHeld], at[kHeld];
        const auto load = [&](int64_t i0) {
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                const int64_t i = i0 + u * 32 + lane;
                k[u] = 0;
                at[u] = (int32_t)i;
                if (i < end && p == 0) {
                    k[u] = load_l2(tokens + i);
                } else if (i < end) {
                    const int2 v = load_l2(from + i);
                    k[u] = v.x;
                    at[u] = v.y;
                }
            }
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                bad |= k[u] > vocab || (p == 0 && k[u] == vocab);
                if (k[u] < 0 || k[u] > vocab) k[u] = vocab;          // what is no token comes last
            }
        };
        const auto digit = [&](int64_t i, int32_t of) { return i < end ? (of >> shift) & (bins - 1) : bins; };
        for (int i = threadIdx.x; i < kSortWarps * bins / 4; i += kSortThreads) reinterpret_cast<uint4*>(s_hist)[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        for (int64_t i0 = begin; i0 < end; i0 += kHeld * 32) {
            load(i0);
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                if (i0 + u * 32 >= end) break;
                const int d = digit(i0 + u * 32 + lane, k[u]);
                const uint32_t peers = __match_any_sync(0xFFFFFFFFu, d);
                if (d < bins && below(peers) == 0) hist[d] += __popc(peers);
                __syncwarp();
            }
        }
        __syncthreads();
        const int b = threadIdx.x;
        if (b < bins) {
            uint32_t sum = 0;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = s_hist[w * bins + b];
                s_hist[w * bins + b] = sum;
                sum += c;
            }
            ws.count[(cta << kMostBits) + b] = sum;
        }
        cg::this_cluster().sync();
        uint32_t total = 0, before = 0;
        if (b < bins) {
            uint32_t v[kSortCtas];
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) v[c] = (uint32_t)load_l2(ws.count + (c << kMostBits) + b);
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) {
                before += c < cta ? v[c] : 0u;
                total += v[c];
            }
        }
        uint32_t scan = total;                           // of the bins before this one
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, scan, o);
            if (lane >= o) scan += v;
        }
        if (lane == 31) s_warp[warp] = scan;
        __syncthreads();
        for (int w = 0; w < warp; ++w) before += s_warp[w];
        if (b < bins) s_base[b] = before + scan - total;
        __syncthreads();
        for (int64_t i0 = begin; i0 < end; i0 += kHeld * 32) {
            if (a_warp > kHeld * 32) load(i0);
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                if (i0 + u * 32 >= end) break;
                const int d = digit(i0 + u * 32 + lane, k[u]);
                const uint32_t peers = __match_any_sync(0xFFFFFFFFu, d);
                uint32_t place = 0;
                if (d < bins) place = s_base[d] + hist[d] + below(peers);
                __syncwarp();
                if (d < bins) {
                    if (below(peers) == 0) hist[d] += __popc(peers);
                    to[place] = make_int2(k[u], at[u]);
                }
                __syncwarp();
            }
        }
        cg::this_cluster().sync();
    }
    if (bad && status) atomicOr(status, SR_STATUS_BAD_TARGET);
}

// Few tokens (4096 or fewer: 1200 in 6 us, sorted by one CTA 14): the place of each is the number of those that belong before it.  A CTA has 32 tokens and all keys in shared memory; eight threads
// share the keys of a token.  Gradients of 256 columns fp32 into 4096 rows, ranked and sorted: 2048 tokens 13 and 18 us, 4096 18 and 20, 6144 27 and 21; of 2048 bf16
// into 151936 rows, whose zeros hide the sort, 111 and 113, 123 and 113, 126 and 114.
constexpr int kFewTokens = 4096, kRanked = 32;
__global__ void __launch_bounds__(kThreads)
rank_tokens_kernel(const int32_t* tokens, int n, int vocab, int2* sorted, int32_t* status) {
    extern __shared__ __align__(16) int32_t s_key[];    // [n up to a multiple of 32]
    __shared__ int s_rank[kRanked];
    grid_begin();
    const int padded = (n + 31) & ~31;
    bool bad = false;
    for (int i0 = threadIdx.x; i0 < padded; i0 += 8 * kThreads) {
        int32_t k[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) k[u] = i0 + u * kThreads < n ? tokens[i0 + u * kThreads] : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (i0 + u * kThreads >= padded) break;
            bad |= k[u] >= vocab;
            s_key[i0 + u * kThreads] = k[u] < 0 || k[u] > vocab ? vocab : k[u];
        }
    }
    if (threadIdx.x < kRanked) s_rank[threadIdx.x] = 0;
    __syncthreads();
    constexpr int kParts = kThreads / kRanked;
    const int t = threadIdx.x % kRanked, i = blockIdx.x * kRanked + t, part = threadIdx.x / kRanked;
    if (i < n) {
        // keys before the token count when they are not larger, those behind it when they are smaller
        const int mine = s_key[i], lo = padded / kParts * part, hi = lo + padded / kParts;
        const int middle = max(lo, min(hi, i & ~3));
        int rank = 0;
        const auto count = [&](int from, int to, auto before) {
#pragma unroll 4
            for (int j = from; j < to; j += 4) {
                const int4 k = *reinterpret_cast<const int4*>(s_key + j);
                rank += before(k.x) + before(k.y) + before(k.z) + before(k.w);
            }
        };
        const auto not_larger = [&](int k) { return (int)(k <= mine); };
        const auto smaller = [&](int k) { return (int)(k < mine); };
        count(lo, middle, not_larger);
        if (middle < hi && middle == (i & ~3)) {
            for (int j = middle; j < middle + 4; ++j) rank += j < i ? not_larger(s_key[j]) : smaller(s_key[j]);
            count(middle + 4, hi, smaller);
        } else {
            count(middle, hi, smaller);
        }
        atomicAdd(&s_rank[t], rank);
    }
    __syncthreads();
    if (i < n && part == 0) {
        sorted[s_rank[t]] = make_int2(s_key[i], i);
    }
    if (bad && status && blockIdx.x == 0) atomicOr(status, SR_STATUS_BAD_TARGET);
}

// ------------------------------------------------------------------------------------------------- sums
// Pieces of the sorted tokens, the same number of tokens each (a multiple of 8).
struct Pieces {
    int length, n;
};
constexpr int kBatch = 8;
Pieces pieces_of(int n_tokens, int width) {
    // A wave of the GPU (148 x 8 groups of 2048 columns), or more where that leaves a frequent token's run in too many pieces: a piece is
    // summed a batch after the other, and so are the pieces of a run that is a tenth of all tokens (131072 of 64 columns 102 -> 65 us).
    const int64_t even = (int64_t)n_tokens * width / (2048 * 1184);
    const int64_t by_run = n_tokens > 16384 ? (int64_t)(sqrt((double)n_tokens) / 4) : n_tokens > 2048 ? 2 * kBatch : kBatch;
    const int length = (int)std::min<int64_t>((std::max(even, by_run) + kBatch - 1) / kBatch * kBatch, 512);
    return Pieces{length, n_tokens > 0 ? (n_tokens - 1) / length + 1 : 0};
}

struct SumArgs {
    EmbedGradArgs g;
    const int2* sorted;              // (token, position)
    float* partial;                  // [pieces][2][width]: of the run that came from the piece before, and of the one that goes on
    Pieces pieces;
};

template <typename Table, int kCols>
__device__ __forceinline__ void write_row(const EmbedGradArgs& g, int token, int c, const float (&sum)[kCols]) {
    Table* to = static_cast<Table*>(g.d_table) + (int64_t)token * g.table_pitch + c;
    float x[kCols];
    if (g.accumulate) {
        Cols<Table, kCols> had;
        had.load(to);
#pragma unroll
        for (int e = 0; e < kCols; ++e) x[e] = fmaf(g.scale, sum[e], had.at(e));
    } else {
#pragma unroll
        for (int e = 0; e < kCols; ++e) x[e] = g.scale * sum[e];
    }
    Cols<Table, kCols> o;
    o.set(x);
    o.store(to);
}

// Writes zeros to the rows [begin, end) that no token took.
constexpr int kMostZeroRows = 1024;
template <typename Table, bool kWide>
__device__ __forceinline__ void zero_rows(const SumArgs& a, int begin, int end) {
    __shared__ uint32_t s_taken[kMostZeroRows / 32];
    __shared__ int s_from;
    const EmbedGradArgs& g = a.g;
    if (threadIdx.x < kMostZeroRows / 32) s_taken[threadIdx.x] = 0u;
    if (threadIdx.x < 32) {                              // the first sorted token of these rows: 32 probes at a time
        int lo = 0, hi = g.n_tokens;                     // all before lo are smaller, none from hi on is
        while (lo < hi) {
            const int step = (hi - lo - 1) / 32 + 1, at = (int)min((int64_t)hi - 1, (int64_t)lo + (int64_t)step * (threadIdx.x + 1) - 1);
            const int smaller = __popc(__ballot_sync(0xFFFFFFFFu, a.sorted[at].x < begin));
            const int64_t from = (int64_t)lo + (int64_t)step * smaller;
            hi = (int)min((int64_t)hi, from + step - 1);
            lo = (int)min((int64_t)hi, from);
            if (smaller == 32) lo = hi;
        }
        if (threadIdx.x == 0) s_from = lo;
    }
    __syncthreads();
    for (int64_t i = s_from + (int64_t)threadIdx.x; i < g.n_tokens; i += kThreads) {
        const int token = a.sorted[i].x;
        if (token >= end) break;
        atomicOr(&s_taken[(token - begin) >> 5], 1u << ((token - begin) & 31));
    }
    __syncthreads();
    for (int r = threadIdx.x >> 5; r < end - begin; r += kThreads / 32)       // a warp to a row
        if (!((s_taken[r >> 5] >> (r & 31)) & 1u))
            zero_row<kWide>(reinterpret_cast<char*>(static_cast<Table*>(g.d_table) + (int64_t)(begin + r) * g.table_pitch), g.width * (int)sizeof(Table), threadIdx.x & 31);
}

// The first `sum_ctas` CTAs sum pieces, the others write zeros, `zero_rows_each` rows each from row `zero_first` on.
template <typename Grad, typename Table, int kCols>
__global__ void __launch_bounds__(kThreads)
embed_sums_kernel(const __grid_constant__ SumArgs a, int across, int tiles, int sum_ctas, int zero_first, int zero_rows_each) {
    grid_begin();
    const EmbedGradArgs& g = a.g;
    if ((int)blockIdx.x >= sum_ctas) {
        const int64_t begin = zero_first + (int64_t)((int)blockIdx.x - sum_ctas) * zero_rows_each;
        zero_rows<Table, kCols * sizeof(Table) >= 16>(a, (int)begin, (int)min((int64_t)g.vocab, begin + zero_rows_each));
        return;
    }
    const int tile = blockIdx.x % tiles, piece = (blockIdx.x / tiles) * (kThreads / across) + threadIdx.x / across;
    const int c = (tile * across + (threadIdx.x & (across - 1))) * kCols;
    if (piece >= a.pieces.n || c >= g.width) return;
    const int64_t begin = (int64_t)piece * a.pieces.length, end = min((int64_t)g.n_tokens, begin + a.pieces.length);
    const Grad* const d = static_cast<const Grad*>(g.d_out) + c;
    bool came = begin > 0 && a.sorted[begin - 1].x == a.sorted[begin].x;
    float sum[kCols];
#pragma unroll
    for (int e = 0; e < kCols; ++e) sum[e] = 0.0f;
    int token[kBatch + 1], pos[kBatch];                  // of a batch; pieces begin on multiples of it
    const auto load_ids = [&](int64_t i0) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int2 one = i0 + k < end ? a.sorted[i0 + k] : make_int2(g.vocab, 0);
            token[k] = one.x;
            pos[k] = one.y;
        }
        token[kBatch] = i0 + kBatch < g.n_tokens ? a.sorted[i0 + kBatch].x : g.vocab;
    };
    load_ids(begin);
    for (int64_t i0 = begin; i0 < end; i0 += kBatch) {
        Cols<Grad, kCols> v[kBatch];
        int here[kBatch + 1];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (token[k] < g.vocab) v[k].load(d + (int64_t)pos[k] * g.pitch);
            here[k] = token[k];
        }
        here[kBatch] = token[kBatch];
        if (end - i0 < kBatch) {                         // the last one: the token behind it
            const int behind = end < g.n_tokens ? a.sorted[end].x : g.vocab;
#pragma unroll
            for (int k = 1; k <= kBatch; ++k)
                if (i0 + k >= end) here[k] = behind;
        }
        if (i0 + kBatch < end) load_ids(i0 + kBatch);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (i0 + k >= end || here[k] >= g.vocab) return;         // nothing but what is no token from here on
#pragma unroll
            for (int e = 0; e < kCols; ++e) sum[e] += v[k].at(e);
            const bool last = i0 + k + 1 == end, ends = here[k + 1] != here[k];
            if (!last && !ends) continue;
            if (ends && !came) {
                write_row<Table, kCols>(g, here[k], c, sum);
            } else {
                Cols<float, kCols> part;
                part.set(sum);
                part.store(a.partial + ((int64_t)piece * 2 + (came ? 0 : 1)) * g.width + c);
            }
            came = false;
#pragma unroll
            for (int e = 0; e < kCols; ++e) sum[e] = 0.0f;
        }
    }
}

// Runs that go on behind their first piece.
template <typename Table, int kCols>
__global__ void __launch_bounds__(kThreads)
embed_join_kernel(const __grid_constant__ SumArgs a, int across, int tiles) {
    grid_begin();
    const EmbedGradArgs& g = a.g;
    const int tile = blockIdx.x % tiles, piece = (blockIdx.x / tiles) * (kThreads / across) + threadIdx.x / across;
    const int c = (tile * across + (threadIdx.x & (across - 1))) * kCols;
    if (piece + 1 >= a.pieces.n || c >= g.width) return;
    const int64_t begin = (int64_t)piece * a.pieces.length, end = begin + a.pieces.length;       // not the last piece: it is whole
    const int token = a.sorted[end - 1].x;
    if (token >= g.vocab || a.sorted[end].x != token) return;
    if (a.sorted[begin].x == token && begin > 0 && a.sorted[begin - 1].x == token) return;                // began further ahead
    float sum[kCols];
    Cols<float, kCols> first;
    first.load(a.partial + ((int64_t)piece * 2 + 1) * g.width + c);
#pragma unroll
    for (int e = 0; e < kCols; ++e) sum[e] = first.at(e);
    // how many of the pieces from `next` on, up to a batch, begin with the run's token
    const auto count = [&](int next) {
        int n = 0;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) n += next + k < a.pieces.n && a.sorted[(int64_t)(next + k) * a.pieces.length].x == token;
        return n;
    };
    int next = piece + 1, n = count(next);
    while (n > 0) {
        Cols<float, kCols> part[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            part[k].zero();
            if (k < n) part[k].load(a.partial + (int64_t)(next + k) * 2 * g.width + c);
        }
        next += kBatch;
        const int more = n == kBatch ? count(next) : 0;
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
#pragma unroll
            for (int e = 0; e < kCols; ++e) sum[e] += part[k].at(e);
        n = more;
    }
    write_row<Table, kCols>(g, token, c, sum);
}

// ------------------------------------------------------------------------------------------------- launches
// The most elements, a power of two up to `most`, that lie together in both buffers: all rows begin on their vectors and are made of whole ones.
int cols_of(int most, const void* p, int64_t pitch, int size_p, const void* q, int64_t q_pitch, int size_q, int width) {
    const auto fits = [](const void* x, int64_t row, int size, int cols) {
        const int bytes = std::min(16, cols * size);
        return (reinterpret_cast<uintptr_t>(x) % bytes) == 0 && (row * size) % bytes == 0;
    };
    int cols = most;
    while (cols > 1 && (width % cols || !fits(p, pitch, size_p, cols) || !fits(q, q_pitch, size_q, cols))) cols /= 2;
    return cols;
}

template <typename Table, typename Out, int kCols>
int embed_with(const EmbedArgs& a, cudaStream_t s) {
    const Spread sp = spread(a.width, kCols, kThreads);
    const auto ctas = [&](int rows) { return (((int64_t)a.n_tokens - 1) / (kThreads / sp.across * rows) + 1) * sp.tiles; };
    // as many rows to a thread as leave the GPU a wave of CTAs
    if (ctas(8) >= 148 * 6) {
        if (ctas(8) > INT32_MAX) return SR_ERR_BAD_SIZE;
        SR_LAUNCH("embed_kernel", (embed_kernel<Table, Out, kCols, 8>), (int)ctas(8), kThreads, 0, s, a, sp.across, sp.tiles);
    } else if (ctas(2) >= 148 * 6) {
        SR_LAUNCH("embed_kernel", (embed_kernel<Table, Out, kCols, 2>), (int)ctas(2), kThreads, 0, s, a, sp.across, sp.tiles);
    } else {
        SR_LAUNCH("embed_kernel", (embed_kernel<Table, Out, kCols, 1>), (int)ctas(1), kThreads, 0, s, a, sp.across, sp.tiles);
    }
    return SR_OK;
}
template <typename Table, typename Out>
int embed_types(const EmbedArgs& a, cudaStream_t s) {
    constexpr int kMost = 16 / (int)(sizeof(Table) > sizeof(Out) ? sizeof(Table) : sizeof(Out));
    const int cols = cols_of(kMost, a.table, a.table_pitch, sizeof(Table), a.out, a.pitch, sizeof(Out), a.width);
    if (cols == 1 && a.width >= 64) {
        const Spread sp = spread(a.width + 16 / (int)sizeof(Out) - 1, 16 / (int)sizeof(Out), 32);        // one vector more where a row begins inside its first
        const int64_t ctas = (((int64_t)a.n_tokens - 1) / (kThreads / sp.across * kShiftRows) + 1) * sp.tiles;
        if (ctas > INT32_MAX) return SR_ERR_BAD_SIZE;
        SR_LAUNCH("embed_shift_kernel", (embed_shift_kernel<Table, Out>), (int)ctas, kThreads, 0, s, a, sp.across, sp.tiles);
        return SR_OK;
    }
    switch (cols) {
        case 8: if constexpr (kMost == 8) return embed_with<Table, Out, 8>(a, s); else break;
        case 4: return embed_with<Table, Out, 4>(a, s);
        case 2: return embed_with<Table, Out, 2>(a, s);
        default: break;
    }
    return embed_with<Table, Out, 1>(a, s);
}

struct GradScratch {
    SortScratch sort;
    float* partial;
    size_t bytes;
};
GradScratch grad_scratch(void* ws, int n_tokens, int width) {
    char* const base = static_cast<char*>(ws);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        char* const p = base + at;
        at += align_up(bytes, 256);
        return p;
    };
    GradScratch g;
    for (int k = 0; k < 2; ++k) g.sort.sorted[k] = reinterpret_cast<int2*>(take((size_t)n_tokens * sizeof(int2)));
    g.sort.count = reinterpret_cast<uint32_t*>(take((size_t)kSortCtas * (sizeof(uint32_t) << kMostBits)));
    g.partial = reinterpret_cast<float*>(take((size_t)pieces_of(n_tokens, width).n * 2 * width * sizeof(float)));
    g.bytes = at;
    return g;
}

template <typename Grad, typename Table, int kCols>
int embed_grad_with(const SumArgs& a, int zeroed, cudaStream_t s) {
    const Spread sp = spread(a.g.width, kCols, kThreads);
    const int64_t sum_ctas = a.pieces.n > 0 ? (((int64_t)a.pieces.n - 1) / (kThreads / sp.across) + 1) * sp.tiles : 0;       // below n_tokens * width / 256
    int zero_each = 0, zero_ctas = 0;
    if (!a.g.accumulate && zeroed < a.g.vocab) {         // the rows from `zeroed` on
        zero_each = std::min((a.g.vocab - zeroed - 1) / (148 * 8) + 1, kMostZeroRows);
        zero_ctas = (a.g.vocab - zeroed - 1) / zero_each + 1;
    }
    if (sum_ctas + zero_ctas == 0) return SR_OK;
    SR_LAUNCH("embed_sums_kernel", (embed_sums_kernel<Grad, Table, kCols>), (int)(sum_ctas + zero_ctas), kThreads, 0, s, a, sp.across, sp.tiles, (int)sum_ctas, zeroed, zero_each);
    if (a.pieces.n > 1) SR_LAUNCH("embed_join_kernel", (embed_join_kernel<Table, kCols>), (int)sum_ctas, kThreads, 0, s, a, sp.across, sp.tiles);
    return SR_OK;
}

template <typename Grad, typename Table>
int embed_grad_types(const EmbedGradArgs& g, void* ws, cudaStream_t s) {
    constexpr int kMost = 16 / (int)(sizeof(Table) > sizeof(Grad) ? sizeof(Table) : sizeof(Grad));
    const GradScratch scratch = grad_scratch(ws, g.n_tokens, g.width);
    int sorted = 0, zeroed = 0;                                          // which of the two buffers; rows of the table that are zeroed by then
    const int cols = cols_of(kMost, g.d_out, g.pitch, sizeof(Grad), g.d_table, g.table_pitch, sizeof(Table), g.width);
    if (g.n_tokens > kFewTokens) {
        int key_bits = 1;
        while ((g.vocab >> key_bits) != 0) ++key_bits;                   // `vocab` itself stands for what is no token
        const int passes = (key_bits - 1) / kMostBits + 1, bits = (key_bits - 1) / passes + 1;
        const size_t smem = (size_t)kSortWarps * sizeof(uint32_t) << bits;
        SR_CUDA_TRY(cudaFuncSetAttribute(sort_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)((size_t)kSortWarps * sizeof(uint32_t) << kMostBits)));
        SR_CUDA_TRY(cudaFuncSetAttribute(sort_tokens_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        ZeroRows zero = {static_cast<char*>(g.d_table), g.table_pitch * (int64_t)sizeof(Table), g.width * (int)sizeof(Table), 0, cols * sizeof(Table) >= 16};
        if (!g.accumulate) {                                             // what takes as long as sorting, less the time to look through the tokens; 4 MB a us
            const double bytes = (9.0 + g.n_tokens / 6000.0) * 4e6;
            zeroed = zero.rows = (int)std::min<double>(g.vocab, bytes / zero.width);
        }
        const int ctas = kSortCtas + (zeroed > 0 ? kZeroCtas : 0);
        const int rc = launch_as(true, kSortCtas, "sort_tokens_kernel", sort_tokens_kernel, ctas, kSortThreads, smem, s, g.tokens, g.n_tokens, g.vocab, passes, bits, scratch.sort, zero,
                                 g.status);
        if (rc != SR_OK) return rc;
        sorted = (passes - 1) & 1;
    } else if (g.n_tokens > 0) {
        SR_LAUNCH("rank_tokens_kernel", rank_tokens_kernel, (g.n_tokens - 1) / kRanked + 1, kThreads, (size_t)((g.n_tokens + 31) & ~31) * sizeof(int32_t), s, g.tokens, g.n_tokens, g.vocab,
                  scratch.sort.sorted[0], g.status);
    }
    const SumArgs a{g, scratch.sort.sorted[sorted], scratch.partial, pieces_of(g.n_tokens, g.width)};
    switch (cols) {
        case 8: if constexpr (kMost == 8) return embed_grad_with<Grad, Table, 8>(a, zeroed, s); else break;
        case 4: return embed_grad_with<Grad, Table, 4>(a, zeroed, s);
        case 2: return embed_grad_with<Grad, Table, 2>(a, zeroed, s);
        default: break;
    }
    return embed_grad_with<Grad, Table, 1>(a, zeroed, s);
}

}  // namespace

int launch_embed(const EmbedArgs& a, cudaStream_t s) {
    if (a.n_tokens == 0) return SR_OK;
    if (a.dtype == SR_DTYPE_F32) return embed_types<float, float>(a, s);
    if (a.dtype == SR_DTYPE_BF16) return a.table_dtype == SR_DTYPE_F32 ? embed_types<float, __nv_bfloat16>(a, s) : embed_types<__nv_bfloat16, __nv_bfloat16>(a, s);
    return a.table_dtype == SR_DTYPE_F32 ? embed_types<float, __half>(a, s) : embed_types<__half, __half>(a, s);
}

size_t embed_grad_workspace_bytes(int32_t n_tokens, int32_t vocab, int32_t width) {
    (void)vocab;
    return grad_scratch(nullptr, n_tokens, width).bytes;
}

int launch_embed_grad(const EmbedGradArgs& g, void* ws, cudaStream_t s) {
    if (g.dtype == SR_DTYPE_F32) return embed_grad_types<float, float>(g, ws, s);
    if (g.dtype == SR_DTYPE_BF16) return g.table_dtype == SR_DTYPE_F32 ? embed_grad_types<__nv_bfloat16, float>(g, ws, s) : embed_grad_types<__nv_bfloat16, __nv_bfloat16>(g, ws, s);
    return g.table_dtype == SR_DTYPE_F32 ? embed_grad_types<__half, float>(g, ws, s) : embed_grad_types<__half, __half>(g, ws, s);
}

}  // namespace sr
