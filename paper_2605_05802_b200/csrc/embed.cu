// Embedding of tokens and the gradient of its table (sr_tokens.h).
//
// Both move rows: the forward call reads the rows that are taken and writes one a token, bound by HBM.  The gradient adds up, for
// every row of the table, the rows of the tokens that took it.  Tokens are sorted first, so that a row's terms stand together in
// ascending order and nothing depends on the order of atomics; the sorted tokens are cut into pieces of equal length, each
// summed by one group of threads with the columns spread over them, and runs that cross pieces leave fp32 partial sums, which are added in order.
#include <cooperative_groups.h>

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

// ------------------------------------------------------------------------------------------------- sorting
// A stable radix sort of (token, position) by one cluster: digits of up to 10 bits, two passes for vocabularies of up to a million.
// A warp has consecutive tokens and counts them in a histogram of its own, so that ranks follow the order of the tokens;
// the CTAs' histograms meet in global memory, with the cluster's barrier (release, acquire) around them.
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMostBits = 10;
constexpr int kSortCtas = 8;

struct SortScratch {
    int32_t* key[2];
    int32_t* pos[2];
    uint32_t* count;        // [kSortCtas][1 << kMostBits]
};

// What other CTAs of the cluster have written, from L2; not moved over a barrier.
__device__ __forceinline__ int32_t load_l2(const void* p) {
    int32_t v;
    asm volatile("ld.global.cg.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t below(uint32_t peers) { return __popc(peers & ((1u << (threadIdx.x & 31)) - 1u)); }

__global__ void __launch_bounds__(kSortThreads)
sort_tokens_kernel(const int32_t* tokens, int n, int vocab, int passes, int bits, SortScratch ws, int32_t* status) {
    extern __shared__ uint32_t s_hist[];                // [kSortWarps][bins]
    __shared__ uint32_t s_base[1 << kMostBits], s_warp[kSortWarps];
    grid_begin();
    const int ctas = gridDim.x, cta = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bins = 1 << bits;
    const int64_t a_warp = (((int64_t)n - 1) / (ctas * kSortThreads) + 1) * 32;       // tokens, a multiple of 32
    const int64_t begin = ((int64_t)cta * kSortWarps + warp) * a_warp, end = min((int64_t)n, begin + a_warp);
    uint32_t* const hist = s_hist + warp * bins;
    bool bad = false;
    for (int p = 0; p < passes; ++p) {
        const int32_t *key = p ? ws.key[(p - 1) & 1] : tokens, *pos = p ? ws.pos[(p - 1) & 1] : nullptr;
        const int shift = p * bits;
        const auto key_at = [&](int64_t i) {
            const int32_t k = load_l2(key + i);
            bad |= k > vocab || (p == 0 && k == vocab);
            return k < 0 || k > vocab ? vocab : k;                   // what is no token comes last
        };
        for (int i = threadIdx.x; i < kSortWarps * bins; i += kSortThreads) s_hist[i] = 0u;
        __syncthreads();
        for (int64_t i0 = begin; i0 < end; i0 += 32) {
            const int64_t i = i0 + lane;
            const bool real = i < end;
            const int32_t k = real ? key_at(i) : 0;
            const int d = real ? (k >> shift) & (bins - 1) : bins;
            const uint32_t peers = __match_any_sync(0xFFFFFFFFu, d);
            if (real && below(peers) == 0) hist[d] += __popc(peers);
            __syncwarp();
        }
        __syncthreads();
        const int b = threadIdx.x;
        if (b < bins) {
            uint32_t sum = 0;
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = s_hist[w * bins + b];
                s_hist[w * bins + b] = sum;
                sum += c;
            }
            ws.count[(cta << kMostBits) + b] = sum;
        }
        cg::this_cluster().sync();
        uint32_t total = 0, before = 0;
        if (b < bins)
            for (int c = 0; c < ctas; ++c) {
                const uint32_t v = (uint32_t)load_l2(ws.count + (c << kMostBits) + b);
                before += c < cta ? v : 0u;
                total += v;
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
        for (int64_t i0 = begin; i0 < end; i0 += 32) {
            const int64_t i = i0 + lane;
            const bool real = i < end;
            const int32_t k = real ? key_at(i) : 0;
            const int32_t at = real ? (p ? load_l2(pos + i) : (int32_t)i) : 0;
            const int d = real ? (k >> shift) & (bins - 1) : bins;
            const uint32_t peers = __match_any_sync(0xFFFFFFFFu, d);
            uint32_t to = 0;
            if (real) to = s_base[d] + hist[d] + below(peers);
            __syncwarp();
            if (real) {
                if (below(peers) == 0) hist[d] += __popc(peers);
                ws.key[p & 1][to] = k;
                ws.pos[p & 1][to] = at;
            }
            __syncwarp();
        }
        cg::this_cluster().sync();
    }
    if (bad && status) atomicOr(status, SR_STATUS_BAD_TARGET);
}

// ------------------------------------------------------------------------------------------------- sums
// Pieces of the sorted tokens, the same number of tokens each (a multiple of 8).
struct Pieces {
    int length, n;
};
constexpr int kBatch = 8;
Pieces pieces_of(int n_tokens, int width) {
    // a wave of the GPU (148 x 8 groups of 2048 columns), not shorter than 8 tokens and not longer than 512
    const int64_t even = (int64_t)n_tokens * width / (2048 * 1184);
    const int length = (int)std::min<int64_t>(std::max<int64_t>((even + kBatch - 1) / kBatch * kBatch, kBatch), 512);
    return Pieces{length, n_tokens > 0 ? (n_tokens - 1) / length + 1 : 0};
}

struct SumArgs {
    EmbedGradArgs g;
    const int32_t *key, *pos;        // sorted
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

template <typename Grad, typename Table, int kCols>
__global__ void __launch_bounds__(kThreads)
embed_sums_kernel(const __grid_constant__ SumArgs a, int across, int tiles) {
    grid_begin();
    const EmbedGradArgs& g = a.g;
    const int tile = blockIdx.x % tiles, piece = (blockIdx.x / tiles) * (kThreads / across) + threadIdx.x / across;
    const int c = (tile * across + (threadIdx.x & (across - 1))) * kCols;
    if (piece >= a.pieces.n || c >= g.width) return;
    const int64_t begin = (int64_t)piece * a.pieces.length, end = min((int64_t)g.n_tokens, begin + a.pieces.length);
    const Grad* const d = static_cast<const Grad*>(g.d_out) + c;
    bool came = begin > 0 && a.key[begin - 1] == a.key[begin];
    float sum[kCols];
#pragma unroll
    for (int e = 0; e < kCols; ++e) sum[e] = 0.0f;
    for (int64_t i0 = begin; i0 < end; i0 += kBatch) {
        int token[kBatch + 1];
#pragma unroll
        for (int k = 0; k <= kBatch; ++k) token[k] = i0 + k < g.n_tokens ? a.key[i0 + k] : g.vocab;
        Cols<Grad, kCols> v[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (token[k] < g.vocab) v[k].load(d + (int64_t)a.pos[i0 + k] * g.pitch);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (token[k] >= g.vocab) return;             // nothing but what is no token from here on
#pragma unroll
            for (int e = 0; e < kCols; ++e) sum[e] += v[k].at(e);
            const bool last = i0 + k + 1 == end, ends = token[k + 1] != token[k];
            if (!last && !ends) continue;
            if (ends && !came) {
                write_row<Table, kCols>(g, token[k], c, sum);
            } else {
                float* const to = a.partial + ((int64_t)piece * 2 + (came ? 0 : 1)) * g.width + c;
#pragma unroll
                for (int e = 0; e < kCols; ++e) to[e] = sum[e];
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
    const int token = a.key[end - 1];
    if (token >= g.vocab || a.key[end] != token) return;
    if (a.key[begin] == token && begin > 0 && a.key[begin - 1] == token) return;                // began further ahead
    float sum[kCols];
    const float* from = a.partial + ((int64_t)piece * 2 + 1) * g.width + c;
#pragma unroll
    for (int e = 0; e < kCols; ++e) sum[e] = from[e];
    for (int next = piece + 1; next < a.pieces.n && a.key[(int64_t)next * a.pieces.length] == token; ++next) {
        from = a.partial + (int64_t)next * 2 * g.width + c;
#pragma unroll
        for (int e = 0; e < kCols; ++e) sum[e] += from[e];
    }
    write_row<Table, kCols>(g, token, c, sum);
}

template <typename Table, int kCols>
__global__ void __launch_bounds__(kThreads)
zero_rows_kernel(Table* table, int vocab, int width, int64_t pitch) {
    grid_begin();
    Cols<Table, kCols> zero;
    zero.zero();
    for (int64_t row = blockIdx.x; row < vocab; row += gridDim.x)
        for (int c = threadIdx.x * kCols; c < width; c += kThreads * kCols) zero.store(table + row * pitch + c);
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
    constexpr int kMost = 16 / (int)sizeof(Out);
    switch (cols_of(kMost, a.table, a.table_pitch, sizeof(Table), a.out, a.pitch, sizeof(Out), a.width)) {
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
    for (int k = 0; k < 2; ++k) {
        g.sort.key[k] = reinterpret_cast<int32_t*>(take((size_t)n_tokens * 4));
        g.sort.pos[k] = reinterpret_cast<int32_t*>(take((size_t)n_tokens * 4));
    }
    g.sort.count = reinterpret_cast<uint32_t*>(take((size_t)kSortCtas * (sizeof(uint32_t) << kMostBits)));
    g.partial = reinterpret_cast<float*>(take((size_t)pieces_of(n_tokens, width).n * 2 * width * sizeof(float)));
    g.bytes = at;
    return g;
}

template <typename Grad, typename Table, int kCols>
int embed_grad_with(const SumArgs& a, cudaStream_t s) {
    const Spread sp = spread(a.g.width, kCols, kThreads);
    const int64_t blocks = ((int64_t)a.pieces.n - 1) / (kThreads / sp.across) + 1;       // times the tiles: below n_tokens * width / 256
    SR_LAUNCH("embed_sums_kernel", (embed_sums_kernel<Grad, Table, kCols>), (int)(blocks * sp.tiles), kThreads, 0, s, a, sp.across, sp.tiles);
    SR_LAUNCH("embed_join_kernel", (embed_join_kernel<Table, kCols>), (int)(blocks * sp.tiles), kThreads, 0, s, a, sp.across, sp.tiles);
    return SR_OK;
}

template <typename Table, int kCols>
int zero_rows(const EmbedGradArgs& g, cudaStream_t s) {
    SR_LAUNCH("zero_rows_kernel", (zero_rows_kernel<Table, kCols>), std::min(g.vocab, 148 * 16), kThreads, 0, s, static_cast<Table*>(g.d_table), g.vocab, g.width, g.table_pitch);
    return SR_OK;
}

template <typename Grad, typename Table>
int embed_grad_types(const EmbedGradArgs& g, void* ws, cudaStream_t s) {
    constexpr int kMost = 16 / (int)sizeof(Grad);
    const int cols = cols_of(kMost, g.d_out, g.pitch, sizeof(Grad), g.d_table, g.table_pitch, sizeof(Table), g.width);
    if (!g.accumulate) {
        const int rc = cols == 8 ? zero_rows<Table, 8>(g, s) : cols == 4 ? zero_rows<Table, 4>(g, s) : cols == 2 ? zero_rows<Table, 2>(g, s) : zero_rows<Table, 1>(g, s);
        if (rc != SR_OK) return rc;
    }
    if (g.n_tokens == 0) return SR_OK;
    const GradScratch scratch = grad_scratch(ws, g.n_tokens, g.width);
    int key_bits = 1;
    while ((g.vocab >> key_bits) != 0) ++key_bits;                       // `vocab` itself stands for what is no token
    const int passes = (key_bits - 1) / kMostBits + 1, bits = (key_bits - 1) / passes + 1;
    const int ctas = g.n_tokens > 8192 ? kSortCtas : 1;
    const size_t smem = (size_t)kSortWarps * sizeof(uint32_t) << bits;
    SR_CUDA_TRY(cudaFuncSetAttribute(sort_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)((size_t)kSortWarps * sizeof(uint32_t) << kMostBits)));
    const int rc = launch_as(true, ctas, "sort_tokens_kernel", sort_tokens_kernel, ctas, kSortThreads, smem, s, g.tokens, g.n_tokens, g.vocab, passes, bits, scratch.sort, g.status);
    if (rc != SR_OK) return rc;
    const SumArgs a{g, scratch.sort.key[(passes - 1) & 1], scratch.sort.pos[(passes - 1) & 1], scratch.partial, pieces_of(g.n_tokens, g.width)};
    switch (cols) {
        case 8: if constexpr (kMost == 8) return embed_grad_with<Grad, Table, 8>(a, s); else break;
        case 4: return embed_grad_with<Grad, Table, 4>(a, s);
        case 2: return embed_grad_with<Grad, Table, 2>(a, s);
        default: break;
    }
    return embed_grad_with<Grad, Table, 1>(a, s);
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
