// Logits adjusted by penalties for tokens seen before, biases and masks of allowed tokens, and their gradient (sr_tokens.h).
//
// A CTA has a slice of 8192 tokens of the vocabulary and a run of rows.  Shared memory holds what the rules say of its tokens: a bit for each
// that a history or a bias touches, how often it was seen and which entry of the bias list is its own.  Histories are read whole by every CTA
// of their rows, which costs 4 bytes a token from L2 and no hashing, sorting or limit of their length; where a row goes on where
// the one before it ended (a rollout scored as a whole), only what is new is added.  The slice itself then streams through
// registers once: vectors that nothing touches and no mask cuts pass as they are.  Counts are whole numbers and the bias
// entry is the largest index, so no order of atomics enters a result.
#include <algorithm>

#include "tokens.cuh"

namespace sr {
namespace {

constexpr int kThreads = 256;
constexpr int kSlice = 8192;
constexpr int kWords = kSlice / 32;
constexpr uint32_t kInPrompt = 0x80000000u;      // of a count: seen in the prompt; the rest: how often behind it

template <typename T>
__device__ __forceinline__ T banned_value(bool backward) { return from_float<T>(backward ? 0.0f : -INFINITY); }
template <typename T>
__device__ __forceinline__ uint32_t banned_word(bool backward) {
    if (backward) return 0u;
    return sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u;
}

// Bits l .. l + 31 of a row of words.  Reads the word behind only where bits of it are among the first `need`.
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int l, int need) {
    const int w = l >> 5, sh = l & 31;
    const uint32_t lo = words[w];
    return sh + need <= 32 ? lo >> sh : __funnelshift_r(lo, words[w + 1], sh);
}

struct Shared {
    uint32_t* touched;      // [kWords + 1]
    uint32_t* count;        // [kSlice], forward with histories
    uint32_t* entry;        // [kSlice], forward with biases: 1 + index in the row's list
};

// What a row's rules are beside the tables in shared memory.
struct RowRules {
    float repetition, presence, frequency;
    const float* bias;              // of the row's list
    const uint32_t* mask;           // of the slice's first token, or NULL
};

template <bool kBackward>
__device__ __forceinline__ float touched_value(const AdjustArgs& a, const Shared& sm, const RowRules& r, int l, float v, float x) {
    if (kBackward) return x > 0.0f ? v / r.repetition : v * r.repetition;
    if (sm.count) {
        const uint32_t c = sm.count[l], n = c & ~kInPrompt;
        if (c && a.repetition) v = v > 0.0f ? v / r.repetition : v * r.repetition;
        if (n) v = fmaf(-r.frequency, (float)n, v) - r.presence;
    }
    if (sm.entry) {
        const uint32_t e = sm.entry[l];
        if (e) v += r.bias[e - 1];
    }
    return v;
}

// Adds entries [from, to) of a list to the tables; all of them lie inside the list's array.
template <typename Take>
__device__ __forceinline__ void scan_ids(const AdjustArgs& a, const int32_t* ids, int64_t from, int64_t to, uint32_t first, uint32_t n, bool& bad, Take take) {
    const auto one = [&](int64_t i, int32_t id) {
        bad |= id >= a.vocab;
        const uint32_t l = (uint32_t)id - first;
        if (id >= 0 && l < n) take(i, l);
    };
    int64_t i = from + threadIdx.x;
    for (; i + 3 * kThreads < to; i += 4 * kThreads) {
        int32_t id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = ids[i + k * kThreads];
#pragma unroll
        for (int k = 0; k < 4; ++k) one(i + k * kThreads, id[k]);
    }
    for (; i < to; i += kThreads) one(i, ids[i]);
}

// The part of [start, start + len) inside [0, n).
__device__ __forceinline__ void inside(int64_t start, int64_t len, int64_t n, int64_t& from, int64_t& to) {
    from = max(start, (int64_t)0);
    to = start >= n ? from : min(n, start + len);
    if (len <= 0 || to < from) to = from;
}

// kSparse: out is in, and only vectors that change are read and written.
template <typename T, bool kBackward, bool kSparse>
__global__ void __launch_bounds__(kThreads)
adjust_kernel(const __grid_constant__ AdjustArgs a, int slices, int rows_per_cta) {
    extern __shared__ __align__(16) uint32_t s_tables[];
    constexpr int E = Vec<T>::kElems;
    constexpr int kVecs = kSlice / E / kThreads;
    constexpr uint32_t kAll = (1u << E) - 1u;
    grid_begin();
    const int slice = blockIdx.x % slices;
    const int64_t row0 = (int64_t)(blockIdx.x / slices) * rows_per_cta;
    const int row_end = (int)min((int64_t)a.n_rows, row0 + rows_per_cta);
    const int first = slice * kSlice, n = min(kSlice, a.vocab - first);
    const bool histories = a.history_start != nullptr, biases = !kBackward && a.bias_value != nullptr;
    Shared sm;
    sm.touched = s_tables;
    sm.count = !kBackward && histories ? s_tables + kWords + 4 : nullptr;
    sm.entry = biases ? s_tables + kWords + 4 + (histories ? kSlice : 0) : nullptr;

    bool bad = false, negative = false, no_mask = false;
    int64_t had_start = 0, had_bias = 0;
    int32_t had_len = 0, had_prompt = 0, had_bias_len = 0;
    for (int row = (int)row0; row < row_end; ++row) {
        const T* in = static_cast<const T*>(a.in) + (int64_t)row * a.pitch + first;
        T* out = static_cast<T*>(a.out) + (int64_t)row * a.out_pitch + first;
        const T* raw = kBackward && a.logits ? static_cast<const T*>(a.logits) + (int64_t)row * a.logits_pitch + first : nullptr;
        RowRules r;
        r.mask = nullptr;
        if (a.allowed) {
            const int m = a.mask_row ? a.mask_row[row] : row;
            if (m >= a.n_masks) no_mask = true;
            else if (m >= 0) r.mask = a.allowed + (int64_t)m * a.mask_pitch + (first >> 5);
        }
        // vectors on 16 bytes of both rows, and the elements before and behind them
        const bool alike = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
        const int off = (int)(reinterpret_cast<uintptr_t>(out) & 15) / (int)sizeof(T);
        const int head = alike ? min(n, off ? E - off : 0) : n, vecs = (n - head) / E;
        const uint4* from = reinterpret_cast<const uint4*>(in + head);
        uint4* to = reinterpret_cast<uint4*>(out + head);
        uint4 q[kVecs];
        uint32_t m[kVecs];
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int j = threadIdx.x + k * kThreads;
            m[k] = j < vecs && r.mask ? bits_at(r.mask, head + j * E, E) & kAll : kAll;
        }
        if (!kSparse) {
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int j = threadIdx.x + k * kThreads;
                q[k] = j < vecs && m[k] ? load_once(from + j) : make_uint4(0u, 0u, 0u, 0u);
            }
        }

        // the tables
        int64_t start = 0, bias_start = 0;
        int32_t len = 0, prompt = 0, bias_len = 0;
        if (histories) {
            start = a.history_start[row];
            len = a.history_len[row];
            negative |= len < 0;
            prompt = !kBackward && a.prompt_len ? a.prompt_len[row] : 0;
        }
        if (biases) {
            bias_start = a.bias_start[row];
            bias_len = a.bias_len[row];
            negative |= bias_len < 0;
        }
        const bool goes_on = row > row0 && start == had_start && prompt == had_prompt && len >= had_len && bias_start == had_bias && bias_len == had_bias_len;
        if (!goes_on || len > had_len) {
            if (row > row0) __syncthreads();             // the row before is done with them
            if (!goes_on) {
                had_len = 0;
                for (int i = threadIdx.x; i <= kWords; i += kThreads) sm.touched[i] = 0u;
                for (int i = threadIdx.x; sm.count && i < kSlice / 4; i += kThreads) reinterpret_cast<uint4*>(sm.count)[i] = make_uint4(0u, 0u, 0u, 0u);
                for (int i = threadIdx.x; sm.entry && i < kSlice / 4; i += kThreads) reinterpret_cast<uint4*>(sm.entry)[i] = make_uint4(0u, 0u, 0u, 0u);
                __syncthreads();
                if (biases) {
                    int64_t lo, hi;
                    inside(bias_start, bias_len, a.n_bias, lo, hi);
                    scan_ids(a, a.bias_token, lo, hi, (uint32_t)first, (uint32_t)n, bad, [&](int64_t i, uint32_t l) {
                        atomicMax(&sm.entry[l], (uint32_t)(i - bias_start) + 1u);
                        atomicOr(&sm.touched[l >> 5], 1u << (l & 31));
                    });
                }
            }
            if (histories) {
                int64_t lo, hi;
                const int32_t done = max(had_len, 0);
                inside(start + done, (int64_t)len - done, a.n_history, lo, hi);
                const int64_t behind = start + max(prompt, 0);
                scan_ids(a, a.history, lo, hi, (uint32_t)first, (uint32_t)n, bad, [&](int64_t i, uint32_t l) {
                    if (!kBackward) {
                        if (i >= behind) atomicAdd(&sm.count[l], 1u);
                        else atomicOr(&sm.count[l], kInPrompt);
                    }
                    atomicOr(&sm.touched[l >> 5], 1u << (l & 31));
                });
            }
            __syncthreads();
        }
        had_start = start; had_len = len; had_prompt = prompt; had_bias = bias_start; had_bias_len = bias_len;

        r.repetition = a.repetition ? a.repetition[row] : 1.0f;
        r.presence = a.presence ? a.presence[row] : 0.0f;
        r.frequency = a.frequency ? a.frequency[row] : 0.0f;
        r.bias = a.bias_value + bias_start;

        // elements outside the vectors
        for (int i = threadIdx.x; i < n - vecs * E; i += kThreads) {
            const int l = i < head ? i : i + vecs * E;
            const bool is_allowed = !r.mask || (bits_at(r.mask, l, 1) & 1u);
            const bool is_touched = (sm.touched[l >> 5] >> (l & 31)) & 1u;
            if (!is_allowed) out[l] = banned_value<T>(kBackward);
            else if (is_touched) out[l] = from_float<T>(touched_value<kBackward>(a, sm, r, l, to_float(in[l]), kBackward ? to_float(raw[l]) : 0.0f));
            else if (!kSparse) out[l] = in[l];
        }
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int j = threadIdx.x + k * kThreads, l = head + j * E;
            if (j >= vecs) break;
            uint32_t t = bits_at(sm.touched, l, E) & m[k];
            if (kSparse) {
                if (m[k] == kAll && t == 0u) continue;
                q[k] = m[k] ? load_once(from + j) : make_uint4(0u, 0u, 0u, 0u);
            }
            if (t) {
                float v[E];
                unpack(q[k], v, T());
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if ((t >> e) & 1u) v[e] = touched_value<kBackward>(a, sm, r, l + e, v[e], kBackward ? to_float(raw[l + e]) : 0.0f);
                q[k] = pack(v, T());
            }
            if (m[k] != kAll) {
                uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t keep;
                    if (E == 4) keep = (m[k] >> i) & 1u ? 0xFFFFFFFFu : 0u;
                    else keep = ((m[k] >> (2 * i)) & 1u ? 0x0000FFFFu : 0u) | ((m[k] >> (2 * i + 1)) & 1u ? 0xFFFF0000u : 0u);
                    w[i] = (w[i] & keep) | (banned_word<T>(kBackward) & ~keep);
                }
                q[k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            store_once(to + j, q[k]);
        }
    }
    if (a.status) {
        const int bits = (bad ? SR_STATUS_BAD_TARGET : 0) | (negative ? SR_STATUS_NEG_LEN : 0) | (no_mask ? SR_STATUS_BAD_INDEX : 0);
        if (bits) atomicOr(a.status, bits);
    }
}

template <typename T, bool kBackward>
int launch_form(const AdjustArgs& a, bool in_place, cudaStream_t s) {
    const int slices = (a.vocab - 1) / kSlice + 1;
    // Few rows get a CTA each a slice; many are dealt out in runs, so that a rollout's rows find its history at hand, but
    // leave every SM a few turns.
    const int64_t units = (int64_t)slices * a.n_rows;
    int64_t rows = std::min<int64_t>(std::max<int64_t>(units / (148 * 24), 1), 64);
    rows = std::max(rows, (units - 1) / (INT32_MAX - slices) + 1);           // CTAs are numbered in 31 bits
    const int64_t ctas = (int64_t)slices * ((a.n_rows - 1) / rows + 1);
    const size_t tables = kBackward ? 0 : (size_t)((a.history_start != nullptr) + (a.bias_value != nullptr)) * kSlice;
    const size_t smem = (kWords + 4 + tables) * sizeof(uint32_t);
    const auto kernel = in_place ? adjust_kernel<T, kBackward, true> : adjust_kernel<T, kBackward, false>;
    if (smem > 48 * 1024) SR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    SR_LAUNCH("adjust_kernel", kernel, (int)ctas, kThreads, smem, s, a, slices, (int)rows);
    return SR_OK;
}

}  // namespace

int launch_adjust(const AdjustArgs& a, bool backward, cudaStream_t s) {
    if (a.n_rows == 0) return SR_OK;
    const bool in_place = a.in == a.out;
    if (a.dtype == SR_DTYPE_F32) return backward ? launch_form<float, true>(a, in_place, s) : launch_form<float, false>(a, in_place, s);
    if (a.dtype == SR_DTYPE_BF16) return backward ? launch_form<__nv_bfloat16, true>(a, in_place, s) : launch_form<__nv_bfloat16, false>(a, in_place, s);
    return backward ? launch_form<__half, true>(a, in_place, s) : launch_form<__half, false>(a, in_place, s);
}

}  // namespace sr
