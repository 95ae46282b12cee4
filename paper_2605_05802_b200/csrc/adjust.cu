// Logits adjusted by penalties for tokens seen before, biases and masks of allowed tokens, and their gradient (sr_tokens.h).
//
// A CTA has a slice of the vocabulary (16 KB of a row) and a run of rows.  Every thread owns the same four vectors of 16 bytes in each row, and with
// them their tokens: a bit of a register says which of them a history or a bias touches, shared memory how often each was seen and
// which entry of the bias list is its own.  Histories are read whole by every CTA of their rows, which costs 4 bytes a token from L2 and
// no hashing, sorting or limit of their length; where a row goes on where the one before it ended (a rollout scored as a whole), the
// owner of the new token notes it, and the CTA's threads go from row to row without a barrier.  Vectors pass through registers once, the
// next row's on their way meanwhile; those of which no token is allowed are not read.  Counts are whole numbers and a token's bias is the
// largest index in the list, so no order of atomics enters a result.
#include <stdlib.h>

#include <algorithm>

#include "tokens.cuh"

namespace sr {
namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 4;                         // a thread's, of a row of the slice
constexpr int kIdsAhead = 1536;                  // of the next row's history, and of its biases each: copied while this row is written
constexpr int kBiasesAhead = 512;
constexpr uint32_t kInPrompt = 0x80000000u;      // of a count: seen in the prompt,
constexpr uint32_t kBiased = 0x40000000u;        // in the bias list; the rest: how often behind the prompt
constexpr int kMostLength = 0x3FFFFFFF;          // of a history
template <typename T>
constexpr int kSliceOf = kThreads * kVecs * Vec<T>::kElems;

template <typename T>
__device__ __forceinline__ T banned_value(bool backward) { return from_float<T>(backward ? 0.0f : -INFINITY); }
template <typename T>
__device__ __forceinline__ uint32_t banned_word(bool backward) {
    if (backward) return 0u;
    return sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u;
}

// Bits l .. l + 31 of a row of words, the first `need` of them; the word behind is read only where one of those is in it.
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int l, int need) {
    const int w = l >> 5, sh = l & 31;
    const uint32_t lo = words[w];
    return sh + need <= 32 ? lo >> sh : __funnelshift_r(lo, words[w + 1], sh);
}

// The part of [start, start + len) inside [0, n): where it begins, and its length.
__device__ __forceinline__ int inside(int64_t start, int len, int64_t n, int64_t& from) {
    from = max(start, (int64_t)0);
    return start >= n || len <= 0 ? 0 : (int)max(min(n, start + len) - from, (int64_t)0);
}

// Copies to shared memory that a thread waits for before it uses what it has copied itself; in groups.
__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy_word(void* to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(shared_at(to)), "l"(from) : "memory"); }
__device__ __forceinline__ void copy_vector(void* to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(shared_at(to)), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void copies_wait_but_one() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

// What a row brings along; written to shared memory a batch of rows at a time, by one warp.
struct Record {
    int64_t start, bias_start;
    int32_t len, prompt, bias_len;
    int32_t from;                   // positions from here on are new; -1: nothing is as in the row before
    int32_t id;                     // the one new token, where there is one
    int32_t mask_behind;            // the mask of the row after the next
    float repetition, shrink, presence, frequency;      // shrink: its reciprocal
};
constexpr int kBatch = 16;

// kSparse: out is in, and only vectors that change are read and written.
// kShift: rows lie in different ways against 16 bytes, or in and out do.  The touched tokens are then bits of shared memory, which all
// threads read, and a barrier stands before and behind each change of them.
template <typename T, bool kBackward, bool kSparse, bool kShift>
__global__ void __launch_bounds__(kThreads, 3)
adjust_kernel(const __grid_constant__ AdjustArgs a, int runs, int rows_per_cta) {
    constexpr int E = Vec<T>::kElems, kSlice = kSliceOf<T>, kWords = kThreads + 1;        // kSlice / 32 + 1 of them in kShift
    constexpr uint32_t kAll = (1u << E) - 1u;
    extern __shared__ __align__(16) uint32_t s_tables[];
    __shared__ uint32_t s_touched[2][kWords];
    __shared__ Record s_record[kBatch];
    __shared__ uint4 s_vector[kThreads];                 // each thread's own, and so are the ids
    __shared__ int32_t s_ids[kIdsAhead], s_bias_ids[kBackward ? 1 : kBiasesAhead];
    __shared__ float s_bias_values[2][kBackward ? 1 : kBiasesAhead];
    __shared__ uint4 s_raw[kBackward ? kVecs * kThreads : 1];            // the logits of touched vectors, a row ahead
    grid_begin();
    const int tid = threadIdx.x;
    const bool histories = a.history_start != nullptr, biases = !kBackward && a.bias_value != nullptr;
    uint32_t* const count = s_tables;                                                     // [kSlice], forward
    uint32_t* const entry = s_tables + kSlice;                                            // [kSlice], with biases: 1 + index in the row's list, of what lies inside its array
    const int first = (int)(blockIdx.x / runs) * kSlice, n = min(kSlice, a.vocab - first);
    const int64_t row0 = (int64_t)(blockIdx.x % runs) * rows_per_cta;
    const int row_end = (int)min((int64_t)a.n_rows, row0 + rows_per_cta);
    const T* in = static_cast<const T*>(a.in) + row0 * a.pitch + first;
    T* out = static_cast<T*>(a.out) + row0 * a.out_pitch + first;
    const T* raw = kBackward ? static_cast<const T*>(a.logits) + row0 * a.logits_pitch + first : nullptr;
    int flags = 0;

    // elements before the first boundary of 16 bytes of both, and the vectors behind them
    int head = 0, vecs = 0;
    const auto split = [&](const T* x, const T* y, int& h, int& v) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
        const int off = (int)(p & 15) / (int)sizeof(T);
        h = kShift && ((p ^ q) & 15) != 0 ? n : min(n, off ? E - off : 0);
        v = (n - h) / E;
    };
    if (!kShift) split(in, out, head, vecs);
    uint32_t word = 0u;                                  // touched tokens of the thread's vectors, E bits of each
    // Place of a token that lies in no vector: 0 .. 7 before them, 8 .. 15 behind; the threads of that number have them.
    const auto outside = [&](int l) { return l < head ? l : 8 + l - head - vecs * E; };
    bool odd = false;                                    // whether the thread's is touched

    if (!kBackward && (histories || biases)) {
        for (int i = tid; i < kSlice / 4; i += kThreads) {
            reinterpret_cast<uint4*>(count)[i] = make_uint4(0u, 0u, 0u, 0u);
            if (biases) reinterpret_cast<uint4*>(entry)[i] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
    for (int i = tid; i < 2 * kWords; i += kThreads) s_touched[0][i] = 0u;

    // A turn begins with the next row's masks and vectors and ends with this row's: the first one has none.
    constexpr uint32_t kEvery = E * kVecs == 32 ? 0xFFFFFFFFu : (1u << (E * kVecs & 31)) - 1u;
    uint4 q[kVecs];
    const auto mask_at = [&](int m) { return a.allowed + (int64_t)m * a.mask_pitch + (first >> 5); };
    const auto mask_of = [&](int64_t row) {              // -1: none
        if (!a.allowed || row >= row_end) return -1;
        const int m = a.mask_row ? a.mask_row[row] : (int)row;
        if (m >= a.n_masks) flags |= SR_STATUS_BAD_INDEX;
        return m < a.n_masks ? m : -1;
    };
    // Words with the bits of the thread's vectors, and those bits.
    struct MaskWords {
        uint32_t lo[kVecs], hi[kVecs];
    };
    const auto words_of = [&](int m, int h, int v) {
        MaskWords w = {};
        if (m >= 0) {
            const uint32_t* const words = mask_at(m);
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int l = h + (tid + k * kThreads) * E;
                if (tid + k * kThreads < v) {
                    w.lo[k] = words[l >> 5];
                    if ((l & 31) + E > 32) w.hi[k] = words[(l >> 5) + 1];
                }
            }
        }
        return w;
    };
    const auto bits_of = [&](const MaskWords& w, int m, int h) {
        uint32_t bits = 0u;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) bits |= (__funnelshift_r(w.lo[k], w.hi[k], h + (tid + k * kThreads) * E) & kAll) << (k * E);
        return m < 0 ? kEvery : bits;
    };
    int mask = -1, next_mask = mask_of(row0);            // of the row and the one behind it
    uint32_t allowed = kEvery, next_allowed = kShift ? kEvery : bits_of(words_of(next_mask, head, vecs), next_mask, head);      // of the thread's vectors
    int at = kBatch;                                     // of the records
    bool ids_ahead = false;                              // this row's are on their way to shared memory
    int half = 0;                                        // of s_touched and s_bias_values, for the row at hand
    uint32_t raw_ahead = 0u;                             // touched tokens whose logits are on their way
#pragma unroll 1
    for (int row = (int)row0 - 1; row < row_end; ++row) {
        const T* const next_in = row < row0 ? in : in + a.pitch;
        int next_head = head, next_vecs = vecs;          // the same for all rows but in kShift
        uint4 ahead[kVecs];
#pragma unroll
        for (int k = 0; k < kVecs; ++k) ahead[k] = make_uint4(0u, 0u, 0u, 0u);
        if (row + 1 < row_end) {
            if (kShift) {
                split(next_in, row < row0 ? out : out + a.out_pitch, next_head, next_vecs);
                next_allowed = bits_of(words_of(next_mask, next_head, next_vecs), next_mask, next_head);
            }
            if (!kSparse) {
                const uint4* p = reinterpret_cast<const uint4*>(next_in + next_head) + tid;
#pragma unroll
                for (int k = 0; k < kVecs; ++k)
                    if (tid + k * kThreads < next_vecs && ((next_allowed >> (k * E)) & kAll) != 0u) ahead[k] = load_once(p + k * kThreads);
            }
        }
        int mask_behind = -1;
        if (row < row0) mask_behind = mask_of(row0 + 1);
        MaskWords words_behind = {};
        if (!kShift && row < row0 && a.allowed) words_behind = words_of(mask_behind, head, vecs);
        if (row >= row0) {
            if (at == kBatch) {                          // records of the rows from here on, by the first warp
                if (row > row0) __syncthreads();
                if (tid < 32) {
                    Record r = {};
                    const int64_t mine = (int64_t)row + tid;
                    const bool real = tid < kBatch && mine < row_end;
                    r.repetition = 1.0f;
                    if (real) {                          // all on their way before one is looked at
                        if (a.repetition) r.repetition = a.repetition[mine];
                        if (histories) {
                            r.start = a.history_start[mine];
                            r.len = a.history_len[mine];
                            if (!kBackward && a.prompt_len) r.prompt = a.prompt_len[mine];
                        }
                        if (!kBackward) {
                            if (a.presence) r.presence = a.presence[mine];
                            if (a.frequency) r.frequency = a.frequency[mine];
                            if (biases) {
                                r.bias_start = a.bias_start[mine];
                                r.bias_len = a.bias_len[mine];
                            }
                        }
                        r.mask_behind = mask_of(mine + 2);
                        if (r.len < 0 || r.bias_len < 0) flags |= SR_STATUS_NEG_LEN;
                        r.len = min(max(r.len, 0), kMostLength);
                        r.prompt = max(r.prompt, 0);
                        r.shrink = __fdiv_rn(1.0f, r.repetition);
                    }
                    const Record last = s_record[kBatch - 1];        // of the rows before
                    __syncwarp();
                    Record before;
                    before.start = __shfl_up_sync(0xFFFFFFFFu, r.start, 1);
                    before.bias_start = __shfl_up_sync(0xFFFFFFFFu, r.bias_start, 1);
                    before.len = __shfl_up_sync(0xFFFFFFFFu, r.len, 1);
                    before.prompt = __shfl_up_sync(0xFFFFFFFFu, r.prompt, 1);
                    before.bias_len = __shfl_up_sync(0xFFFFFFFFu, r.bias_len, 1);
                    if (tid == 0) before = last;
                    const bool same = mine > row0 && r.start == before.start && r.prompt == before.prompt && r.len >= before.len && r.bias_start == before.bias_start &&
                                      r.bias_len == before.bias_len;
                    r.from = same ? before.len : -1;
                    r.id = -1;
                    if (real && same && r.len == before.len + 1) {
                        const int64_t pos = r.start + before.len;
                        if (pos >= 0 && pos < a.n_history) r.id = a.history[pos];
                        if (r.id >= a.vocab) flags |= SR_STATUS_BAD_TARGET;
                    }
                    if (tid < kBatch) s_record[tid] = r;
                }
                __syncthreads();
                at = 0;
            }
            const Record& r = s_record[at++];
            mask_behind = r.mask_behind;
            if (!kShift && a.allowed) words_behind = words_of(mask_behind, head, vecs);

            // the tables of this row
            if (r.from < 0 || r.len > r.from + 1 || (kShift && r.len > r.from)) {
                if (kShift && row > row0) __syncthreads();           // the row before is done with them
                if (r.from < 0) half ^= 1;
                if (row > row0) {
                    if (r.from >= 0) {
                        if (!kShift) {                   // more than one new token: the owners' bits meet theirs
                            s_touched[half][tid] = word;
                            if (odd) atomicOr(&s_touched[half][kThreads], 1u << tid);
                        }
                    } else if (kShift) {
                        for (int i = tid; !kBackward && (histories || biases) && i < n; i += kThreads) {
                            count[i] = 0u;
                            if (biases) entry[i] = 0u;
                        }
                        for (int i = tid; i < kWords; i += kThreads) s_touched[half][i] = 0u;
                    } else if (!kBackward) {
                        const auto forget = [&](int l) {
                            count[l] = 0u;
                            if (biases) entry[l] = 0u;
                        };
#pragma unroll 1
                        for (uint32_t left = word; left != 0u; left &= left - 1u) {
                            const int b = __ffs(left) - 1;
                            forget(head + (tid + b / E * kThreads) * E + b % E);
                        }
                        if (odd) forget(tid < 8 ? tid : head + vecs * E + tid - 8);
                    }
                    __syncthreads();
                }
                // ids of the bias list, then of the history, in the slice
                const bool copied = ids_ahead && r.from < 0;
                if (copied) copies_wait();
#pragma unroll 1
                for (int pass = biases && r.from < 0 ? 0 : 1; pass < 1 + histories; ++pass) {
                    int64_t from;
                    const int done = pass == 0 ? 0 : max(r.from, 0);
                    const int64_t start = (pass == 0 ? r.bias_start : r.start) + done;
                    const int ids_n = inside(start, (pass == 0 ? r.bias_len : r.len) - done, pass == 0 ? a.n_bias : a.n_history, from);
                    const int32_t* const ids = (pass == 0 ? a.bias_token : a.history) + from;
                    const int behind = pass == 0 ? 0 : (int)(r.prompt - done - (from - start));      // the first id behind the prompt
                    const auto one = [&](int c, int32_t id) {
                        const uint32_t l = (uint32_t)id - (uint32_t)first;
                        if (id < 0 || l >= (uint32_t)n) {
                            if (id >= a.vocab) flags |= SR_STATUS_BAD_TARGET;
                            return;
                        }
                        if (!kBackward) {
                            if (pass == 0) {
                                atomicMax(&entry[l], (uint32_t)c + 1u);
                                atomicOr(&count[l], kBiased);
                            } else if (c >= behind) {
                                atomicAdd(&count[l], 1u);
                            } else {
                                atomicOr(&count[l], kInPrompt);
                            }
                        }
                        const int v = (int)l - head;
                        if (kShift) atomicOr(&s_touched[half][l >> 5], 1u << (l & 31));
                        else if (v < 0 || v >= vecs * E) atomicOr(&s_touched[half][kThreads], 1u << outside((int)l));
                        else atomicOr(&s_touched[half][(v / E) & (kThreads - 1)], 1u << ((v / E / kThreads) * E + v % E));
                    };
                    int c = tid;
                    if (copied) {
                        const int32_t* const held = pass == 0 ? s_bias_ids : s_ids;
                        const int held_n = min(ids_n, pass == 0 ? kBiasesAhead : kIdsAhead);
#pragma unroll 1
                        for (; c < held_n; c += kThreads) one(c, held[c]);
                    } else if (pass == 0) {
                        for (int k = tid; k < min(ids_n, kBiasesAhead); k += kThreads) s_bias_values[half][k] = a.bias_value[from + k];
                    }
#pragma unroll 1
                    for (; c < ids_n; c += 4 * kThreads) {
                        int32_t id[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) id[k] = c + k * kThreads < ids_n ? ids[c + k * kThreads] : -1;
#pragma unroll
                        for (int k = 0; k < 4; ++k) one(c + k * kThreads, id[k]);
                    }
                }
                __syncthreads();
                if (!kShift) {
                    word = s_touched[half][tid];
                    odd = tid < 16 && ((s_touched[half][kThreads] >> tid) & 1u);
                    s_touched[half ^ 1][tid] = 0u;       // for the next time: everybody has read it before the barriers above
                    if (tid == 0) s_touched[half ^ 1][kThreads] = 0u;
                }
            } else if (!kShift && r.id >= first && r.id - first < n) {
                const int l = r.id - first, v = l - head;            // one new token: its owner notes it
                bool mine;
                if (v < 0 || v >= vecs * E) {
                    mine = outside(l) == tid;
                    odd |= mine;
                } else {
                    mine = ((v / E) & (kThreads - 1)) == tid;
                    if (mine) word |= 1u << ((v / E / kThreads) * E + v % E);
                }
                if (mine && !kBackward) {
                    if (r.from >= r.prompt) count[l] += 1u;
                    else count[l] |= kInPrompt;
                }
            }
            if (kShift) {
                word = 0u;
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {
                    const int j = tid + k * kThreads;
                    if (j < vecs) word |= (bits_at(s_touched[half], head + j * E, E) & kAll) << (k * E);
                }
            }

            // on their way while this row is written: the ids of the next, where it begins anew
            ids_ahead = at < kBatch && row + 1 < row_end && s_record[at < kBatch ? at : 0].from < 0;
            if (ids_ahead) {
                const Record& next = s_record[at];
                int64_t from;
                if (histories) {
                    const int ids_n = min(inside(next.start, next.len, a.n_history, from), kIdsAhead);
#pragma unroll 1
                    for (int c = tid; c < ids_n; c += kThreads) copy_word(&s_ids[c], a.history + from + c);
                }
                if (biases) {
                    const int ids_n = min(inside(next.bias_start, next.bias_len, a.n_bias, from), kBiasesAhead);
#pragma unroll 1
                    for (int c = tid; c < ids_n; c += kThreads) {
                        copy_word(&s_bias_ids[c], a.bias_token + from + c);
                        copy_word(&s_bias_values[half ^ 1][c], a.bias_value + from + c);
                    }
                }
            }
            copies_end();

            // This row.  16-bit logits are multiplied by the reciprocal, whose 2^-24 their last rounding (2^-9, 2^-12) hides.
            const float repetition = r.repetition, shrink = r.shrink;
            const auto changed = [&](int l, float v, bool positive) {
                const auto repeated = [&] { return kBackward ? positive : v > 0.0f; };
                if (kBackward) return sizeof(T) == 4 ? (repeated() ? v / repetition : v * repetition) : v * (repeated() ? shrink : repetition);
                const uint32_t c = count[l], times = c & ~(kInPrompt | kBiased);
                if (c & ~kBiased) v = sizeof(T) == 4 ? (repeated() ? v / repetition : v * repetition) : v * (repeated() ? shrink : repetition);
                const float less = fmaf(-r.frequency, (float)times, v) - r.presence;
                v = times ? less : v;
                if (c & kBiased) {
                    const int e = (int)entry[l] - 1;
                    v += e < kBiasesAhead ? s_bias_values[half][e] : a.bias_value[max(r.bias_start, (int64_t)0) + e];
                }
                return v;
            };
            // elements in no vector
#pragma unroll 1
            for (int i = tid; kShift ? i < n - vecs * E : i < 16; i += kThreads) {
                const int l = kShift ? (i < head ? i : i + vecs * E) : i < 8 ? i : head + vecs * E + i - 8;
                if (!kShift && (i < 8 ? l >= head : l >= n)) continue;
                if (mask >= 0 && !((mask_at(mask)[l >> 5] >> (l & 31)) & 1u)) out[l] = banned_value<T>(kBackward);
                else if (kShift ? (s_touched[half][l >> 5] >> (l & 31)) & 1u : odd) out[l] = from_float<T>(changed(l, to_float(in[l]), kBackward && to_float(raw[l]) > 0.0f));
                else if (!kSparse) out[l] = in[l];
            }
            if (kSparse) {
                const uint4* p = reinterpret_cast<const uint4*>(in + head) + tid;
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {        // vectors with a token that stays and one that changes
                    const uint32_t m = (allowed >> (k * E)) & kAll, t = (word >> (k * E)) & kAll;
                    if (tid + k * kThreads < vecs && m != 0u && (m != kAll || t != 0u)) q[k] = load_once(p + k * kThreads);
                }
            }
            const uint32_t left = word & allowed;        // tokens that change, one after the other in the thread's part of shared memory
            if (left != 0u) {
                T* const mine = reinterpret_cast<T*>(s_vector + tid);
                if (kBackward) copies_wait_but_one();
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {
                    if (((left >> (k * E)) & kAll) == 0u) continue;
                    s_vector[tid] = q[k];
                    const int l0 = head + (tid + k * kThreads) * E;
                    const T* const raw_held = reinterpret_cast<const T*>(s_raw + (kBackward ? k * kThreads + tid : 0));
#pragma unroll 1
                    for (uint32_t b = (left >> (k * E)) & kAll; b != 0u; b &= b - 1u) {
                        const int e = __ffs(b) - 1;
                        bool positive = false;           // the logit whose gradient this is
                        if (kBackward) positive = to_float((raw_ahead >> (k * E)) & 1u ? raw_held[e] : raw[l0 + e]) > 0.0f;
                        mine[e] = from_float<T>(changed(l0 + e, to_float(mine[e]), positive));
                    }
                    q[k] = s_vector[tid];
                }
            }
            if (kBackward) {                             // the next row's logits of what is touched already
                raw_ahead = 0u;
                if (word != 0u && !kShift && row + 1 < row_end && (reinterpret_cast<uintptr_t>(raw + a.logits_pitch + head) & 15) == 0) {
                    const uint4* const p = reinterpret_cast<const uint4*>(raw + a.logits_pitch + head) + tid;
#pragma unroll
                    for (int k = 0; k < kVecs; ++k) {
                        if (((word & next_allowed) >> (k * E) & kAll) == 0u) continue;
                        copy_vector(&s_raw[k * kThreads + tid], p + k * kThreads);
                        raw_ahead |= kAll << (k * E);
                    }
                }
                copies_end();
            }
            uint4* const to = reinterpret_cast<uint4*>(out + head) + tid;
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                if (tid + k * kThreads >= vecs) break;
                const uint32_t m = (allowed >> (k * E)) & kAll;
                if (kSparse && m == kAll && ((word >> (k * E)) & kAll) == 0u) continue;
                if (m != kAll) {
                    uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t keep;
                        if (E == 4) keep = (m >> i) & 1u ? 0xFFFFFFFFu : 0u;
                        else keep = ((m >> (2 * i)) & 1u ? 0x0000FFFFu : 0u) | ((m >> (2 * i + 1)) & 1u ? 0xFFFF0000u : 0u);
                        w[i] = (w[i] & keep) | (banned_word<T>(kBackward) & ~keep);
                    }
                    q[k] = make_uint4(w[0], w[1], w[2], w[3]);
                }
                store_once(to + k * kThreads, q[k]);
            }
            in += a.pitch;
            out += a.out_pitch;
            if (kBackward) raw += a.logits_pitch;
        }
#pragma unroll
        for (int k = 0; k < kVecs; ++k) q[k] = ahead[k];
        mask = next_mask;
        allowed = next_allowed;
        next_mask = mask_behind;
        if (!kShift) next_allowed = bits_of(words_behind, mask_behind, head);
        head = next_head;
        vecs = next_vecs;
    }
    if (a.status && flags) atomicOr(a.status, flags);
}

template <typename T, bool kBackward>
int launch_type(const AdjustArgs& a, cudaStream_t s) {
    constexpr int kSlice = kSliceOf<T>;
    const int slices = (a.vocab - 1) / kSlice + 1;
    // Few rows get a CTA each a slice; many are dealt out in runs, so that a rollout's rows find its history at hand, but
    // leave every SM a few turns.
    const int64_t units = (int64_t)slices * a.n_rows;
    static const char* tune = getenv("TUNE_WAVES");
    static const char* tune2 = getenv("TUNE_SLOTS");
    const int waves = tune ? atoi(tune) : 3, slots = tune2 ? atoi(tune2) : 296;
    int64_t rows = std::min<int64_t>((units - 1) / (slots * waves) + 1, 64);
    rows = std::max(rows, (units - 1) / (INT32_MAX - slices) + 1);           // CTAs are numbered in 31 bits
    const int64_t runs = (a.n_rows - 1) / rows + 1, ctas = slices * runs;
    const size_t smem = kBackward ? 0 : (size_t)(a.bias_value ? 2 : a.history_start ? 1 : 0) * kSlice * sizeof(uint32_t);
    const auto apart = [&](int64_t pitch) { return a.n_rows > 1 && pitch * (int64_t)sizeof(T) % 16 != 0; };
    const bool alike = ((reinterpret_cast<uintptr_t>(a.in) ^ reinterpret_cast<uintptr_t>(a.out)) & 15) == 0;
    const bool shift = !alike || apart(a.pitch) || apart(a.out_pitch);
    const auto kernel = a.in == a.out ? (shift ? adjust_kernel<T, kBackward, true, true> : adjust_kernel<T, kBackward, true, false>)
                                      : (shift ? adjust_kernel<T, kBackward, false, true> : adjust_kernel<T, kBackward, false, false>);
    if (smem > 24 * 1024) SR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    SR_LAUNCH("adjust_kernel", kernel, (int)ctas, kThreads, smem, s, a, (int)runs, (int)rows);
    return SR_OK;
}

}  // namespace

int launch_adjust(const AdjustArgs& a, bool backward, cudaStream_t s) {
    if (a.n_rows == 0) return SR_OK;
    if (a.dtype == SR_DTYPE_F32) return backward ? launch_type<float, true>(a, s) : launch_type<float, false>(a, s);
    if (a.dtype == SR_DTYPE_BF16) return backward ? launch_type<__nv_bfloat16, true>(a, s) : launch_type<__nv_bfloat16, false>(a, s);
    return backward ? launch_type<__half, true>(a, s) : launch_type<__half, false>(a, s);
}

}  // namespace sr
