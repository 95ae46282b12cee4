// Logits adjusted by penalties for tokens seen before, biases and masks of allowed tokens, and their gradient (sr_tokens.h).
//
// A CTA has a slice of the vocabulary (16 KB of a row) and a run of rows.  Every thread owns the same four vectors of 16 bytes in each row, and with
// them their tokens: the bits of a register say which of them a history or a bias touches, shared memory how often each was seen and
// which entry of the bias list is its own.  Histories are read whole by every CTA of their rows, which costs 4 bytes a token from L2 and
// no hashing, sorting or limit of their length.  Where a row goes on where the one before it ended (a rollout scored as a whole), the
// owner of the new token notes it, and the CTA's threads go from row to row without a barrier; where a row begins anew, its ids have been
// copied to shared memory while the row before was written.  Vectors go through a ring of rows in shared memory, copied ahead by the thread that
// changes and writes them; those of which no token is allowed are not read.  Counts are whole numbers and a token's bias is the largest
// index in the list, so no order of atomics enters a result.
//
// Rollouts as a whole are bound by HBM: 4096 rows of 151936 bf16 in 411 us, 6.1 TB/s of logits read and written; the gradient of 2048 with masks,
// half of which allow a handful, in 181 us (their banned vectors are not read: what is left runs at 5.2 TB/s, and takes a copy 143).  Rows with histories of their own are
// bound by latency and issue: 512 of them 73 us with penalties (a copy 48), 131 with 300 biases each and masks too (36 without what masks ban), of 600 to 900
// instructions a warp and row, a copy's 220 among them; two changed tokens side by side make no difference.  In place, where only what changes is read and written, 4096 rows with penalties
// take 302 us, 512 with biases and masks 138.  Rows of in and out that begin at different distances from 16 bytes go element by element: 4096 of
// 50257 bf16 1030 us, 158 where all begin on 16 bytes, 236 where both are contiguous (off 16 bytes alike).  Before: tables looked up for every vector (4096 rows 618 us), rows in registers (446; their
// code outgrew the instruction cache with every change unrolled), 512 threads (429), slices of twice the size (580).
#include <algorithm>

#include "rows_ahead.cuh"
#include "tokens.cuh"

namespace sr {
namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 4;                         // a thread's, of a row of the slice
constexpr int kIdsAhead = 1024;                  // of the next row's history, and of its biases: copied while this row is written
constexpr int kBiasesAhead = 256;
constexpr int kMostLength = 0x3FFFFFFF;          // of a history
constexpr int kMostBiases = 0xFFFF;              // of a list
// A token's count, 16 bits: seen in the prompt, in the bias list, and how often behind the prompt.  From kMany on, give or take what
// the CTA's threads add at once, occurrences are counted in a table of few such tokens.
constexpr uint32_t kInPrompt = 0x8000u, kBiased = 0x4000u, kTimes = 0x3FFFu, kMany = 0x2000u;
constexpr int kFrequent = 64;
template <typename T>
constexpr int kSliceOf = kThreads * kVecs * Vec<T>::kElems;

template <typename T>
__device__ __forceinline__ T banned_value(bool backward) { return from_float<T>(backward ? 0.0f : -INFINITY); }
template <typename T>
__device__ __forceinline__ uint32_t banned_word(bool backward) {
    if (backward) return 0u;
    return sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u;
}

// Word i of a vector without the tokens whose bits are 0.
template <typename T, bool kBackward>
__device__ __forceinline__ uint32_t cut(uint32_t w, uint32_t bits, int i) {
    uint32_t keep;
    if (sizeof(T) == 4) keep = 0u - ((bits >> i) & 1u);
    else asm("prmt.b32 %0, %1, %2, 0xDD88;" : "=r"(keep) : "r"(bits << (7 - 2 * i)), "r"(bits << (14 - 2 * i)));      // signs of bytes, twice each
    return (w & keep) | (banned_word<T>(kBackward) & ~keep);
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
template <int kLater>                     // groups that may still be on their way
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLater) : "memory"); }

// What a row brings along; written to shared memory a batch of rows at a time, by one warp.
struct Record {
    int64_t start, bias_start;      // as given,
    int32_t len, prompt, bias_len;
    int64_t from_at, bias_at;       // and of the history (from `from` on) and the list what lies inside their arrays,
    int32_t n, bias_n, behind;      // with the first of its ids that is behind the prompt
    int32_t from;                   // positions of the history from here on are new; -1: nothing is as in the row before
    int32_t id;                     // the one new token, where there is one
    int32_t mask, mask_ahead;       // this row's, and that of the row whose mask is looked up in this row's turn
    float repetition, shrink, presence, frequency;      // shrink: its reciprocal
};
constexpr int kBatch = 8;

// Tokens that are seen thousands of times, out of line: a call that hardly any row makes.
__device__ __noinline__ void count_frequent(uint32_t* table, int l) {
    for (int i = 0; i < kFrequent; ++i) {
        const int slot = (l + i) % kFrequent;
        const uint32_t had = atomicCAS(&table[slot], 0u, (uint32_t)l + 1u);
        if (had != 0u && had != (uint32_t)l + 1u) continue;
        atomicAdd(&table[kFrequent + slot], 1u);
        return;
    }
}
__device__ __noinline__ uint32_t times_frequent(const uint32_t* table, uint32_t times, int l, int id, const int32_t* history, int64_t n_history, const Record& r, uint32_t more) {
    for (int i = 0; i < kFrequent; ++i) {
        const int slot = (l + i) % kFrequent;
        if (table[slot] == (uint32_t)l + 1u) return times + table[kFrequent + slot];
        if (table[slot] == 0u) return times;          // a further one would have found room here: there was none
    }
    int64_t from;                   // more of them than the table holds
    const int skip = min(r.prompt, r.len), n = inside(r.start + skip, r.len - skip, n_history, from);
    times = 0;
    for (int k = 0; k < n; ++k) times += history[from + k] == id;
    return times - more;            // those that the caller adds
}

// Where things lie in dynamic shared memory (bytes).  kStages: rows of the ring, one of which is changed and written while the others are on their way.
template <typename T, int kStages, bool kBackward>
struct Layout {
    static constexpr int kSlice = kSliceOf<T>, kRow = kVecs * kThreads * 16;
    static constexpr int kRaw = kStages * kRow, kCount = kRaw + (kBackward ? kRow : 0), kEntry = kCount + (kBackward ? 0 : kSlice * 2),
                         kBiasIds = kEntry + kSlice * 2, kBiasValues = kBiasIds + kBiasesAhead * 4, kAll = kBiasValues + 2 * kBiasesAhead * 4;
    static constexpr int bytes(bool counts, bool biases) { return kBackward ? kCount : biases ? kAll : counts ? kEntry : kCount; }
};

// kSparse: out is in, and only vectors that change are read and written.
// kShift: not all rows of in and out begin on 16 bytes.  The touched tokens are then bits of shared memory, which all threads read; the new tokens of
// a batch's rows are looked up in their records until a barrier lets them into the tables (4096 rows of 151935 bf16: 543 us, with barriers at every new token 622).
template <typename T, int kStages, bool kBackward, bool kSparse, bool kShift>
__global__ void __launch_bounds__(kThreads, kStages == 3 ? 3 : 4)
adjust_kernel(const __grid_constant__ AdjustArgs a, int runs, int rows_per_cta) {
    using Lay = Layout<T, kStages, kBackward>;
    constexpr int E = Vec<T>::kElems, kSlice = Lay::kSlice, kBits = E * kVecs;
    static_assert(kBits <= 32, "a bit for each token of a thread's vectors");
    constexpr int kWords = kThreads + 1;                 // at least kSlice / 32 + 1
    constexpr uint32_t kEvery = (uint32_t)((1ull << kBits) - 1u), kAll = (1u << E) - 1u;
    extern __shared__ __align__(16) unsigned char s_bytes[];
    __shared__ uint32_t s_touched[2][kWords];
    __shared__ Record s_record[kBatch];
    __shared__ int32_t s_ids[kIdsAhead];                 // a thread's own
    __shared__ uint32_t s_frequent[kBackward ? 1 : 2 * kFrequent];                        // 1 + token, and its further occurrences
    grid_begin();
    const int tid = threadIdx.x;
    const bool histories = a.history_start != nullptr, biases = !kBackward && a.bias_value != nullptr, counts = !kBackward && (histories || biases);
    uint4* const s_raw = reinterpret_cast<uint4*>(s_bytes + Lay::kRaw);                   // backward: the logits of touched vectors, a row ahead; a thread's own
    uint16_t* const count = reinterpret_cast<uint16_t*>(s_bytes + Lay::kCount);           // [kSlice]
    uint16_t* const entry = reinterpret_cast<uint16_t*>(s_bytes + Lay::kEntry);           // [kSlice]: 1 + index in the row's list, of what lies inside its array
    int32_t* const s_bias_ids = reinterpret_cast<int32_t*>(s_bytes + Lay::kBiasIds);      // a thread's own
    float* const s_bias_values = reinterpret_cast<float*>(s_bytes + Lay::kBiasValues);    // [2][kBiasesAhead]
    const int first = (int)(blockIdx.x / runs) * kSlice, n = min(kSlice, a.vocab - first);
    const int64_t row0 = (int64_t)(blockIdx.x % runs) * rows_per_cta;
    const int row_end = (int)min((int64_t)a.n_rows, row0 + rows_per_cta);
    const T* in = static_cast<const T*>(a.in) + row0 * a.pitch + first;
    T* out = static_cast<T*>(a.out) + row0 * a.out_pitch + first;
    const T* raw = kBackward ? static_cast<const T*>(a.logits) + row0 * a.logits_pitch + first : nullptr;
    int flags = 0;

    // elements before the first boundary of 16 bytes of both, and the vectors behind them
    int head = 0, vecs = n / E;
    const auto split = [&](const T* x, const T* y, int& h, int& v) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
        const int off = (int)(p & 15) / (int)sizeof(T);
        h = ((p ^ q) & 15) != 0 ? n : min(n, off ? E - off : 0);
        v = (n - h) / E;
    };
    uint32_t word = 0u;                                  // touched tokens of the thread's vectors
    bool odd = false;                                    // whether the token is that thread `tid` has behind the vectors
    const auto bits_of_vector = [&](uint32_t w, int k) { return (w >> (k * E)) & kAll; };

    if (counts) {
        for (int i = tid; i < kSlice / 8; i += kThreads) {
            reinterpret_cast<uint4*>(count)[i] = make_uint4(0u, 0u, 0u, 0u);
            if (biases) reinterpret_cast<uint4*>(entry)[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        for (int i = tid; i < 2 * kFrequent; i += kThreads) s_frequent[i] = 0u;
    }
    bool frequent = false;                               // whether the thread has counted there
    for (int i = tid; i < 2 * kWords; i += kThreads) s_touched[0][i] = 0u;

    // Masks: that of a row, -1 for none; the words with the bits of the thread's vectors; those bits.
    const auto mask_at = [&](int m) { return a.allowed + (int64_t)m * a.mask_pitch + (first >> 5); };
    const auto mask_of = [&](int64_t row) {
        if (!a.allowed || row >= row_end) return -1;
        const int m = a.mask_row ? a.mask_row[row] : (int)row;
        if (m >= a.n_masks) flags |= SR_STATUS_BAD_INDEX;
        return m < a.n_masks ? m : -1;
    };
    struct MaskWords {
        uint32_t lo[kVecs], hi[kShift ? kVecs : 1];
    };
    const auto words_of = [&](int m, int h, int v) {
        MaskWords w = {};
        if (m >= 0) {
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int j = tid + k * kThreads, l = (kShift ? h : 0) + j * E;
                if (j >= v) continue;
                w.lo[k] = mask_at(m)[l >> 5];
                if (kShift && (l & 31) + E > 32) w.hi[k] = mask_at(m)[(l >> 5) + 1];
            }
        }
        return w;
    };
    const auto bits_of = [&](const MaskWords& w, int m, int h) {
        uint32_t bits = 0u;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int sh = ((kShift ? h : 0) + (tid + k * kThreads) * E) & 31;
            bits |= ((kShift ? __funnelshift_r(w.lo[k], w.hi[k], sh) : w.lo[k] >> sh) & kAll) << (k * E);
        }
        return m < 0 ? kEvery : bits;
    };

    // The turn of a row looks up the mask of the row kDepth behind it, has the vectors of the row before that one copied into the ring,
    // and changes and writes its own.  The first turns are those of no row.
    constexpr int kDepth = kStages;
    uint32_t allowed[kDepth];                            // of the thread's vectors, from this row on
    constexpr int kEdges = 16;                           // more than there are elements before and behind the vectors of a row, if it has any
    T edge[kDepth];                                      // kShift: that of the thread, copied ahead like the vectors
    int head_ahead = 0, vecs_ahead = vecs;               // of the row that is looked up; the same for all but in kShift
    if (kShift) split(in, out, head_ahead, vecs_ahead);
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
        allowed[d] = kEvery;
        edge[d] = from_float<T>(0.0f);
    }
    {
        const int m = mask_of(row0);
        if (a.allowed) allowed[kDepth - 1] = bits_of(words_of(m, head_ahead, vecs_ahead), m, head_ahead);
    }
    int at = kBatch;                                     // of the records
    constexpr int kFull = kVecs * kThreads;              // vectors of a whole slice
    uint4* const ring = reinterpret_cast<uint4*>(s_bytes) + tid;
    int fill = 0, take = 0;                              // its rows that are next
    const T* in_ahead = in;
    int half = 0;                                        // of s_touched and s_bias_values, for the row at hand
    // the ids of a row that begins anew, on their way to shared memory while the one before it is written
    const auto copy_ids = [&](int64_t from_at, int n, int64_t bias_at, int bias_n) {
        if (histories) {
#pragma unroll 1
            for (int c = tid; c < min(n, kIdsAhead); c += kThreads) copy_word(&s_ids[c], a.history + from_at + c);
        }
        if (biases) {
#pragma unroll 1
            for (int c = tid; c < min(bias_n, kBiasesAhead); c += kThreads) {
                copy_word(&s_bias_ids[c], a.bias_token + bias_at + c);
                copy_word(&s_bias_values[(half ^ 1) * kBiasesAhead + c], a.bias_value + bias_at + c);
            }
        }
    };
    bool ids_ahead = true;                               // whether this row's are
    {
        const int64_t start = histories ? a.history_start[row0] : 0, bias_start = biases ? a.bias_start[row0] : 0;
        const int len = histories ? a.history_len[row0] : 0, bias_len = biases ? a.bias_len[row0] : 0;
        int64_t from_at, bias_at;
        const int ids_n = inside(start, min(len, kMostLength), a.n_history, from_at), bias_n = inside(bias_start, min(bias_len, kMostBiases), a.n_bias, bias_at);
        copy_ids(from_at, ids_n, bias_at, bias_n);
        copies_end();
    }
    uint32_t raw_ahead = 0u;                             // touched vectors whose logits are on their way
    const auto flag = [&](int l, uint32_t bit) { atomicOr(reinterpret_cast<uint32_t*>(count) + (l >> 1), bit << ((l & 1) * 16)); };
    const auto add_one = [&](int l) {
        if ((count[l] & kTimes) < kMany) {
            atomicAdd(reinterpret_cast<uint32_t*>(count) + (l >> 1), 1u << ((l & 1) * 16));
            return;
        }
        frequent = true;
        count_frequent(s_frequent, l);
    };
    // kShift: records from here to the row's own have new tokens that are not in the tables yet
    int waiting = kBatch;
    const auto note = [&](const Record& r) {             // one of them, by one thread
        if (r.id < first || r.id - first >= n) return;
        const int l = r.id - first;
        if (!kBackward) {
            if (r.from < r.prompt) flag(l, kInPrompt);
            else add_one(l);
        }
        atomicOr(&s_touched[half][l >> 5], 1u << (l & 31));
    };
#pragma unroll 1
    for (int row = (int)row0 - (kDepth - 1); row < row_end; ++row) {
        int mask_ahead = -1;
        if (row >= row0) {
            if (at == kBatch) {                          // records of the rows from here on, by the first warp
                if (row > row0) __syncthreads();
                if (kShift && row > row0 && tid >= waiting && tid < kBatch) note(s_record[tid]);
                if (kShift) __syncwarp();
                waiting = 0;
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
                        r.mask = mask_of(mine);
                        r.mask_ahead = mask_of(mine + kDepth);
                        if (r.len < 0 || r.bias_len < 0) flags |= SR_STATUS_NEG_LEN;
                        if (r.bias_len > kMostBiases) flags |= SR_STATUS_BAD_INDEX;
                        r.len = min(max(r.len, 0), kMostLength);
                        r.bias_len = min(r.bias_len, kMostBiases);
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
                    const int done = max(r.from, 0);
                    r.n = inside(r.start + done, r.len - done, a.n_history, r.from_at);
                    r.behind = (int)(r.prompt - (r.from_at - r.start));
                    r.bias_n = inside(r.bias_start, r.bias_len, a.n_bias, r.bias_at);
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
            mask_ahead = r.mask_ahead;

            // the tables of this row
            if (r.from < 0 || r.len > r.from + 1) {
                if (kShift && row > row0) __syncthreads();           // the row before is done with them
                if (r.from < 0) half ^= 1;
                if (row > row0) {
                    if (r.from >= 0) {
                        if (kShift) {
                            if (tid >= waiting && tid < at - 1) note(s_record[tid]);
                        } else {                         // more than one new token: the owners' bits meet theirs
                            s_touched[half][tid] = word;
                            if (odd) atomicOr(&s_touched[half][kWords - 1], 1u << tid);
                        }
                    } else {
                        if (kShift) {
                            for (int i = tid; counts && i < kSlice / 8; i += kThreads) {
                                reinterpret_cast<uint4*>(count)[i] = make_uint4(0u, 0u, 0u, 0u);
                                if (biases) reinterpret_cast<uint4*>(entry)[i] = make_uint4(0u, 0u, 0u, 0u);
                            }
                            for (int i = tid; i < kWords; i += kThreads) s_touched[half][i] = 0u;
                        } else if (!kBackward) {
#pragma unroll
                            for (int k = 0; k < kVecs; ++k) {
                                if (bits_of_vector(word, k) == 0u) continue;
                                const int l0 = (tid + k * kThreads) * E;
#pragma unroll
                                for (int e = 0; e < E; e += 2) {
                                    *reinterpret_cast<uint32_t*>(count + l0 + e) = 0u;
                                    if (biases) *reinterpret_cast<uint32_t*>(entry + l0 + e) = 0u;
                                }
                            }
                            if (odd) {
                                count[vecs * E + tid] = 0u;
                                if (biases) entry[vecs * E + tid] = 0u;
                            }
                        }
                    }
                    if (__syncthreads_or(frequent) && r.from < 0) {
                        for (int i = tid; !kBackward && i < 2 * kFrequent; i += kThreads) s_frequent[i] = 0u;
                        frequent = false;
                        __syncthreads();
                    }
                }
                // ids of the bias list, then of the history, in the slice
                const bool copied = ids_ahead && r.from < 0;
                if (copied) copies_wait<kSparse ? 0 : kBackward ? 2 : 1>();
#pragma unroll 1
                for (int pass = biases && r.from < 0 ? 0 : 1; pass < 1 + histories; ++pass) {
                    const int ids_n = pass == 0 ? r.bias_n : r.n, behind = r.behind;
                    const int32_t* const ids = pass == 0 ? a.bias_token + r.bias_at : a.history + r.from_at;
                    const auto one = [&](int c, int32_t id) {
                        const uint32_t l = (uint32_t)id - (uint32_t)first;
                        if (id < 0 || l >= (uint32_t)n) {
                            if (id >= a.vocab) flags |= SR_STATUS_BAD_TARGET;
                            return;
                        }
                        if (!kBackward) {
                            if (pass == 0) {             // the largest index, in 16 bits of a word
                                uint32_t* const w = reinterpret_cast<uint32_t*>(entry) + (l >> 1);
                                const uint32_t sh = (l & 1) * 16, mine = (uint32_t)c + 1u;
                                for (uint32_t had = *w; ((had >> sh) & 0xFFFFu) < mine;) {
                                    const uint32_t now = atomicCAS(w, had, (had & ~(0xFFFFu << sh)) | mine << sh);
                                    if (now == had) break;
                                    had = now;
                                }
                                flag((int)l, kBiased);
                            } else if (c >= behind) {
                                add_one((int)l);
                            } else {
                                flag((int)l, kInPrompt);
                            }
                        }
                        if (kShift) {
                            atomicOr(&s_touched[half][l >> 5], 1u << (l & 31));
                        } else if ((int)l >= vecs * E) {
                            atomicOr(&s_touched[half][kWords - 1], 1u << (l - vecs * E));
                        } else {
                            atomicOr(&s_touched[half][l / E % kThreads], 1u << (l / E / kThreads * E + l % E));
                        }
                    };
                    int c = tid;
                    if (copied) {
                        const int32_t* const held = pass == 0 ? s_bias_ids : s_ids;
                        const int held_n = min(ids_n, pass == 0 ? kBiasesAhead : kIdsAhead);
#pragma unroll 1
                        for (; c < held_n; c += kThreads) one(c, held[c]);
                    } else if (pass == 0) {
                        for (int k = tid; k < min(ids_n, kBiasesAhead); k += kThreads) s_bias_values[half * kBiasesAhead + k] = a.bias_value[r.bias_at + k];
                    }
#pragma unroll 1
                    for (; c < ids_n; c += 4 * kThreads) {
                        int32_t id[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) id[k] = c + k * kThreads < ids_n ? ids[c + k * kThreads] : -1;
#pragma unroll 1
                        for (int k = 0; k < 4; ++k) one(c + k * kThreads, k == 0 ? id[0] : k == 1 ? id[1] : k == 2 ? id[2] : id[3]);
                    }
                }
                __syncthreads();
                waiting = at;
                if (!kShift) {
                    word = s_touched[half][tid];
                    odd = tid < E && ((s_touched[half][kWords - 1] >> tid) & 1u);
                    s_touched[half ^ 1][tid] = 0u;       // for the next time: all have read it before the barriers above
                    if (tid == 0) s_touched[half ^ 1][kWords - 1] = 0u;
                }
            } else if (!kShift && r.id >= first && r.id - first < n) {
                const int l = r.id - first;              // one new token: its owner notes it
                bool mine;
                if (l >= vecs * E) {
                    mine = l - vecs * E == tid;
                    odd |= mine;
                } else {
                    mine = l / E % kThreads == tid;
                    if (mine) word |= 1u << (l / E / kThreads * E + l % E);
                }
                if (mine && !kBackward) {                // others change other halves of a word meanwhile: atomics too
                    if (r.from >= r.prompt) add_one(l);
                    else flag(l, kInPrompt);
                }
            }
            if (kShift) {
                split(in, out, head, vecs);
                word = 0u;
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {
                    const int j = tid + k * kThreads;
                    if (j < vecs) word |= (bits_at(s_touched[half], head + j * E, E) & kAll) << (k * E);
                }
                for (int i = waiting; i < at; ++i) {
                    const int id = s_record[i].id, v = id - first - head;
                    if (id >= first && id - first < n && v >= 0 && v < vecs * E && v / E % kThreads == tid) word |= 1u << (v / E / kThreads * E + v % E);
                }
            }

            ids_ahead = at < kBatch && row + 1 < row_end && s_record[at < kBatch ? at : 0].from < 0;
            if (ids_ahead) copy_ids(s_record[at].from_at, s_record[at].n, s_record[at].bias_at, s_record[at].bias_n);
        }
        copies_end();

        // vectors of the last row that was looked up, and the mask of the next one
        MaskWords words = {};
        if (!kSparse) {
            if (row_ahead(row, kDepth - 1, row_end)) {
                const uint4* const p = reinterpret_cast<const uint4*>(in_ahead + head_ahead) + tid;
                uint4* const to = ring + fill * kFull;
#pragma unroll
                for (int k = 0; k < kVecs; ++k)
                    if (tid + k * kThreads < vecs_ahead && bits_of_vector(allowed[kDepth - 1], k) != 0u) copy_vector(to + k * kThreads, p + k * kThreads);
                const int edges = n - vecs_ahead * E;
                if (kShift && edges <= kEdges && tid < edges) edge[kDepth - 1] = in_ahead[tid < head_ahead ? tid : tid + vecs_ahead * E];
                in_ahead += a.pitch;
                fill = fill == kStages - 1 ? 0 : fill + 1;
            }
        }
        copies_end();
        if (row < row0) mask_ahead = mask_of((int64_t)row + kDepth);
        if (kShift && row_ahead(row, kDepth, row_end)) {
            const int64_t ahead = (int64_t)row + kDepth;
            split(static_cast<const T*>(a.in) + ahead * a.pitch + first, static_cast<T*>(a.out) + ahead * a.out_pitch + first, head_ahead, vecs_ahead);
        }
        if (a.allowed) words = words_of(mask_ahead, head_ahead, vecs_ahead);

        if (row >= row0) {
            const Record& r = s_record[at - 1];
            // This row.  16-bit logits are multiplied by the reciprocal, whose 2^-24 their last rounding (2^-9, 2^-12) hides.
            const auto changed = [&](int l, float v, bool positive) {
                const float repetition = r.repetition;
                const auto repeated = [&](bool larger) { return sizeof(T) == 4 ? (larger ? v / repetition : v * repetition) : v * (larger ? r.shrink : repetition); };
                if (kBackward) return repeated(positive);
                uint32_t c = count[l], times = c & kTimes, more = 0u;
                for (int i = waiting; kShift && i < at; ++i) {
                    if (s_record[i].id != first + l) continue;
                    if (s_record[i].from < s_record[i].prompt) c |= kInPrompt;
                    else ++more;
                }
                c |= more;                               // whether it was seen at all
                if (c & ~kBiased) v = repeated(v > 0.0f);
                if (times >= kMany) times = times_frequent(s_frequent, times, l, first + l, a.history, a.n_history, r, more);
                times += more;
                const float less = fmaf(-r.frequency, (float)times, v) - r.presence;
                v = times ? less : v;
                if (c & kBiased) {
                    const int e = (int)entry[l] - 1;
                    v += e < kBiasesAhead ? s_bias_values[half * kBiasesAhead + e] : a.bias_value[r.bias_at + e];
                }
                return v;
            };
            const auto touched_at = [&](int l) {
                bool is = (s_touched[half][l >> 5] >> (l & 31)) & 1u;
                for (int i = waiting; i < at; ++i) is |= s_record[i].id == first + l;
                return is;
            };
            // elements in no vector
#pragma unroll 1
            for (int i = tid; (kShift || vecs != kFull) && i < n - vecs * E; i += kThreads) {
                const int l = i < head ? i : i + vecs * E;
                const T v = kShift && !kSparse && n - vecs * E <= kEdges ? edge[0] : in[l];
                if (r.mask >= 0 && !((mask_at(r.mask)[l >> 5] >> (l & 31)) & 1u)) out[l] = banned_value<T>(kBackward);
                else if (kShift ? touched_at(l) : odd) out[l] = from_float<T>(changed(l, to_float(v), kBackward && to_float(raw[l]) > 0.0f));
                else if (!kSparse) out[l] = v;
            }
            uint4* const mine = ring + take * kFull;     // the thread's vectors
            take = take == kStages - 1 ? 0 : take + 1;
            if (kSparse) {
                const uint4* p = reinterpret_cast<const uint4*>(in + head) + tid;
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {        // those with a token that stays and one that changes
                    const uint32_t m = bits_of_vector(allowed[0], k), t = bits_of_vector(word, k);
                    if (tid + k * kThreads < vecs && m != 0u && (m != kAll || t != 0u)) copy_vector(mine + k * kThreads, p + k * kThreads);
                }
                copies_end();
                copies_wait<0>();
            } else if (!kBackward) {
                copies_wait<2 * kStages - 2>();
            } else {
                copies_wait<3 * kStages - 3>();
            }
            const uint32_t left = word & allowed[0];     // tokens that change, one after the other
            if (kBackward && !kShift && raw_ahead != 0u) copies_wait<2>();       // used or not: the next row's go to the same place
#pragma unroll 1
            for (uint32_t b = left; b != 0u; b &= b - 1u) {
                const int bit = __ffs(b) - 1, v = bit / E * kThreads, l = head + (tid + v) * E + bit % E;
                T* const x = reinterpret_cast<T*>(mine + v) + bit % E;
                bool positive = false;                   // the logit whose gradient this is
                if (kBackward) positive = to_float((raw_ahead >> bit) & 1u ? reinterpret_cast<const T*>(s_raw + tid + v)[bit % E] : raw[l]) > 0.0f;
                *x = from_float<T>(changed(l, to_float(*x), positive));
            }
            uint4* const to = reinterpret_cast<uint4*>(out + head) + tid;
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                if (tid + k * kThreads >= vecs) break;
                const uint32_t m = bits_of_vector(allowed[0], k);
                if (kSparse && m == kAll && bits_of_vector(word, k) == 0u) continue;
                uint4 q = mine[k * kThreads];
                if (m != kAll) {
                    q.x = cut<T, kBackward>(q.x, m, 0);
                    q.y = cut<T, kBackward>(q.y, m, 1);
                    q.z = cut<T, kBackward>(q.z, m, 2);
                    q.w = cut<T, kBackward>(q.w, m, 3);
                }
                store_once(to + k * kThreads, q);
            }
            if (kBackward && !kShift) {                  // the next row's logits of what is touched already
                raw_ahead = 0u;
                if (word != 0u && row + 1 < row_end && (reinterpret_cast<uintptr_t>(raw + a.logits_pitch) & 15) == 0) {
                    const uint4* const p = reinterpret_cast<const uint4*>(raw + a.logits_pitch) + tid;
#pragma unroll
                    for (int k = 0; k < kVecs; ++k) {
                        if (bits_of_vector(word & (kDepth > 1 ? allowed[kDepth > 1] : kEvery), k) == 0u) continue;
                        copy_vector(&s_raw[k * kThreads + tid], p + k * kThreads);
                        raw_ahead |= kAll << (k * E);
                    }
                }
            }
            in += a.pitch;
            out += a.out_pitch;
            if (kBackward) raw += a.logits_pitch;
        }
        if (kBackward) copies_end();
#pragma unroll
        for (int d = 0; d + 1 < kDepth; ++d) {
            allowed[d] = allowed[d + 1];
            if (kShift) edge[d] = edge[d + 1];
        }
        if (a.allowed) allowed[kDepth - 1] = bits_of(words, mask_ahead, head_ahead);
    }
    if (a.status && flags) atomicOr(a.status, flags);
}

// Whether rows mostly have histories of their own: many ids a row.  That goes by the length of the array, since the rows' own lengths lie on the device.
// Around the limit little hangs on it: with 1 to 64 ids a row and all rows beginning anew, 512 of 151936 bf16 take 58 to 64 us as rows that go on and 54 to 55
// as rows that begin anew, 2048 of 50024 76 to 85 and 77 to 82; rollouts of 64 rows behind prompts of 4000, 49 ids a row, are taken for rows that begin anew: 64 us, otherwise 70.
bool begin_anew(const AdjustArgs& a) { return a.n_history > 8 * (int64_t)a.n_rows; }

template <typename T, int kStages, bool kBackward, bool kSparse, bool kShift>
int launch_form(const AdjustArgs& a, cudaStream_t s) {
    constexpr int kSlice = kSliceOf<T>;
    const int slices = (a.vocab - 1) / kSlice + 1;
    // Few rows get a CTA each a slice; many are dealt out in runs, so that a rollout's rows find its history at hand, but leave every SM a few
    // turns: two, or three where rows begin anew and runs gain less (512 rows with biases and masks 143 -> 132 us; 601 rows of whole
    // rollouts 28 -> 31).  Turns are counted with four CTAs an SM, with three for the ring of three rows, before runs are rounded to whole rows and at most 64 of
    // them.  What is launched takes more: biases leave room for three CTAs only (512 rows of 151936 1634 CTAs, 3.7 turns of 444; 601 of 50021 1057, 2.4), and
    // roundings begin another turn (the gradient of 1200 x 4096 600 CTAs on 592 places, of 2048 x 151936 1197; 4096 rows without masks 1216 on 444).
    // Slices go from the lowest ids on: with most vocabularies these are the tokens that are seen most often, and whose CTAs take longest.
    const int64_t units = (int64_t)slices * a.n_rows;
    int64_t rows = std::min<int64_t>((units - 1) / (148 * (kStages == 3 ? 3 : 4) * (begin_anew(a) ? 3 : 2)) + 1, 64);
    rows = std::max(rows, (units - 1) / (INT32_MAX - slices) + 1);           // CTAs are numbered in 31 bits
    const int64_t runs = (a.n_rows - 1) / rows + 1, ctas = slices * runs;
    using Lay = Layout<T, kStages, kBackward>;
    const int smem = Lay::bytes(a.history_start != nullptr, a.bias_value != nullptr);
    const auto kernel = adjust_kernel<T, kStages, kBackward, kSparse, kShift>;
    SR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay::kAll));
    SR_LAUNCH("adjust_kernel", kernel, (int)ctas, kThreads, (size_t)smem, s, a, (int)runs, (int)rows);
    return SR_OK;
}
template <typename T, bool kBackward>
int launch_type(const AdjustArgs& a, cudaStream_t s) {
    const auto on_16 = [&](const void* p, int64_t pitch) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (a.n_rows == 1 || pitch * (int64_t)sizeof(T) % 16 == 0); };
    const bool shift = !on_16(a.in, a.pitch) || !on_16(a.out, a.out_pitch);
    if (a.in == a.out) return shift ? launch_form<T, 1, kBackward, true, true>(a, s) : launch_form<T, 1, kBackward, true, false>(a, s);
    // Rows that begin anew wait for their tables, not for memory: a ring of two rows leaves room for a fourth CTA (with penalties and three turns instead of
    // two, 512 rows of 151936 bf16 77 -> 61 us, 2048 292 -> 236).  Rows that go on where others ended stream: three rows, three CTAs.  That pays for the largest
    // calls (4096 rows of 151936 414 -> 410 us) and costs 4 to 9 % of smaller ones (2048 210 -> 221, 512 55 -> 60; 8192 of 50024 290 -> 306).
    // Biases take the room of a fourth CTA in any case, and the gradient has no counts that would (2048 rows 206 -> 180).
    const bool streams = !kBackward && a.bias_value == nullptr && !begin_anew(a);
    if (streams) return shift ? launch_form<T, 3, false, false, true>(a, s) : launch_form<T, 3, false, false, false>(a, s);
    return shift ? launch_form<T, 2, kBackward, false, true>(a, s) : launch_form<T, 2, kBackward, false, false>(a, s);
}

}  // namespace

int launch_adjust(const AdjustArgs& a, bool backward, cudaStream_t s) {
    if (a.n_rows == 0) return SR_OK;
    if (a.dtype == SR_DTYPE_F32) return backward ? launch_type<float, true>(a, s) : launch_type<float, false>(a, s);
    if (a.dtype == SR_DTYPE_BF16) return backward ? launch_type<__nv_bfloat16, true>(a, s) : launch_type<__nv_bfloat16, false>(a, s);
    return backward ? launch_type<__half, true>(a, s) : launch_type<__half, false>(a, s);
}

}  // namespace sr
