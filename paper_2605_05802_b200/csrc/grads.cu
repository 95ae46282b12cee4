// Global gradient norm and clipping over a list of tensors.
//
// The list travels as a kernel argument: no copy to the device, nothing to keep between calls, and a captured call holds its
// own.  Tensors are cut into pieces of 16 KB and the pieces dealt out evenly, as runs, to a grid that fills the GPU; a CTA
// searches the tensor of its first piece and walks on from there.  Both kernels are bound by HBM: the norm reads every
// gradient once, clipping reads and writes it (the factor is known only when all squares are added up).  1.9 GB of bf16: 885 us for
// both, 6.4 TB/s (pieces of 32 KB: 900); 392 small fp32 tensors, 65 MB: 38 us.  Loads of the norm leave in L2 what fits: clipping
// finds it there (with loads that do not, 41 us).
//
// Squares of 32 bytes a thread are added in fp32, and such sums in fp64.  Where a sum of squares leaves the range
// in which fp32 squares keep their digits (gradients around 2^60 and above, or 2^-50 and below), its elements are squared
// again in fp64.
#include "logits.cuh"

namespace sr {
namespace {

constexpr int kGradThreads = 256;
constexpr int kVecsInFlight = 4;
constexpr int kPieceBytes = kGradPiece;
static_assert(kPieceBytes == kGradThreads * kVecsInFlight * 16, "a piece is what a CTA has in flight");
constexpr int kGradCtas = 148 * 6;

// kCap tensors; a kernel argument may have 32764 bytes.
template <int kCap>
struct GradList {
    const void* src[kCap];
    void* dst[kCap];
    int64_t count[kCap];
    int32_t piece[kCap + 1];         // first piece of each tensor, and the number of pieces
    uint8_t dtype[kCap];
    int32_t n;
};
constexpr int kFew = 32, kMany = 768;
static_assert(sizeof(GradList<kMany>) < 32000, "kernel argument");

// Calls body(tensor, first element, elements) for every piece of this CTA, in order.
template <int kCap, typename Body>
__device__ __forceinline__ void for_pieces(const GradList<kCap>& list, Body body) {
    const int total = list.piece[list.n];
    const int begin = (int)((long long)total * blockIdx.x / gridDim.x), end = (int)((long long)total * (blockIdx.x + 1) / gridDim.x);
    if (begin >= end) return;
    int lo = 0, hi = list.n;                       // last tensor whose first piece is not behind `begin`
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list.piece[mid] <= begin) lo = mid;
        else hi = mid;
    }
    for (int p = begin; p < end; ++p) {
        while (list.piece[lo + 1] <= p) ++lo;
        const int size = list.dtype[lo] == SR_DTYPE_F32 ? 4 : 2;
        const int64_t at = (int64_t)(p - list.piece[lo]) * (kPieceBytes / size);
        body(lo, at, (int)min((int64_t)(kPieceBytes / size), list.count[lo] - at));
    }
}

// Sum of squares of N elements in fp64.
template <int N>
__device__ __forceinline__ double square_sum(const float (&x)[N]) {
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < N; ++k) s[k & 3] = fmaf(x[k], x[k], s[k & 3]);
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    if (sum > 0x1p-100f && sum < 0x1p120f) return (double)sum;
    double exact = 0.0;
#pragma unroll
    for (int k = 0; k < N; ++k) exact += (double)x[k] * (double)x[k];
    return exact;
}

template <typename T>
__device__ __forceinline__ double piece_square_sum(const T* p, int n) {
    constexpr int E = Vec<T>::kElems;
    const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15) / (int)sizeof(T);
    const int head = min(n, off ? E - off : 0), vecs = (n - head) / E, tail = n - head - vecs * E;
    double sum = 0.0;
    if ((int)threadIdx.x < head + tail) {
        const float x[1] = {to_float(p[(int)threadIdx.x < head ? threadIdx.x : vecs * E + threadIdx.x])};
        sum += square_sum(x);
    }
    const uint4* body = reinterpret_cast<const uint4*>(p + head);
    uint4 q[kVecsInFlight];
#pragma unroll
    for (int k = 0; k < kVecsInFlight; ++k) {
        const int i = threadIdx.x + k * kGradThreads;
        q[k] = i < vecs ? body[i] : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < kVecsInFlight; k += 2) {
        if ((q[k].x | q[k].y | q[k].z | q[k].w | q[k + 1].x | q[k + 1].y | q[k + 1].z | q[k + 1].w) == 0u) continue;
        float a[E], b[E], x[2 * E];
        unpack(q[k], a, T());
        unpack(q[k + 1], b, T());
#pragma unroll
        for (int j = 0; j < E; ++j) { x[j] = a[j]; x[E + j] = b[j]; }
        sum += square_sum(x);
    }
    return sum;
}

// Sum over a CTA in thread 0, in an order that depends on the thread count alone.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double s_warp[32];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (unsigned w = 1; w < blockDim.x >> 5; ++w) v += s_warp[w];
    return v;
}

template <int kCap>
__global__ void __launch_bounds__(kGradThreads)
grad_squares_kernel(const __grid_constant__ GradList<kCap> list, double* partial) {
    grid_begin();
    double sum = 0.0;
    for_pieces(list, [&](int i, int64_t at, int n) {
        if (list.dtype[i] == SR_DTYPE_F32) sum += piece_square_sum(static_cast<const float*>(list.src[i]) + at, n);
        else if (list.dtype[i] == SR_DTYPE_BF16) sum += piece_square_sum(static_cast<const __nv_bfloat16*>(list.src[i]) + at, n);
        else sum += piece_square_sum(static_cast<const __half*>(list.src[i]) + at, n);
    });
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(1024)
grad_norm_kernel(const double* partial, int n, float* norm) {
    grid_begin();
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += 1024) sum += partial[i];
    sum = block_sum(sum);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

template <typename T>
__device__ __forceinline__ void scale_piece(const T* p, T* out, int n, float factor) {
    constexpr int E = Vec<T>::kElems;
    const bool vec = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    if (!vec) {
        for (int i = threadIdx.x; i < n; i += kGradThreads) out[i] = from_float<T>(to_float(p[i]) * factor);
        return;
    }
    const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15) / (int)sizeof(T);
    const int head = min(n, off ? E - off : 0), vecs = (n - head) / E, tail = n - head - vecs * E;
    if ((int)threadIdx.x < head + tail) {
        const int i = (int)threadIdx.x < head ? threadIdx.x : vecs * E + threadIdx.x;
        out[i] = from_float<T>(to_float(p[i]) * factor);
    }
    const uint4* body = reinterpret_cast<const uint4*>(p + head);
    uint4* to = reinterpret_cast<uint4*>(out + head);
    uint4 q[kVecsInFlight];
#pragma unroll
    for (int k = 0; k < kVecsInFlight; ++k) {
        const int i = threadIdx.x + k * kGradThreads;
        if (i < vecs) q[k] = body[i];
    }
#pragma unroll
    for (int k = 0; k < kVecsInFlight; ++k) {
        const int i = threadIdx.x + k * kGradThreads;
        if (i >= vecs) break;
        float x[E];
        unpack(q[k], x, T());
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] *= factor;
        to[i] = pack(x, T());
    }
}

template <int kCap>
__global__ void __launch_bounds__(kGradThreads)
clip_grads_kernel(const __grid_constant__ GradList<kCap> list, const float* norm, float max_norm, int32_t* status) {
    grid_begin();
    const float total = *norm;
    const bool finite = isfinite(total);
    if (!finite && status && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(status, SR_STATUS_NONFINITE);
    const float factor = finite ? fminf(1.0f, __fdiv_rn(max_norm, total + 1e-6f)) : 1.0f;
    for_pieces(list, [&](int i, int64_t at, int n) {
        if (factor == 1.0f && list.dst[i] == list.src[i]) return;
        if (list.dtype[i] == SR_DTYPE_F32) scale_piece(static_cast<const float*>(list.src[i]) + at, static_cast<float*>(list.dst[i]) + at, n, factor);
        else if (list.dtype[i] == SR_DTYPE_BF16) scale_piece(static_cast<const __nv_bfloat16*>(list.src[i]) + at, static_cast<__nv_bfloat16*>(list.dst[i]) + at, n, factor);
        else scale_piece(static_cast<const __half*>(list.src[i]) + at, static_cast<__half*>(list.dst[i]) + at, n, factor);
    });
}

// Calls launch_list(list, CTAs) for the tensors, as many at a time as one kernel argument holds.  Their pieces are at most
// INT32_MAX: the caller has counted them.
template <int kCap, typename Launch>
int for_lists(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n_tensors, void* const* out, Launch launch_list) {
    GradList<kCap> list;
    for (int at = 0; at < n_tensors;) {
        int64_t pieces = 0;
        int n = 0;
        for (; at < n_tensors && n < kCap; ++at) {
            if (counts[at] == 0) continue;
            list.src[n] = grads[at];
            list.dst[n] = out ? out[at] : const_cast<void*>(grads[at]);
            list.count[n] = counts[at];
            list.dtype[n] = (uint8_t)dtypes[at];
            list.piece[n++] = (int32_t)pieces;
            pieces += grad_pieces(counts[at], dtypes[at]);
        }
        if (n == 0) break;
        list.piece[n] = (int32_t)pieces;
        list.n = n;
        const int rc = launch_list(list, (int)(pieces < kGradCtas ? pieces : kGradCtas));
        if (rc != SR_OK) return rc;
    }
    return SR_OK;
}

}  // namespace

size_t grad_norm_workspace_bytes(int32_t n_tensors) {
    const size_t lists = n_tensors <= kFew ? 1 : ((size_t)n_tensors + kMany - 1) / kMany;
    return lists * kGradCtas * sizeof(double);
}

int launch_grad_norm(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n_tensors, float* norm, void* ws, cudaStream_t s) {
    double* const partial = static_cast<double*>(ws);
    int used = 0;
    const auto squares = [&](const auto& list, int ctas) {
        const int rc = launch("grad_squares_kernel", grad_squares_kernel<sizeof(list.dtype)>, ctas, kGradThreads, 0, s, list, partial + used);
        used += ctas;
        return rc;
    };
    const int rc = n_tensors <= kFew ? for_lists<kFew>(grads, counts, dtypes, n_tensors, nullptr, squares) : for_lists<kMany>(grads, counts, dtypes, n_tensors, nullptr, squares);
    if (rc != SR_OK) return rc;
    SR_LAUNCH("grad_norm_kernel", grad_norm_kernel, 1, 1024, 0, s, partial, used, norm);
    return SR_OK;
}

int launch_clip_grads(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n_tensors, const float* norm, float max_norm,
                      void* const* out, int32_t* status, cudaStream_t s) {
    const auto clip = [&](const auto& list, int ctas) {
        return launch("clip_grads_kernel", clip_grads_kernel<sizeof(list.dtype)>, ctas, kGradThreads, 0, s, list, norm, max_norm, status);
    };
    return n_tensors <= kFew ? for_lists<kFew>(grads, counts, dtypes, n_tensors, out, clip) : for_lists<kMany>(grads, counts, dtypes, n_tensors, out, clip);
}

}  // namespace sr
