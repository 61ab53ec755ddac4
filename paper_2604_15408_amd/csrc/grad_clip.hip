// The norm over many tensors and their clipping, for gfx950:
//     norm = |s| sqrt(sum of g^2 over all tensors),   out = g s min(1, max_norm / (norm + 1e-6)).
//
// The tensors are cut into chunks of at most kChunk values, listed in a table that the host lays out once; a work-group takes
// chunk after chunk, whatever tensor it belongs to, so thousands of small tensors and a few large ones are the same work.
// grad_squares_kernel reads every value once and leaves one sum of squares for each work-group in the workspace;
// grad_scale_kernel: every work-group adds those up (the same order everywhere, so all have the same factor), and rewrites its chunks.
// Squares are formed and added in fp64: they are exact there (24-bit values), no gradient's square overflows or vanishes,
// and with one conversion and one fma a value the kernel stays bound by memory.
//
// us (both kernels): 151 M bf16 values into fp32 189 (squares 50: 6.0 TB/s; scaling 138: 6.6 TB/s of reads and writes), fp32 into fp32 297;
// 5.5 M fp32 values 14.2 to 14.9 (5.5 and 9.1 in the kernels by the profiler); 0.7 M bf16 into fp32 8.
#include "common.h"
#include "linear_kernel.h"

namespace ragged {
namespace {

constexpr int kChunk = 16384;                                  // values of a chunk (151 M bf16 into fp32: 8192 as fast, 32768 213 us)
// Outputs of more values than this go past the caches, which keeps the gradients there for the second reading: 151 M values 242 -> 206 us;
// that one then leaves them to others as well: 194.
// Fewer are left there for the optimiser (38 M into fp32 55 us, 53 past them).  Every chunk counts as a whole one: of thousands of small
// tensors, which are more than 2048 chunks with fewer values, the outputs go past the caches as well.
constexpr int64_t kClipBypass = 32 << 20;
constexpr int kClipGroups = 1024;                              // work-groups (and partial sums) at most
static_assert(kClipGroups * 8 <= RAGGED_GRAD_WORKSPACE, "one fp64 sum for each work-group");

struct GradChunk {
    const void* src;
    void* dst;                                                 // null: the chunk counts for the norm only
    int32_t n, src_dt, dst_dt, pad;
};
static_assert(sizeof(GradChunk) == RAGGED_GRAD_CHUNK_BYTES, "the table's layout");

// Values of a tensor, aligned to themselves only, in global memory (an address that comes out of a table could be anywhere for the compiler).
__device__ __forceinline__ float half_value(uint16_t w) { return (float)__builtin_bit_cast(_Float16, w); }
__device__ __forceinline__ float bfloat_value(uint16_t w) { return __builtin_bit_cast(float, (uint32_t)w << 16); }
__device__ __forceinline__ uint16_t half_word(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ uint16_t bfloat_word(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
template <int DT>
struct Grad {
    typedef uint16_t word;
    static __device__ __forceinline__ float value(uint16_t w) { return DT == RAGGED_F16 ? half_value(w) : bfloat_value(w); }
    static __device__ __forceinline__ uint16_t rounded(float v) { return DT == RAGGED_F16 ? half_word(v) : bfloat_word(v); }
};
template <>
struct Grad<RAGGED_F32> {
    typedef float word;
    static __device__ __forceinline__ float value(float w) { return w; }
    static __device__ __forceinline__ float rounded(float v) { return v; }
};
template <int DT, int W>
struct GradLine {
    typedef typename Grad<DT>::word word;
    typedef word line __attribute__((ext_vector_type(W), aligned(sizeof(word))));
    typedef __attribute__((address_space(1))) line global_line;
    typedef __attribute__((address_space(1))) word global_word;
    static __device__ __forceinline__ line load(const void* p, int i) {
        return *(const global_line*)((const global_word*)p + i);
    }
    static __device__ __forceinline__ line load_last(const void* p, int i) {
        return __builtin_nontemporal_load((const global_line*)((const global_word*)p + i));
    }
    static __device__ __forceinline__ word load1(const void* p, int i) { return ((const global_word*)p)[i]; }
    static __device__ __forceinline__ void store1(void* p, int i, word w) { ((global_word*)p)[i] = w; }
    template <bool BYPASS>
    static __device__ __forceinline__ void store(void* p, int i, line w) {
        if constexpr (BYPASS) __builtin_nontemporal_store(w, (global_line*)((global_word*)p + i));
        else *(global_line*)((global_word*)p + i) = w;
    }
};
// Lines a thread requests before it uses the first.
constexpr int kClipAhead = 4;

// Sum over the work-group in a fixed order, result in every thread.
__device__ __forceinline__ double group_sum(double v, double* lds) {
#pragma unroll
    for (int apart = 32; apart > 0; apart /= 2) v += __shfl_xor(v, apart);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <int DT>
__device__ __forceinline__ double chunk_squares(const void* src, int n) {
    constexpr int W = DT == RAGGED_F32 ? 4 : 8;                // 16 bytes
    typedef GradLine<DT, W> Line;
    double sum = 0.0;
    auto add = [&](const typename Line::line& w) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const double v = Grad<DT>::value(w[e]);
            sum = fma(v, v, sum);
        }
    };
    const int whole = n / W * W;
    int i = W * threadIdx.x;
    constexpr int kStep = W * kBlockThreads;
    for (; i + (kClipAhead - 1) * kStep < whole; i += kClipAhead * kStep) {
        typename Line::line w[kClipAhead];
#pragma unroll
        for (int u = 0; u < kClipAhead; ++u) w[u] = Line::load(src, i + u * kStep);
#pragma unroll
        for (int u = 0; u < kClipAhead; ++u) add(w[u]);
    }
    for (; i < whole; i += kStep) add(Line::load(src, i));
    if (whole + (int)threadIdx.x < n) {
        const double v = Grad<DT>::value(Line::load1(src, whole + threadIdx.x));
        sum = fma(v, v, sum);
    }
    return sum;
}

__global__ __launch_bounds__(kBlockThreads)
void grad_squares_kernel(const GradChunk* __restrict__ table, int chunks, double* __restrict__ partial) {
    __shared__ double lds[4];
    double sum = 0.0;
    GradChunk next = blockIdx.x < (unsigned)chunks ? table[blockIdx.x] : GradChunk{};
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const GradChunk t = next;
        if (c + (int)gridDim.x < chunks) next = table[c + gridDim.x];
        sum += t.src_dt == RAGGED_F32 ? chunk_squares<RAGGED_F32>(t.src, t.n)
             : t.src_dt == RAGGED_F16 ? chunk_squares<RAGGED_F16>(t.src, t.n) : chunk_squares<RAGGED_BF16>(t.src, t.n);
    }
    sum = group_sum(sum, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// The factor as fp32, with a power of two of its own where it lies below fp32's normal numbers: gradients of 1e38 clipped to a norm of 1 have 1e-40,
// in fp32 off by 2^-17 of itself, and outputs that are ordinary numbers.  (One instruction more a value; both kernels are bound by memory.)
struct Factor {
    float times;                                               // then in [1/2, 1)
    int power;
    static __device__ __forceinline__ Factor from(double f) {
        if (fabs(f) >= 0x1p-126) return {(float)f, 0};
        int power;
        const float times = (float)frexp(f, &power);
        return {times, power};
    }
    __device__ __forceinline__ float of(float v) const { return __builtin_ldexpf(v * times, power); }
};

template <int SRC, int DST, bool BYPASS>
__device__ __forceinline__ void chunk_scale(const void* src, void* dst, int n, Factor by) {
    constexpr int W = DST == RAGGED_F32 ? 4 : 8;               // 16 bytes of output
    typedef GradLine<SRC, W> In;
    typedef GradLine<DST, W> Out;
    auto scale = [&](const typename In::line& w, int i) {
        typename Out::line v;
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = Grad<DST>::rounded(by.of(Grad<SRC>::value(w[e])));
        Out::template store<BYPASS>(dst, i, v);
    };
    const int whole = n / W * W;
    int i = W * threadIdx.x;
    constexpr int kStep = W * kBlockThreads;
    for (; i + (kClipAhead - 1) * kStep < whole; i += kClipAhead * kStep) {
        typename In::line w[kClipAhead];
#pragma unroll
        for (int u = 0; u < kClipAhead; ++u) w[u] = BYPASS ? In::load_last(src, i + u * kStep) : In::load(src, i + u * kStep);
#pragma unroll
        for (int u = 0; u < kClipAhead; ++u) scale(w[u], i + u * kStep);
    }
    for (; i < whole; i += kStep) scale(In::load(src, i), i);
    if (whole + (int)threadIdx.x < n)
        Out::store1(dst, whole + threadIdx.x, Grad<DST>::rounded(by.of(Grad<SRC>::value(In::load1(src, whole + threadIdx.x)))));
}
template <int SRC, bool BYPASS>
__device__ __forceinline__ void chunk_scale(const GradChunk& t, Factor by) {
    if (t.dst_dt == RAGGED_F32) chunk_scale<SRC, RAGGED_F32, BYPASS>(t.src, t.dst, t.n, by);
    else chunk_scale<SRC, SRC, BYPASS>(t.src, t.dst, t.n, by);
}

template <bool BYPASS>
__global__ __launch_bounds__(kBlockThreads)
void grad_scale_kernel(const GradChunk* __restrict__ table, int chunks, const double* __restrict__ partial, int parts, float scale,
                       float max_norm, double* __restrict__ norm_out) {
    __shared__ double lds[4];
    double sum = 0.0;
    int c = chunks - 1 - (int)blockIdx.x;                      // from the end: what the first kernel read last is still cached
    GradChunk next = c >= 0 ? table[c] : GradChunk{};
    double part[kClipGroups / kBlockThreads];
#pragma unroll
    for (int i = 0; i < kClipGroups / kBlockThreads; ++i) part[i] = threadIdx.x + i * kBlockThreads < parts ? partial[threadIdx.x + i * kBlockThreads] : 0.0;
#pragma unroll
    for (int i = 0; i < kClipGroups / kBlockThreads; ++i) sum += part[i];
    const double norm = sqrt(group_sum(sum, lds)) * fabs((double)scale);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    // a norm that is no number or infinite clips nothing: the caller sees it in the norm
    double clip = isfinite(norm) ? (double)max_norm / (norm + 1e-6) : 1.0;
    clip = clip < 1.0 ? clip : 1.0;
    const Factor by = Factor::from(clip * (double)scale);
    for (; c >= 0; c -= gridDim.x) {
        const GradChunk t = next;
        if (c >= (int)gridDim.x) next = table[c - gridDim.x];
        if (!t.dst || (t.dst == t.src && by.times == 1.0f)) continue;
        if (t.src_dt == RAGGED_F32) chunk_scale<RAGGED_F32, BYPASS>(t, by);
        else if (t.src_dt == RAGGED_F16) chunk_scale<RAGGED_F16, BYPASS>(t, by);
        else chunk_scale<RAGGED_BF16, BYPASS>(t, by);
    }
}

int value_bytes(int dt) { return dt == RAGGED_F32 ? 4 : 2; }

}  // namespace

int64_t grad_chunks(const ragged_grad_tensor& t) { return (t.numel + kChunk - 1) / kChunk; }

void grad_table(const ragged_grad_tensor* tensors, int n, void* table) {
    GradChunk* out = static_cast<GradChunk*>(table);
    for (int i = 0; i < n; ++i) {
        const ragged_grad_tensor& t = tensors[i];
        for (int64_t at = 0; at < t.numel; at += kChunk) {
            const int64_t left = t.numel - at;
            *out++ = GradChunk{static_cast<const char*>(t.src) + at * value_bytes(t.src_dt),
                               t.dst ? static_cast<char*>(t.dst) + at * value_bytes(t.dst_dt) : nullptr,
                               (int32_t)(left < kChunk ? left : kChunk), t.src_dt, t.dst_dt, 0};
        }
    }
}

hipError_t launch_grad_clip(const void* table, int chunks, float scale, float max_norm, void* workspace, double* norm, hipStream_t stream) {
    const GradChunk* const t = static_cast<const GradChunk*>(table);
    double* const partial = static_cast<double*>(workspace);
    const int groups = chunks < 1 ? 1 : chunks < kClipGroups ? chunks : kClipGroups;
    const hipError_t err = launch_kernel(grad_squares_kernel, dim3(groups), dim3(kBlockThreads), stream, t, chunks, partial);
    if (err != hipSuccess) return err;
    const auto kernel = (int64_t)chunks * kChunk > kClipBypass ? grad_scale_kernel<true> : grad_scale_kernel<false>;
    return launch_kernel(kernel, dim3(groups), dim3(kBlockThreads), stream, t, chunks, static_cast<const double*>(partial), groups, scale, max_norm,
                         norm);
}

}  // namespace ragged
