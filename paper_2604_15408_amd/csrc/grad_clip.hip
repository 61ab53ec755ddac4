// The norm over many tensors and their clipping, for gfx950:
//     norm = |s| sqrt(sum of g^2 over all tensors),   out = g s min(1, max_norm / (norm + 1e-6)).
//
// The tensors are cut into chunks of at most kChunk values, listed in a table that the host lays out once; a work-group takes
// chunk after chunk, whatever tensor it belongs to, so thousands of small tensors and a few large ones are the same work.
// grad_squares_kernel reads every value once and leaves one sum of squares for each work-group in the workspace;
// grad_scale_kernel: every work-group adds those up (the same order everywhere, so all have the same factor), and rewrites its chunks.
// Squares are formed and added in fp64: they are exact there (24-bit values), no gradient's square overflows or vanishes,
// and with one conversion and one fma a value the kernel stays bound by memory.
#include "common.h"
#include "linear_kernel.h"

namespace ragged {
namespace {

constexpr int kChunk = 16384;                                  // values of a chunk
constexpr int kClipGroups = 2048;                              // work-groups (and partial sums) at most
static_assert(kClipGroups * 8 <= RAGGED_GRAD_WORKSPACE, "one fp64 sum for each work-group");

struct GradChunk {
    const void* src;
    void* dst;                                                 // null: the chunk counts for the norm only
    int32_t n, src_dt, dst_dt, pad;
};
static_assert(sizeof(GradChunk) == RAGGED_GRAD_CHUNK_BYTES, "the table's layout");

// Eight values of a tensor that is aligned to its own values only.
typedef uint16_t u16x8 __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x8 __attribute__((ext_vector_type(8), aligned(4)));
__device__ __forceinline__ float half_value(uint16_t w) { return (float)__builtin_bit_cast(_Float16, w); }
__device__ __forceinline__ float bfloat_value(uint16_t w) { return __builtin_bit_cast(float, (uint32_t)w << 16); }
__device__ __forceinline__ uint16_t half_word(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ uint16_t bfloat_word(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

template <int DT>
__device__ __forceinline__ void load8(const void* p, int64_t i, float (&v)[8]) {
    if (DT == RAGGED_F32) {
        const f32x8 w = *reinterpret_cast<const f32x8*>(static_cast<const float*>(p) + i);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = w[e];
    } else {
        const u16x8 w = *reinterpret_cast<const u16x8*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = DT == RAGGED_F16 ? half_value(w[e]) : bfloat_value(w[e]);
    }
}
template <int DT>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
    if (DT == RAGGED_F32) return static_cast<const float*>(p)[i];
    const uint16_t w = static_cast<const uint16_t*>(p)[i];
    return DT == RAGGED_F16 ? half_value(w) : bfloat_value(w);
}
template <int DT>
__device__ __forceinline__ void store1(void* p, int64_t i, float v) {
    if (DT == RAGGED_F32) static_cast<float*>(p)[i] = v;
    else static_cast<uint16_t*>(p)[i] = DT == RAGGED_F16 ? half_word(v) : bfloat_word(v);
}
template <int DT>
__device__ __forceinline__ void store8(void* p, int64_t i, const float (&v)[8]) {
    if (DT == RAGGED_F32) {
        f32x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = v[e];
        *reinterpret_cast<f32x8*>(static_cast<float*>(p) + i) = w;
    } else {
        u16x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = DT == RAGGED_F16 ? half_word(v[e]) : bfloat_word(v[e]);
        *reinterpret_cast<u16x8*>(static_cast<uint16_t*>(p) + i) = w;
    }
}

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
    double sum = 0.0;
    const int whole = n & ~7;
    for (int i = 8 * threadIdx.x; i < whole; i += 8 * kBlockThreads) {
        float v[8];
        load8<DT>(src, i, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma((double)v[e], (double)v[e], sum);
    }
    if (whole + (int)threadIdx.x < n) {
        const double v = load1<DT>(src, whole + threadIdx.x);
        sum = fma(v, v, sum);
    }
    return sum;
}

__global__ __launch_bounds__(kBlockThreads)
void grad_squares_kernel(const GradChunk* __restrict__ table, int chunks, double* __restrict__ partial) {
    __shared__ double lds[4];
    double sum = 0.0;
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const GradChunk t = table[c];
        sum += t.src_dt == RAGGED_F32 ? chunk_squares<RAGGED_F32>(t.src, t.n)
             : t.src_dt == RAGGED_F16 ? chunk_squares<RAGGED_F16>(t.src, t.n) : chunk_squares<RAGGED_BF16>(t.src, t.n);
    }
    sum = group_sum(sum, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <int SRC, int DST>
__device__ __forceinline__ void chunk_scale(const void* src, void* dst, int n, float factor) {
    const int whole = n & ~7;
    for (int i = 8 * threadIdx.x; i < whole; i += 8 * kBlockThreads) {
        float v[8];
        load8<SRC>(src, i, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= factor;
        store8<DST>(dst, i, v);
    }
    if (whole + (int)threadIdx.x < n) store1<DST>(dst, whole + threadIdx.x, load1<SRC>(src, whole + threadIdx.x) * factor);
}
template <int SRC>
__device__ __forceinline__ void chunk_scale(const GradChunk& t, float factor) {
    if (t.dst_dt == RAGGED_F32) chunk_scale<SRC, RAGGED_F32>(t.src, t.dst, t.n, factor);
    else chunk_scale<SRC, SRC == RAGGED_F32 ? RAGGED_F32 : SRC>(t.src, t.dst, t.n, factor);
}

__global__ __launch_bounds__(kBlockThreads)
void grad_scale_kernel(const GradChunk* __restrict__ table, int chunks, const double* __restrict__ partial, int parts, float scale,
                       float max_norm, double* __restrict__ norm_out) {
    __shared__ double lds[4];
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kBlockThreads) sum += partial[i];
    const double norm = sqrt(group_sum(sum, lds)) * fabs((double)scale);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    // a norm that is no number or infinite clips nothing: the caller sees it in the norm
    double clip = isfinite(norm) ? (double)max_norm / (norm + 1e-6) : 1.0;
    clip = clip < 1.0 ? clip : 1.0;
    const float factor = (float)(clip * (double)scale);
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const GradChunk t = table[c];
        if (!t.dst || (t.dst == t.src && factor == 1.0f)) continue;
        if (t.src_dt == RAGGED_F32) chunk_scale<RAGGED_F32>(t, factor);
        else if (t.src_dt == RAGGED_F16) chunk_scale<RAGGED_F16>(t, factor);
        else chunk_scale<RAGGED_BF16>(t, factor);
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
    return launch_kernel(grad_scale_kernel, dim3(groups), dim3(kBlockThreads), stream, t, chunks, static_cast<const double*>(partial), groups,
                         scale, max_norm, norm);
}

}  // namespace ragged
