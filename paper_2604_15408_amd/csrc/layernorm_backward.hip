// The backward pass of LayerNorm over packed rows, for gfx950.  With xh = (x - mean) rstd and w = gamma dy, all of one row,
//     dx = rstd (w - mean(w) - xh mean(w xh)) [+ res],   dgamma = sum over rows of dy xh,   dbeta = sum over rows of dy.
//
// layernorm_backward_kernel: 16, 32 or 64 lanes a row as in the forward pass, the row's x and dy in registers, so that mean and
//   variance are formed again from x (which is read anyway: nothing needs to be kept from the forward pass).  A lane has the same
//   columns in all the rows that it takes and adds up their share of dgamma and dbeta in registers; a work-group adds those of its
//   lanes up through LDS and leaves one partial sum for each column in the workspace.
// layernorm_sums_kernel: adds up the partial sums of the work-groups, always in the same order.
// Bound by memory: x, dy and res in, dx out.  25 216 x 1024 fp16 with residual (206 MB) 37 us over and over, of which 33 the rows, 42 from HBM.
#include <type_traits>

#include "common.h"
#include "lane_sums.h"
#include "linear_kernel.h"

namespace ragged {
namespace {

constexpr int kLnbGroups = 512;                                // work-groups at most: two on a CU
constexpr int kSumThreads = 1024, kSumColumns = 32;

template <int AUX>
__device__ __forceinline__ LinearLine<8> load_chunk(__amdgpu_buffer_rsrc_t rsrc, uint32_t voff) {
    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff, 0, AUX);
    return __builtin_bit_cast(LinearLine<8>, v);
}

// LAST: loads and stores that leave the caches to others.  Nothing of the inputs is used again; from HBM, with residual, 25 216 x 1024 47 us
// without and 42 with it, 12 608 x 2048 49 and 44, without residual 25 216 x 768 30.5 and 28, and with a kernel that reads dx next 56.5 / 52.4,
// 58.6 / 54.6, 37.4 / 35.8.  Smaller tensors, mostly still in the caches from the kernel that wrote them, gain nothing (25 216 x 192 17.5 / 18.2).
constexpr int64_t kLnbLast = 32 << 20;                         // bytes of dx from which on
template <typename In, int L, int NC, bool LAST>
__global__ __launch_bounds__(kBlockThreads)
void layernorm_backward_kernel(const uint16_t* __restrict__ x, const uint16_t* __restrict__ gamma, const uint16_t* dy, const uint16_t* res,
                               uint16_t* dx, float* __restrict__ partial, int rows_cap, const int32_t* __restrict__ rows_dev, int C,
                               float eps) {                    // dx may be dy or res: no restrict
    typedef LinearLine<8> Chunk;
    constexpr int kRows = kWaveSize / L;                       // rows of a wavefront at a time
    constexpr int kGroupRows = kBlockThreads / L;              // rows of a work-group at a time
    constexpr int kAux = LAST ? 2 : 0;                         // the non-temporal bit of a buffer access
    __shared__ float sums[NC * 8 * kBlockThreads];
    int given = rows_cap;
    if (rows_dev) { const int r = *rows_dev; given = r < given ? r : given; }
    const int rows = __builtin_amdgcn_readfirstlane(given);
    if ((int64_t)blockIdx.x * kGroupRows >= rows) return;      // (its partial sums are not read)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & (kWaveSize - 1), sub = lane % L;
    const uint32_t row_bytes = (uint32_t)C * 2u;
    auto there = [&](int i) { return 8 * (sub + L * i) < C; };
    // of chunk i, `first` bytes behind its buffer's start; a chunk that is not there lies outside of every buffer
    auto offset = [&](int i, uint32_t first) -> uint32_t { return there(i) ? first + 16u * (sub + L * i) : 1u << 31; };
    const uint32_t lane_row = lane / L * row_bytes;
    Chunk g_raw[NC];
    {
        const __amdgpu_buffer_rsrc_t r = buf_rsrc(gamma, row_bytes);
#pragma unroll
        for (int i = 0; i < NC; ++i) g_raw[i] = Chunk::load(r, offset(i, 0));
    }
    float dg[NC][8] = {}, db[NC][8] = {};
    const float inv_c = 1.0f / (float)C;
    for (int64_t row = (int64_t)blockIdx.x * kGroupRows + wave * kRows; row < rows; row += (int64_t)gridDim.x * kGroupRows) {
        const uint32_t records = (uint32_t)(rows - row < kRows ? rows - row : kRows) * row_bytes;
        const __amdgpu_buffer_rsrc_t x_rsrc = buf_rsrc(x + row * C, records), dy_rsrc = buf_rsrc(dy + row * C, records);
        Chunk x_raw[NC], dy_raw[NC], res_raw[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            x_raw[i] = load_chunk<kAux>(x_rsrc, offset(i, lane_row));
            dy_raw[i] = load_chunk<kAux>(dy_rsrc, offset(i, lane_row));
        }
        if (res) {
            const __amdgpu_buffer_rsrc_t res_rsrc = buf_rsrc(res + row * C, records);
#pragma unroll
            for (int i = 0; i < NC; ++i) res_raw[i] = load_chunk<kAux>(res_rsrc, offset(i, lane_row));
        }
        float v[NC][8], sum = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            x_raw[i].unpack(In{}, v[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v[i][e];
        }
        const float mean = lanes_sum_f32<L>(sum) / (float)C;
        float square = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const float centre = there(i) ? mean : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] -= centre;
                square = __builtin_fmaf(v[i][e], v[i][e], square);
            }
        }
        // (a lane behind the last row adds nothing to the sums, whatever eps is)
        const float rstd = row + lane / L < rows ? 1.0f / sqrtf(lanes_sum_f32<L>(square) / (float)C + eps) : 0.f;
        float w[NC][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            float gm[8];
            g_raw[i].unpack(In{}, gm);
            dy_raw[i].unpack(In{}, w[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] *= rstd;                               // xh
                dg[i][e] = __builtin_fmaf(w[i][e], v[i][e], dg[i][e]);
                db[i][e] += w[i][e];
                w[i][e] *= gm[e];
                s1 += w[i][e];
                s2 = __builtin_fmaf(w[i][e], v[i][e], s2);
            }
        }
        s1 = lanes_sum_f32<L>(s1) * inv_c;
        s2 = lanes_sum_f32<L>(s2) * inv_c;
        const __amdgpu_buffer_rsrc_t dx_rsrc = buf_rsrc(dx + row * C, records);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            float out[8], add[8] = {};
            if (res) res_raw[i].unpack(In{}, add);
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = __builtin_fmaf(rstd, w[i][e] - s1 - v[i][e] * s2, add[e]);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, Chunk::pack(In{}, out)), dx_rsrc, offset(i, lane_row), 0, kAux);
        }
    }
    // the lanes of the work-group that share a column: one value each, column sub + L i of lane-row threadIdx / L
    const int lane_rows = kGroupRows, my = threadIdx.x / L;
    float* const out = partial + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (which) __syncthreads();
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[(my * NC * L + L * i + sub) * 8 + e] = which ? db[i][e] : dg[i][e];
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += kBlockThreads) {
            float total = sums[c];
            for (int r = 1; r < lane_rows; ++r) total += sums[r * NC * L * 8 + c];
            out[which * C + c] = total;
        }
    }
}

// sums[j] = sum over the work-groups that had rows of partial[group][j], j < 2 C: dgamma, then dbeta
__global__ __launch_bounds__(kSumThreads)
void layernorm_sums_kernel(const float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta, int groups, int group_rows,
                           int rows_cap, const int32_t* __restrict__ rows_dev, int C) {
    constexpr int kSlices = kSumThreads / kSumColumns;
    __shared__ float part[kSlices][kSumColumns];
    int rows = rows_cap;
    if (rows_dev) { const int r = *rows_dev; rows = r < rows ? r : rows; }
    rows = rows < 0 ? 0 : rows;
    const int64_t with_rows = ((int64_t)rows + group_rows - 1) / group_rows;
    const int n = with_rows < groups ? (int)with_rows : groups;
    const int slice = threadIdx.x / kSumColumns, col = threadIdx.x % kSumColumns, j = blockIdx.x * kSumColumns + col;
    float total = 0.f;
    if (j < 2 * C) {
#pragma unroll 8
        for (int g = slice; g < n; g += kSlices) total += partial[(int64_t)g * 2 * C + j];
    }
    part[slice][col] = total;
    __syncthreads();
    if (slice == 0 && j < 2 * C) {
        float sum = part[0][col];
#pragma unroll
        for (int s = 1; s < kSlices; ++s) sum += part[s][col];
        (j < C ? dgamma[j] : dbeta[j - C]) = sum;
    }
}

struct LnbShape { int lanes, groups; };
LnbShape lnb_shape(int64_t rows_cap, int C) {
    const int lanes = C <= 256 ? 16 : C <= 768 ? 32 : 64;
    const int64_t per = kBlockThreads / lanes, all = (rows_cap + per - 1) / per;
    return {lanes, (int)(all < kLnbGroups ? all : kLnbGroups)};
}

}  // namespace

int64_t layernorm_backward_workspace(int64_t rows_cap, int C) { return (int64_t)lnb_shape(rows_cap, C).groups * 2 * C * 4; }

hipError_t launch_layernorm_backward(const void* x, const void* gamma, const void* dy, const void* res, void* dx, float* dgamma, float* dbeta,
                                     void* workspace, int rows_cap, const int32_t* rows_dev, int C, float eps, ragged_dtype dt,
                                     hipStream_t stream) {
    const LnbShape shape = lnb_shape(rows_cap, C);
    float* const partial = static_cast<float*>(workspace);
    auto launch = [&](auto kernel) {
        return launch_kernel(kernel, dim3(shape.groups), dim3(kBlockThreads), stream, static_cast<const uint16_t*>(x),
                             static_cast<const uint16_t*>(gamma), static_cast<const uint16_t*>(dy), static_cast<const uint16_t*>(res),
                             static_cast<uint16_t*>(dx), partial, rows_cap, rows_dev, C, eps);
    };
    const int chunks = (C / 8 + shape.lanes - 1) / shape.lanes;
    auto form = [&](auto in, auto last) {
        typedef decltype(in) In;
        constexpr bool LAST = decltype(last)::value;
#define LNB_FORM(L, NC) if (shape.lanes == L && chunks == NC) return launch(layernorm_backward_kernel<In, L, NC, LAST>);
        LNB_FORM(16, 1) LNB_FORM(16, 2) LNB_FORM(32, 2) LNB_FORM(32, 3) LNB_FORM(64, 2) LNB_FORM(64, 3)
        return launch(layernorm_backward_kernel<In, 64, 4, LAST>);
#undef LNB_FORM
    };
    auto typed = [&](auto in) {
        return (int64_t)rows_cap * C * 2 > kLnbLast ? form(in, std::true_type{}) : form(in, std::false_type{});
    };
    const hipError_t err = dt == RAGGED_F16 ? typed(F16{}) : typed(BF16{});
    if (err != hipSuccess) return err;
    return launch_kernel(layernorm_sums_kernel, dim3((2 * C + kSumColumns - 1) / kSumColumns), dim3(kSumThreads), stream,
                         static_cast<const float*>(partial), dgamma, dbeta, shape.groups, kBlockThreads / shape.lanes, rows_cap, rows_dev, C);
}

}  // namespace ragged
