// The gradients of attention over a packed ragged buffer, for gfx950.  With c the scale, L the row statistics of the forward pass
// and delta_i = sum over d of dO_id O_id,
//     P_ij = exp(c q_i.k_j - L_i),   dP_ij = dO_i.v_j,   dS_ij = P_ij (dP_ij - delta_i),
//     dV = P^T dO,   dK = c dS^T Q,   dQ = c dS K.
//
// One launch, no atomics, no workspace: a work-group owns 64 rows of one (image, head), either as KEYS, whose dK and dV it sums up
// over all query tiles, or as QUERIES, whose dQ it sums up over all key tiles.  Both form P and dP again from 16-bit rows
// (seven products instead of the five that a pass over both at once would need), which is what lets every sum have one owner and one order.
//
// The two roles are one piece of code with the operands exchanged.  A wavefront owns 16 rows ("columns" below: the MFMA's column
// dimension); tiles of the other side's 64 rows stream through a ring in LDS by direct loads, two operands at a time:
//     keys:    columns are keys,    tile A = Q, B = dO:   S = Q K^T,   dP = dO V^T;   dV^T += dO^T P,   dK^T += Q^T dS
//     queries: columns are queries, tile A = K, B = V :   S^T = K Q^T, dP^T = V dO^T;                   dQ^T += K^T dS^T
// As in the forward pass the first products leave each lane with the scores of ONE column and tile rows 4 (lane/16) + r of every 16,
// which is the B operand that the second products want, and those read the same row-major tiles transposed: P and dS never leave
// registers.  LDS layout, swizzle and operand addresses are those of the forward kernel (attn.hip).
//
// P and dS are rounded to the input type for the second products, as the gradients themselves are in the end: a sum of n terms
// whose signs are mixed is off by about as much as its own rounding.  Sums are fp32.
#include "attn_parts.h"
#include "common.h"
#include "mfma_lds.h"

namespace ragged {
namespace {

constexpr int kGroupPairs = 512;        // (image, head) pairs of a dispatch batch, as in the forward pass
constexpr int kRingBytes = 2 * 2 * kTileBytes;

struct BackwardArgs {
    const uint16_t *q, *k, *v, *o, *d_o;
    uint16_t *dq, *dk, *dv;
    const float* lse;                   // [rows, H]
    const int32_t* cu_seqlens;
    int H, pairs, group, in_tok, out_tok, grad_tok;
    uint32_t h_magic;
    float scale;
};

// Sum over d of a[d] b[d], 16 values.
template <typename In>
__device__ __forceinline__ float dot16(const uint4 (&a)[2], const uint4 (&b)[2]) {
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const typename In::vec8 x = as_vec8<typename In::vec8>(a[h]), y = as_vec8<typename In::vec8>(b[h]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf((float)x[e], (float)y[e], sum);
    }
    return sum;
}

// Eight fp32 values of a lane as one operand of a product.
__device__ __forceinline__ f16x8 operand(F16, const f32x4& lo, const f32x4& hi) {
    f16x8 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = (_Float16)lo[e]; v[4 + e] = (_Float16)hi[e]; }
    return v;
}
__device__ __forceinline__ bf16x8 operand(BF16, const f32x4& lo, const f32x4& hi) {
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = (__bf16)lo[e]; v[4 + e] = (__bf16)hi[e]; }
    return v;
}

__device__ __forceinline__ void store_row(F16, uint16_t* dst, const f32x4 (&acc)[4], float times) {
    float v[16];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[4 * dt + r] = acc[dt][r] * times;
    store16(reinterpret_cast<_Float16*>(dst), v);
}
__device__ __forceinline__ void store_row(BF16, uint16_t* dst, const f32x4 (&acc)[4], float times) {
    float v[16];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[4 * dt + r] = acc[dt][r] * times;
    store16(reinterpret_cast<__bf16*>(dst), v);
}

// One work-group's rows m0 .. m0 + 63 of an image's head as KEYS or as queries.
template <typename In, bool KEYS>
__device__ __forceinline__ void own_rows(const BackwardArgs& p, uint4* ring, float2 (*stats)[kBN], int s, int n, int h, int m0) {
    typedef typename In::vec8 vec8;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int64_t head = (int64_t)h * kHeadDim;
    const int own = m0 + wave * 16 + col;                      // this lane's row inside the image
    const bool active = m0 + wave * 16 < n;
    const float c2 = p.scale * kLog2e;
    // what streams: Q and dO past keys, K and V past queries
    const int tok_a = p.in_tok, tok_b = KEYS ? p.out_tok : p.in_tok;
    const uint16_t* const base_a = (KEYS ? p.q : p.k) + (int64_t)s * tok_a + head;
    const uint16_t* const base_b = (KEYS ? p.d_o : p.v) + (int64_t)s * tok_b + head;
    const uint32_t ring0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)ring);
    const int tiles = (n + kBN - 1) / kBN;
    const int load_row = 16 * wave + (lane >> 3);
    const uint32_t load_chunk = 16u * ((lane & 7) ^ ((lane >> 4) & 3));
    auto issue = [&](int t, int slot) {
        const int rem = n - t * kBN;
        const int need = rem >= kBN ? kBN : 32 * ((rem + 31) >> 5);       // rows the tile's products touch
        if (16 * wave >= need) return;
        const uint32_t dst = ring0 + slot * 2 * kTileBytes + wave * 2048;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int rel = load_row + 8 * i;
            rel = rel < rem ? rel : rem - 1;                   // past the end: the last real row again
            dma16(dst + i * 1024, (uint32_t)rel * tok_a * 2u + load_chunk, base_a + (int64_t)t * kBN * tok_a);
            dma16(dst + i * 1024 + kTileBytes, (uint32_t)rel * tok_b * 2u + load_chunk, base_b + (int64_t)t * kBN * tok_b);
        }
    };
    issue(0, 0);

    // ---- this lane's column: two operands, 16 head-dim elements (16 g ..) of each (zeros past the end)
    uint4 own_a[2] = {}, own_b[2] = {};                        // k, v or q, dO
    float lse2 = 0.f, delta = 0.f;                             // queries: statistics of the column
    if (own < n) {
        const int64_t row = (int64_t)s + own;
        const uint4* a = reinterpret_cast<const uint4*>((KEYS ? p.k : p.q) + row * p.in_tok + head + 16 * g);
        const uint4* b = reinterpret_cast<const uint4*>(KEYS ? p.v + row * p.in_tok + head + 16 * g : p.d_o + row * p.out_tok + head + 16 * g);
        own_a[0] = a[0]; own_a[1] = a[1];
        own_b[0] = b[0]; own_b[1] = b[1];
        if (!KEYS) {
            const uint4* o = reinterpret_cast<const uint4*>(p.o + row * p.out_tok + head + 16 * g);
            const uint4 o_row[2] = {o[0], o[1]};
            delta = dot16<In>(own_b, o_row);
            lse2 = p.lse[row * p.H + h] * kLog2e;
        }
    }
    if (!KEYS) delta = quad_sum(delta);
    const vec8 col_a[2] = {as_vec8<vec8>(own_a[0]), as_vec8<vec8>(own_a[1])};
    const vec8 col_b[2] = {as_vec8<vec8>(own_b[0]), as_vec8<vec8>(own_b[1])};

    // ---- keys: statistics of the queries of a tile, four threads a row; behind the last one exp2(.. - inf) = 0
    uint4 st_o[2], st_do[2];
    float st_lse;
    auto request_stats = [&](int t) {
        const int row = t * kBN + (tid >> 2);
        const int64_t at = (int64_t)s + (row < n ? row : n - 1);
        const uint4* o = reinterpret_cast<const uint4*>(p.o + at * p.out_tok + head + 16 * (tid & 3));
        const uint4* d = reinterpret_cast<const uint4*>(p.d_o + at * p.out_tok + head + 16 * (tid & 3));
        st_o[0] = o[0]; st_o[1] = o[1];
        st_do[0] = d[0]; st_do[1] = d[1];
        st_lse = p.lse[at * p.H + h];
    };
    auto write_stats = [&](int t) {
        float d = dot16<In>(st_o, st_do);
        d += __shfl_xor(d, 1);
        d += __shfl_xor(d, 2);
        if ((tid & 3) == 0) stats[t & 1][tid >> 2] = t * kBN + (tid >> 2) < n ? make_float2(st_lse * kLog2e, d) : make_float2(INFINITY, 0.f);
    };
    if (KEYS) {
        request_stats(0);
        write_stats(0);
    }

    // LDS addresses of this lane inside a tile, as in the forward kernel
    const uint32_t row_rel = col * 128 + 16 * ((2 * g) ^ ((col >> 1) & 3));
    const int tr_row = 4 * g + (col >> 2);
    const uint32_t tr_rel = tr_row * 128 + 16 * ((2 * (col & 3)) ^ ((tr_row >> 1) & 3));

    f32x4 acc_a[4], acc_b[4];                                  // dK^T or dQ^T; dV^T
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) acc_a[dt] = acc_b[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int t = 0; t < tiles; ++t) {
        const int slot = t & 1;
        wait_vm<0>();
        __syncthreads();                                       // tile t is there; everyone is past the reads of tile t - 1
        if (t + 1 < tiles) {
            issue(t + 1, slot ^ 1);
            if (KEYS) request_stats(t + 1);
        }
        if (active) {
            const uint32_t tile = ring0 + slot * 2 * kTileBytes;
            const int rem = n - t * kBN;
            const int blocks = rem >= 32 + 1 ? 2 : 1;          // of 32 rows
#pragma unroll
            for (int bb = 0; bb < 2; ++bb) {
                if (bb >= blocks) break;
                f32x4 pr[2], ds[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int kt = 2 * bb + u;
                    const uint32_t ra = tile + row_rel + kt * 16 * 128;
                    f32x4 sc = In::mfma(as_vec8<vec8>(lds_read16(ra)), col_a[0], f32x4{0.f, 0.f, 0.f, 0.f});
                    sc = In::mfma(as_vec8<vec8>(lds_read16((ra ^ 16u))), col_a[1], sc);
                    const uint32_t rb = ra + kTileBytes;
                    f32x4 dp = In::mfma(as_vec8<vec8>(lds_read16(rb)), col_b[0], f32x4{0.f, 0.f, 0.f, 0.f});
                    dp = In::mfma(as_vec8<vec8>(lds_read16((rb ^ 16u))), col_b[1], dp);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = 16 * kt + 4 * g + r;
                        float l2 = lse2, dl = delta;
                        if (KEYS) {
                            const float2 st = stats[slot][row];
                            l2 = st.x;
                            dl = st.y;
                        }
                        float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], c2, -l2));
                        if (!KEYS) e = row < rem ? e : 0.f;
                        pr[u][r] = e;
                        ds[u][r] = e * (dp[r] - dl);
                    }
                }
                const vec8 ds_op = operand(In{}, ds[0], ds[1]);
                vec8 p_op;
                if (KEYS) p_op = operand(In{}, pr[0], pr[1]);
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    const uint32_t a = tile + (((dt & 2) ? tr_rel ^ 16u : tr_rel) + 8 * (dt & 1) + bb * 32 * 128);
                    const uint2 lo = __builtin_bit_cast(uint2, lds_read_tr(a)), hi = __builtin_bit_cast(uint2, lds_read_tr(a + 16 * 128));
                    acc_a[dt] = In::mfma(as_vec8<vec8>(make_uint4(lo.x, lo.y, hi.x, hi.y)), ds_op, acc_a[dt]);
                    if (KEYS) {
                        const uint2 lo2 = __builtin_bit_cast(uint2, lds_read_tr(a + kTileBytes)),
                                    hi2 = __builtin_bit_cast(uint2, lds_read_tr(a + kTileBytes + 16 * 128));
                        acc_b[dt] = In::mfma(as_vec8<vec8>(make_uint4(lo2.x, lo2.y, hi2.x, hi2.y)), p_op, acc_b[dt]);
                    }
                }
            }
        }
        if (KEYS && t + 1 < tiles) write_stats(t + 1);
    }
    // this lane owns elements 16 g .. 16 g + 15 of its row
    if (own < n) {
        const int64_t at = ((int64_t)s + own) * p.grad_tok + head + 16 * g;
        store_row(In{}, (KEYS ? p.dk : p.dq) + at, acc_a, p.scale);
        if (KEYS) store_row(In{}, p.dv + at, acc_b, 1.0f);
    }
}

template <typename In>
__global__ __launch_bounds__(kBlockThreads)
void attn_backward_kernel(BackwardArgs p) {
    __shared__ __attribute__((aligned(1024))) uint4 ring[kRingBytes / 16];     // [slot][A | B]
    __shared__ float2 stats[2][kBN];                           // of a tile's queries: L log2 e, delta
    const int pair = blockIdx.z * p.group + blockIdx.x;
    if (pair >= p.pairs) return;
    uint32_t img, h;
    divmod((uint32_t)pair, (uint32_t)p.H, p.h_magic, img, h);
    const int s = p.cu_seqlens[img], n = __builtin_amdgcn_readfirstlane(p.cu_seqlens[img + 1] - s);
    const int m0 = (blockIdx.y >> 1) * kBN;
    if (m0 >= n) return;
    if (blockIdx.y & 1) own_rows<In, false>(p, ring, stats, s, n, (int)h, m0);
    else own_rows<In, true>(p, ring, stats, s, n, (int)h, m0);
}

}  // namespace

hipError_t launch_attn_backward(const void* q, const void* k, const void* v, const void* o, const void* d_o, const float* lse, void* dq, void* dk,
                                void* dv, const int32_t* cu_seqlens, int B, int max_seqlen, int H, int64_t in_tok, int64_t out_tok,
                                int64_t grad_tok, float scale, ragged_dtype dt, hipStream_t stream) {
    const int pairs = B * H, tiles = (max_seqlen + kBN - 1) / kBN;
    const int pairs8 = (pairs + kXcds - 1) / kXcds * kXcds;
    const int group = pairs8 < kGroupPairs ? pairs8 : kGroupPairs, batches = (pairs + group - 1) / group;
    const BackwardArgs p{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v),
                         static_cast<const uint16_t*>(o), static_cast<const uint16_t*>(d_o), static_cast<uint16_t*>(dq),
                         static_cast<uint16_t*>(dk), static_cast<uint16_t*>(dv), lse, cu_seqlens, H, pairs, group, (int)in_tok, (int)out_tok,
                         (int)grad_tok, div_magic((uint32_t)H), scale};
    const dim3 grid(group, 2 * tiles, batches);
    return dt == RAGGED_F16 ? launch_kernel(attn_backward_kernel<F16>, grid, dim3(kBlockThreads), stream, p)
                            : launch_kernel(attn_backward_kernel<BF16>, grid, dim3(kBlockThreads), stream, p);
}

}  // namespace ragged
