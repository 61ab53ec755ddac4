// The gradients of attention over a packed ragged buffer, for gfx950.  With c the scale, L the row statistics of the forward pass
// and delta_i = sum over d of dO_id O_id,
//     P_ij = exp(c q_i.k_j - L_i),   dP_ij = dO_i.v_j,   dS_ij = P_ij (dP_ij - delta_i),
//     dV = P^T dO,   dK = c dS^T Q,   dQ = c dS K.
//
// One launch, no atomics, no workspace.  A sequence of at most 64 rows is one work-group's (whole_sequence, few_keys: five products, dS
// turned through LDS).  Of a longer one a work-group owns 128 rows (64 in small launches), either as KEYS, whose dK and dV it sums up over all query tiles, or as
// QUERIES, whose dQ it sums up over all key tiles (own_rows).  Both form P and dP again from 16-bit rows (seven products instead of the
// five that a pass over both at once would need), which is what lets every sum have one owner and one order.
//
// The two roles are one piece of code with the operands exchanged.  A wavefront owns 32 rows ("columns" below: the MFMA's column
// dimension, two blocks of 16); tiles of the other side's 64 rows stream through a ring in LDS by direct loads:
//     keys:    columns are keys,    tile A = Q, B = dO:   S = Q K^T,   dP = dO V^T;   dV^T += dO^T P,   dK^T += Q^T dS
//     queries: columns are queries, tile A = K, B = V :   S^T = K Q^T, dP^T = V dO^T;                   dQ^T += K^T dS^T
// As in the forward pass the first products leave each lane with the scores of ONE column and tile rows 4 (lane/16) + r of every 16,
// which is the B operand that the second products want, and those read the same row-major tiles transposed: P and dS never leave
// registers.  LDS layout, swizzle and operand addresses are those of the forward kernel (attn.hip).  Two column blocks share every
// operand read from LDS: with one the LDS pipe was the bound (32 x 577 tokens, 12 heads, bf16: 258 us with 16 columns a wavefront).
//
// delta is the diagonal of dO O^T, two MFMAs for 16 rows.  Past keys the rows of o stream through the ring as a third operand and the
// statistics of a tile are formed from LDS between two barriers: read by the lanes from memory in front of the loop they cost
// a work-group of keys a quarter of its time (same case 112 us for the keys alone, 82 without).  - delta is where the sum dP starts.
//
// P and dS are rounded to the input type for the second products, as the gradients themselves are in the end: a sum of n terms
// whose signs are mixed is off by about as much as its own rounding (2.4 thousandths in bf16, 0.30 in fp16; a rounding of the exact gradients 1.7
// and 0.21, which both kept as hi + lo would reach in 1.7 to 1.8 times the time).  Sums are fp32.
//
// fp16 has the bits for that and not the range: P = 1/n is below its normal numbers beyond 16 384 keys, dS overflows at 65 504 where dQ and dK
// need not, and vanishes where gradients are small.  So P is rounded as 2^15 P, and dS as F dS; both are taken out of the fp32 sums.
// |dS| <= |dP - delta| <= 2 |dO| |v|, and F is the power of two with which 2 |dO| |v| is below 2^14, |dO| and |v| being the lengths of several
// rows as one vector.  From 33 to 64 rows that is all of them; up to 32 F comes from the largest |P dP| instead, which is there, as is, if F were
// below 1, the largest |dS| of 33 to 64 rows.  Of a longer sequence it is 4 rows, spread evenly over it, so that F is the same in every
// work-group and launch (past queries a query's own dO), and 1 at least: with N(0, 1) rows F = 16 and |F (dP - delta)| is up to 2^9.  Where far larger
// dS come all the same, the sums of a column end as infinities or no numbers, all of them: such columns are gone through again with 2^-16 F, down to
// 2^-24, with which no dS overflows; the others have been stored.  F is in the exponent that P is formed with, so that the loop has one
// multiplication more past keys (from F P to 2^15 P), and none past queries.  Launches of fp16 take 2 to 8 % more for it, most of it for the
// sample (64 x 128 28.5 -> 30.4 us, 128 x about 100 38.2 -> 41.1, 64 x 197 55.6 -> 58, 32 x 577 144 -> 149, 256 x 30 19.4 -> 20.4).
//
// us now (gradients alone, H = 12, by the card): 32 x 577 bf16 138 to 150 (82 GFLOP in five products, 115 in the seven of this form: 0.77 to
// 0.83 PFLOP/s, where a loop of products alone sustains 1.3), 64 x 197 bf16 52, fp16 58 (155 MB of rows: 26 us at the rate of a copy), 32 x about
// 40 bf16 6.4.
#include <type_traits>

#include "attn_parts.h"
#include "common.h"
#include "lane_sums.h"
#include "mfma_lds.h"

namespace ragged {
namespace {

// Launches of at most this many work-groups of 128 rows take work-groups of 64 (CB = 1): CUs would be idle.  us with 64 / 128 rows, bf16: 2 x 197
// tokens, 3 heads 7.7 / 9.8, 4 x 197, 12 heads (192 groups) 9.5 / 10.7, 8 x 197 (384) 12.7 / 12.8, 16 x 128 (384) 10.1 / 10.4; beyond, 32 x 197 at
// keep 0.5 (1536) 15.3 / 13.1, 64 x 197 64 / 53, 32 x 577 186 / 143 (fp16 the same way: 8.4 / 10.4, 10.6 / 11.4, 13.8 / 14.0, 10.8 / 11.4; 16.4 / 13.9,
// 71 / 57, 197 / 155).
constexpr int kSmallGroups = 512;
// (image, head) pairs of a dispatch batch: all the work-groups of a batch come before the next one's, those of a pair on one XCD.  As many
// pairs as have their rows in three quarters of that XCD's 4 MB L2, so that the work-groups of a pair read them there; those of 512, as in
// the forward pass, would be streamed again and again (64 x 197 tokens: 512 pairs 59 us, 256 61, 128 55; 32 x 577: 512 159, 128 154, 64 144).
constexpr int kGroupPairs = 512, kGroupPairsMin = 32;
constexpr int64_t kGroupBytes = 3 << 20;
// Up to 512 pairs whose work-groups are no more than this start about together in any order, and in one batch those of them that have
// rows are dealt out evenly: 32 x about 40 of 197 tokens 6.7 us and 7.6 in batches of 128, 32 x about 100 12.8 and 13.4, 8 x 900 83 and 86.
constexpr int kAtOnce = 2048;
constexpr int kSlotBytes = 3 * kTileBytes;      // tiles A and B; keys: the rows of o besides
constexpr int kLseBytes = kBN * 4;
constexpr int kVotes = 2 * kSlotBytes + 2 * kLseBytes + 2 * kBN * 4;         // ring, L of a tile's queries, statistics (L log2 e, - delta) and
constexpr int kLdsBytes = kVotes + kBlockThreads / kWaveSize * 8;            // a word or two of each wavefront

struct BackwardArgs {
    const uint16_t *q, *k, *v, *o, *d_o;
    uint16_t *dq, *dk, *dv;
    const float* lse;                   // [rows, H]
    int H, in_tok, out_tok, grad_tok;
    float scale;
};

// dma16 for four bytes a lane: lane i's go to lds_dst + 4 i.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma4(uint32_t lds_dst, uint32_t voff, const void* base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(lds_dst), "v"(voff), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ void lds_write8(uint32_t addr, uint2 v) {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
    *reinterpret_cast<lds_u32x2*>(static_cast<uintptr_t>(addr)) = u32x2{v.x, v.y};
}

// delta of 16 rows: the diagonal of dO O^T.  A lane brings 16 head-dim elements (16 g ..) of row lane % 16 of both and gets the sum of
// that row if its group is the row's own (g = row / 4), as exact products added up in fp32.
template <typename In>
__device__ __forceinline__ float diagonal(const uint4 (&a)[2], const uint4 (&b)[2], int col) {
    f32x4 d = In::mfma(as_vec8<typename In::vec8>(a[0]), as_vec8<typename In::vec8>(b[0]), f32x4{0.f, 0.f, 0.f, 0.f});
    d = In::mfma(as_vec8<typename In::vec8>(a[1]), as_vec8<typename In::vec8>(b[1]), d);
    const float lo = col & 1 ? d[1] : d[0], hi = col & 1 ? d[3] : d[2];
    return col & 2 ? hi : lo;
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

// fp16's powers of two: 2^kFitP for P, 2^fit for dS, fit from squares of the lengths of what dO and v are to be sized by (0: nothing to go by, 1).
template <typename In> constexpr bool kFit = std::is_same<In, F16>::value;
constexpr int kFitP = 15, kFitLast = -24, kFitStep = 16, kFitMost = 60;
__device__ __forceinline__ float power2(int e) { return __builtin_bit_cast(float, (uint32_t)(127 + e) << 23); }
__device__ __forceinline__ int exponent(float v) { return (int)(__builtin_bit_cast(uint32_t, v) >> 23 & 255) - 127; }
__device__ __forceinline__ int fit_within(int fit) { return fit < kFitLast ? kFitLast : fit > kFitMost ? kFitMost : fit; }
__device__ __forceinline__ int fit_of(float squares_do, float squares_v) {
    const float a = squares_do == 0.f ? 1.f : squares_do, b = squares_v == 0.f ? 1.f : squares_v;
    return fit_within(12 - (exponent(a * b) >> 1));            // 2 sqrt(a b) < 2^(exponent / 2 + 2)
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_f32<0x128>(v));
    v = fmaxf(v, dpp_f32<0x124>(v));
    v = fmaxf(v, dpp_f32<0x122>(v));
    return quad_max(fmaxf(v, dpp_f32<0x121>(v)));
}
__device__ __forceinline__ float squares(const uint4& w) {
    const f16x8 v = as_vec8<f16x8>(w);
    float even = 0.f, odd = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        even = __builtin_fmaf((float)v[e], (float)v[e], even);
        odd = __builtin_fmaf((float)v[e + 1], (float)v[e + 1], odd);
    }
    return even + odd;
}

// A lane's 16 sums, times the scale (and what they were formed with taken out), as elements of a row.
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

// One work-group's rows m0 .. m0 + 64 CB - 1 of an image's head as KEYS or as queries; a wavefront has CB blocks of 16 columns.
template <typename In, bool KEYS, int CB>
__device__ __forceinline__ void own_rows(const BackwardArgs& p, uint4* lds, int s, int n, int h, int m0) {
    typedef typename In::vec8 vec8;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int64_t head = (int64_t)h * kHeadDim;
    const int first = m0 + wave * 16 * CB;                     // the wavefront's rows inside the image
    const bool active = first < n;
    const float c2 = p.scale * kLog2e;
    // what streams: Q and dO past keys, K and V past queries
    const int tok_a = p.in_tok, tok_b = KEYS ? p.out_tok : p.in_tok;
    const uint16_t* const base_a = (KEYS ? p.q : p.k) + (int64_t)s * tok_a + head;
    const uint16_t* const base_b = (KEYS ? p.d_o : p.v) + (int64_t)s * tok_b + head;
    const uint32_t ring0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)lds);
    const uint32_t lse0 = ring0 + 2 * kSlotBytes;
    float* const lse_lds = reinterpret_cast<float*>(lds) + 2 * kSlotBytes / 4;
    f32x4* const stats = reinterpret_cast<f32x4*>(lse_lds + 2 * kBN);         // [2][kBN / 4]
    uint32_t* const votes = reinterpret_cast<uint32_t*>(lds) + kVotes / 4;
    const uint16_t* const base_o = p.o + (int64_t)s * tok_b + head;           // (keys)
    const int tiles = (n + kBN - 1) / kBN;
    const int load_row = 16 * wave + (lane >> 3);
    const uint32_t load_chunk = 16u * ((lane & 7) ^ ((lane >> 4) & 3));
    auto issue = [&](int t, int slot, int rem) {
        const int need = rem >= kBN ? kBN : 32 * ((rem + 31) >> 5);       // rows the tile's products touch
        if (16 * wave >= need) return;
        const uint32_t dst = ring0 + slot * kSlotBytes + wave * 2048;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int rel = load_row + 8 * i;
            rel = rel < rem ? rel : rem - 1;                   // past the end: the last real row again
            dma16(dst + i * 1024, (uint32_t)rel * tok_a * 2u + load_chunk, base_a + (int64_t)t * kBN * tok_a);
            dma16(dst + i * 1024 + kTileBytes, (uint32_t)rel * tok_b * 2u + load_chunk, base_b + (int64_t)t * kBN * tok_b);
            if (KEYS) dma16(dst + i * 1024 + 2 * kTileBytes, (uint32_t)rel * tok_b * 2u + load_chunk, base_o + (int64_t)t * kBN * tok_b);
        }
        if (KEYS && wave == 0)
            dma4(lse0 + slot * kLseBytes, (uint32_t)(lane < rem ? lane : rem - 1) * p.H * 4u, p.lse + ((int64_t)s + t * kBN) * p.H + h);
    };
    issue(0, 0, n);

    // ---- this lane's columns: two operands, 16 head-dim elements (16 g ..) of each (zeros past the end)
    vec8 col_a[CB][2], col_b[CB][2];                           // k, v or q, dO
    float lse2[CB], minus_delta[CB];                           // queries: statistics of the columns
    int fit[CB];                                               // fp16; keys: one for the sequence, queries: one for each column
    bool todo[CB];                                             // columns that are there and not stored yet
    uint4 own_a[CB][2] = {}, own_b[CB][2] = {}, own_o[CB][2] = {};
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        lse2[cb] = 0.f;
        const int own = first + 16 * cb + col;
        todo[cb] = own < n;
        if (own < n) {
            const int64_t row = (int64_t)s + own;
            const uint4* a = reinterpret_cast<const uint4*>((KEYS ? p.k : p.q) + row * p.in_tok + head + 16 * g);
            const uint4* b = reinterpret_cast<const uint4*>(KEYS ? p.v + row * p.in_tok + head + 16 * g : p.d_o + row * p.out_tok + head + 16 * g);
            own_a[cb][0] = a[0]; own_a[cb][1] = a[1];
            own_b[cb][0] = b[0]; own_b[cb][1] = b[1];
            if (!KEYS) {
                const uint4* o = reinterpret_cast<const uint4*>(p.o + row * p.out_tok + head + 16 * g);
                own_o[cb][0] = o[0]; own_o[cb][1] = o[1];
                lse2[cb] = p.lse[row * p.H + h];
            }
        }
    }
    // fp16: squares of 4 rows of the sequence, from the first to the last: v by 8 lanes each, dO by the other 32
    float size_v = 0.f, size_do = 0.f;
    if constexpr (kFit<In>) {
        uint4 sample = {};
        if (KEYS || lane < 32) {
            const int64_t row = (int64_t)s + (lane >> 3 & 3) * (n - 1) / 3, at = head + 8 * (lane & 7);
            sample = *reinterpret_cast<const uint4*>(lane < 32 ? p.v + row * p.in_tok + at : p.d_o + row * p.out_tok + at);
        }
        const float sum = lanes_sum_f32<32>(squares(sample));
        size_v = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sum), 0));
        size_do = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sum), 32));
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        minus_delta[cb] = 0.f;
        lse2[cb] *= kLog2e;
        if (!KEYS) minus_delta[cb] = -__shfl(diagonal<In>(own_b[cb], own_o[cb], col), 16 * (col >> 2) + col);
        fit[cb] = 0;
        if constexpr (kFit<In>) {
            // (4 times the square of a query's own row: what 4 such rows would have in the sample)
            fit[cb] = KEYS ? fit_of(size_do, size_v)
                           : fit_of(4.f * quad_sum(squares(own_b[cb][0]) + squares(own_b[cb][1])), size_v);
            fit[cb] = fit[cb] < 0 ? 0 : fit[cb];               // (large rows need not count: one that nobody looks at does not)
            if (!KEYS) lse2[cb] -= (float)fit[cb];
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            col_a[cb][ks] = as_vec8<vec8>(own_a[cb][ks]);
            col_b[cb][ks] = as_vec8<vec8>(own_b[cb][ks]);
        }
    }

    // LDS addresses of this lane inside a tile, as in the forward kernel
    const uint32_t row_rel = col * 128 + 16 * ((2 * g) ^ ((col >> 1) & 3));
    const int tr_row = 4 * g + (col >> 2);
    const uint32_t tr_rel = tr_row * 128 + 16 * ((2 * (col & 3)) ^ ((tr_row >> 1) & 3));

    // The columns count as used here: a load that the compiler still believes in flight inside the loop makes it wait there for all
    // memory traffic, the next tile's among it.
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) asm volatile("" : "+v"(col_a[cb][ks]), "+v"(col_b[cb][ks]));
        asm volatile("" : "+v"(lse2[cb]), "+v"(minus_delta[cb]));
    }
    f32x4 acc_a[CB][4], acc_b[CB][4];                          // dK^T or dQ^T; dV^T
    float p_times = 1.f;                                       // fp16, keys: from F P to 2^15 P

    // keys: the statistics of a tile's queries, 16 of them by each wavefront; behind the last query exp2(.. - inf) = 0
    auto write_stats = [&](int t, int slot) {
        const uint32_t rb = ring0 + slot * kSlotBytes + kTileBytes + row_rel + wave * 16 * 128, ro = rb + kTileBytes;
        const uint4 d[2] = {lds_read16(rb), lds_read16(rb ^ 16u)}, o[2] = {lds_read16(ro), lds_read16(ro ^ 16u)};
        const float delta = diagonal<In>(d, o, col);
        if (g == col >> 2) {
            const bool there = t * kBN + 16 * wave + col < n;
            const float own_lse = lse_lds[slot * kBN + 16 * wave + col] * kLog2e;
            reinterpret_cast<float*>(stats)[16 * wave + col] = there ? kFit<In> ? own_lse - (float)fit[0] : own_lse : INFINITY;
            reinterpret_cast<float*>(stats)[kBN + 16 * wave + col] = there ? -delta : 0.f;
        }
    };

    // 32 rows of a tile: MASK where some of them may lie behind the last key, NU = 1 where the second 16 all do
    auto block = [&](uint32_t tile, int bb, int rem, auto mask, auto subtiles) {
        constexpr bool MASK = decltype(mask)::value;
        constexpr int NU = decltype(subtiles)::value;
        f32x4 pr[CB][2], ds[CB][2];                            // P and dS (fp16: 2^15 P, F dS)
        if (NU == 1) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) pr[cb][1] = ds[cb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int kt = 2 * bb + u;
            const uint32_t ra = tile + row_rel + kt * 16 * 128, rb = ra + kTileBytes;
            const vec8 a0 = as_vec8<vec8>(lds_read16(ra)), a1 = as_vec8<vec8>(lds_read16(ra ^ 16u));
            const vec8 b0 = as_vec8<vec8>(lds_read16(rb)), b1 = as_vec8<vec8>(lds_read16(rb ^ 16u));
            f32x4 row_lse, row_delta;
            if (KEYS) {
                row_lse = stats[4 * kt + g];
                row_delta = stats[kBN / 4 + 4 * kt + g];
            }
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const f32x4 from = KEYS ? row_delta : f32x4{minus_delta[cb], minus_delta[cb], minus_delta[cb], minus_delta[cb]};
                f32x4 sc = In::mfma(a0, col_a[cb][0], f32x4{0.f, 0.f, 0.f, 0.f});
                f32x4 dp = In::mfma(b0, col_b[cb][0], from);   // dP - delta: delta is where the sum starts
                sc = In::mfma(a1, col_a[cb][1], sc);
                dp = In::mfma(b1, col_b[cb][1], dp);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], c2, KEYS ? -row_lse[r] : -lse2[cb]));
                    if (MASK && !KEYS) e = 16 * kt + 4 * g + r < rem ? e : 0.f;
                    pr[cb][u][r] = e;
                    if (kFit<In> && KEYS) {                    // (kept apart from its conversion: one fma and conversion each takes longer)
                        float scaled = e * p_times;
                        asm("" : "+v"(scaled));
                        pr[cb][u][r] = scaled;
                    }
                    ds[cb][u][r] = e * dp[r];
                }
            }
        }
        vec8 ds_op[CB], p_op[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            ds_op[cb] = operand(In{}, ds[cb][0], ds[cb][1]);
            if (KEYS) p_op[cb] = operand(In{}, pr[cb][0], pr[cb][1]);
        }
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
            const uint32_t a = tile + (((dt & 2) ? tr_rel ^ 16u : tr_rel) + 8 * (dt & 1) + bb * 32 * 128);
            const uint2 lo = __builtin_bit_cast(uint2, lds_read_tr(a)), hi = __builtin_bit_cast(uint2, lds_read_tr(a + 16 * 128));
            const vec8 at = as_vec8<vec8>(make_uint4(lo.x, lo.y, hi.x, hi.y));
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) acc_a[cb][dt] = In::mfma(at, ds_op[cb], acc_a[cb][dt]);
            if (KEYS) {
                const uint2 lo2 = __builtin_bit_cast(uint2, lds_read_tr(a + kTileBytes)),
                            hi2 = __builtin_bit_cast(uint2, lds_read_tr(a + kTileBytes + 16 * 128));
                const vec8 bt = as_vec8<vec8>(make_uint4(lo2.x, lo2.y, hi2.x, hi2.y));
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) acc_b[cb][dt] = In::mfma(bt, p_op[cb], acc_b[cb][dt]);
            }
        }
    };
    for (;;) {
        float zero = 0.f;
        if (kFit<In>) asm volatile("v_mov_b32 %0, 0" : "=v"(zero));                          // (made here, not kept in four registers)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) acc_a[cb][dt] = acc_b[cb][dt] = f32x4{zero, zero, zero, zero};
        if (kFit<In> && KEYS) p_times = power2(kFitP - fit[0]);
        for (int t = 0; t < tiles; ++t) {
            const int slot = t & 1;
            wait_vm<0>();
            __syncthreads();                                       // tile t is there; everyone is past the reads of tile t - 1
            if (t + 1 < tiles) issue(t + 1, slot ^ 1, n - (t + 1) * kBN);
            if (KEYS) {
                if (t * kBN + 16 * wave < n + 16) write_stats(t, slot);
                __syncthreads();
            }
            if (active) {
                const uint32_t tile = ring0 + slot * kSlotBytes;
                const int rem = n - t * kBN;
                typedef std::integral_constant<int, 1> Half;
                typedef std::integral_constant<int, 2> Whole;
                // a last block of at most 16 rows has a form of its own: 64 x 197 tokens 57.4 -> 54.7 us (CB = 1, a chain of latencies, gains nothing)
                const int whole = rem >= kBN ? 2 : CB == 1 ? (rem + 31) >> 5 : (rem + 15) >> 5;
                if (KEYS || rem >= kBN) {
#pragma nounroll
                    for (int bb = 0; bb < whole; ++bb) block(tile, bb, rem, std::false_type{}, Whole{});
                } else {
#pragma nounroll
                    for (int bb = 0; bb < whole; ++bb) block(tile, bb, rem, std::true_type{}, Whole{});
                }
                if constexpr (CB > 1) {
                    if (32 * whole < rem && rem < kBN) block(tile, whole, rem, std::true_type{}, Half{});
                }
            }
        }
        // this lane owns elements 16 g .. 16 g + 15 of its rows
        bool left = false;
        int here = lane;
        asm volatile("" : "+v"(here));                             // (addresses formed here, not kept through the loop)
        const int64_t lane_at = ((int64_t)s + (first + (here & 15))) * p.grad_tok + head + 16 * (here >> 4);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            if (!todo[cb]) continue;
            if (kFit<In> && fit[cb] > kFitLast && !(fabsf(acc_a[cb][0][0]) < INFINITY)) {
                left = true;                                       // (the same in the four lanes of the column)
                continue;
            }
            todo[cb] = false;
            const int64_t at = lane_at + (int64_t)(16 * cb) * p.grad_tok;
            store_row(In{}, (KEYS ? p.dk : p.dq) + at, acc_a[cb], p.scale * power2(-fit[cb]));
            if (KEYS) store_row(In{}, p.dv + at, acc_b[cb], kFit<In> ? power2(-kFitP) : 1.0f);
        }
        if (!kFit<In>) return;
        const uint64_t any = __ballot(left);
        if (lane == 0) votes[wave] = any != 0;
        __syncthreads();                                           // everyone is past the last tile, too
        if ((votes[0] | votes[1] | votes[2] | votes[3]) == 0) return;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {                          // (past queries the columns that are done are only gone through)
            const int lower = fit_within(fit[cb] - kFitStep);
            if (!KEYS) lse2[cb] += (float)(fit[cb] - lower);
            fit[cb] = lower;
        }
        int rows = n;
        asm volatile("" : "+s"(rows));                             // (nor these)
        issue(0, 0, rows);
    }
}

// A whole sequence of at most kFewKeys rows: as whole_sequence, but delta is the sum over the keys of P dP in fp32, over the lanes of a
// wavefront and then over the two that have keys; o is not read.  The same sum from the rounded o is off by u |dO| |o|, and the fewer the
// keys the more that is beside the rounding of dS: with two keys dQ and dK were off by 3.3 thousandths in bf16, now by 2.4, as everywhere
// above 40.  It costs a second round through LDS, us in bf16 with o / with P dP: 32 x 12 tokens 4.4 / 4.6, 32 x 30 4.9 / 5.3, 256 x 30
// 19.9 / 19.5; of all sequences up to 64 rows (four wavefronts, 64 queries each) 1 us of 6 to 12, hence the threshold.
constexpr int kFewKeys = 32;
template <typename In>
__device__ __forceinline__ void few_keys(const BackwardArgs& p, uint4* lds, int s, int n, int h) {
    typedef typename In::vec8 vec8;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int64_t head = (int64_t)h * kHeadDim;
    const float c2 = p.scale * kLog2e;
    const uint32_t q0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)lds);
    const uint32_t do0 = q0 + kTileBytes, k0 = q0 + 2 * kTileBytes, ds0 = q0 + 3 * kTileBytes, lse0 = q0 + 4 * kTileBytes;
    const f32x4* const lse_lds = reinterpret_cast<const f32x4*>(lds + 4 * kTileBytes / 16);
    f32x4* const parts = reinterpret_cast<f32x4*>(lds + (4 * kTileBytes + kLseBytes) / 16);           // [wavefront][kFewKeys / 4]
    uint32_t* const votes = reinterpret_cast<uint32_t*>(lds) + kVotes / 4;
    static_assert(4 * kTileBytes + kLseBytes + 2 * kFewKeys * 4 <= kVotes && kFewKeys == 32, "Q, dO, K, dS, L and the parts of delta");
    const bool active = wave < 2;                              // 16 keys each, the second's may all be past the end (its part of dS is zeros)
    if (active) {
        const uint32_t chunk = 16u * ((lane & 7) ^ ((lane >> 4) & 3));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int rel = 16 * wave + 8 * i + (lane >> 3);
            rel = rel < n ? rel : n - 1;                       // past the end: the last real row again
            const uint32_t in = (uint32_t)rel * p.in_tok * 2u + chunk, out = (uint32_t)rel * p.out_tok * 2u + chunk;
            const uint32_t at = wave * 2048 + i * 1024;
            dma16(q0 + at, in, p.q + (int64_t)s * p.in_tok + head);
            dma16(do0 + at, out, p.d_o + (int64_t)s * p.out_tok + head);
            dma16(k0 + at, in, p.k + (int64_t)s * p.in_tok + head);
        }
        if (wave == 0) dma4(lse0, (uint32_t)(lane < n ? lane : n - 1) * p.H * 4u, p.lse + (int64_t)s * p.H + h);
    }
    // this lane's key: k and v, head-dim elements 16 g .. (zeros past the end)
    const int own = 16 * wave + col;
    uint4 own_k[2] = {}, own_v[2] = {};
    if (own < n) {
        const int64_t at = ((int64_t)s + own) * p.in_tok + head + 16 * g;
        const uint4 *k = reinterpret_cast<const uint4*>(p.k + at), *v = reinterpret_cast<const uint4*>(p.v + at);
        own_k[0] = k[0]; own_k[1] = k[1];
        own_v[0] = v[0]; own_v[1] = v[1];
    }
    const vec8 kf[2] = {as_vec8<vec8>(own_k[0]), as_vec8<vec8>(own_k[1])}, vf[2] = {as_vec8<vec8>(own_v[0]), as_vec8<vec8>(own_v[1])};
    const uint32_t row_rel = col * 128 + 16 * ((2 * g) ^ ((col >> 1) & 3));
    const int tr_row = 4 * g + (col >> 2);
    const uint32_t tr_rel = tr_row * 128 + 16 * ((2 * (col & 3)) ^ ((tr_row >> 1) & 3));
    auto transposed = [&](uint32_t tile, int dt) {
        const uint32_t a = tile + (((dt & 2) ? tr_rel ^ 16u : tr_rel) + 8 * (dt & 1));
        const uint2 lo = __builtin_bit_cast(uint2, lds_read_tr(a)), hi = __builtin_bit_cast(uint2, lds_read_tr(a + 16 * 128));
        return as_vec8<vec8>(make_uint4(lo.x, lo.y, hi.x, hi.y));
    };
    wait_vm<0>();
    __syncthreads();
    f32x4 pr[2], ds[2], part[2];                               // 16 queries each
    if (active) {
        float most = 0.f;                                      // fp16: the largest |P dP|
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const uint32_t ra = q0 + row_rel + kt * 2048, rb = do0 + row_rel + kt * 2048;
            pr[kt] = In::mfma(as_vec8<vec8>(lds_read16(ra)), kf[0], f32x4{0.f, 0.f, 0.f, 0.f});
            ds[kt] = In::mfma(as_vec8<vec8>(lds_read16(rb)), vf[0], f32x4{0.f, 0.f, 0.f, 0.f});
            pr[kt] = In::mfma(as_vec8<vec8>(lds_read16(ra ^ 16u)), kf[1], pr[kt]);
            ds[kt] = In::mfma(as_vec8<vec8>(lds_read16(rb ^ 16u)), vf[1], ds[kt]);
            const f32x4 row_lse = lse_lds[4 * kt + g];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(pr[kt][r], c2, __builtin_fmaf(-kLog2e, row_lse[r], kFit<In> ? kFitP : 0)));
                const bool there = own < n && 16 * kt + 4 * g + r < n;
                pr[kt][r] = there ? e : 0.f;
                ds[kt][r] = there ? ds[kt][r] : 0.f;
                const float share = pr[kt][r] * ds[kt][r];
                part[kt][r] = lanes_sum_f32<16>(share);
                most = fmaxf(most, fabsf(share));
            }
            if (col == 0) parts[wave * (kFewKeys / 4) + 4 * kt + g] = part[kt];
        }
        if constexpr (kFit<In>) {
            most = wave_max(most);
            if (lane == 0) votes[wave] = as_u32(most);
        }
    }
    __syncthreads();
    int fit = 0;
    if constexpr (kFit<In>) {
        const float most = fmaxf(as_f32(votes[0]), as_f32(votes[1]));
        // |dS| <= |P dP| + P |delta| <= 33 times the largest |P dP|, which is below 2^(exponent + 1 - kFitP)
        fit = fit_within(most == 0.f ? 0 : 8 + kFitP - exponent(most));
    }
    if (active) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const f32x4 delta = parts[4 * kt + g] + parts[kFewKeys / 4 + 4 * kt + g];
#pragma unroll
            for (int r = 0; r < 4; ++r) {                      // fp16: delta and P come with 2^kFitP
                const float from = kFit<In> ? __builtin_fmaf(ds[kt][r], power2(fit - kFitP), -power2(fit - 2 * kFitP) * delta[r]) : ds[kt][r] - delta[r];
                ds[kt][r] = n > 1 ? pr[kt][r] * from : 0.f;    // (a single key has P = 1 whatever it is)
            }
        }
        const vec8 p_op = operand(In{}, pr[0], pr[1]), ds_op = operand(In{}, ds[0], ds[1]);
        // dS by keys: row own, queries 16 kt + 4 g .. + 3 in the same swizzled order as the other tiles
        const uint4 w = __builtin_bit_cast(uint4, ds_op);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const uint32_t at = ds0 + own * 128 + 16 * ((2 * kt + (g >> 1)) ^ ((own >> 1) & 3)) + 8 * (g & 1);
            lds_write8(at, kt ? make_uint2(w.z, w.w) : make_uint2(w.x, w.y));
        }
        f32x4 acc_k[4], acc_v[4];
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
            acc_k[dt] = In::mfma(transposed(q0, dt), ds_op, f32x4{0.f, 0.f, 0.f, 0.f});
            acc_v[dt] = In::mfma(transposed(do0, dt), p_op, f32x4{0.f, 0.f, 0.f, 0.f});
        }
        if (own < n) {
            const int64_t at = ((int64_t)s + own) * p.grad_tok + head + 16 * g;
            store_row(In{}, p.dk + at, acc_k, p.scale * power2(-fit));
            store_row(In{}, p.dv + at, acc_v, kFit<In> ? power2(-kFitP) : 1.0f);
        }
    }
    __syncthreads();
    // dQ^T = K^T dS^T: in the transposed read this wavefront's columns are the queries 16 (col / 4) + 4 wave + col % 4
    const int query = 16 * (col >> 2) + 4 * wave + (col & 3);
    const vec8 ds_op = transposed(ds0, wave);
    f32x4 acc_q[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) acc_q[dt] = In::mfma(transposed(k0, dt), ds_op, f32x4{0.f, 0.f, 0.f, 0.f});
    if (query < n) store_row(In{}, p.dq + ((int64_t)s + query) * p.grad_tok + head + 16 * g, acc_q, p.scale * power2(-fit));
}

// A whole sequence of 33 to 64 rows: P and dS are formed once, dS goes through LDS to the products that want it by queries.
template <typename In>
__device__ __forceinline__ void whole_sequence(const BackwardArgs& p, uint4* lds, int s, int n, int h) {
    typedef typename In::vec8 vec8;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int64_t head = (int64_t)h * kHeadDim;
    const float c2 = p.scale * kLog2e;
    const uint32_t q0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)lds);
    const uint32_t do0 = q0 + kTileBytes, o0 = q0 + 2 * kTileBytes, k0 = q0 + 3 * kTileBytes, ds0 = q0 + 4 * kTileBytes;
    const uint32_t lse0 = q0 + 2 * kSlotBytes;
    float* const lse_lds = reinterpret_cast<float*>(lds) + 2 * kSlotBytes / 4;
    f32x4* const stats = reinterpret_cast<f32x4*>(lse_lds + 2 * kBN);
    float* const sums = reinterpret_cast<float*>(lds) + kVotes / 4;                     // [2][wavefront]
    const uint32_t chunk = 16u * ((lane & 7) ^ ((lane >> 4) & 3));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int rel = 16 * wave + 8 * i + (lane >> 3);
        rel = rel < n ? rel : n - 1;                           // past the end: the last real row again
        const uint32_t in = (uint32_t)rel * p.in_tok * 2u + chunk, out = (uint32_t)rel * p.out_tok * 2u + chunk;
        const uint32_t at = wave * 2048 + i * 1024;
        dma16(q0 + at, in, p.q + (int64_t)s * p.in_tok + head);
        dma16(do0 + at, out, p.d_o + (int64_t)s * p.out_tok + head);
        dma16(o0 + at, out, p.o + (int64_t)s * p.out_tok + head);
        dma16(k0 + at, in, p.k + (int64_t)s * p.in_tok + head);
    }
    if (wave == 0) dma4(lse0, (uint32_t)(lane < n ? lane : n - 1) * p.H * 4u, p.lse + (int64_t)s * p.H + h);
    // this lane's key: k and v, head-dim elements 16 g .. (zeros past the end)
    const int own = 16 * wave + col;
    uint4 own_k[2] = {}, own_v[2] = {};
    if (own < n) {
        const int64_t at = ((int64_t)s + own) * p.in_tok + head + 16 * g;
        const uint4 *k = reinterpret_cast<const uint4*>(p.k + at), *v = reinterpret_cast<const uint4*>(p.v + at);
        own_k[0] = k[0]; own_k[1] = k[1];
        own_v[0] = v[0]; own_v[1] = v[1];
    }
    const vec8 kf[2] = {as_vec8<vec8>(own_k[0]), as_vec8<vec8>(own_k[1])}, vf[2] = {as_vec8<vec8>(own_v[0]), as_vec8<vec8>(own_v[1])};
    const uint32_t row_rel = col * 128 + 16 * ((2 * g) ^ ((col >> 1) & 3));
    const int tr_row = 4 * g + (col >> 2);
    const uint32_t tr_rel = tr_row * 128 + 16 * ((2 * (col & 3)) ^ ((tr_row >> 1) & 3));
    wait_vm<0>();
    __syncthreads();
    const uint32_t rb = do0 + row_rel + wave * 2048, ro = o0 + row_rel + wave * 2048;
    const uint4 d[2] = {lds_read16(rb), lds_read16(rb ^ 16u)}, o[2] = {lds_read16(ro), lds_read16(ro ^ 16u)};
    const float delta = diagonal<In>(d, o, col);
    if (g == col >> 2) {
        reinterpret_cast<float*>(stats)[own] = own < n ? __builtin_fmaf(lse_lds[own], kLog2e, kFit<In> ? -kFitP : 0) : INFINITY;
        reinterpret_cast<float*>(stats)[kBN + own] = own < n ? -delta : 0.f;
    }
    if constexpr (kFit<In>) {                                  // of all rows of dO (the last one again past the end) and of v
        const float of_do = lanes_sum_f32<kWaveSize>(squares(d[0]) + squares(d[1])),
                    of_v = lanes_sum_f32<kWaveSize>(squares(own_v[0]) + squares(own_v[1]));
        if (lane == 0) {
            sums[wave] = of_do;
            sums[4 + wave] = of_v;
        }
    }
    __syncthreads();
    int fit = 0;
    if constexpr (kFit<In>)
        fit = fit_of((sums[0] + sums[1]) + (sums[2] + sums[3]), (sums[4] + sums[5]) + (sums[6] + sums[7]));
    // 32 queries: P (fp16: 2^kFitP P) and, times `by`, dS
    auto scores = [&](int bb, f32x4 (&pr)[2], f32x4 (&ds)[2], float by) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int kt = 2 * bb + u;
            const uint32_t ra = q0 + row_rel + kt * 2048, rb = do0 + row_rel + kt * 2048;
            const f32x4 row_lse = stats[4 * kt + g];
            pr[u] = In::mfma(as_vec8<vec8>(lds_read16(ra)), kf[0], f32x4{0.f, 0.f, 0.f, 0.f});
            ds[u] = In::mfma(as_vec8<vec8>(lds_read16(rb)), vf[0], stats[kBN / 4 + 4 * kt + g]);
            pr[u] = In::mfma(as_vec8<vec8>(lds_read16(ra ^ 16u)), kf[1], pr[u]);
            ds[u] = In::mfma(as_vec8<vec8>(lds_read16(rb ^ 16u)), vf[1], ds[u]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                pr[u][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(pr[u][r], c2, -row_lse[r]));
                const float e = kFit<In> ? pr[u][r] * by : pr[u][r];
                ds[u][r] = own < n ? e * ds[u][r] : 0.f;
            }
        }
    };
    if (kFit<In> && fit < 0) {                                 // rows that large need not count (nobody looks at some): by the largest |dS| itself
        float most = 0.f;
#pragma nounroll
        for (int bb = 0; bb < 2; ++bb) {
            f32x4 pr[2], ds[2];
            scores(bb, pr, ds, power2(-kFitP));
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(ds[e / 4][e % 4]));
        }
        most = wave_max(most);
        __syncthreads();                                       // everyone has read the sums
        if (lane == 0) sums[wave] = most;
        __syncthreads();
        most = fmaxf(fmaxf(sums[0], sums[1]), fmaxf(sums[2], sums[3]));
        fit = fit_within(most == 0.f ? 0 : 14 - exponent(most));
    }
    f32x4 acc_k[4], acc_v[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) acc_k[dt] = acc_v[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto transposed = [&](uint32_t tile, int dt, int bb) {
        const uint32_t a = tile + (((dt & 2) ? tr_rel ^ 16u : tr_rel) + 8 * (dt & 1) + bb * 32 * 128);
        const uint2 lo = __builtin_bit_cast(uint2, lds_read_tr(a)), hi = __builtin_bit_cast(uint2, lds_read_tr(a + 16 * 128));
        return as_vec8<vec8>(make_uint4(lo.x, lo.y, hi.x, hi.y));
    };
#pragma unroll
    for (int bb = 0; bb < 2; ++bb) {
        f32x4 pr[2], ds[2];
        scores(bb, pr, ds, power2(fit - kFitP));
        const vec8 p_op = operand(In{}, pr[0], pr[1]), ds_op = operand(In{}, ds[0], ds[1]);
        // dS by keys: row own, queries 16 kt + 4 g .. + 3 in the same swizzled order as the other tiles
        const uint4 w = __builtin_bit_cast(uint4, ds_op);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t at = ds0 + own * 128 + 16 * ((2 * (2 * bb + u) + (g >> 1)) ^ ((own >> 1) & 3)) + 8 * (g & 1);
            lds_write8(at, u ? make_uint2(w.z, w.w) : make_uint2(w.x, w.y));
        }
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
            acc_k[dt] = In::mfma(transposed(q0, dt, bb), ds_op, acc_k[dt]);
            acc_v[dt] = In::mfma(transposed(do0, dt, bb), p_op, acc_v[dt]);
        }
    }
    if (own < n) {
        const int64_t at = ((int64_t)s + own) * p.grad_tok + head + 16 * g;
        store_row(In{}, p.dk + at, acc_k, p.scale * power2(-fit));
        store_row(In{}, p.dv + at, acc_v, kFit<In> ? power2(-kFitP) : 1.0f);
    }
    __syncthreads();
    // dQ^T += K^T dS^T: in the transposed read this wavefront's columns are the queries 16 (col / 4) + 4 wave + col % 4
    const int query = 16 * (col >> 2) + 4 * wave + (col & 3);
    f32x4 acc_q[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) acc_q[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int bb = 0; bb < 2; ++bb) {
        const vec8 ds_op = transposed(ds0, wave, bb);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) acc_q[dt] = In::mfma(transposed(k0, dt, bb), ds_op, acc_q[dt]);
    }
    if (query < n) store_row(In{}, p.dq + ((int64_t)s + query) * p.grad_tok + head + 16 * g, acc_q, p.scale * power2(-fit));
}

template <typename In, int CB>
__global__ __launch_bounds__(kBlockThreads, 3)             // three work-groups on a CU: 168 registers, 49 KB of LDS
void attn_backward_kernel(const int32_t* __restrict__ cu_seqlens, int H, uint32_t h_magic, int pairs, int group, int own_tiles, BackwardArgs p) {
    // (what a work-group needs to find out whether it has rows at all arrives in scalar registers with its wavefronts)
    __shared__ __attribute__((aligned(1024))) uint4 lds[kLdsBytes / 16];
    const int pair = blockIdx.z * group + blockIdx.x;
    if (pair >= pairs) return;
    uint32_t img, h;
    divmod((uint32_t)pair, (uint32_t)H, h_magic, img, h);
    const int s = cu_seqlens[img], n = __builtin_amdgcn_readfirstlane(cu_seqlens[img + 1] - s);
    const int y = (int)blockIdx.y, tile = y >= own_tiles ? y - own_tiles : y;     // keys, which take longer, first
    const int m0 = tile * 64 * CB;
    if (m0 >= n) return;
    if (__builtin_expect(n <= kBN, 1)) {
        if (y == 0) {
            if (n <= kFewKeys) few_keys<In>(p, lds, s, n, (int)h);
            else whole_sequence<In>(p, lds, s, n, (int)h);
        }
        return;
    }
    if (y != tile) own_rows<In, false, CB>(p, lds, s, n, (int)h, m0);
    else own_rows<In, true, CB>(p, lds, s, n, (int)h, m0);
}

}  // namespace

hipError_t launch_attn_backward(const void* q, const void* k, const void* v, const void* o, const void* d_o, const float* lse, void* dq, void* dk,
                                void* dv, const int32_t* cu_seqlens, int B, int max_seqlen, int H, int64_t in_tok, int64_t out_tok,
                                int64_t grad_tok, float scale, ragged_dtype dt, hipStream_t stream) {
    const int pairs = B * H;
    const int own = (int64_t)pairs * 2 * ((max_seqlen + 127) / 128) <= kSmallGroups ? 64 : 128, tiles = (max_seqlen + own - 1) / own;
    int group = kGroupPairs;
    const bool at_once = pairs <= kGroupPairs && pairs * 2 * tiles <= kAtOnce;
    while (!at_once && group > kGroupPairsMin && (int64_t)group / kXcds * max_seqlen * (5 * kHeadDim * 2) > kGroupBytes) group /= 2;
    while ((pairs + group - 1) / group > kMaxGridYZ) group *= 2;              // (ends: the C ABI layer has checked it for 512)
    const int pairs8 = (pairs + kXcds - 1) / kXcds * kXcds;
    if (group > pairs8) group = pairs8;
    const int batches = (pairs + group - 1) / group;
    const BackwardArgs p{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v),
                         static_cast<const uint16_t*>(o), static_cast<const uint16_t*>(d_o), static_cast<uint16_t*>(dq),
                         static_cast<uint16_t*>(dk), static_cast<uint16_t*>(dv), lse, H, (int)in_tok, (int)out_tok, (int)grad_tok, scale};
    const dim3 grid(group, 2 * tiles, batches);
    auto typed = [&](auto in) {
        typedef decltype(in) In;
        return launch_kernel(own == 64 ? attn_backward_kernel<In, 1> : attn_backward_kernel<In, 2>, grid, dim3(kBlockThreads), stream, cu_seqlens, H, div_magic((uint32_t)H), pairs, group, tiles, p);
    };
    return dt == RAGGED_F16 ? typed(F16{}) : typed(BF16{});
}

}  // namespace ragged
