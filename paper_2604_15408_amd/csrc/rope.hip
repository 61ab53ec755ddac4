// Rotary positions on packed rows, for gfx950: every pair (a, b) of a head's rotated part becomes
//     (m (a cos t - b sin t), m (a sin t + b cos t)),   t = coordinate * frequency of the pair (negated for the inverse), m the amplitude.
//
// One launch for the query and the key rows.  What bounds it is memory: a row of 24 heads of 64 is 3 KB in and 3 KB out, and its 32
// angles serve all of its heads.  A work-group takes a few rows: it requests their values, turns the rows' coordinates into
// cosines and sines in LDS while those are on their way, and rotates.
//
// Angles.  coordinate * frequency can be 10^6 radians, where the distance of fp32 numbers is 0.06.  The product is formed in fp64 as a
// number of turns (error 2^-53 of it), brought to [-1/2, 1/2] by subtracting the nearest whole number, and only then rounded to fp32.
#include "common.h"
#include "linear_kernel.h"

namespace ragged {
namespace {

// kChunksHalf, kChunksInterleaved: 16 bytes at a time, where the pairs of a head fill whole chunks; kSinglePairs: any other number of pairs.
enum { kChunksHalf = 0, kChunksInterleaved = 1, kSinglePairs = 2 };
constexpr int kRopeAhead = 4;                                  // units a thread requests before the angles are there
constexpr int kRopeRows = 16;                                  // rows of a work-group at most
constexpr int kRopeAngles = 2048;                              // angles of a work-group at most (16 KB of LDS)
constexpr int kRopeFill = 512;                                 // work-groups below which rows are not gathered into fewer

struct RopeArgs {
    const uint16_t* q;
    const uint16_t* k;                                         // may be null: no key heads
    uint16_t* q_out;                                           // may be q, with the same stride
    uint16_t* k_out;
    const int32_t* rows_dev;
    const float* coords;                                       // [n_coords, axes]
    const int32_t* index;                                      // [rows] or null
    const double* freqs;                                       // [pairs]
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;    // elements from row to row
    int rows_cap, rows_per, Hq, D, pairs, interleaved;
    int unit_heads, per_head;                                  // heads of a row (queries, then keys), units of a head
    int rotated;                                               // units of a head that rotate; the others copy
    int axes, n_coords;
    uint32_t row_magic, head_magic, pair_magic, axis_magic, coord_magic;
    float amplitude;
    int inverse;
};

// Two values of a pair, turned.
__device__ __forceinline__ void turn(float& a, float& b, float2 cs) {
    const float u = a * cs.x - b * cs.y;
    b = a * cs.y + b * cs.x;
    a = u;
}

template <typename In, int FORM>
__global__ __launch_bounds__(kBlockThreads)
void rope_kernel(RopeArgs p) {
    typedef LinearLine<8> Chunk;
    typedef LinearLine<2> Word;
    __shared__ float2 angle[kRopeAngles];                      // [row][pair]: m cos t, m sin t
    int rows = p.rows_cap;
    if (p.rows_dev) { const int r = *p.rows_dev; rows = r < rows ? r : rows; }
    const int row0 = blockIdx.x * p.rows_per;
    if (row0 >= rows) return;
    const int n = rows - row0 < p.rows_per ? rows - row0 : p.rows_per;
    const uint32_t units = (uint32_t)n * p.unit_heads * p.per_head;
    const uint32_t row_units = (uint32_t)p.unit_heads * p.per_head;

    // unit u: row, head and what it covers of the head
    struct Place { const uint16_t* src; uint16_t* dst; uint32_t row, piece; };
    auto place = [&](uint32_t u) {
        Place at;
        uint32_t rest, head;
        divmod(u, row_units, p.row_magic, at.row, rest);
        divmod(rest, (uint32_t)p.per_head, p.head_magic, head, at.piece);
        const int64_t row = row0 + at.row;
        const bool key = head >= (uint32_t)p.Hq;
        const int64_t off = (int64_t)(key ? head - p.Hq : head) * p.D;
        at.src = (key ? p.k + row * p.k_stride : p.q + row * p.q_stride) + off;
        at.dst = (key ? p.k_out + row * p.k_out_stride : p.q_out + row * p.q_out_stride) + off;
        return at;
    };
    struct Values { Chunk a, b; };                             // (the forms that take less use the first words of it)
    auto load = [&](const Place& at) {
        Values v{};
        const uint32_t j = at.piece;
        if (FORM == kSinglePairs) {
            if (j >= (uint32_t)p.rotated) v.a.w[0] = *reinterpret_cast<const uint32_t*>(at.src + 2 * j);
            else if (p.interleaved) v.a.w[0] = *reinterpret_cast<const uint32_t*>(at.src + 2 * j);
            else v.a.w[0] = at.src[j] | (uint32_t)at.src[j + p.pairs] << 16;
        } else if (FORM == kChunksInterleaved) {
            v.a = *reinterpret_cast<const Chunk*>(at.src + 8 * j);
        } else if (j < (uint32_t)p.rotated) {
            v.a = *reinterpret_cast<const Chunk*>(at.src + 8 * j);
            v.b = *reinterpret_cast<const Chunk*>(at.src + 8 * j + p.pairs);
        } else {
            v.a = *reinterpret_cast<const Chunk*>(at.src + 8 * j + p.pairs);
        }
        return v;
    };
    auto finish = [&](const Place& at, Values v) {
        const uint32_t j = at.piece;
        const bool copy = j >= (uint32_t)p.rotated;
        const float2* cs = angle + at.row * p.pairs;
        if (FORM == kSinglePairs) {
            if (!copy) {
                Word w{{v.a.w[0]}};
                float x[2];
                w.unpack(In{}, x);
                turn(x[0], x[1], cs[j]);
                w = Word::pack(In{}, x);
                v.a.w[0] = w.w[0];
                if (!p.interleaved) {
                    at.dst[j] = (uint16_t)w.w[0];
                    at.dst[j + p.pairs] = (uint16_t)(w.w[0] >> 16);
                    return;
                }
            }
            *reinterpret_cast<uint32_t*>(at.dst + 2 * j) = v.a.w[0];
        } else if (FORM == kChunksInterleaved) {
            if (!copy) {
                float x[8];
                v.a.unpack(In{}, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) turn(x[2 * e], x[2 * e + 1], cs[4 * j + e]);
                v.a = Chunk::pack(In{}, x);
            }
            *reinterpret_cast<Chunk*>(at.dst + 8 * j) = v.a;
        } else if (copy) {
            *reinterpret_cast<Chunk*>(at.dst + 8 * j + p.pairs) = v.a;
        } else {
            float x[8], y[8];
            v.a.unpack(In{}, x);
            v.b.unpack(In{}, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) turn(x[e], y[e], cs[8 * j + e]);
            *reinterpret_cast<Chunk*>(at.dst + 8 * j) = Chunk::pack(In{}, x);
            *reinterpret_cast<Chunk*>(at.dst + 8 * j + p.pairs) = Chunk::pack(In{}, y);
        }
    };

    Values ahead[kRopeAhead];
#pragma unroll
    for (int i = 0; i < kRopeAhead; ++i) {
        const uint32_t u = threadIdx.x + i * kBlockThreads;
        if (u < units) ahead[i] = load(place(u));
    }
    const uint32_t angles = (uint32_t)n * p.pairs;
    for (uint32_t j = threadIdx.x; j < angles; j += kBlockThreads) {
        uint32_t row, pair, axis, rest, turns, at;
        divmod(j, (uint32_t)p.pairs, p.pair_magic, row, pair);
        divmod(pair, (uint32_t)(p.pairs / p.axes), p.axis_magic, axis, rest);
        divmod(p.index ? (uint32_t)p.index[row0 + row] : (uint32_t)(row0 + row), (uint32_t)p.n_coords, p.coord_magic, turns, at);
        constexpr double kPerTurn = 0.15915494309189533577;    // 1 / (2 pi)
        double t = (double)p.coords[(int64_t)at * p.axes + axis] * (p.freqs[pair] * kPerTurn);
        t -= rint(t);
        float s, c;
        sincospif(2.0f * (float)t, &s, &c);
        angle[j] = make_float2(p.amplitude * c, (p.inverse ? -p.amplitude : p.amplitude) * s);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRopeAhead; ++i) {
        const uint32_t u = threadIdx.x + i * kBlockThreads;
        if (u < units) finish(place(u), ahead[i]);
    }
    for (uint32_t u = threadIdx.x + kRopeAhead * kBlockThreads; u < units; u += kBlockThreads) {
        const Place at = place(u);
        finish(at, load(at));
    }
}

}  // namespace

hipError_t launch_rope(const void* q, const void* k, void* q_out, void* k_out, int rows_cap, const int32_t* rows_dev, int Hq, int Hk, int D,
                       int64_t q_stride, int64_t k_stride, int64_t q_out_stride, int64_t k_out_stride, const float* coords, int n_coords,
                       int axes, const int32_t* index, const double* freqs, int pairs, int interleaved, float amplitude, int inverse,
                       ragged_dtype dt, hipStream_t stream) {
    RopeArgs p{};
    p.q = static_cast<const uint16_t*>(q);
    p.k = static_cast<const uint16_t*>(k);
    p.q_out = static_cast<uint16_t*>(q_out);
    p.k_out = static_cast<uint16_t*>(k_out);
    p.rows_dev = rows_dev;
    p.coords = coords;
    p.index = index;
    p.freqs = freqs;
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.q_out_stride = q_out_stride;
    p.k_out_stride = k_out_stride;
    p.rows_cap = rows_cap;
    p.Hq = Hq;
    p.D = D;
    p.pairs = pairs;
    p.interleaved = interleaved;
    p.axes = axes;
    p.n_coords = n_coords;
    p.amplitude = amplitude;
    p.inverse = inverse;
    // 16 bytes at a time where the rotated part is whole chunks
    const int form = interleaved ? (pairs % 4 == 0 ? kChunksInterleaved : kSinglePairs) : (pairs % 8 == 0 ? kChunksHalf : kSinglePairs);
    p.rotated = form == kChunksHalf ? pairs / 8 : form == kChunksInterleaved ? pairs / 4 : pairs;
    const int copied = form == kSinglePairs ? (D - 2 * pairs) / 2 : (D - 2 * pairs) / 8;
    const bool in_place = q_out == q && k_out == k;            // what is not rotated is there already
    p.per_head = p.rotated + (in_place ? 0 : copied);
    p.unit_heads = Hq + (k ? Hk : 0);
    const int row_units = p.unit_heads * p.per_head;
    // as many rows as a thread's units ahead allow, fewer where there would be too few work-groups
    int per = kRopeAhead * kBlockThreads / row_units;
    per = per < rows_cap / kRopeFill ? per : rows_cap / kRopeFill;
    per = per < kRopeAngles / pairs ? per : kRopeAngles / pairs;
    per = per < kRopeRows ? per : kRopeRows;
    p.rows_per = per < 1 ? 1 : per;
    p.row_magic = div_magic((uint32_t)row_units);
    p.head_magic = div_magic((uint32_t)p.per_head);
    p.pair_magic = div_magic((uint32_t)pairs);
    p.axis_magic = div_magic((uint32_t)(pairs / axes));
    p.coord_magic = div_magic((uint32_t)n_coords);
    const dim3 grid((unsigned)(((int64_t)rows_cap + p.rows_per - 1) / p.rows_per));
    auto typed = [&](auto in) {
        typedef decltype(in) In;
        return form == kChunksHalf ? launch_kernel(rope_kernel<In, kChunksHalf>, grid, dim3(kBlockThreads), stream, p)
             : form == kChunksInterleaved ? launch_kernel(rope_kernel<In, kChunksInterleaved>, grid, dim3(kBlockThreads), stream, p)
                                          : launch_kernel(rope_kernel<In, kSinglePairs>, grid, dim3(kBlockThreads), stream, p);
    };
    return dt == RAGGED_F16 ? typed(F16{}) : typed(BF16{});
}

}  // namespace ragged
