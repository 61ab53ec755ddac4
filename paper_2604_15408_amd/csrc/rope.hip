// Rotary positions on packed rows, for gfx950: every pair (a, b) of a head's rotated part becomes
//     (m (a cos t - b sin t), m (a sin t + b cos t)),   t = coordinate * frequency of the pair (negated for the inverse), m the amplitude.
//
// One launch for the query and the key rows.  What bounds it is memory: a row of 24 heads of 64 is 3 KB in and 3 KB out, and its 32
// angles serve all of its heads.  A work-group takes a few rows: it requests their values, turns the rows' coordinates into
// cosines and sines in LDS while those are on their way, and rotates.
//
// Angles.  coordinate * frequency can be 10^6 radians, where the distance of fp32 numbers is 0.06.  The product is formed in fp64 as a
// number of turns (three roundings, of 1 / (2 pi) and of two products: off by 3 * 2^-53 of it at most), brought to [-1/2, 1/2] by subtracting
// the nearest whole number, and only then rounded to fp32.
#include "common.h"
#include "linear_kernel.h"

namespace ragged {
namespace {

// W values at a time: as many as the pairs of a head (half) or its rotated part (interleaved) can be shared out in, up to 16 bytes.
enum { kHalf = 0, kInterleaved = 1 };
template <int W> struct Words { typedef uint32_t type __attribute__((ext_vector_type(W / 2))); };
template <> struct Words<2> { typedef uint32_t type; };
template <> struct Words<1> { typedef uint16_t type; };
constexpr int kRopeAhead = 4;                                  // units a thread requests before the angles are there
constexpr int kRopeRows = 64;                                  // rows of a work-group at most
constexpr int kRopeAngles = 2048;                              // angles of a work-group at most (16 KB of LDS)
// Output beyond half of the last-level cache goes past it, and so do the inputs, which nothing reads again: 168 MB alone 51 us instead of 75 over
// and over, 70 instead of 77 from HBM, and with a kernel that reads it next 104 instead of 102.  Below, the next kernel finds it there (57 MB: 27 us and 38 with its reader either way).
constexpr int64_t kRopeBypass = 128 << 20;                     // bytes
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
    int rows_cap, rows_per, Hq, D, pairs;
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

// Values of a row as fp32 and back, rounded once.
template <typename In, int W>
__device__ __forceinline__ void widen(const typename Words<W>::type& w, float (&v)[W]) {
    if constexpr (W == 1) {
        float two[2];
        LinearLine<2>{{(uint32_t)w}}.unpack(In{}, two);
        v[0] = two[0];
    } else {
        const LinearLine<W> l = __builtin_bit_cast(LinearLine<W>, w);
        l.unpack(In{}, v);
    }
}
template <typename In, int W>
__device__ __forceinline__ typename Words<W>::type narrow(const float (&v)[W]) {
    if constexpr (W == 1) {
        const float two[2] = {v[0], 0.f};
        return (uint16_t)LinearLine<2>::pack(In{}, two).w[0];
    } else {
        return __builtin_bit_cast(typename Words<W>::type, LinearLine<W>::pack(In{}, v));
    }
}

template <typename In, int LAYOUT, int W, bool BYPASS = false>
__global__ __launch_bounds__(kBlockThreads)
void rope_kernel(RopeArgs p) {
    typedef typename Words<W>::type Line;
    constexpr int CW = LAYOUT == kHalf && W < 8 ? 2 * W : W;   // values at a time of what is copied
    typedef typename Words<CW>::type CopyLine;
    __shared__ float2 angle[kRopeAngles];                      // [row][pair]: m cos t, m sin t
    int rows = p.rows_cap;
    if (p.rows_dev) { const int r = *p.rows_dev; rows = r < rows ? r : rows; }
    const int64_t group_row0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * p.rows_per;
    if (group_row0 >= rows) return;
    const int row0 = (int)group_row0;
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
    // interleaved: what rotates and what is copied lie in one row of equal lines; half: a unit has two lines, a copied one a line of its own width
    struct Values { Line a, b; };
    static_assert(sizeof(CopyLine) <= sizeof(Values), "a copied unit's values are kept in place of a pair's");
    auto get = [&](auto* src) {
        if constexpr (BYPASS) return __builtin_nontemporal_load(src);
        else return *src;
    };
    auto load = [&](const Place& at) {
        Values v;
        const uint32_t j = at.piece;
        if (LAYOUT == kInterleaved) {
            v.a = get(reinterpret_cast<const Line*>(at.src + W * j));
        } else if (j < (uint32_t)p.rotated) {
            v.a = get(reinterpret_cast<const Line*>(at.src + W * j));
            v.b = get(reinterpret_cast<const Line*>(at.src + W * j + p.pairs));
        } else {
            const CopyLine c = get(reinterpret_cast<const CopyLine*>(at.src + 2 * p.pairs + CW * (j - p.rotated)));
            __builtin_memcpy(&v, &c, sizeof(c));
        }
        return v;
    };
    auto put = [&](uint16_t* dst, auto line) {
        typedef decltype(line) T;
        if constexpr (BYPASS) __builtin_nontemporal_store(line, reinterpret_cast<T*>(dst));
        else *reinterpret_cast<T*>(dst) = line;
    };
    auto finish = [&](const Place& at, const Values& v) {
        const uint32_t j = at.piece;
        if (j >= (uint32_t)p.rotated) {
            if (LAYOUT == kInterleaved) {
                put(at.dst + W * j, v.a);
            } else {
                CopyLine c;
                __builtin_memcpy(&c, &v, sizeof(c));
                put(at.dst + 2 * p.pairs + CW * (j - p.rotated), c);
            }
            return;
        }
        const float2* cs = angle + at.row * p.pairs;
        float x[W], y[W];
        widen<In, W>(v.a, x);
        if constexpr (LAYOUT == kHalf) {
            widen<In, W>(v.b, y);
#pragma unroll
            for (int e = 0; e < W; ++e) turn(x[e], y[e], cs[W * j + e]);
            put(at.dst + W * j + p.pairs, narrow<In, W>(y));
        } else {
#pragma unroll
            for (int e = 0; e < W / 2; ++e) turn(x[2 * e], x[2 * e + 1], cs[W / 2 * j + e]);
        }
        put(at.dst + W * j, narrow<In, W>(x));
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
    p.axes = axes;
    p.n_coords = n_coords;
    p.amplitude = amplitude;
    p.inverse = inverse;
    const int shared = interleaved ? 2 * pairs : pairs;
    const int w = shared % 8 == 0 ? 8 : shared % 4 == 0 ? 4 : shared % 2 == 0 ? 2 : 1;
    const int cw = interleaved || w == 8 ? w : 2 * w;
    p.rotated = shared / w;
    const bool in_place = q_out == q && k_out == k;            // what is not rotated is there already
    p.per_head = p.rotated + (in_place ? 0 : (D - 2 * pairs) / cw);
    p.unit_heads = Hq + (k ? Hk : 0);
    const int row_units = p.unit_heads * p.per_head;
    // As few rows as keep 15 of 16 threads busy (or those that keep most), but not so many that there would be too few work-groups.
    // 18 464 rows of 96 units from HBM: 2, 5 and 10 rows 27.0, 27.4 and 29.6 us; 32 774 of 320: 1, 2 and 3 rows 93, 97 and 77.
    int most = rows_cap / kRopeFill < kRopeAngles / pairs ? rows_cap / kRopeFill : kRopeAngles / pairs;
    most = most < kRopeRows ? most : kRopeRows;
    p.rows_per = 1;
    double best = 0.0;
    for (int per = 1; per <= most && (per == 1 || per * row_units <= kRopeAhead * kBlockThreads); ++per) {
        const int units = per * row_units, slots = (units + kBlockThreads - 1) / kBlockThreads * kBlockThreads;
        const double busy = (double)units / slots;
        if (busy > best) { best = busy; p.rows_per = per; }
        if (busy >= 0.9375) break;
    }
    p.row_magic = div_magic((uint32_t)row_units);
    p.head_magic = div_magic((uint32_t)p.per_head);
    p.pair_magic = div_magic((uint32_t)pairs);
    p.axis_magic = div_magic((uint32_t)(pairs / axes));
    p.coord_magic = div_magic((uint32_t)n_coords);
    const bool bypass = (int64_t)rows_cap * p.unit_heads * D * 2 > kRopeBypass;
    const int64_t groups = ((int64_t)rows_cap + p.rows_per - 1) / p.rows_per;
    constexpr int64_t kGridX = 1 << 20;                        // (threads along a dimension of the grid have to fit 32 bits)
    const dim3 grid((unsigned)(groups < kGridX ? groups : kGridX), (unsigned)((groups + kGridX - 1) / kGridX));
    auto typed = [&](auto in) {
        typedef decltype(in) In;
        auto launch = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(kBlockThreads), stream, p); };
        if (w == 8 && bypass) return launch(interleaved ? rope_kernel<In, kInterleaved, 8, true> : rope_kernel<In, kHalf, 8, true>);
        if (interleaved) return launch(w == 8 ? rope_kernel<In, kInterleaved, 8> : w == 4 ? rope_kernel<In, kInterleaved, 4> : rope_kernel<In, kInterleaved, 2>);
        return launch(w == 8 ? rope_kernel<In, kHalf, 8> : w == 4 ? rope_kernel<In, kHalf, 4> : w == 2 ? rope_kernel<In, kHalf, 2> : rope_kernel<In, kHalf, 1>);
    };
    return dt == RAGGED_F16 ? typed(F16{}) : typed(BF16{});
}

}  // namespace ragged
