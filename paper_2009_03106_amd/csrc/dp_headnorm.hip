// Norms of queries and keys for each head with the position rotation in the same pass, and their backward pass with the
// per-example gradients of the gains:
//     r = 1 / sqrt(mean(x^2) + eps),  y = R(p) (x r (*) w)
//     u = R(p)^T dy,  dx = r (u (*) w - x r mean(u (*) w (*) x r)),  gain_rows[i] = sum_{t, h} u (*) x r
// Bound by memory: a row is read once into registers (two rows in the backward pass) and one is written.
//
// A row of D numbers is the registers of L lanes of a wave, as pairs that turn together; the 64 / L rows of a wave are `hw`
// heads of `tw` tokens, hw tw = 64 / L.  The sines and cosines of a token's angles serve all of its heads.
#include <algorithm>
#include <type_traits>
#include "dp_elems.h"
#include "dp_internal.h"

namespace dpk {

namespace {

// What a launch works on: how rows are dealt to lanes.
struct Rows {
    int L, hw, tw;             // lanes of a row, heads and tokens of a wave at a time (powers of two)
    int its0, its;             // steps over the heads: of the first descriptor, of both
    int split;                 // waves that share a token's steps
};

// A lane has two pieces of eight numbers (16 bytes; float32: 32), eight pairs.
//   halves: columns 8 l and rot / 2 + 8 l, as far as the numbers turn
//   PAIRS (neighbours turn together), and behind the numbers that turn: the first pieces of all lanes, then the second ones, so that
//           the lanes' pieces lie next to each other in every access (48 us for 122 MB of 24 + 8 heads of 64 float32; with the 16 numbers
//           of a lane next to each other 58)
// na, nb: how many of each piece there are: eight, or none for lanes behind the row (kWhole), also four (kFours), any number (kAny).
enum Fill { kAny, kFours, kWhole };
struct Pieces { int a, b, na, nb; };
template <bool PAIRS, Fill F> __device__ __forceinline__ Pieces pieces(const HeadnormArgs& a, int l) {
    const int half = a.rot / 2, turning = PAIRS ? 0 : (half + 7) / 8;      // lanes with pairs that are half of `rot` apart
    Pieces p;
    if (!PAIRS && l < turning) {
        p.a = 8 * l;
        p.b = half + 8 * l;
        p.na = p.nb = F == kWhole ? 8 : min(8, half - 8 * l);
    } else {
        const int first = PAIRS ? 0 : a.rot, lanes = (a.D - first + 15) / 16, k = l - turning;
        p.a = first + 8 * k;
        p.b = first + 8 * (lanes + k);
        p.na = k >= lanes ? 0 : F == kWhole ? 8 : min(8, a.D - p.a);
        p.nb = k >= lanes ? 0 : F == kWhole ? 8 : min(8, max(0, a.D - p.b));
    }
    return p;
}

// n numbers of the row at `row`, from column c on.  A piece that is not whole is the end of eight numbers (where the row has as many
// before its end), moved to the front: one load, and selects.
template <int DT, Fill F> __device__ __forceinline__ void load_some(const void* p, int64_t row, int c, int n, float (&v)[8]) {
    if constexpr (F == kWhole) {
        Raw8<DT> r{};
        if (n) r = load_raw8<DT>(p, row + c);
        widen8<DT>(r, v);
    } else if constexpr (F == kFours) {
        float f[4] = {}, g[4] = {};
        if (n) {                                       // the second four: these again, where there are no more
            load_piece<DT>(p, row + c, f);
            load_piece<DT>(p, row + c + (n & 8) / 2, g);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[j] = f[j]; v[4 + j] = n == 8 ? g[j] : 0.f; }
    } else if (n == 0 || c + n >= 8) {
        const int over = 8 - n;
        Raw8<DT> r{};
        if (n) r = load_raw8<DT>(p, row + c - over);
        widen8<DT>(r, v);
        if (__ballot(over & 7)) {
            const bool four = over & 4, two = over & 2, one = over & 1;
#pragma unroll
            for (int j = 0; j < 8; ++j) { const float u = j < 4 ? v[(j + 4) & 7] : 0.f; v[j] = four ? u : v[j]; }
#pragma unroll
            for (int j = 0; j < 8; ++j) { const float u = j < 6 ? v[(j + 2) & 7] : 0.f; v[j] = two ? u : v[j]; }
#pragma unroll
            for (int j = 0; j < 8; ++j) { const float u = j < 7 ? v[(j + 1) & 7] : 0.f; v[j] = one ? u : v[j]; }
        }
    } else {
        load_first<DT>(p, row + c, n, v);
    }
}
template <int DT, Fill F, bool PAST> __device__ __forceinline__ void store_some(void* p, int64_t at, int n, const float (&v)[8]) {
    if (n == 8) {
        store8<DT, PAST>(p, at, v);
    } else if constexpr (F == kFours) {
        const float f[4] = {v[0], v[1], v[2], v[3]};
        if (n == 4) store_piece<DT>(p, at, f);
    } else if constexpr (F == kAny) {
        store_first<DT>(p, at, n, f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]});
    }
}

// sine and cosine of position * freq.  The angle is taken in quarter turns and in 64 bits, without the nearest whole number of them:
// what is left is at most an eighth of a turn, and the series below are exact to float32 there (the first terms left out:
// x^11 / 11! < 2e-9, x^12 / 12! < 2e-10 for x up to pi / 4).  Added to 1.5 2^52, a number below 2^51 is rounded to a whole one, whose
// last bits are the sum's.
__device__ __forceinline__ void sincos_of(int position, double freq, float& s, float& c) {
    const double quarters = (double)position * (freq * 0.63661977236758134308), big = 6755399441055744.0, sum = quarters + big;
    const float x = (float)(quarters - (sum - big)) * 1.5707963f;
    const int q = (int)__double_as_longlong(sum) & 3;
    const float z = x * x;
    const float sx = x + x * z * (-1.6666667e-1f + z * (8.3333333e-3f + z * (-1.9841270e-4f + z * 2.7557319e-6f)));
    const float cx = 1.0f + z * (-0.5f + z * (4.1666667e-2f + z * (-1.3888889e-3f + z * (2.4801587e-5f + z * -2.7557319e-7f))));
    s = q & 1 ? cx : sx;
    c = q & 1 ? sx : cx;
    if (q & 2) s = -s;
    if (q == 1 || q == 2) c = -c;
}

// the turn of each pair of a lane; those behind the rotated ones do not turn
template <bool PAIRS> struct Turn {
    float s[8], c[8];
    int a, b;                  // PAIRS: how many pairs of each piece turn; halves: whether the lane's do
    __device__ __forceinline__ void of(const HeadnormArgs& h, const Pieces& p, int position, bool live) {
        a = PAIRS ? (h.rot - p.a) / 2 : p.a < h.rot / 2;
        b = (h.rot - p.b) / 2;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            s[v] = 0.f;
            c[v] = 1.f;
            const int j = !PAIRS ? p.a + v : v < 4 ? p.a / 2 + v : p.b / 2 + v - 4;
            if (live && j < h.rot / 2) sincos_of(position, h.freqs[j], s[v], c[v]);
        }
    }
};

template <int DT, bool PAIRS, Fill F> struct Row {
    float lo[8], hi[8];        // (lo[i], hi[i]) turn together; PAIRS: neighbours within lo, and within hi

    // zeros where there are none
    __device__ __forceinline__ void load(const Pieces& c, const void* p, int64_t at, bool live) {
        load_some<DT, F>(p, at, c.a, live ? c.na : 0, lo);
        load_some<DT, F>(p, at, c.b, live ? c.nb : 0, hi);
    }
    template <bool PAST> __device__ __forceinline__ void store(const Pieces& c, void* p, int64_t at) const {
        store_some<DT, F, PAST>(p, at + c.a, c.na, lo);
        store_some<DT, F, PAST>(p, at + c.b, c.nb, hi);
    }
    // to numbers of 32 or 64 bits, or (add) onto them
    template <class S> __device__ __forceinline__ void to_lds(const Pieces& c, S* row, bool add) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i < c.na) row[c.a + i] = add ? row[c.a + i] + lo[i] : lo[i];
            if (i < c.nb) row[c.b + i] = add ? row[c.b + i] + hi[i] : hi[i];
        }
    }
    __device__ __forceinline__ void from_lds(const Pieces& c, const float* row) {
        if constexpr (F != kAny) {                     // on 16 bytes; where there is none, the zeros behind the longest row
            const auto at = [&](int column, bool there) { return reinterpret_cast<const float4*>(row + (there ? column : kMaxHeadDim)); };
            const float4 *p = at(c.a, c.na), *q = at(c.b, c.nb);
            const float4 f[4] = {p[0], F == kWhole ? p[1] : *at(c.a + 4, c.na > 4), q[0], F == kWhole ? q[1] : *at(c.b + 4, c.nb > 4)};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                lo[4 * i] = f[i].x; lo[4 * i + 1] = f[i].y; lo[4 * i + 2] = f[i].z; lo[4 * i + 3] = f[i].w;
                hi[4 * i] = f[2 + i].x; hi[4 * i + 1] = f[2 + i].y; hi[4 * i + 2] = f[2 + i].z; hi[4 * i + 3] = f[2 + i].w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lo[i] = i < c.na ? row[c.a + i] : 0.f;
                hi[i] = i < c.nb ? row[c.b + i] : 0.f;
            }
        }
    }
    // The pairs that turn, by the angles whose sines and cosines these are (sign -1: back).  Numbers behind them are left alone: through a
    // sine of 0 an infinite one would become its neighbour's NaN.
    __device__ __forceinline__ void rotate(const Turn<PAIRS>& t, float sign) {
        const auto one = [&](float& x, float& y, int k, bool turns) {
            const float sk = sign * t.s[k], u = x * t.c[k] - y * sk, v = x * sk + y * t.c[k];
            x = turns ? u : x;
            y = turns ? v : y;
        };
        if constexpr (PAIRS) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { one(lo[2 * i], lo[2 * i + 1], i, i < t.a); one(hi[2 * i], hi[2 * i + 1], 4 + i, i < t.b); }
        } else if (t.a) {
#pragma unroll
            for (int i = 0; i < 8; ++i) one(lo[i], hi[i], i, true);
        }
    }
};

__device__ __forceinline__ float row_sum(float v, int L) {
    for (int off = L >> 1; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

struct Token { int b, t, position; bool live; };
__device__ __forceinline__ Token token_of(const HeadnormArgs& a, int n) {      // fewer than 2^30
    Token k;
    k.live = n < a.B * a.T;
    const int at = k.live ? n : 0;
    k.b = at / a.T;
    k.t = at - k.b * a.T;
    if (a.lengths) k.live = k.live && k.t < a.lengths[k.b];
    k.position = a.positions ? a.positions[k.b * a.positions_b + k.t] : k.t;
    return k;
}

// A wave takes tw tokens at a time and its share of the steps over their heads.
template <int DT, bool PAIRS, Fill F, bool PAST>
__global__ __launch_bounds__(kThreads) void k_headnorm(HeadnormArgs a, Rows w) {
    const int lane = threadIdx.x & (kWave - 1), l = lane & (w.L - 1), g = lane / w.L;
    const int64_t wave = (int64_t)blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t step = (int64_t)gridDim.x * (kThreads / kWave) / w.split;
    const int part = (int)(wave % w.split);
    const int it0 = (int)((int64_t)w.its * part / w.split), it1 = (int)((int64_t)w.its * (part + 1) / w.split);
    const Pieces pc = pieces<PAIRS, F>(a, l);
    const float mean = 1.0f / a.D;
    for (int64_t n0 = wave / w.split * w.tw; n0 < a.B * a.T; n0 += step * w.tw) {
        const Token k = token_of(a, (int)n0 + g / w.hw);
        Turn<PAIRS> turn;
        turn.of(a, pc, k.position, k.live);
#pragma unroll 1
        for (int which = it0 >= w.its0; which <= (it1 > w.its0); ++which) {
            const HeadsArgs& hd = a.heads[which];
            const int first = which ? w.its0 : 0, from = max(it0, first), to = which ? it1 : min(it1, w.its0);
            Row<0, PAIRS, F> gain;
            gain.load(pc, hd.gain, 0, true);
            const int64_t in = k.b * hd.x_b + k.t * hd.x_t, out = k.b * hd.o_b + k.t * hd.o_t;
            for (int it = from; it < to; ++it) {
                const int h = (it - first) * w.hw + (g & (w.hw - 1));
                const bool live = k.live && h < hd.H;
                Row<DT, PAIRS, F> x;
                x.load(pc, hd.x, in + h * hd.x_h, live);
                float sq = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sq += x.lo[i] * x.lo[i] + x.hi[i] * x.hi[i];
                const float r = rsqrtf(row_sum(sq, w.L) * mean + a.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x.lo[i] *= r * gain.lo[i];
                    x.hi[i] *= r * gain.hi[i];
                }
                x.rotate(turn, 1.0f);
                if (live) x.template store<PAST>(pc, hd.out, out + h * hd.o_h);
            }
        }
    }
}

// Backward.  A workgroup has some tokens of an example and all of one descriptor's heads: the gains' gradients of a lane's columns
// stay in its registers, in float32.  `split` of its waves share a token's heads.  The sums go to partial[example][chunk][D] of the
// descriptor.
// (The next row's loads ahead of the present row's work made it slower, 89 us instead of 79 for 64 x 512 tokens of 12 + 12 heads of 64
// bf16: the other waves' loads fill that time already, and the registers are theirs.)
struct Back {
    Rows w;
    int tokens, chunks;        // of a workgroup, of an example
    float* partial;
};
struct BackPlan {
    Back of[2];
    int first;                 // workgroups from here on have the second descriptor's heads
    int64_t steps;             // rows that a group of lanes has, at most
};

// Where a wave has more than kChain steps, they join its sums in LDS every kChain steps, and those have 64 bits (S): however long the
// sequence and many the heads, no more than kChain additions and six between the lanes follow each other in float32.  (Shorter ones
// need no more than that anyway, and would pay for it: 33 x 1088 tokens of 2 + 1 heads of 128 bf16 25.1 us instead of 24.1.  Long ones
// take as long as with one chain: 1 x 109226 of 5 + 1 heads of 128 bf16 132 us, 256 x 2048 of 32 + 8 3.23 ms.)
constexpr int kChain = 64;
constexpr int kZeros = 8;                              // behind the gains in LDS
// Tokens [t0, end) of example b by a workgroup: dx, and in sums[wave] the waves' shares of the gain's gradient.
template <int DT, bool PAIRS, Fill F, bool PAST, class S>
__device__ __forceinline__ void back_rows(const HeadnormArgs& a, const HeadsArgs& hd, const Rows& w, int b, int64_t t0, int end, float* gains, S (*sums)[kMaxHeadDim]) {
    constexpr bool kLong = std::is_same_v<S, double>;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = lane & (w.L - 1), g = lane / w.L;
    const int part = wave % w.split, it0 = w.its * part / w.split, it1 = w.its * (part + 1) / w.split;
    const int step = kThreads / kWave / w.split * w.tw;
    const Pieces pc = pieces<PAIRS, F>(a, l);
    const float mean = 1.0f / a.D;
    if (hd.H > 0)                                      // a descriptor without heads need not have a gain
        for (int j = threadIdx.x; j < a.D; j += kThreads) gains[j] = global_in<float>(hd.gain)[j];
    if (threadIdx.x < kZeros) gains[kMaxHeadDim + threadIdx.x] = 0.f;
    __syncthreads();
    Row<0, PAIRS, F> acc = {};
    int chain = 0;                                     // steps that acc has
    bool some = false;                                 // whether sums[wave] has any
    const auto gather = [&] {                          // the rows of a wave, in a fixed order, into its sums
#pragma unroll
        for (int i = 0; i < 8; ++i)
            for (int off = w.L; off < kWave; off <<= 1) {
                acc.lo[i] += __shfl_xor(acc.lo[i], off, kWave);
                acc.hi[i] += __shfl_xor(acc.hi[i], off, kWave);
            }
        if (g == 0) acc.to_lds(pc, sums[wave], kLong && some);
    };
    Turn<PAIRS> turn;
    const int64_t x0 = b * hd.x_b, u0 = b * hd.dy_b, o0 = b * hd.o_b;
    for (int64_t n = t0 + wave / w.split * w.tw; n < end; n += step) {
        const int64_t t = n + g / w.hw;                // the lane's token
        const bool here = t < end;
        turn.of(a, pc, !here ? 0 : a.positions ? a.positions[b * a.positions_b + t] : (int)t, here);
        for (int it = it0; it < it1; ++it) {
            if (kLong && chain++ == kChain) {
                gather();
                acc = {};
                some = true;
                chain = 1;
            }
            const int h = it * w.hw + (g & (w.hw - 1));
            const bool live = here && h < hd.H;
            Row<DT, PAIRS, F> x, u;
            x.load(pc, hd.x, x0 + t * hd.x_t + h * hd.x_h, live);
            u.load(pc, hd.dy, u0 + t * hd.dy_t + h * hd.dy_h, live);
            float sq = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sq += x.lo[i] * x.lo[i] + x.hi[i] * x.hi[i];
            const float r = rsqrtf(row_sum(sq, w.L) * mean + a.eps);
            u.rotate(turn, -1.0f);
            Row<0, PAIRS, F> gain;
            asm volatile("" ::: "memory");             // else the reads move out of the loops, and into registers
            gain.from_lds(pc, gains);
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x.lo[i] *= r;
                x.hi[i] *= r;
                acc.lo[i] += u.lo[i] * x.lo[i];
                acc.hi[i] += u.hi[i] * x.hi[i];
                u.lo[i] *= gain.lo[i];
                u.hi[i] *= gain.hi[i];
                dot += u.lo[i] * x.lo[i] + u.hi[i] * x.hi[i];
            }
            dot = row_sum(dot, w.L) * mean;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x.lo[i] = r * (u.lo[i] - x.lo[i] * dot);
                x.hi[i] = r * (u.hi[i] - x.hi[i] * dot);
            }
            if (live) x.template store<PAST>(pc, hd.out, o0 + t * hd.o_t + h * hd.o_h);
        }
    }
    gather();
    __syncthreads();
}

__device__ __forceinline__ int length_of(const HeadnormArgs& a, int b) { return a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T; }

template <int DT, bool PAIRS, Fill F, bool PAST, class S>
__global__ __launch_bounds__(kThreads, 3) void k_headnorm_back(HeadnormArgs a, BackPlan plan) {
    __shared__ S sums[kThreads / kWave][kMaxHeadDim];
    __shared__ __align__(16) float gains[kMaxHeadDim + kZeros]; // not in registers, which decide how many waves there are
    const int which = (int)blockIdx.x >= plan.first;
    const Back& bk = plan.of[which];
    const int wg = blockIdx.x - (which ? plan.first : 0), b = wg / bk.chunks;
    const int64_t t0 = (int64_t)(wg - b * bk.chunks) * bk.tokens;
    const int end = (int)min(t0 + bk.tokens, (int64_t)length_of(a, b));
    back_rows<DT, PAIRS, F, PAST>(a, a.heads[which], bk.w, b, t0, end, gains, sums);
    for (int j = threadIdx.x; j < a.D; j += kThreads)
        bk.partial[(int64_t)wg * a.D + j] = (float)((sums[0][j] + sums[1][j]) + (sums[2][j] + sums[3][j]));
}

// An example of few rows: a workgroup has all of them (at most kFewSteps for a wave), and nothing is left to add up.
template <int DT, bool PAIRS, Fill F>
__global__ __launch_bounds__(kThreads, 3) void k_headnorm_back_few(HeadnormArgs a, BackPlan plan, int accumulate, float* __restrict__ sqnorm) {
    __shared__ float sums[kThreads / kWave][kMaxHeadDim];
    __shared__ __align__(16) float gains[kMaxHeadDim + kZeros];
    __shared__ double red[kThreads / kWave];
    const int b = blockIdx.x, end = length_of(a, b);
    double sq = 0.0;
#pragma unroll 1
    for (int which = 0; which < a.n_heads; ++which) {
        back_rows<DT, PAIRS, F, false>(a, a.heads[which], plan.of[which].w, b, 0, end, gains, sums);
        for (int j = threadIdx.x; j < a.D; j += kThreads) {
            const float f = (sums[0][j] + sums[1][j]) + (sums[2][j] + sums[3][j]);
            a.heads[which].gain_rows[(int64_t)b * a.D + j] = f;
            sq += (double)f * f;
        }
    }
    sq = block_sum_256_f64(sq, red);
    if (threadIdx.x == 0) sqnorm[b] = (float)(accumulate ? sqnorm[b] + sq : sq);
}

// A workgroup per example: the chunks' sums (W columns next to each other for a thread, up to 64 threads along the columns, the
// others take other chunks), and the squared norm of the rows.
constexpr int kFoldThreads = 1024;                     // for many chunks; 256 for up to 64 (2500 x 100 tokens of 4 + 1 heads of 64 bf16: 128 us instead of 148)
template <int W, int THREADS>
__global__ __launch_bounds__(THREADS) void k_headnorm_fold(HeadnormArgs a, BackPlan plan, int accumulate, float* __restrict__ sqnorm) {
    constexpr int kWaves = THREADS / kWave;
    __shared__ double part[kWaves][kWave * W];
    __shared__ double red[kWaves];
    const int b = blockIdx.x, columns = a.D / W, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    int ct = 1;                                        // threads along the columns, a power of two
    while (ct < columns && ct < kWave) ct *= 2;
    const int groups = THREADS / ct, g = threadIdx.x / ct;
    double sq = 0.0;
    for (int c0 = 0; c0 < columns; c0 += ct) {
        const int c = c0 + (lane & (ct - 1));
        double s[2][W] = {};
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which >= a.n_heads || c >= columns) continue;
            const Back& bk = plan.of[which];
            const float* p = bk.partial + (int64_t)b * bk.chunks * a.D + c * W;
            int k = g;
            for (; k + 3 * groups < bk.chunks; k += 4 * groups) {
                float f[4][W];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int v = 0; v < W; ++v) f[i][v] = p[(int64_t)(k + i * groups) * a.D + v];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int v = 0; v < W; ++v) s[which][v] += f[i][v];
            }
            for (; k < bk.chunks; k += groups)
#pragma unroll
                for (int v = 0; v < W; ++v) s[which][v] += p[(int64_t)k * a.D + v];
        }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which >= a.n_heads) break;
#pragma unroll
            for (int v = 0; v < W; ++v) {
                for (int off = ct; off < kWave; off <<= 1) s[which][v] += __shfl_xor(s[which][v], off, kWave);
                if (lane < ct) part[wave][lane * W + v] = s[which][v];
            }
            __syncthreads();
            const int j = c0 * W + threadIdx.x;        // the column that this thread adds up over the waves
            if ((int)threadIdx.x < ct * W && j < a.D) {
                double sum = 0.0;
#pragma unroll
                for (int k = 0; k < kWaves; ++k) sum += part[k][threadIdx.x];
                const float f = (float)sum;
                a.heads[which].gain_rows[(int64_t)b * a.D + j] = f;
                sq += (double)f * f;
            }
            __syncthreads();
        }
    }
    sq = wave_sum_f64(sq);
    if (lane == 0) red[wave] = sq;
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int k = 1; k < kWaves; ++k) sq += red[k];
    sqnorm[b] = (float)(accumulate ? sqnorm[b] + sq : sq);
}

int pow2_up(int n) {
    int p = 1;
    while (p < n) p *= 2;
    return p;
}

// lanes of a row: at most 34 have something of 512 numbers
int lanes_of(const HeadnormArgs& a) {
    return pow2_up(a.pairs ? ceil_div(a.D, 16) : ceil_div(a.rot / 2, 8) + ceil_div(a.D - a.rot, 16));
}
// What the lanes' pieces are.  24 + 8 heads of 72, 80 MB, forward and backward: fours 36 and 60 us in float32, 48 and 114 in bf16; any
// number 46 and 88, 64 and 132.  (Numbers one by one, a row per wave, instead of any number: 173 us instead of 87 for the backward
// pass of 58 x 305 tokens of 8 + 8 heads of 110 bf16.)
Fill fill_of(const HeadnormArgs& a) {
    if (a.D % 16 == 0 && (a.pairs || a.rot % 16 == 0)) return kWhole;
    return a.D % 4 == 0 && (a.pairs || a.rot % 8 == 0) ? kFours : kAny;
}

constexpr int kTurns = 4;
// Heads and tokens of a wave.  Heads lie next to each other, but the rows of a token have the same angles: as many heads at a time as
// leave each lane `turns` steps over a token's heads, the number that leaves fewest rows idle (a tenth at most, if there is such a
// one).  A token's angles cost about as much as working on a row.
Rows rows_of(int H0, int H1, int L, int turns) {
    const int W = kWave / L;
    Rows w{};
    w.L = L;
    int64_t least = INT64_MAX;
    for (int hw = W; hw >= 1; hw /= 2) {
        const int i0 = ceil_div(H0, hw), i1 = ceil_div(H1, hw);
        const int64_t taken = (int64_t)hw * (i0 + i1);
        if (taken > least || (hw > 1 && i0 + i1 < turns)) continue;
        least = taken;
        w.hw = hw; w.tw = W / hw; w.its0 = i0; w.its = i0 + i1;
        if (taken * 10 <= (int64_t)(H0 + H1) * 11) break;
    }
    w.split = 1;
    return w;
}

// Chunks of an example's tokens in the backward pass.  The chip holds 768 workgroups at a time (three for each of the 256 compute
// units by registers, four for some types), and a launch takes about as many rounds of 768 as it has, of the steps of a wave (a row
// for each of its groups of lanes), about two more for each token's angles, and about four for its beginning and its end.
// 11 x 1688 tokens, padded, of 32 + 8 heads of 96 fp16: 77 us, 84 in rounds of 1024.  2 x 54613 tokens of 5 + 1 heads of 128 bf16: 124
// us, 140 with the angles not counted.  1 x 109226 of them: 134 us, 168 with a third of the chunks at most.
constexpr int kAtATime = 768, kMostRounds = 6, kBackChunks = 1536, kEndSteps = 4, kAngleSteps = 2, kFewChunks = 64;
int most_chunks(int B, int T) { return std::max(1, std::min({kBackChunks, T, kMostRounds * kAtATime / B})); }

// A wave gets about per_wave steps: descriptors with more heads get shorter chunks; where tokens are few, two or four waves of a
// workgroup share their heads.
struct BackCost { int64_t workgroups; int steps; };
BackCost cut_back(const HeadnormArgs& a, int64_t per_wave, BackPlan& p) {
    constexpr int waves = kThreads / kWave;
    const int most = most_chunks(a.B, a.T);
    BackCost c{};
    for (int i = 0; i < a.n_heads; ++i) {
        Back& k = p.of[i];
        k.w.split = 1;
        while (k.w.split < waves && k.w.split * 2 <= k.w.its && k.w.its / k.w.split > per_wave) k.w.split *= 2;
        const int granule = waves / k.w.split * k.w.tw, its = ceil_div(std::max(1, k.w.its), k.w.split) + kAngleSteps;      // tokens that a workgroup has at a time, steps for them
        const int64_t rounds = std::max<int64_t>({1, per_wave / its, ceil_div(ceil_div(a.T, granule), most)});
        k.tokens = (int)std::min<int64_t>(a.T, granule * rounds);
        k.chunks = ceil_div(a.T, k.tokens);
        c.workgroups += (int64_t)a.B * k.chunks;
        c.steps = std::max<int>(c.steps, ceil_div(k.tokens, granule) * its);
        p.steps = std::max<int64_t>(i ? p.steps : 0, (int64_t)ceil_div(k.tokens, granule) * ceil_div(k.w.its, k.w.split));
    }
    return c;
}
BackPlan plan_back(const HeadnormArgs& a, int L, float* partial) {
    BackPlan p{};
    int64_t steps = 0;                                  // of all waves together
    for (int i = 0; i < a.n_heads; ++i) {
        p.of[i].w = rows_of(a.heads[i].H, 0, L, kTurns);
        p.of[i].partial = partial + (int64_t)i * a.B * most_chunks(a.B, a.T) * a.D;
        steps += (int64_t)a.B * ceil_div(a.T, p.of[i].w.tw) * (p.of[i].w.its + kAngleSteps);
    }
    int64_t best = INT64_MAX, best_per_wave = 1;
    for (int r = a.lengths ? 2 : 1; r <= kMostRounds; ++r) {            // (lengths: the ends of at least two rounds even out)
        constexpr int waves = kThreads / kWave;
        const int64_t per_wave = std::max<int64_t>(1, (steps + kAtATime * waves * r - 1) / (kAtATime * waves * r));
        const BackCost c = cut_back(a, per_wave, p);
        const int64_t cost = (c.workgroups + kAtATime - 1) / kAtATime * (c.steps + kEndSteps);
        if (cost >= best) continue;
        best = cost;
        best_per_wave = per_wave;
    }
    cut_back(a, best_per_wave, p);
    p.first = a.B * p.of[0].chunks;
    return p;
}

// Whether the outputs go past the last-level cache: where the inputs fit it, but not with the outputs, which would push them out.
// 159 MB and as much of outputs, 30 x 32 heads of 128 bf16: 54 us instead of 71; 24 + 8 heads of 32 float32: 79 instead of 83;
// backward, 99 MB of each: 62 us instead of 73.  Larger inputs do not stay there either way: 399 MB of 24 + 8 heads of 32 float32 took
// 235 us past the cache and 191 through it, of 128 bf16 156 and 160.  Pieces that are not whole are stored in parts of cache
// lines, which the cache puts together.
bool past_cache(const HeadnormArgs& a, int dt) {
    int64_t in = 0, out = 0;
    for (int i = 0; i < a.n_heads; ++i) {
        const HeadsArgs& h = a.heads[i];
        const int64_t bytes = (int64_t)a.B * a.T * h.H * a.D * (dt == 0 ? 4 : 2);
        in += h.dy ? 2 * bytes : bytes;
        if (h.out != h.x && h.out != h.dy) out += bytes;
    }
    return fill_of(a) == kWhole && in <= kLastLevelCache && in + out > kLastLevelCache;
}
// Many examples of few rows, which fill at least half of the chip with a workgroup each: the steps of a wave as above, those of the
// fewest.  Whether there are few enough.  bf16, 4 + 1 heads of 64: 4000 examples of one token 67 us, in two launches 98; 2000 of 48 (9
// steps) 55 and 69; 256 of 48 17 and 16; 800 of 100 (18 steps) 55 and 51.
constexpr int kFewSteps = 10;
bool plan_few(const HeadnormArgs& a, int L, BackPlan& p) {
    if (a.B < kAtATime / 2) return false;
    constexpr int waves = kThreads / kWave;
    int64_t all = 0;
    for (int i = 0; i < a.n_heads; ++i) {
        int64_t least = INT64_MAX;
        for (int turns = 1; turns <= kTurns; turns *= 2) {
            Rows w = rows_of(a.heads[i].H, 0, L, turns);
            for (w.split = 1; w.split <= waves && w.split <= std::max(1, w.its); w.split *= 2) {
                const int64_t steps = (int64_t)ceil_div(a.T, waves / w.split * w.tw) * (ceil_div(w.its, w.split) + kAngleSteps);
                if (steps >= least) continue;
                least = steps;
                p.of[i].w = w;
            }
        }
        all += least;
    }
    return all <= kFewSteps;
}

template <Fill F> using FillIs = std::integral_constant<Fill, F>;
template <int DT, class L> void by_layout(const HeadnormArgs& a, L&& launch) {
    constexpr std::false_type no{};
    constexpr std::true_type yes{};
    const auto with = [&](auto pairs) {
        switch (fill_of(a)) {
        case kAny:   launch(pairs, FillIs<kAny>{}, no); break;
        case kFours: launch(pairs, FillIs<kFours>{}, no); break;
        default:
            if (past_cache(a, DT)) launch(pairs, FillIs<kWhole>{}, yes);
            else                   launch(pairs, FillIs<kWhole>{}, no);
        }
    };
    if (a.pairs) with(yes);
    else         with(no);
}
template <int DT> void forward(const HeadnormArgs& a, const Rows& w, int grid, hipStream_t st) {
    by_layout<DT>(a, [&](auto pairs, auto fill, auto past) { k_headnorm<DT, pairs, fill, past><<<grid, kThreads, 0, st>>>(a, w); });
}
template <int DT> void backward_few(const HeadnormArgs& a, const BackPlan& p, bool accumulate, float* sqnorm, hipStream_t st) {
    by_layout<DT>(a, [&](auto pairs, auto fill, auto) { k_headnorm_back_few<DT, pairs, fill><<<a.B, kThreads, 0, st>>>(a, p, accumulate, sqnorm); });
}
template <int DT> void backward(const HeadnormArgs& a, const BackPlan& p, hipStream_t st) {
    const int grid = a.B * (p.of[0].chunks + p.of[1].chunks);
    by_layout<DT>(a, [&](auto pairs, auto fill, auto past) {
        if (p.steps > kChain) k_headnorm_back<DT, pairs, fill, past, double><<<grid, kThreads, 0, st>>>(a, p);
        else                  k_headnorm_back<DT, pairs, fill, past, float><<<grid, kThreads, 0, st>>>(a, p);
    });
}

}  // namespace

bool headnorm_fits(int64_t B, int64_t T, int64_t H0, int64_t H1) {
    const int64_t tokens = int64_t(1) << 30, heads = int64_t(1) << 20;
    if (!launch_holds(B, kFoldThreads) || T > tokens || H0 > heads || H1 > heads) return false;
    return B == 0 || T <= tokens / B;
}
size_t headnorm_ws_bytes(int n_heads, int B, int T, int D) { return (size_t)B * most_chunks(B, T) * n_heads * D * sizeof(float); }

hipError_t launch_headnorm(const HeadnormArgs& a, int dt, hipStream_t st) {
    Rows w = rows_of(a.heads[0].H, a.heads[1].H, lanes_of(a), kTurns);
    // a wave for every tw tokens; where that leaves the chip empty, several waves share a token's heads
    const int64_t groups = ((int64_t)a.B * a.T + w.tw - 1) / w.tw;
    w.split = (int)std::max<int64_t>(1, std::min<int64_t>(w.its, 4096 / groups));
    const int64_t wgs = (groups * w.split + kThreads / kWave - 1) / (kThreads / kWave);
    int grid = (int)std::min<int64_t>(wgs, 1 << 14);
    // whole tokens: a multiple of split waves
    while ((int64_t)grid * (kThreads / kWave) % w.split) ++grid;
    if (dt == 0)      forward<0>(a, w, grid, st);
    else if (dt == 1) forward<1>(a, w, grid, st);
    else              forward<2>(a, w, grid, st);
    return hipGetLastError();
}

hipError_t launch_headnorm_sqnorm(const HeadnormArgs& a, int dt, bool accumulate, float* sqnorm, void* ws, hipStream_t st) {
    BackPlan few{};
    if (plan_few(a, lanes_of(a), few)) {
        if (dt == 0)      backward_few<0>(a, few, accumulate, sqnorm, st);
        else if (dt == 1) backward_few<1>(a, few, accumulate, sqnorm, st);
        else              backward_few<2>(a, few, accumulate, sqnorm, st);
        return hipGetLastError();
    }
    const BackPlan p = plan_back(a, lanes_of(a), static_cast<float*>(ws));
    if (dt == 0)      backward<0>(a, p, st);
    else if (dt == 1) backward<1>(a, p, st);
    else              backward<2>(a, p, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const auto fold = [&](auto kernel, int threads) { kernel<<<a.B, threads, 0, st>>>(a, p, accumulate, sqnorm); };
    if (std::max(p.of[0].chunks, p.of[1].chunks) <= kFewChunks) fold(a.D % 4 == 0 ? k_headnorm_fold<4, 256> : k_headnorm_fold<1, 256>, 256);
    else fold(a.D % 4 == 0 ? k_headnorm_fold<4, kFoldThreads> : k_headnorm_fold<1, kFoldThreads>, kFoldThreads);
    return hipGetLastError();
}

}  // namespace dpk
