// Relative position bias by buckets:  scores[b, h, q, k] + table[bucket(k - q - q_start[b]), h], and the gradient of the
// table for each example, the sums of dS over the pairs of each bucket.
// Both are bound by memory: an element is read (and written) once, for one addition.
#include <algorithm>
#include "dp_elems.h"
#include "dp_internal.h"

namespace dpk {

namespace {

// what is live of example b: queries [0, nq), keys [0, nk), and with causal k <= q + start
struct Window { int nq, nk; int64_t start; };
__device__ __forceinline__ Window window_of(const PosbiasArgs& a, int b) {
    Window w;
    w.nq = a.q_lens ? min(max(a.q_lens[b], 0), a.Tq) : a.Tq;
    w.nk = a.k_lens ? min(max(a.k_lens[b], 0), a.Tk) : a.Tk;
    w.start = a.q_start ? a.q_start[b] : 0;
    return w;
}
// bucket of a distance; outside [0, n_buckets): none
__device__ __forceinline__ int bucket_of(const PosbiasArgs& a, int64_t distance) {
    const int64_t reach = a.reach;
    return a.buckets[min(max(distance, -reach), reach) + reach];
}

// ---- adding
// A thread adds to blocks of 8 queries x 8 keys, four queries at a time: four loads of 16 bytes (float32: 32), 11 biases, four
// stores.  A workgroup has CT threads next to each other along the keys and RG along the queries, for `steps` rows of blocks
// each, and keeps the biases of all its distances in LDS, so that the two dependent look-ups are made once for a distance and
// not once for an element.  One element after the other, with both look-ups, took 172 us for 32 x 12 x 512 x 512 bf16.
struct AddTiles { int ct, rg, steps, row_tiles, col_tiles; };      // ct, rg: logarithms
constexpr int kAddSteps = 8;
constexpr int kAddDistances = 8 * (kThreads + kAddSteps);          // 8 (CT + RG steps) with CT RG = 256 threads
template <int DT, bool PAST>
__global__ __launch_bounds__(kThreads) void k_posbias_add(PosbiasArgs a, const void* scores, const float* __restrict__ table, void* out, AddTiles tl) {
    __shared__ __align__(16) float bias[kAddDistances];
    const int CT = 1 << tl.ct, RG = 1 << tl.rg;
    const int tile = blockIdx.x % (tl.row_tiles * tl.col_tiles), bh = blockIdx.x / (tl.row_tiles * tl.col_tiles), h = bh % a.H, b = bh / a.H;
    const int col0 = tile % tl.col_tiles * CT, row0 = tile / tl.col_tiles * RG * tl.steps;       // in blocks
    const Window w = window_of(a, b);
    // the distances k - q of the tile: from the first key and the last query on
    const int64_t least = (int64_t)8 * col0 - (8 * ((int64_t)row0 + RG * tl.steps) - 1) - w.start;
    if (8 * row0 >= w.nq || 8 * col0 >= w.nk || (a.causal && least > 0)) return;
    const int ct = threadIdx.x & (CT - 1), rg = threadIdx.x >> tl.ct;
    const int k0 = (col0 + ct) * 8, nk = min(8, w.nk - k0);
    // every load lies within the tensor: those of the last keys begin `over` earlier (rows of at least 8 keys)
    const bool narrow = a.Tk < 8, last = k0 + 8 > a.Tk;
    const int over = (a.Tk + 7) / 8 * 8 - a.Tk;
    const int64_t in0 = b * a.s_b + h * a.s_h + (last && !narrow ? k0 - over : k0), out0 = b * a.o_b + h * a.o_h + k0;
    // Four queries of this thread: step s is half a block of eight.
    struct Step { int q0, nq, seen; };
    const auto step_of = [&](int s) {
        Step t;
        t.q0 = (row0 + (s >> 1) * RG + rg) * 8 + 4 * (s & 1);
        t.nq = s < 2 * tl.steps && nk > 0 ? min(4, w.nq - t.q0) : 0;
        // the live keys of a query are its first ones: `seen` of the block's for the first query, one more for each other
        t.seen = a.causal ? (int)min(max(t.q0 + w.start - k0 + 1, (int64_t)-8), (int64_t)8) : 8;
        if (t.seen + 3 <= 0) t.nq = 0;
        return t;
    };
    Raw8<DT> r[4];
    const auto load = [&](const Step& t) {
        const int64_t at = in0 + t.q0 * a.s_q;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < t.nq && !narrow) r[i] = load_raw8<DT>(scores, at + i * a.s_q);
    };
    Step t = step_of(0);
    load(t);                                           // on their way while the biases are looked up
    const auto bias_of = [&](int j) { return j >= 0 && j < a.n_buckets ? table[j * a.H + h] : 0.f; };
    const float before = bias_of(a.buckets[0]), behind = bias_of(a.buckets[2 * a.reach]);      // of all distances beyond the reach
    const int distances = 8 * (CT + RG * tl.steps);
    for (int t0 = threadIdx.x; t0 < distances; t0 += 4 * kThreads) {
        int j[4];
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t d = least + t0 + i * kThreads;
            j[i] = d > -a.reach && d < a.reach ? a.buckets[d + a.reach] : -1;
            v[i] = d <= -a.reach ? before : d >= a.reach ? behind : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j[i] >= 0 && j[i] < a.n_buckets) v[i] = table[j[i] * a.H + h];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t0 + i * kThreads < distances) bias[t0 + i * kThreads] = v[i];
    }
    __syncthreads();
#pragma unroll 1
    for (int s = 0; s < 2 * tl.steps; ++s) {
        if (s > 0) {
            t = step_of(s);
            load(t);
        }
        const int q0 = t.q0, nq = t.nq, seen = t.seen, block = (s >> 1) * RG + rg, half = 4 * (s & 1);
        if (nq <= 0) continue;
        if (narrow) {
            for (int i = 0; i < nq; ++i)
                for (int j = 0; j < min(nk, seen + i); ++j)
                    store_one<DT>(out, out0 + (q0 + i) * a.o_q + j, load_one<DT>(scores, in0 + (q0 + i) * a.s_q + j) + bias[8 * (ct + RG * tl.steps - 1 - block) + 7 + j - half - i]);
            continue;
        }
        float c[12];                                   // c[3 + j - i]: the bias of key j and query i of these four
        const float4* cp = reinterpret_cast<const float4*>(bias + 8 * (ct + RG * tl.steps - 1 - block) + 4 - half);
#pragma unroll
        for (int i = 0; i < 3; ++i) { const float4 f = cp[i]; c[4 * i] = f.x; c[4 * i + 1] = f.y; c[4 * i + 2] = f.z; c[4 * i + 3] = f.w; }
        const int64_t to = out0 + q0 * a.o_q;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= nq) break;
            float v[8];
            widen8<DT>(r[i], v);
            if (over) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = last && (over & 4) ? v[j + 4] : v[j];
#pragma unroll
                for (int j = 0; j < 6; ++j) v[j] = last && (over & 2) ? v[j + 2] : v[j];
#pragma unroll
                for (int j = 0; j < 7; ++j) v[j] = last && (over & 1) ? v[j + 1] : v[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += c[3 + j - i];
            const int n = min(nk, seen + i);
            if (n >= 8) store8<DT, PAST>(out, to + i * a.o_q, v);
            else        store_first<DT>(out, to + i * a.o_q, max(n, 0), f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]});
        }
    }
}

// As many threads along the keys as there are blocks (a row's accesses are then next to each other), up to the whole workgroup;
// rows of blocks one after the other while there are more than eight workgroups for each of the 256 compute units.
AddTiles plan_add(int64_t BH, int Tq, int Tk) {
    AddTiles t{};
    const int R = (Tq + 7) / 8, C = (Tk + 7) / 8;
    t.ct = 3;
    while (t.ct < 8 && (1 << t.ct) < C) ++t.ct;
    t.rg = 8 - t.ct;
    t.col_tiles = (C + (1 << t.ct) - 1) >> t.ct;
    const auto tiles = [&](int steps) { return (R + (steps << t.rg) - 1) / (steps << t.rg); };
    t.steps = 1;
    while (t.steps < kAddSteps && BH * t.col_tiles * tiles(2 * t.steps) >= 2048) t.steps *= 2;
    t.row_tiles = tiles(t.steps);
    return t;
}

// ---- the gradient
// A lane adds up blocks of 8 queries x 8 keys along a diagonal of blocks: block (rb, rb + m) for one m and rb = r0, r0 + 1, ...
// All of them have their elements on the same 15 diagonals, k - q = 8 m + e with -7 <= e <= 7, so the sums stay in the lane's
// registers, and a group of LC lanes with neighbouring m reads LC pieces of 16 bytes (8 of float32: 32) next to each other
// of every query.  Everything is added in 64 bits; only the diagonal of a block of 16-bit elements (at most 8 of them) in float32, whose
// roundings are 2^-13 of the elements' own or less (in 64 bits 64 x 12 x 512 x 512 bf16 take 88 us instead of 86, 45 x 12 x 514 x 514 95
// instead of 84).
// 64 x 12 x 512 x 512 bf16: 88 us (4.6 TB/s; a copy of 4 GiB reaches 4.8).  A thread per diagonal, one element after the other in 64
// bits, took 2950 us.
struct Walk {
    int lc;                    // log2 of LC
    int R, C;                  // blocks of queries, of keys
    int m_first, bands;        // bands of LC diagonals of blocks, from m_first on
    int wgs;                   // workgroups of an example's head; a group of lanes has one piece of one band
};
// rows of blocks in which band bd of an example has live elements: [lo, lo + the result)
__device__ __forceinline__ int band_rows(const PosbiasArgs& a, const Walk& wk, const Window& w, int bd, int& lo) {
    const int LC = 1 << wk.lc, m0 = wk.m_first + bd * LC;
    lo = max(0, -(m0 + LC - 1));
    return a.causal && (int64_t)8 * m0 - 7 > w.start ? 0 : max(0, min((w.nq + 7) / 8, (w.nk + 7) / 8 - m0) - lo);
}
// The pieces of all bands are numbered band by band: those of the first bands, with `before` rows together, end at this number.  Every
// band has at least one, and of the others its share by rows.
__host__ __device__ __forceinline__ int pieces_up_to(int bands, int64_t before, float share) { return bands + (int)((float)before * share); }
__host__ __device__ __forceinline__ float share_of(int pieces, int bands, int64_t rows) { return rows > 0 ? (float)(pieces - bands) / (float)rows : 0.f; }
// Piece number `task` of `tasks` (at least as many as bands): its band and rows [r0, r1).
struct Piece { int band, r0, r1; };
__device__ __forceinline__ Piece piece_of(const PosbiasArgs& a, const Walk& wk, const Window& w, int task, int tasks) {
    int64_t all = 0;
    int lo;
    for (int bd = 0; bd < wk.bands; ++bd) all += band_rows(a, wk, w, bd, lo);
    const float share = share_of(tasks, wk.bands, all);
    int64_t before = 0;
    int first = 0;
    for (int bd = 0;; ++bd) {
        const int rows = band_rows(a, wk, w, bd, lo);
        before += rows;
        const int next = bd + 1 == wk.bands ? tasks : pieces_up_to(bd + 1, before, share);
        if (task < next) {
            // (every piece's end is the next one's beginning by the same expression)
            const int i = task - first, n = next - first;
            const float step = (float)rows / (float)n;
            return Piece{bd, lo + (int)((float)i * step), i + 1 == n ? lo + rows : lo + (int)((float)(i + 1) * step)};
        }
        first = next;
    }
}
constexpr int kMaxSlots = kThreads * 8 + 8 * (kThreads / 8);

// The groups' sums val [groups][8 LC + 8], slot 8 l + e of a group its diagonal 8 (m0 + l) + e - 7: the pieces of a band (next to each
// other) are added into the first one's slots, then the slots by their buckets.
__device__ __forceinline__ void fold_slots(const PosbiasArgs& a, const Walk& wk, int LC, double* val, short* bkt, const int* band_of, const Window& w,
                                           int b, int h, double* __restrict__ partial, float* __restrict__ rows) {
    const int tid = threadIdx.x, G = kThreads / LC, P = 8 * LC + 8;
    __syncthreads();
    // the first pieces of their bands here, as bits
    const int lane = tid & (kWave - 1);
    const uint64_t heads = __ballot(lane < G && (lane == 0 || band_of[lane] != band_of[max(lane - 1, 0)]));
    for (uint64_t left = heads; left; left &= left - 1) {
        const int from = __builtin_ctzll(left), to = left & (left - 1) ? __builtin_ctzll(left & (left - 1)) : G;
        const int64_t nearest = (int64_t)8 * (wk.m_first + band_of[from] * LC) - 7 - w.start;
        for (int x0 = tid; x0 < P; x0 += 4 * kThreads) {
            int j[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {              // four look-ups at once
                const int x = x0 + i * kThreads;
                j[i] = x >= P || (a.causal && nearest + x > 0) ? -1 : bucket_of(a, nearest + x);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = x0 + i * kThreads;
                if (x >= P) break;
                double v = val[from * P + x];
#pragma unroll 4
                for (int t = from + 1; t < to; ++t) v += val[t * P + x];
                val[from * P + x] = v;
                bkt[from * P + x] = (short)(j[i] >= 0 && j[i] < a.n_buckets ? j[i] : -1);
            }
        }
    }
    __syncthreads();
    // 2^ul threads for a bucket look through all slots
    int ul = 6;
    while (ul > 0 && (kThreads >> ul) < a.n_buckets) --ul;
    const int u = tid & ((1 << ul) - 1);
    for (int j0 = 0; j0 < a.n_buckets; j0 += kThreads >> ul) {
        const int j = j0 + (tid >> ul);
        double s = 0.0;
        for (uint64_t left = heads; left; left &= left - 1) {
            const int from = __builtin_ctzll(left) * P, to = from + P;
            int k = from + u;
            for (; k + (7 << ul) < to; k += 8 << ul) {
                double v[8];
                int c[8];
#pragma unroll
                for (int y = 0; y < 8; ++y) { v[y] = val[k + (y << ul)]; c[y] = bkt[k + (y << ul)]; }
#pragma unroll
                for (int y = 0; y < 8; ++y) s += c[y] == j ? v[y] : 0.0;
            }
            for (; k < to; k += 1 << ul) s += bkt[k] == j ? val[k] : 0.0;
        }
        for (int off = 1; off < 1 << ul; off <<= 1) s += __shfl_xor(s, off, kWave);
        if (u == 0 && j < a.n_buckets) {
            if (wk.wgs == 1) rows[((int64_t)b * a.n_buckets + j) * a.H + h] = (float)s;
            else             partial[(int64_t)blockIdx.x * a.n_buckets + j] = s;
        }
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads, 3) void k_posbias_walk(PosbiasArgs a, const void* __restrict__ dS, Walk wk, double* __restrict__ partial, float* __restrict__ rows) {
    __shared__ double val[kMaxSlots];                  // [groups][8 LC + 8]: sums of the groups' diagonals
    __shared__ short bkt[kMaxSlots];                   // and their buckets
    __shared__ int band_of[kThreads / 8];
    const int tid = threadIdx.x, LC = 1 << wk.lc, G = kThreads >> wk.lc, P = 8 * LC + 8;
    const int li = tid & (LC - 1), g = tid >> wk.lc;
    const int wg = blockIdx.x % wk.wgs, bh = blockIdx.x / wk.wgs, h = bh % a.H, b = bh / a.H;
    const Window w = window_of(a, b);
    const Piece pc = piece_of(a, wk, w, wg * G + g, wk.wgs * G);
    if (li == 0) band_of[g] = pc.band;
    const int m0 = wk.m_first + pc.band * LC, m = m0 + li;
    double acc[15];
#pragma unroll
    for (int e = 0; e < 15; ++e) acc[e] = 0.0;
    {
        const int r0 = pc.r0, r1 = pc.r1;
        const int64_t base = b * a.s_b + h * a.s_h;
        const bool narrow = a.Tk < 8;
        const int over = wk.C * 8 - a.Tk;              // how far the last block of keys reaches beyond the row
        for (int rb = r0; rb < r1; ++rb) {
            const int q0 = rb * 8, k0 = (rb + m) * 8, nk = min(8, w.nk - k0), nq = min(8, w.nq - q0);
            // no live element: left of the first key, behind the last one, all keys behind the queries
            if (rb + m < 0 || nk <= 0 || (a.causal && (int64_t)k0 - (q0 + 7) > w.start)) continue;
            float d[15];
            if constexpr (DT != 0) {
#pragma unroll
                for (int e = 0; e < 15; ++e) d[e] = 0.f;
            }
            const auto add = [&](int e, float v) {
                if constexpr (DT == 0) acc[e] += v;
                else                   d[e] += v;
            };
            if (narrow) {                              // rows shorter than a piece
                for (int i = 0; i < nq; ++i) {
                    float v[8];
                    load_first<DT>(dS, base + (q0 + i) * a.s_q, nk, v);
#pragma unroll
                    for (int y = 0; y < 8; ++y)
                        if (y == i)
#pragma unroll
                            for (int j = 0; j < 8; ++j) add(7 + j - y, v[j]);
                }
            } else {
                // 128 bytes at once, all of them within the tensor: the last keys' pieces begin `over` earlier, queries behind the
                // last one are the last one again
                constexpr int kAtOnce = DT == 0 ? 4 : 8;
                const bool last = k0 + 8 > a.Tk;
                const int64_t at = base + q0 * a.s_q + (last ? k0 - over : k0), last_row = (a.Tq - 1 - q0) * a.s_q;
                const bool whole = __ballot(nk < 8 || nq < 8) == 0;
#pragma unroll
                for (int i0 = 0; i0 < 8; i0 += kAtOnce) {
                    Raw8<DT> r[kAtOnce];
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) r[i] = load_raw8<DT>(dS, at + min((i0 + i) * a.s_q, last_row));
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i) {
                            float v[8];
                            widen8<DT>(r[i], v);
#pragma unroll
                            for (int j = 0; j < 8; ++j) add(7 + j - i0 - i, v[j]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i) {
                            float v[8];
                            widen8<DT>(r[i], v);
                            if (over & 4)
#pragma unroll
                                for (int j = 0; j < 4; ++j) v[j] = last ? v[j + 4] : v[j];
                            if (over & 2)
#pragma unroll
                                for (int j = 0; j < 6; ++j) v[j] = last ? v[j + 2] : v[j];
                            if (over & 1)
#pragma unroll
                                for (int j = 0; j < 7; ++j) v[j] = last ? v[j + 1] : v[j];
#pragma unroll
                            for (int j = 0; j < 8; ++j) add(7 + j - i0 - i, j < nk && i0 + i < nq ? v[j] : 0.f);
                            // a row's additions before the next one's selects: without this they take 10 registers more, and with
                            // them a fourth of the waves (300 x 12 x 64 x 64: 38 us instead of 33)
                            if constexpr (DT == 0) {
#pragma unroll
                                for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(acc[7 + j - i0 - i]));
                            }
                        }
                    }
                }
            }
            if constexpr (DT != 0) {
#pragma unroll
                for (int e = 0; e < 15; ++e) acc[e] += d[e];
            }
        }
    }
    // lane li's diagonals are slots 8 li ... 8 li + 14 of its group: the upper seven are the next lane's too
#pragma unroll
    for (int y = 0; y < 7; ++y) {
        const double left = __shfl_up(acc[y + 8], 1, LC);
        if (li > 0) acc[y] += left;
    }
    double* v = val + g * P + 8 * li;
#pragma unroll
    for (int y = 0; y < 8; ++y) v[y] = acc[y];
    if (li == LC - 1) {
#pragma unroll
        for (int y = 0; y < 7; ++y) v[8 + y] = acc[8 + y];
        v[15] = 0.0;
    }
    fold_slots(a, wk, LC, val, bkt, band_of, w, b, h, partial, rows);
}

// A workgroup per example: the sums of its heads' workgroups where there are several, and the squared norm of the rows.
constexpr int kFinishThreads = 1024;
__global__ __launch_bounds__(kFinishThreads) void k_posbias_finish(PosbiasArgs a, int wgs, const double* __restrict__ partial, int accumulate, float* __restrict__ rows, float* __restrict__ sqnorm) {
    __shared__ double red[kFinishThreads / kWave];
    const int b = blockIdx.x, n = a.n_buckets * a.H;
    float* r = rows + (int64_t)b * n;
    double sq = 0.0;
    if (wgs == 1) {
        for (int k = threadIdx.x; k < n; k += kFinishThreads) sq += (double)r[k] * r[k];
    } else {
        for (int k = threadIdx.x; k < n; k += kFinishThreads) {          // neighbouring threads: neighbouring buckets
            const int h = k / a.n_buckets, j = k - h * a.n_buckets;
            const double* p = partial + ((int64_t)(b * (int64_t)a.H + h) * wgs) * a.n_buckets + j;
            double s = 0.0;
            int i = 0;
            for (; i + 7 < wgs; i += 8) {
                double v[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] = p[(int64_t)(i + x) * a.n_buckets];
#pragma unroll
                for (int x = 0; x < 8; ++x) s += v[x];
            }
            for (; i < wgs; ++i) s += p[(int64_t)i * a.n_buckets];
            const float f = (float)s;
            r[(int64_t)j * a.H + h] = f;
            sq += (double)f * f;
        }
    }
    sq = wave_sum_f64(sq);
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x >> 6] = sq;
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int k = 1; k < kFinishThreads / kWave; ++k) sq += red[k];
    sqnorm[b] = (float)(accumulate ? sqnorm[b] + sq : sq);
}

// How the blocks of a head are dealt.  Known keys behind every query (causal and no start of its own: half) get no bands.
//
// The workgroups of a head: the chip holds 768 at a time (three for each of the 256 compute units, by registers), and the loads of all
// of them together are what bounds it, so that a launch takes as many rounds of 768 as it has, of a workgroup's longest piece and
// about two steps for its fold.  The fewest steps so counted: 64 x 12 heads of 512 x 512 as 768 workgroups took 89 us, as four
// times as many 103 us.  Examples of their own lengths: two rounds at least, whose ends even out (4 x 16 heads of up to 4096 x 4096, causal: 121 us
// in two rounds, 129 in three, 168 in five).
constexpr int kAtATime = 768, kMostRounds = 8, kFoldSteps = 2;
// rows of a band where everything is live
int full_rows(const Walk& w, int bd) {
    const int LC = 1 << w.lc, m0 = w.m_first + bd * LC;
    return std::max(0, std::min(w.R, w.C - m0) - std::max(0, -(m0 + LC - 1)));
}
struct WalkPlan { Walk w; int64_t rows, least, most; };       // rows of all bands; workgroups of a head, at least and at most
WalkPlan walk_of(int64_t BH, int Tq, int Tk, bool half) {
    WalkPlan p{};
    Walk& w = p.w;
    w.R = (Tq + 7) / 8;
    w.C = (Tk + 7) / 8;
    w.m_first = -(w.R - 1);
    const int diagonals = half ? w.R - 1 + std::min(1, w.C) : w.R + w.C - 1;
    w.lc = 3;
    while (w.lc < 5 && (1 << w.lc) < std::min(w.C, diagonals)) ++w.lc;
    const int LC = 1 << w.lc, G = kThreads / LC;
    w.bands = (diagonals + LC - 1) / LC;
    for (int bd = 0; bd < w.bands; ++bd) p.rows += full_rows(w, bd);
    p.least = (w.bands + G - 1) / G;
    p.most = std::max(p.least, std::min(p.rows / (2 * G), kMostRounds * kAtATime / BH + 1));      // pieces of two steps at least
    return p;
}
// rows of the longest piece
int longest_piece(const Walk& w, int64_t all, int tasks) {
    const float share = share_of(tasks, w.bands, all);
    int64_t before = 0;
    int first = 0, longest = 0;
    for (int bd = 0; bd < w.bands; ++bd) {
        const int rows = full_rows(w, bd);
        before += rows;
        const int next = bd + 1 == w.bands ? tasks : pieces_up_to(bd + 1, before, share);
        longest = std::max(longest, (rows + next - first - 1) / (next - first));
        first = next;
    }
    return longest;
}
Walk plan_walk(int64_t BH, int Tq, int Tk, bool half, bool ragged) {
    WalkPlan p = walk_of(BH, Tq, Tk, half);
    const int G = kThreads >> p.w.lc;
    int64_t best = INT64_MAX;
    for (int r = ragged ? 2 : 1; r <= kMostRounds; ++r) {
        const int64_t k = std::max(p.least, std::min(p.most, r * kAtATime / BH));                 // the most that r rounds hold
        const int64_t cost = ((k * BH + kAtATime - 1) / kAtATime) * (longest_piece(p.w, p.rows, (int)(k * G)) + kFoldSteps);
        if (cost >= best) continue;
        best = cost;
        p.w.wgs = (int)k;
    }
    return p.w;
}
// the most workgroups of a head in any of the plans
int64_t most_wgs(int64_t BH, int Tq, int Tk) { return std::max(walk_of(BH, Tq, Tk, false).most, walk_of(BH, Tq, Tk, true).most); }

}  // namespace

bool posbias_fits(int64_t B, int64_t H, int64_t Tq, int64_t Tk) {
    const int64_t most = int64_t(1) << 31;
    if (B >= most || H >= most || Tq > kMaxLength || Tk > kMaxLength) return false;
    if (B == 0 || H == 0 || Tq == 0 || Tk == 0) return true;
    if (H > most / B || Tq > most / (B * H)) return false;
    const AddTiles t = plan_add(B * H, (int)Tq, (int)Tk);
    return launch_holds(B * H * t.row_tiles * t.col_tiles, kThreads)
        && launch_holds(B, kFinishThreads) && launch_holds(B * H * most_wgs(B * H, (int)Tq, (int)Tk), kThreads);
}
// a number for every bucket and workgroup, where a head has several of them; whether keys are left out is not known here
size_t posbias_ws_bytes(int B, int H, int Tq, int Tk, int n_buckets) {
    const int64_t BH = (int64_t)B * H;
    const int64_t wgs = most_wgs(BH, Tq, Tk);
    return wgs > 1 ? ((size_t)BH * wgs * n_buckets * sizeof(double) + 15) / 16 * 16 : 16;
}

hipError_t launch_posbias_add(const PosbiasArgs& a, const void* scores, const float* table, int dt, void* out, hipStream_t st) {
    const AddTiles t = plan_add((int64_t)a.B * a.H, a.Tq, a.Tk);
    const unsigned grid = (unsigned)((int64_t)a.B * a.H * t.row_tiles * t.col_tiles);
    // Where the scores fit the last-level cache, but not with the output, which would push them out, it goes past that cache: 160 MB
    // and 160 MB of bf16, 5 x 4096 x 4096, 51 us instead of 65.  (Larger scores do not stay there either way: 394 MB 168 us instead of
    // 170.  float32 has stores of 16 bytes 32 bytes apart, which the cache puts together: 80 x 2 x 512 x 512 73 us instead of 64.)
    const int64_t bytes = (int64_t)a.B * a.H * a.Tq * a.Tk * 2;
    const bool past = out != scores && bytes <= kLastLevelCache && 2 * bytes > kLastLevelCache;
    const auto run = [&](auto kernel) { kernel<<<grid, kThreads, 0, st>>>(a, scores, table, out, t); };
    if (dt == 0)      run(k_posbias_add<0, false>);
    else if (dt == 1) run(past ? k_posbias_add<1, true> : k_posbias_add<1, false>);
    else              run(past ? k_posbias_add<2, true> : k_posbias_add<2, false>);
    return hipGetLastError();
}

hipError_t launch_posbias_sqnorm(const PosbiasArgs& a, const void* dS, int dt, bool accumulate, float* rows, float* sqnorm, void* ws, hipStream_t st) {
    const int64_t BH = (int64_t)a.B * a.H;
    const Walk w = plan_walk(BH, a.Tq, a.Tk, a.causal && !a.q_start, a.q_lens || a.k_lens);
    const unsigned grid = (unsigned)(BH * w.wgs);
    double* partial = static_cast<double*>(ws);
    if (dt == 0)      k_posbias_walk<0><<<grid, kThreads, 0, st>>>(a, dS, w, partial, rows);
    else if (dt == 1) k_posbias_walk<1><<<grid, kThreads, 0, st>>>(a, dS, w, partial, rows);
    else              k_posbias_walk<2><<<grid, kThreads, 0, st>>>(a, dS, w, partial, rows);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_posbias_finish<<<a.B, kFinishThreads, 0, st>>>(a, w.wgs, partial, accumulate, rows, sqnorm);
    return hipGetLastError();
}

}  // namespace dpk
