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

// A workgroup per piece of 256 keys of eight queries.
constexpr int kAddRows = 8;
template <int DT>
__global__ __launch_bounds__(kThreads) void k_posbias_add(PosbiasArgs a, const void* scores, const float* __restrict__ table, void* out, int pieces, int row_blocks) {
    const int piece = blockIdx.x % pieces, rb = blockIdx.x / pieces;
    const int q0 = rb % row_blocks * kAddRows, bh = rb / row_blocks, h = bh % a.H, b = bh / a.H;
    const Window w = window_of(a, b);
    const int k = piece * kThreads + threadIdx.x;
    if (k >= w.nk) return;
    for (int q = q0; q < min(q0 + kAddRows, w.nq); ++q) {
        const int64_t distance = (int64_t)k - q - w.start;
        if (a.causal && distance > 0) continue;
        const int j = bucket_of(a, distance);
        const float bias = j >= 0 && j < a.n_buckets ? table[j * a.H + h] : 0.f;
        const float s = load_one<DT>(scores, b * a.s_b + h * a.s_h + q * a.s_q + k);
        store_one<DT>(out, b * a.o_b + h * a.o_h + q * a.o_q + k, s + bias);
    }
}

// Diagonal d of a head, 0 <= d < Tq + Tk - 1, holds the pairs with k - q = d - (Tq - 1).  A thread adds one up; the threads
// of a wave have neighbouring ones, whose elements of a query are next to each other.
template <int DT>
__global__ __launch_bounds__(kThreads) void k_posbias_diagonals(PosbiasArgs a, const void* __restrict__ dS, int diagonals, int pieces, double* __restrict__ sums) {
    const int bh = blockIdx.x / pieces, h = bh % a.H, b = bh / a.H;
    const int d = (blockIdx.x % pieces) * kThreads + threadIdx.x;
    if (d >= diagonals) return;
    const Window w = window_of(a, b);
    const int off = d - (a.Tq - 1);
    double acc = 0.0;
    if (!a.causal || off <= w.start) {
        const int64_t base = b * a.s_b + h * a.s_h + off;
        const int last = min(w.nq, w.nk - off);
        for (int q = max(0, -off); q < last; ++q) acc += load_one<DT>(dS, base + q * (a.s_q + 1));
    }
    sums[(int64_t)bh * diagonals + d] = acc;
}

// A workgroup per example and head: the diagonals' sums by buckets.  The lanes of a wave that share a bucket are added by the
// wave, one bucket after the other, into the wave's own sums: a fixed order.
__global__ __launch_bounds__(kThreads) void k_posbias_fold(PosbiasArgs a, const double* __restrict__ sums, int diagonals, float* __restrict__ rows) {
    extern __shared__ double acc[];                    // [waves][n_buckets]
    constexpr int kWaves = kThreads / kWave;
    const int bh = blockIdx.x, h = bh % a.H, b = bh / a.H, wave = threadIdx.x >> 6, lane = threadIdx.x & (kWave - 1);
    for (int j = threadIdx.x; j < kWaves * a.n_buckets; j += kThreads) acc[j] = 0.0;
    __syncthreads();
    const Window w = window_of(a, b);
    for (int d0 = wave * kWave; d0 < diagonals; d0 += kThreads) {
        const int d = d0 + lane;
        int j = -1;
        double v = 0.0;
        if (d < diagonals) {
            v = sums[(int64_t)bh * diagonals + d];
            j = bucket_of(a, (int64_t)d - (a.Tq - 1) - w.start);
            if (j >= a.n_buckets) j = -1;
        }
        for (uint64_t left = __ballot(j >= 0); left;) {
            const int one = __builtin_amdgcn_readlane(j, (int)__builtin_ctzll(left));
            const double s = wave_sum_f64(j == one ? v : 0.0);
            if (lane == 0) acc[wave * a.n_buckets + one] += s;
            left &= ~__ballot(j == one);
        }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < a.n_buckets; j += kThreads) {
        double s = acc[j];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) s += acc[k * a.n_buckets + j];
        rows[((int64_t)b * a.n_buckets + j) * a.H + h] = (float)s;
    }
}

}  // namespace

bool posbias_fits(int64_t B, int64_t H, int64_t Tq, int64_t Tk) {
    const int64_t most = int64_t(1) << 31;
    if (B >= most || H >= most || Tq >= most / 2 || Tk >= most / 2) return false;
    if (B == 0 || H == 0 || Tq == 0 || Tk == 0) return true;
    if (H > most / B || Tq > most / (B * H)) return false;
    const int64_t pieces_add = (Tk + kThreads - 1) / kThreads, pieces = (Tq + Tk - 1 + kThreads - 1) / kThreads;
    return launch_holds(B * H * ((Tq + kAddRows - 1) / kAddRows) * pieces_add, kThreads) && launch_holds(B * H * pieces, kThreads);
}
size_t posbias_ws_bytes(int B, int H, int Tq, int Tk) { return (size_t)B * H * ((size_t)Tq + Tk - 1) * sizeof(double); }

hipError_t launch_posbias_add(const PosbiasArgs& a, const void* scores, const float* table, int dt, void* out, hipStream_t st) {
    const int pieces = ceil_div(a.Tk, kThreads);
    const int row_blocks = ceil_div(a.Tq, kAddRows);
    const unsigned grid = (unsigned)((int64_t)a.B * a.H * row_blocks * pieces);
    if (dt == 0)      k_posbias_add<0><<<grid, kThreads, 0, st>>>(a, scores, table, out, pieces, row_blocks);
    else if (dt == 1) k_posbias_add<1><<<grid, kThreads, 0, st>>>(a, scores, table, out, pieces, row_blocks);
    else              k_posbias_add<2><<<grid, kThreads, 0, st>>>(a, scores, table, out, pieces, row_blocks);
    return hipGetLastError();
}

hipError_t launch_posbias_rows(const PosbiasArgs& a, const void* dS, int dt, float* rows, void* ws, hipStream_t st) {
    const int diagonals = a.Tq + a.Tk - 1, pieces = ceil_div(diagonals, kThreads);
    const unsigned grid = (unsigned)((int64_t)a.B * a.H * pieces);
    double* sums = static_cast<double*>(ws);
    if (dt == 0)      k_posbias_diagonals<0><<<grid, kThreads, 0, st>>>(a, dS, diagonals, pieces, sums);
    else if (dt == 1) k_posbias_diagonals<1><<<grid, kThreads, 0, st>>>(a, dS, diagonals, pieces, sums);
    else              k_posbias_diagonals<2><<<grid, kThreads, 0, st>>>(a, dS, diagonals, pieces, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_posbias_fold<<<a.B * a.H, kThreads, (size_t)(kThreads / kWave) * a.n_buckets * sizeof(double), st>>>(a, sums, diagonals, rows);
    return hipGetLastError();
}

}  // namespace dpk
