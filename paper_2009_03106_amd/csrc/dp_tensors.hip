// Norm and clipping of a gradient of many tensors:  norm = sqrt(sum_l sum_j x_l[j]^2),
//     out_l = (accumulate ? out_l : 0) + 1 / max(1, norm / C) * x_l.
// Bound by memory: the norm has to be known before the first product, so x is read twice (the second time out of the
// last-level cache where the set fits it) and out is written once.
//
// The tensors are cut into chunks of one size, a workgroup each; the sum of a chunk's squares is one double of the
// workspace.  Squares and sums are doubles: a square of any float32 is exact and in range there, and their two
// instructions per element stay behind the loads.  The order of the additions is fixed.
#include <algorithm>
#include "dp_elems.h"
#include "dp_internal.h"

namespace dpk {

namespace {

// Descriptors travel as kernel arguments, whose block holds 4 KB; longer lists are written to the head of the
// workspace by small launches first.
constexpr int kDirectItems = 112;
struct ItemTable { TensorItem items[kDirectItems]; };

__global__ __launch_bounds__(128) void k_tensors_table(ItemTable t, int n, TensorItem* __restrict__ out) {
    if ((int)threadIdx.x < n) out[threadIdx.x] = t.items[threadIdx.x];
}

// the item that chunk c belongs to: the last one that begins at c or before; 256 candidates at a time
__device__ __forceinline__ int find_item(const TensorItem* __restrict__ items, int n, int c) {
    int lo = 0, len = n;
    while (len > 1) {
        const int step = (len + kThreads - 1) / kThreads;
        const int k = (int)threadIdx.x * step;
        const int before = __syncthreads_count(k < len && items[lo + k].first_chunk <= c);      // at least 1: lo itself
        const int skip = (before - 1) * step;
        lo += skip;
        len = min(step, len - skip);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// by 256 threads, tid this one's number
template <int DT> __device__ __forceinline__ double sum_squares(const void* __restrict__ x, int64_t begin, int64_t end, int tid) {
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    auto add = [&](const Raw8<DT>& r) {
        float v[8];
        widen8<DT>(r, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) { const double d = v[j]; acc[j & 3] = fma(d, d, acc[j & 3]); }
    };
    int64_t k = begin + tid * 8;
    for (; k + 3 * 8 * kThreads + 8 <= end; k += 4 * 8 * kThreads) {       // four loads in flight
        Raw8<DT> r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = load_raw8<DT>(x, k + i * 8 * kThreads);
#pragma unroll
        for (int i = 0; i < 4; ++i) add(r[i]);
    }
    for (; k + 8 <= end; k += 8 * kThreads) add(load_raw8<DT>(x, k));
    for (; k < end; ++k) { const double d = load_one<DT>(x, k); acc[0] = fma(d, d, acc[0]); }      // the last elements: one thread's
    return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

__device__ __forceinline__ double chunk_squares(const TensorItem& it, int64_t begin, int64_t chunk, int tid) {
    const int64_t end = min(it.n, begin + chunk);
    switch (it.dt) {
    case 0: return sum_squares<0>(it.x, begin, end, tid);
    case 1: return sum_squares<1>(it.x, begin, end, tid);
    default: return sum_squares<2>(it.x, begin, end, tid);
    }
}

template <bool DIRECT>
__global__ __launch_bounds__(kThreads) void k_tensors_squares(ItemTable t, const TensorItem* __restrict__ table, int n, int64_t chunk, double* __restrict__ partial) {
    __shared__ double red[4];
    const TensorItem* items = DIRECT ? t.items : table;
    const int c = blockIdx.x, i = find_item(items, n, c);
    const double s = block_sum_256_f64(chunk_squares(items[i], (int64_t)(c - items[i].first_chunk) * chunk, chunk, threadIdx.x), red);
    if (threadIdx.x == 0) partial[c] = s;
}

// the sum of all chunks, by every workgroup that asks in the same order
__device__ __forceinline__ double sum_partials(const double* __restrict__ partial, int chunks, double* red) {
    double s = 0.0;
    int c = threadIdx.x;
    for (; c + 7 * kThreads < chunks; c += 8 * kThreads) {
        double v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = partial[c + k * kThreads];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[k];
    }
    for (; c < chunks; c += kThreads) s += partial[c];
    return block_sum_256_f64(s, red);
}

// norms of the tensors by themselves: a wave adds up an item's chunks
__device__ __forceinline__ void item_norm(const double* __restrict__ partial, int first, int last, float* out) {
    double s = 0.0;
    for (int c = first + (threadIdx.x & (kWave - 1)); c < last; c += kWave) s += partial[c];
    s = wave_sum_f64(s);
    if ((threadIdx.x & (kWave - 1)) == 0) *out = (float)sqrt(s);
}

// workgroup 0: the norm, and in 64 bits for the launch that scales (wide, if not NULL); the others: the norms of four tensors each
template <bool DIRECT>
__global__ __launch_bounds__(kThreads) void k_tensors_fold(ItemTable t, const TensorItem* __restrict__ table, int n, int chunks, const double* __restrict__ partial,
                                                           int accumulate, float* __restrict__ norm, double* __restrict__ wide, float* __restrict__ tensor_norms) {
    __shared__ double red[4];
    const TensorItem* items = DIRECT ? t.items : table;
    if (blockIdx.x == 0) {
        double s = sum_partials(partial, chunks, red);
        if (threadIdx.x == 0) {
            if (accumulate) { const double old = norm[0]; s += old * old; }
            norm[0] = (float)sqrt(s);
            if (wide) wide[0] = sqrt(s);
        }
        return;
    }
    const int i = (blockIdx.x - 1) * (kThreads / kWave) + (threadIdx.x >> 6);
    if (i < n) item_norm(partial, items[i].first_chunk, i + 1 < n ? items[i + 1].first_chunk : chunks, tensor_norms + i);
}

// The factor 1 / max(1, norm / C), as a number that x is multiplied with first and one that follows.  norm / C is a float32 quotient
// of the rounded norm while its reciprocal is a normal number (so a norm that was stored gives the same bits as the one it was
// rounded from).  Beyond that it is taken in 64 bits, from the norm before its rounding where that is infinite, and where the
// factor is below the normal numbers, x is scaled by 2^-126 first: what that rounds is below the result's own steps there.
struct Factor { float first, then; };
__device__ __forceinline__ Factor factor_of(double wide, float C) {
    const float norm = (float)wide, m = norm / C;
    if (m <= 0x1p126f) return Factor{1.0f, 1.0f / fmaxf(m, 1.0f)};
    const double q = (double)C / (isinf(norm) ? wide : (double)norm), f = q > 1.0 ? 1.0 : q;       // NaN: lets it through
    return f < 0x1p-126 ? Factor{0x1p-126f, (float)(f * 0x1p126)} : Factor{1.0f, (float)f};
}

// From the chunk's end, which the last-level cache got last.  Four pieces in flight, of 16 bytes where they are stored, next to each other
// for neighbouring threads.  (340 MB of float32 in 2048 chunks: 176 us for the call, 192 with pieces of 32 bytes one at a time from the
// beginning.  2 GB, most of it bf16: 1213 us, 1284 one at a time.)
template <int DT, int ODT, bool PAST> __device__ __forceinline__ void scale(const void* x, void* out, int64_t begin, int64_t end, Factor f, bool accumulate, int tid) {
    constexpr int V = ODT == 0 ? 4 : 8, U = 4;
    constexpr int64_t step = V * kThreads;
    const auto put = [&](int64_t k, float (&v)[V]) {
        if (accumulate) {
            float o[V];
            load_piece<ODT>(out, k, o);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = o[j] + f.then * (f.first * v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = f.then * (f.first * v[j]);
        }
        store_piece<ODT, PAST>(out, k, v);
    };
    int64_t m = (end - begin + step - 1) / step - 1;   // pieces of all threads together
    if (m >= 0 && begin + (m + 1) * step > end) {      // the last ones, not of all threads
        int64_t k = begin + m-- * step + tid * V;
        if (k + V <= end) {
            float v[V];
            load_piece<DT>(x, k, v);
            put(k, v);
        } else {
            for (; k < end; ++k) {
                const float v = f.then * (f.first * load_one<DT>(x, k));
                store_one<ODT>(out, k, accumulate ? load_one<ODT>(out, k) + v : v);
            }
        }
    }
    int64_t k = begin + m * step + tid * V;
    for (; m >= U - 1; m -= U, k -= U * step) {
        float v[U][V];
#pragma unroll
        for (int i = 0; i < U; ++i) load_piece<DT>(x, k - i * step, v[i]);
#pragma unroll
        for (int i = 0; i < U; ++i) put(k - i * step, v[i]);
    }
    for (; m >= 0; --m, k -= step) {
        float v[V];
        load_piece<DT>(x, k, v);
        put(k, v);
    }
}
template <bool PAST> __device__ __forceinline__ void chunk_scale(const TensorItem& it, int64_t begin, int64_t chunk, Factor f, bool accumulate, int tid) {
    if (f.first == 1.0f && f.then == 1.0f && it.x == it.out && !accumulate) return;                // a factor of 1 leaves every value as it is
    const int64_t end = min(it.n, begin + chunk);
    switch (it.dt * 4 + it.odt) {
    case 0: scale<0, 0, PAST>(it.x, it.out, begin, end, f, accumulate, tid); break;
    case 4: scale<1, 0, PAST>(it.x, it.out, begin, end, f, accumulate, tid); break;
    case 5: scale<1, 1, PAST>(it.x, it.out, begin, end, f, false, tid); break;
    case 8: scale<2, 0, PAST>(it.x, it.out, begin, end, f, accumulate, tid); break;
    default: scale<2, 2, PAST>(it.x, it.out, begin, end, f, false, tid); break;
    }
}
// partial != nullptr: the norm is taken from the chunks' sums by every workgroup for itself, and written.  wide != nullptr: it is there
// in 64 bits.  Neither: norm is the caller's.  PAST: the outputs go past
// the last-level cache, which they would not fit, and leave it to the inputs that are still to be read.
template <bool DIRECT, bool PAST>
__global__ __launch_bounds__(kThreads) void k_tensors_scale(ItemTable t, const TensorItem* __restrict__ table, int n, int64_t chunk, int chunks, int accumulate,
                                                            const double* __restrict__ partial, const double* __restrict__ wide, float* __restrict__ norm, float* __restrict__ tensor_norms, float C) {
    __shared__ double red[4];
    const TensorItem* items = DIRECT ? t.items : table;
    const int c = chunks - 1 - blockIdx.x, i = find_item(items, n, c);        // the last chunks are in the last-level cache (2 GB: 1213 us, 1255 from the first one)
    double total;
    if (partial) {
        total = sqrt(sum_partials(partial, chunks, red));
        if (c == 0 && threadIdx.x == 0) norm[0] = (float)total;
        if (tensor_norms && c == items[i].first_chunk && threadIdx.x < kWave)
            item_norm(partial, c, i + 1 < n ? items[i + 1].first_chunk : chunks, tensor_norms + i);
    } else {
        total = wide ? wide[0] : norm[0];
    }
    chunk_scale<PAST>(items[i], (int64_t)(c - items[i].first_chunk) * chunk, chunk, factor_of(total, C), accumulate, threadIdx.x);
}

// A few chunks of the smallest size: one workgroup takes the norm, with the sums of the launches above in their order, and scales.
// (One dense layer of 64 x 32 with its bias: a launch instead of two, 6.5 us instead of 10.5, most of it the host's.)
constexpr int kFewChunks = 16, kFewThreads = 1024;
__global__ __launch_bounds__(kFewThreads) void k_tensors_few(ItemTable t, int n, int chunks, int accumulate, float* __restrict__ norm, float* __restrict__ tensor_norms, float C) {
    __shared__ double partial[kFewChunks];
    __shared__ double red[kFewThreads / kWave];
    const int tid = threadIdx.x & (kThreads - 1), lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, group = threadIdx.x / kThreads;
    constexpr int kGroups = kFewThreads / kThreads;
    const auto item_of = [&](int c) {
        int i = 0;
        while (i + 1 < n && t.items[i + 1].first_chunk <= c) ++i;
        return i;
    };
    for (int c0 = 0; c0 < chunks; c0 += kGroups) {
        const int c = c0 + group;
        double s = 0.0;
        if (c < chunks) {
            const int i = item_of(c);
            s = chunk_squares(t.items[i], (int64_t)(c - t.items[i].first_chunk) * kTensorChunk, kTensorChunk, tid);
        }
        s = wave_sum_f64(s);
        if (lane == 0) red[wave] = s;
        __syncthreads();
        if (tid == 0 && c < chunks) partial[c] = (red[4 * group] + red[4 * group + 1]) + (red[4 * group + 2] + red[4 * group + 3]);
        __syncthreads();
    }
    const double total = sqrt(wave_sum_f64(lane < chunks ? partial[lane] : 0.0));
    if (threadIdx.x == 0) norm[0] = (float)total;
    if (tensor_norms && wave < n) {
        const int last = wave + 1 < n ? t.items[wave + 1].first_chunk : chunks, c = t.items[wave].first_chunk + lane;
        const double s = wave_sum_f64(c < last ? partial[c] : 0.0);
        if (lane == 0) tensor_norms[wave] = (float)sqrt(s);
    }
    const Factor f = factor_of(total, C);
    for (int c = group; c < chunks; c += kGroups) {
        const int i = item_of(c);
        chunk_scale<false>(t.items[i], (int64_t)(c - t.items[i].first_chunk) * kTensorChunk, kTensorChunk, f, accumulate, tid);
    }
}

// Workspace: the table of items that do not fit the arguments, then the chunks' sums, then the norm in 64 bits.
size_t table_bytes(int64_t n) { return n > kDirectItems ? (size_t)n * sizeof(TensorItem) : 0; }

struct Tables { ItemTable args; const TensorItem* table = nullptr; double* partial = nullptr; };
hipError_t place_items(const TensorItem* items, int n, void* ws, hipStream_t st, Tables& t) {
    t.partial = reinterpret_cast<double*>(static_cast<unsigned char*>(ws) + table_bytes(n));
    if (n <= kDirectItems) {
        std::copy(items, items + n, t.args.items);
        return hipSuccess;
    }
    TensorItem* to = static_cast<TensorItem*>(ws);
    t.table = to;
    for (int at = 0; at < n; at += kDirectItems) {
        const int m = std::min(n - at, kDirectItems);
        std::copy(items + at, items + at + m, t.args.items);
        k_tensors_table<<<1, 128, 0, st>>>(t.args, m, to + at);
    }
    return hipGetLastError();
}

// Whether the outputs are larger than the last-level cache: nothing that reads them behind the call finds them there.
// (340 MB of float32: 164 us past the cache, 194 through it; 600 MB of bf16 304 and 333.  In place of the inputs, or added to sums, it
// makes no difference: 164 and 165, 253 and 252 for that float32, 329 and 330, 696 and 696 for that bf16.  Smaller outputs stay, for the
// optimizer step that reads them next.)
bool past_cache(const TensorItem* items, int n) {
    int64_t bytes = 0;
    for (int i = 0; i < n; ++i) bytes += items[i].n * (items[i].odt == 0 ? 4 : 2);
    return bytes > kLastLevelCache;
}

// Up to here every workgroup of the scaling launch adds up the chunks' sums by itself
constexpr int kOwnFold = 4096;

void squares(const Tables& t, int n, int64_t chunk, int chunks, hipStream_t st) {
    if (t.table) k_tensors_squares<false><<<chunks, kThreads, 0, st>>>(t.args, t.table, n, chunk, t.partial);
    else         k_tensors_squares<true><<<chunks, kThreads, 0, st>>>(t.args, nullptr, n, chunk, t.partial);
}
void fold(const Tables& t, int n, int chunks, bool accumulate, float* norm, double* wide, float* tensor_norms, hipStream_t st) {
    const int grid = 1 + (tensor_norms ? ceil_div(n, kThreads / kWave) : 0);
    if (t.table) k_tensors_fold<false><<<grid, kThreads, 0, st>>>(t.args, t.table, n, chunks, t.partial, accumulate, norm, wide, tensor_norms);
    else         k_tensors_fold<true><<<grid, kThreads, 0, st>>>(t.args, nullptr, n, chunks, t.partial, accumulate, norm, wide, tensor_norms);
}
void scaled(const Tables& t, int n, int64_t chunk, int chunks, bool accumulate, bool past, const double* partial, const double* wide, float* norm, float* tensor_norms, float C, hipStream_t st) {
    const auto run = [&](auto kernel, const TensorItem* table) {
        kernel<<<chunks, kThreads, 0, st>>>(t.args, table, n, chunk, chunks, accumulate, partial, wide, norm, tensor_norms, C);
    };
    if (t.table) run(past ? k_tensors_scale<false, true> : k_tensors_scale<false, false>, t.table);
    else         run(past ? k_tensors_scale<true, true> : k_tensors_scale<true, false>, nullptr);
}

}  // namespace

// Chunks of at least 4096 elements (two 16-byte pieces of float32 for every thread), and larger ones where that makes more than
// 2048 of them (eight workgroups for each of the 256 compute units, and sums that every workgroup still adds up by itself: 31 million
// float32 66 us, in smaller chunks and with a launch for the sums 72).  From 67 million elements on there are eight times as many, of
// the smallest size at least: the ends of the last ones matter less, and of a set beyond the last-level cache what the first pass reads
// last is then a part, where the second one begins (340 MB of float32 164 us, 171 in 2048 chunks, all of which are worked on at once; 2 GB of
// bf16 1072 and 1095).  Of 16 bits that the cache still holds it is about even: 140 MB of bf16 72 us and 70, in place 72 and 70,
// added to float32 sums 157 and 169; 250 MB 141 and 147, 117 and 116, 279 and 301.
int64_t tensor_chunk_elems(int64_t total) {
    const int64_t unit = 8 * kThreads, most = total < (int64_t)kTensorChunk * kTensorChunksLarge ? kTensorChunks : kTensorChunksLarge;
    return std::max<int64_t>(kTensorChunk, (total / most + unit) / unit * unit);
}
size_t tensors_ws_bytes(int64_t n_tensors) {
    return table_bytes(n_tensors) + (size_t)(kTensorChunksLarge + n_tensors + 1) * sizeof(double);
}

hipError_t launch_tensors_norm(const TensorItem* items, int n, int64_t chunk, int chunks, bool accumulate, float* norm, float* tensor_norms, void* ws, hipStream_t st) {
    Tables t;
    const hipError_t e = place_items(items, n, ws, st, t);
    if (e != hipSuccess) return e;
    squares(t, n, chunk, chunks, st);
    fold(t, n, chunks, accumulate, norm, nullptr, tensor_norms, st);
    return hipGetLastError();
}
hipError_t launch_tensors_clip(const TensorItem* items, int n, int64_t chunk, int chunks, bool accumulate, const float* norm, float C, void* ws, hipStream_t st) {
    Tables t;
    const hipError_t e = place_items(items, n, ws, st, t);
    if (e != hipSuccess) return e;
    scaled(t, n, chunk, chunks, accumulate, past_cache(items, n), nullptr, nullptr, const_cast<float*>(norm), nullptr, C, st);
    return hipGetLastError();
}
hipError_t launch_tensors_norm_clip(const TensorItem* items, int n, int64_t chunk, int chunks, bool accumulate, float* norm, float* tensor_norms, float C, void* ws, hipStream_t st) {
    Tables t;
    const hipError_t e = place_items(items, n, ws, st, t);
    if (e != hipSuccess) return e;
    if (chunks <= kFewChunks && chunk == kTensorChunk) {
        k_tensors_few<<<1, kFewThreads, 0, st>>>(t.args, n, chunks, accumulate, norm, tensor_norms, C);
        return hipGetLastError();
    }
    squares(t, n, chunk, chunks, st);
    if (chunks > kOwnFold) {
        double* wide = t.partial + chunks;
        fold(t, n, chunks, false, norm, wide, tensor_norms, st);
        scaled(t, n, chunk, chunks, accumulate, past_cache(items, n), nullptr, wide, norm, nullptr, C, st);
    } else {
        scaled(t, n, chunk, chunks, accumulate, past_cache(items, n), t.partial, nullptr, norm, tensor_norms, C, st);
    }
    return hipGetLastError();
}

}  // namespace dpk
