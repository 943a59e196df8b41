// C-ABI entry points of the norm and clipping of many tensors (include/dpclip.h): argument checks and the cut into chunks.
#include "../../include/dpclip.h"
#include "dp_internal.h"
#include <algorithm>
#include <new>
#include <vector>

using namespace dpk;

namespace {

constexpr int64_t kMaxTensors = int64_t(1) << 20;
constexpr int64_t kMaxElements = int64_t(1) << 48;

size_t elem_bytes(dp_dtype d) { return d == DP_F32 ? 4 : 2; }
bool ok_type(dp_dtype d) { return d == DP_F32 || d == DP_BF16 || d == DP_F16; }
bool is8(dp_dtype d) { return d == DP_F8_E4M3 || d == DP_F8_E5M2 || d == DP_F8_E4M3_E5M2; }
bool element_aligned(const void* p, dp_dtype d) { return reinterpret_cast<uintptr_t>(p) % elem_bytes(d) == 0; }

struct Range { uintptr_t begin, end; bool out; int64_t i; };

// Whether the outputs are apart from each other and from every input but their own (which they may be in place of).
bool outputs_apart(const dp_tensor_desc* t, int64_t n) {
    // the usual cases without a sort: ascending addresses, all in place or all outputs on one side of all inputs
    bool ascending = true, in_place = true;
    uintptr_t end = 0, x_lo = UINTPTR_MAX, x_hi = 0, o_lo = UINTPTR_MAX, o_hi = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (t[i].n == 0) continue;
        const uintptr_t x = (uintptr_t)t[i].x, o = (uintptr_t)t[i].out;
        ascending = ascending && o >= end;
        end = o + (size_t)t[i].n * elem_bytes(t[i].out_dtype);
        in_place = in_place && x == o;
        x_lo = std::min(x_lo, x);
        x_hi = std::max(x_hi, x + (size_t)t[i].n * elem_bytes(t[i].dtype));
        o_lo = std::min(o_lo, o);
        o_hi = std::max(o_hi, end);
    }
    if (ascending && (in_place || o_lo >= x_hi || x_lo >= o_hi)) return true;
    std::vector<Range> r;
    r.reserve(2 * (size_t)n);
    for (int64_t i = 0; i < n; ++i) {
        if (t[i].n == 0) continue;
        const uintptr_t x = (uintptr_t)t[i].x, o = (uintptr_t)t[i].out;
        r.push_back({o, o + (size_t)t[i].n * elem_bytes(t[i].out_dtype), true, i});
        if (x != o) r.push_back({x, x + (size_t)t[i].n * elem_bytes(t[i].dtype), false, i});      // in place: the same range
    }
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    // in order of their beginnings: no output begins before the end of any earlier range, no input before that of an earlier output
    uintptr_t end_any = 0, end_out = 0;
    for (const Range& a : r) {
        if (a.begin < (a.out ? end_any : end_out)) return false;
        end_any = std::max(end_any, a.end);
        if (a.out) end_out = std::max(end_out, a.end);
    }
    return true;
}

// Checks the descriptors and cuts them into chunks.  clip: the outputs count.
dp_status plan_tensors(const dp_tensor_desc* t, int64_t n, bool clip, bool accumulate, std::vector<TensorItem>& items, int64_t& chunk, int& chunks) {
    if (n < 0 || (n > 0 && !t)) return DP_ERR_INVALID_ARG;
    if (n > kMaxTensors) return DP_ERR_UNSUPPORTED;
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (t[i].n < 0) return DP_ERR_INVALID_ARG;
        if (is8(t[i].dtype) || (clip && is8(t[i].out_dtype))) return DP_ERR_UNSUPPORTED;
        if (!ok_type(t[i].dtype)) return DP_ERR_INVALID_ARG;
        if (t[i].n > kMaxElements || (total += t[i].n) > kMaxElements) return DP_ERR_UNSUPPORTED;
        if (t[i].n > 0 && (!t[i].x || !element_aligned(t[i].x, t[i].dtype))) return DP_ERR_INVALID_ARG;
        if (!clip) continue;
        if (t[i].out_dtype != DP_F32 && (t[i].out_dtype != t[i].dtype || accumulate)) return DP_ERR_INVALID_ARG;
        if (t[i].n == 0) continue;
        if (!t[i].out || !element_aligned(t[i].out, t[i].out_dtype)) return DP_ERR_INVALID_ARG;
        if (t[i].x == t[i].out && t[i].dtype != t[i].out_dtype) return DP_ERR_INVALID_ARG;
    }
    if (clip && !outputs_apart(t, n)) return DP_ERR_INVALID_ARG;
    chunk = tensor_chunk_elems(total);
    items.resize((size_t)n);
    int64_t at = 0;
    for (int64_t i = 0; i < n; ++i) {
        items[i] = TensorItem{t[i].x, clip ? t[i].out : nullptr, t[i].n, (int)at, (short)t[i].dtype, (short)(clip ? t[i].out_dtype : t[i].dtype)};
        at += std::max<int64_t>(1, (t[i].n + chunk - 1) / chunk);
    }
    chunks = (int)at;
    return DP_OK;
}

bool scratch_ok(int64_t n, const void* ws, size_t bytes) {
    return ws && bytes >= tensors_ws_bytes(n) && (reinterpret_cast<uintptr_t>(ws) & 15) == 0;
}

// memory for the list of descriptors is all that can throw
template <class F> dp_status guarded(F&& f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return DP_ERR_UNSUPPORTED;
    } catch (...) {
        return DP_ERR_HIP;
    }
}

}  // namespace

extern "C" {

size_t dp_tensors_workspace_bytes(int64_t n_tensors) {
    return n_tensors < 0 || n_tensors > kMaxTensors ? 0 : tensors_ws_bytes(n_tensors);
}

dp_status dp_tensors_norm(const dp_tensor_desc* tensors, int64_t n_tensors, int accumulate, float* norm, float* tensor_norms,
                          void* workspace, size_t workspace_bytes, void* hip_stream) {
    return guarded([&]() -> dp_status {
        std::vector<TensorItem> items;
        int64_t chunk = 0;
        int chunks = 0;
        const dp_status s = plan_tensors(tensors, n_tensors, false, false, items, chunk, chunks);
        if (s != DP_OK) return s;
        if (!norm) return DP_ERR_INVALID_ARG;
        const hipStream_t st = static_cast<hipStream_t>(hip_stream);
        if (n_tensors == 0) return !accumulate && launch_fill_zero(norm, 1, st) != hipSuccess ? DP_ERR_HIP : DP_OK;
        if (!scratch_ok(n_tensors, workspace, workspace_bytes)) return DP_ERR_WORKSPACE;
        const hipError_t e = launch_tensors_norm(items.data(), (int)n_tensors, chunk, chunks, accumulate != 0, norm, tensor_norms, workspace, st);
        return e == hipSuccess ? DP_OK : DP_ERR_HIP;
    });
}

dp_status dp_tensors_clip(const dp_tensor_desc* tensors, int64_t n_tensors, const float* norm, float C, int accumulate,
                          void* workspace, size_t workspace_bytes, void* hip_stream) {
    return guarded([&]() -> dp_status {
        std::vector<TensorItem> items;
        int64_t chunk = 0;
        int chunks = 0;
        const dp_status s = plan_tensors(tensors, n_tensors, true, accumulate != 0, items, chunk, chunks);
        if (s != DP_OK) return s;
        if (!norm || !(C > 0.0f)) return DP_ERR_INVALID_ARG;
        if (n_tensors == 0) return DP_OK;
        if (!scratch_ok(n_tensors, workspace, workspace_bytes)) return DP_ERR_WORKSPACE;
        const hipError_t e = launch_tensors_clip(items.data(), (int)n_tensors, chunk, chunks, accumulate != 0, norm, C, workspace, static_cast<hipStream_t>(hip_stream));
        return e == hipSuccess ? DP_OK : DP_ERR_HIP;
    });
}

dp_status dp_tensors_norm_clip(const dp_tensor_desc* tensors, int64_t n_tensors, float C, int accumulate, float* norm, float* tensor_norms,
                               void* workspace, size_t workspace_bytes, void* hip_stream) {
    return guarded([&]() -> dp_status {
        std::vector<TensorItem> items;
        int64_t chunk = 0;
        int chunks = 0;
        const dp_status s = plan_tensors(tensors, n_tensors, true, accumulate != 0, items, chunk, chunks);
        if (s != DP_OK) return s;
        if (!norm || !(C > 0.0f)) return DP_ERR_INVALID_ARG;
        const hipStream_t st = static_cast<hipStream_t>(hip_stream);
        if (n_tensors == 0) return launch_fill_zero(norm, 1, st) != hipSuccess ? DP_ERR_HIP : DP_OK;
        if (!scratch_ok(n_tensors, workspace, workspace_bytes)) return DP_ERR_WORKSPACE;
        const hipError_t e = launch_tensors_norm_clip(items.data(), (int)n_tensors, chunk, chunks, accumulate != 0, norm, tensor_norms, C, workspace, st);
        return e == hipSuccess ? DP_OK : DP_ERR_HIP;
    });
}

}  // extern "C"
