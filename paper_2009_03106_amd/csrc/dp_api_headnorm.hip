// C-ABI entry points of the norms of queries and keys with the rotation (include/dpclip.h): argument checks and launches.
#include "../../include/dpclip.h"
#include "dp_internal.h"
#include <algorithm>

using namespace dpk;

namespace {

bool element_aligned(const void* p, dp_dtype d) { return reinterpret_cast<uintptr_t>(p) % (d == DP_F32 ? 4 : 2) == 0; }

Strided strided(const dp_headnorm_desc& d, const dp_heads_desc& h, const void* p, int64_t s_b, int64_t s_t, int64_t s_h, int es) {
    return Strided{p, {d.B, d.T, h.H}, {s_b, s_t, s_h}, d.D, es};
}

// backward: dy and gain_rows count
dp_status check(const dp_headnorm_desc* desc, const dp_heads_desc* heads, int64_t n_heads, dp_dtype dtype, bool backward, HeadnormArgs& a) {
    if (!desc || !heads || n_heads < 1 || n_heads > 2) return DP_ERR_INVALID_ARG;
    const dp_headnorm_desc& d = *desc;
    if (d.B < 0 || d.T < 0 || d.D < 1 || d.rot < 0 || d.rot > d.D || d.rot % 2 || !(d.eps > 0.0f) || d.positions_b < 0) return DP_ERR_INVALID_ARG;
    if (d.rotation != DP_ROTATE_HALVES && d.rotation != DP_ROTATE_PAIRS) return DP_ERR_INVALID_ARG;
    if (dtype == DP_F8_E4M3 || dtype == DP_F8_E5M2 || dtype == DP_F8_E4M3_E5M2) return DP_ERR_UNSUPPORTED;
    if (dtype != DP_F32 && dtype != DP_BF16 && dtype != DP_F16) return DP_ERR_INVALID_ARG;
    if (d.D > kMaxHeadDim) return DP_ERR_UNSUPPORTED;
    const int es = dtype == DP_F32 ? 4 : 2;
    for (int64_t i = 0; i < n_heads; ++i) {
        const dp_heads_desc& h = heads[i];
        if (h.H < 0 || h.x_b < 0 || h.x_t < 0 || h.x_h < 0 || h.o_b < 0 || h.o_t < 0 || h.o_h < 0) return DP_ERR_INVALID_ARG;
        if (backward && (h.dy_b < 0 || h.dy_t < 0 || h.dy_h < 0)) return DP_ERR_INVALID_ARG;
        if (too_far(d.B, h.x_b) || too_far(d.T, h.x_t) || too_far(h.H, h.x_h) || too_far(d.B, h.o_b) || too_far(d.T, h.o_t) || too_far(h.H, h.o_h)) return DP_ERR_UNSUPPORTED;
        if (backward && (too_far(d.B, h.dy_b) || too_far(d.T, h.dy_t) || too_far(h.H, h.dy_h))) return DP_ERR_UNSUPPORTED;
    }
    if (too_far(d.B, d.positions_b) || !headnorm_fits(d.B, d.T, heads[0].H, n_heads > 1 ? heads[1].H : 0)) return DP_ERR_UNSUPPORTED;
    a = HeadnormArgs{};
    a.n_heads = (int)n_heads;
    a.B = (int)d.B; a.T = (int)d.T; a.D = (int)d.D; a.rot = (int)d.rot; a.pairs = d.rotation == DP_ROTATE_PAIRS;
    a.eps = d.eps;
    a.positions = d.positions; a.positions_b = d.positions_b;
    a.freqs = d.freqs;
    a.lengths = d.lengths;
    for (int64_t i = 0; i < n_heads; ++i) {
        const dp_heads_desc& h = heads[i];
        a.heads[i] = HeadsArgs{h.x, h.x_b, h.x_t, h.x_h, (int)h.H, h.gain, h.out, h.o_b, h.o_t, h.o_h, backward ? h.dy : nullptr,
                               backward ? h.dy_b : 0, backward ? h.dy_t : 0, backward ? h.dy_h : 0, backward ? h.gain_rows : nullptr};
    }
    if (d.B == 0 || d.T == 0) return DP_OK;
    // what has elements has addresses, and outputs share none with another tensor
    if (d.rot > 0 && !d.freqs && std::max(a.heads[0].H, a.heads[1].H) > 0) return DP_ERR_INVALID_ARG;
    for (int64_t i = 0; i < n_heads; ++i) {
        const dp_heads_desc& h = heads[i];
        if (h.H == 0) continue;
        if (!h.x || !h.gain || !h.out || !element_aligned(h.x, dtype) || !element_aligned(h.out, dtype)) return DP_ERR_INVALID_ARG;
        if (backward && (!h.dy || !element_aligned(h.dy, dtype))) return DP_ERR_INVALID_ARG;
        const Strided out = strided(d, h, h.out, h.o_b, h.o_t, h.o_h, es);
        if (!elements_apart(out)) return DP_ERR_INVALID_ARG;
        for (int64_t k = 0; k < n_heads; ++k) {
            const dp_heads_desc& g = heads[k];
            if (g.H == 0) continue;
            const Strided x = strided(d, g, g.x, g.x_b, g.x_t, g.x_h, es), dy = strided(d, g, g.dy, g.dy_b, g.dy_t, g.dy_h, es);
            if (!(i == k && same_layout(out, x)) && !tensors_apart(out, x)) return DP_ERR_INVALID_ARG;
            if (backward && !(i == k && same_layout(out, dy)) && !tensors_apart(out, dy)) return DP_ERR_INVALID_ARG;
            if (k > i && !tensors_apart(out, strided(d, g, g.out, g.o_b, g.o_t, g.o_h, es))) return DP_ERR_INVALID_ARG;
        }
    }
    // one gain for both: each descriptor's rows are written by themselves, so they need rows of their own
    if (backward && n_heads > 1 && heads[0].gain_rows && heads[1].gain_rows) {
        const Strided r0{heads[0].gain_rows, {1, 1, 1}, {0, 0, 0}, d.B * d.D, 4}, r1{heads[1].gain_rows, {1, 1, 1}, {0, 0, 0}, d.B * d.D, 4};
        if (!tensors_apart(r0, r1)) return DP_ERR_INVALID_ARG;
    }
    return DP_OK;
}

}  // namespace

extern "C" {

size_t dp_headnorm_workspace_bytes(int64_t n_heads, int64_t B, int64_t T, int64_t D) {
    if (n_heads < 1 || n_heads > 2 || B <= 0 || T <= 0 || D < 1 || D > kMaxHeadDim || !headnorm_fits(B, T, 1, 1)) return 0;
    return headnorm_ws_bytes((int)n_heads, (int)B, (int)T, (int)D);
}

dp_status dp_headnorm(const dp_headnorm_desc* desc, const dp_heads_desc* heads, int64_t n_heads, dp_dtype dtype, void* hip_stream) {
    HeadnormArgs a;
    const dp_status s = check(desc, heads, n_heads, dtype, false, a);
    if (s != DP_OK) return s;
    if (a.B == 0 || a.T == 0 || (a.heads[0].H == 0 && a.heads[1].H == 0)) return DP_OK;
    return launch_headnorm(a, (int)dtype, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? DP_OK : DP_ERR_HIP;
}

dp_status dp_headnorm_sqnorm(const dp_headnorm_desc* desc, const dp_heads_desc* heads, int64_t n_heads, dp_dtype dtype,
                             int accumulate, float* sqnorm, void* workspace, size_t workspace_bytes, void* hip_stream) {
    HeadnormArgs a;
    const dp_status s = check(desc, heads, n_heads, dtype, true, a);
    if (s != DP_OK) return s;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (a.B == 0) return DP_OK;
    if (!sqnorm) return DP_ERR_INVALID_ARG;
    for (int i = 0; i < a.n_heads; ++i)
        if (!a.heads[i].gain_rows) return DP_ERR_INVALID_ARG;
    if (a.T == 0 || (a.heads[0].H == 0 && a.heads[1].H == 0)) {
        for (int i = 0; i < a.n_heads; ++i)
            if (launch_fill_zero(a.heads[i].gain_rows, (int64_t)a.B * a.D, st) != hipSuccess) return DP_ERR_HIP;
        if (!accumulate && launch_fill_zero(sqnorm, a.B, st) != hipSuccess) return DP_ERR_HIP;
        return DP_OK;
    }
    if (!workspace || workspace_bytes < headnorm_ws_bytes(a.n_heads, a.B, a.T, a.D) || ((uintptr_t)workspace & 15) != 0) return DP_ERR_WORKSPACE;
    return launch_headnorm_sqnorm(a, (int)dtype, accumulate != 0, sqnorm, workspace, st) == hipSuccess ? DP_OK : DP_ERR_HIP;
}

}  // extern "C"
