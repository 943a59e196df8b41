// C-ABI entry points of the relative position bias (include/dpclip.h): argument checks and launches.
#include "../../include/dpclip.h"
#include "dp_internal.h"

using namespace dpk;

namespace {

constexpr int64_t kMaxReach = int64_t(1) << 20;
constexpr int64_t kMaxTable = int64_t(1) << 30;        // its elements have int offsets in the kernels

bool element_aligned(const void* p, dp_dtype d) { return reinterpret_cast<uintptr_t>(p) % (d == DP_F32 ? 4 : 2) == 0; }

dp_status check(const dp_posbias_desc* d, dp_dtype dtype) {
    if (!d || d->B < 0 || d->H < 0 || d->Tq < 0 || d->Tk < 0 || d->reach < 0 || d->n_buckets < 1) return DP_ERR_INVALID_ARG;
    if (dtype == DP_F8_E4M3 || dtype == DP_F8_E5M2 || dtype == DP_F8_E4M3_E5M2) return DP_ERR_UNSUPPORTED;
    if (dtype != DP_F32 && dtype != DP_BF16 && dtype != DP_F16) return DP_ERR_INVALID_ARG;
    if (d->s_b < 0 || d->s_h < 0 || d->s_q < 0) return DP_ERR_INVALID_ARG;
    if (d->reach > kMaxReach || d->n_buckets > kMaxBuckets || !posbias_fits(d->B, d->H, d->Tq, d->Tk)) return DP_ERR_UNSUPPORTED;
    if (d->n_buckets * d->H > kMaxTable) return DP_ERR_UNSUPPORTED;
    if (too_far(d->B, d->s_b) || too_far(d->H, d->s_h) || too_far(d->Tq, d->s_q)) return DP_ERR_UNSUPPORTED;
    return DP_OK;
}
bool empty(const dp_posbias_desc& d) { return d.B == 0 || d.H == 0 || d.Tq == 0 || d.Tk == 0; }

PosbiasArgs args_of(const dp_posbias_desc& d) {
    return PosbiasArgs{(int)d.B, (int)d.H, (int)d.Tq, (int)d.Tk, d.s_b, d.s_h, d.s_q, d.o_b, d.o_h, d.o_q,
                       d.buckets, (int)d.reach, (int)d.n_buckets, d.q_start, d.q_lens, d.k_lens, d.causal != 0};
}

}  // namespace

extern "C" {

size_t dp_posbias_table_workspace_bytes(int64_t B, int64_t H, int64_t Tq, int64_t Tk, int64_t n_buckets) {
    if (B <= 0 || H <= 0 || Tq <= 0 || Tk <= 0 || n_buckets < 1 || n_buckets > kMaxBuckets || !posbias_fits(B, H, Tq, Tk)) return 0;
    return posbias_ws_bytes((int)B, (int)H, (int)Tq, (int)Tk, (int)n_buckets);
}

size_t dp_posbias_workspace_bytes(int64_t B, int64_t H, int64_t Tq, int64_t Tk) {
    return dp_posbias_table_workspace_bytes(B, H, Tq, Tk, kMaxBuckets);
}

dp_status dp_posbias_add(const dp_posbias_desc* desc, const void* scores, const float* table, dp_dtype dtype, void* out, void* hip_stream) {
    const dp_status s = check(desc, dtype);
    if (s != DP_OK) return s;
    const dp_posbias_desc& d = *desc;
    if (d.o_b < 0 || d.o_h < 0 || d.o_q < 0) return DP_ERR_INVALID_ARG;
    if (too_far(d.B, d.o_b) || too_far(d.H, d.o_h) || too_far(d.Tq, d.o_q)) return DP_ERR_UNSUPPORTED;
    if (empty(d)) return DP_OK;
    if (!scores || !table || !out || !d.buckets || !element_aligned(scores, dtype) || !element_aligned(out, dtype)) return DP_ERR_INVALID_ARG;
    const int es = dtype == DP_F32 ? 4 : 2;
    const Strided in{scores, {d.B, d.H, d.Tq}, {d.s_b, d.s_h, d.s_q}, d.Tk, es}, to{out, {d.B, d.H, d.Tq}, {d.o_b, d.o_h, d.o_q}, d.Tk, es};
    if (!elements_apart(to) || !(same_layout(in, to) || tensors_apart(in, to))) return DP_ERR_INVALID_ARG;
    const hipError_t e = launch_posbias_add(args_of(d), scores, table, (int)dtype, out, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? DP_OK : DP_ERR_HIP;
}

dp_status dp_posbias_sqnorm(const dp_posbias_desc* desc, const void* dS, dp_dtype dtype, int accumulate, float* sqnorm, float* rows,
                            void* workspace, size_t workspace_bytes, void* hip_stream) {
    const dp_status s = check(desc, dtype);
    if (s != DP_OK) return s;
    const dp_posbias_desc& d = *desc;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (d.B == 0) return DP_OK;
    if (!sqnorm) return DP_ERR_INVALID_ARG;
    const int64_t width = d.n_buckets * d.H;
    if (empty(d)) {
        if (width > 0 && !rows) return DP_ERR_INVALID_ARG;
        if (width > 0 && launch_fill_zero(rows, d.B * width, st) != hipSuccess) return DP_ERR_HIP;
        if (!accumulate && launch_fill_zero(sqnorm, d.B, st) != hipSuccess) return DP_ERR_HIP;
        return DP_OK;
    }
    if (!dS || !rows || !d.buckets || !element_aligned(dS, dtype)) return DP_ERR_INVALID_ARG;
    const size_t need = posbias_ws_bytes((int)d.B, (int)d.H, (int)d.Tq, (int)d.Tk, (int)d.n_buckets);
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15) != 0) return DP_ERR_WORKSPACE;
    const hipError_t e = launch_posbias_sqnorm(args_of(d), dS, (int)dtype, accumulate != 0, rows, sqnorm, workspace, st);
    return e == hipSuccess ? DP_OK : DP_ERR_HIP;
}

}  // extern "C"
