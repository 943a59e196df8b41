// Which strided tensors share memory: host checks of the entry points whose tensors need not be contiguous.
#include "dp_internal.h"
#include <algorithm>

namespace dpk {

namespace {

struct Dim { int64_t size, stride; };

// dimensions of more than one element, the outermost first
int by_stride(const Strided& a, Dim (&d)[3]) {
    int n = 0;
    for (int i = 0; i < 3; ++i)
        if (a.size[i] > 1) d[n++] = Dim{a.size[i], a.stride[i]};
    std::sort(d, d + n, [](const Dim& x, const Dim& y) { return x.stride > y.stride; });
    return n;
}
// elements from the first to behind the last one of dimensions [i, n)
int64_t span(const Dim* d, int i, int n, int64_t inner) {
    for (; i < n; ++i) inner += (d[i].size - 1) * d[i].stride;
    return inner;
}

}  // namespace

bool too_far(int64_t size, int64_t stride) { return size > 1 && stride > (int64_t(1) << 48) / (size - 1); }

bool elements_apart(const Strided& a) {
    Dim d[3];
    const int n = by_stride(a, d);
    for (int i = 0; i < n; ++i)
        if (d[i].stride < span(d, i + 1, n, a.inner)) return false;
    return true;
}

bool same_layout(const Strided& a, const Strided& b) {
    if (a.p != b.p || a.inner != b.inner || a.es != b.es) return false;
    for (int i = 0; i < 3; ++i)
        if (a.size[i] != b.size[i] || (a.size[i] > 1 && a.stride[i] != b.stride[i])) return false;
    return true;
}

bool tensors_apart(const Strided& a, const Strided& b) {
    Dim da[3], db[3];
    const int na = by_stride(a, da), nb = by_stride(b, db);
    const intptr_t pa = (intptr_t)a.p, pb = (intptr_t)b.p;
    for (int i = 0;; ++i) {
        const intptr_t ea = pa + (intptr_t)span(da, i, na, a.inner) * a.es, eb = pb + (intptr_t)span(db, i, nb, b.inner) * b.es;
        if (ea <= pb || eb <= pa) return true;
        if (i >= na || i >= nb || da[i].size != db[i].size || da[i].stride * a.es != db[i].stride * b.es) return false;
        // one step of the dimension: both parts lie inside it, so that other steps' parts are further away
        const intptr_t fa = pa + (intptr_t)span(da, i + 1, na, a.inner) * a.es, fb = pb + (intptr_t)span(db, i + 1, nb, b.inner) * b.es;
        if (std::max(fa, fb) - std::min(pa, pb) > (intptr_t)da[i].stride * a.es) return false;
    }
}

}  // namespace dpk
