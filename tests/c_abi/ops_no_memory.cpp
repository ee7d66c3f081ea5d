// Every replica operator's entry with no host memory left: each call is one that
// is refused with a text, for which no allocation succeeds.  No device is touched.
#include <cstdio>
#include <cstdlib>
#include <new>

#include "ar_plan.h"

static bool g_none = false;

void* operator new(std::size_t n) {
    void* const p = g_none ? nullptr : std::malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

template <class F>
static int check(const char* name, F call) {
    g_none = true;
    const ar_status s = call();
    g_none = false;
    std::printf("%s: %d\n", name, int(s));
    return s != AR_ERR_OOM;
}

int main() {
    int64_t bytes = 0;
    void* const p = reinterpret_cast<void*>(int64_t(1) << 40);
    const int64_t* const ids = static_cast<const int64_t*>(p);
    const int64_t big = int64_t(1) << 40;
    int bad = 0;
    bad += check("ar_embed_lookup", [&] {
        return ar_embed_lookup(AR_F32, 10, 8, 4, p, 1, ids, 1.0f, p, 8, nullptr);
    });
    bad += check("ar_embed_grad_workspace",
                 [&] { return ar_embed_grad_workspace(big, 8, 4, &bytes); });
    bad += check("ar_embed_grad", [&] {
        return ar_embed_grad(AR_F32, 10, 8, 4, p, 1, ids, 1.0f, 0, p, 8, p, big, nullptr);
    });
    bad += check("ar_glu_workspace", [&] { return ar_glu_workspace(AR_F32, big, 8, 4, 0, &bytes); });
    bad += check("ar_glu_forward", [&] {
        return ar_glu_forward(AR_F32, AR_ACT_SILU, 4, 8, 4, p, 8, p, p, 8, p, 1, nullptr, nullptr, 0,
                              AR_F32, nullptr, 0, nullptr);
    });
    bad += check("ar_glu_backward", [&] {
        return ar_glu_backward(AR_F32, 4, 8, 4, p, 4, p, 8, p, p, 8, p, p, 4, AR_I32, 0, p, 8, p, p,
                               8, p, big, nullptr);
    });
    bad += check("ar_distill_workspace", [&] { return ar_distill_workspace(big, 8, 4, &bytes); });
    bad += check("ar_distill", [&] {
        return ar_distill(AR_F32, 4, 100, 5, p, 100, AR_F32, p, 5, ids, 5, -1.0f, nullptr,
                          static_cast<float*>(p), nullptr, 0, p, big, nullptr);
    });
    return bad;
}
