// The entries of position bias, routing, balance loss and activations in 8 bits with no
// host memory left: each call is one that is refused with a text, for which no allocation
// succeeds.  No device is touched.
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
    const int64_t big = int64_t(1) << 40;
    int bad = 0;
    bad += check("ar_position_bias", [&] {
        return ar_position_bias(AR_F32, 32, 128, 0, 4, 8, 16, 0, p, 1, p, 128, 16, nullptr);
    });
    bad += check("ar_position_bias_grad_workspace",
                 [&] { return ar_position_bias_grad_workspace(AR_F32, 32, 2, big, 8, 16, &bytes); });
    bad += check("ar_position_bias_grad", [&] {
        return ar_position_bias_grad(AR_F32, 32, 128, 0, 2, 4, 8, 16, 0, p, 512, 128, 16, 0, p, 1, p,
                                     big, nullptr);
    });
    bad += check("ar_route_workspace", [&] { return ar_route_workspace(4, big, 2, &bytes); });
    bad += check("ar_route", [&] {
        return ar_route(AR_F32, 4, 16, 2, p, 1, nullptr, 0, static_cast<int64_t*>(p),
                        static_cast<float*>(p), static_cast<int32_t*>(p), static_cast<float*>(p), p,
                        big, nullptr);
    });
    bad += check("ar_balance", [&] {
        return ar_balance(AR_F32, 4, 16, 2, p, 1, static_cast<int64_t*>(p), static_cast<int32_t*>(p),
                          static_cast<float*>(p), 1.0f, 0, nullptr, static_cast<float*>(p), p, 16,
                          nullptr);
    });
    bad += check("ar_checkpoint_row", [&] { return ar_checkpoint_row(big, &bytes); });
    bad += check("ar_checkpoint_store",
                 [&] { return ar_checkpoint_store(AR_F32, 4, 8, p, 1, p, 48, nullptr); });
    bad += check("ar_checkpoint_load",
                 [&] { return ar_checkpoint_load(AR_F32, 4, 8, p, 48, p, 1, nullptr); });
    return bad;
}
