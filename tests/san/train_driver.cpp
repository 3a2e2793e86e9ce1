// Calls the entry points of normalisations and of AdamW steps with arguments that the host-side checks must refuse (and the queries
// with valid ones), in a build whose HOST code carries AddressSanitizer and UndefinedBehaviorSanitizer.  No kernel is launched
// and no GPU is needed.  Built and run by tests/test_train_cpu.py.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "spo.h"

static int failures = 0;
#define EXPECT(call, want)                                                                                                     \
    do {                                                                                                                       \
        const long long got_ = (long long)(call);                                                                              \
        if (got_ != (long long)(want)) {                                                                                       \
            std::fprintf(stderr, "%s:%d: %s = %lld, expected %lld\n", __FILE__, __LINE__, #call, got_, (long long)(want));      \
            ++failures;                                                                                                        \
        }                                                                                                                      \
    } while (0)

// non-NULL, aligned dummies: never dereferenced on the paths taken here
static float *f = reinterpret_cast<float *>(uintptr_t(4096));
static uint8_t *codes = reinterpret_cast<uint8_t *>(uintptr_t(8192));
static void *ws = reinterpret_cast<void *>(uintptr_t(1) << 20);
static void *odd = reinterpret_cast<void *>((uintptr_t(1) << 20) + 8);
static void *off1 = reinterpret_cast<void *>(uintptr_t(4097)), *off2 = reinterpret_cast<void *>(uintptr_t(4098));
static const size_t big = size_t(1) << 50;
static const int64_t large = int64_t(1) << 62;

static spo_norm_desc norm_desc() {
    spo_norm_desc d{};
    d.struct_size = sizeof d;
    d.kind = SPO_NORM_LAYER;
    d.x_dtype = d.y_dtype = SPO_BF16;
    d.w_dtype = SPO_FP32;
    d.rows = 10;
    d.cols = 100;
    d.x = d.weight = d.bias = f;
    d.eps = 1e-6f;
    return d;
}
static int fwd(const spo_norm_desc *d, void *y = f, int64_t stride = 0) { return spo_norm_fwd(d, y, stride, f, f, nullptr); }
struct Back {
    const float *mean = f, *rstd = f;
    const void *dy = f;
    int dy_dtype = SPO_BF16;
    int64_t dy_stride = 0;
    void *dx = f;
    int dx_dtype = SPO_BF16;
    void *dw = f, *db = f;
    int dw_dtype = SPO_FP32, accumulate = 0;
    void *w = ws;
    size_t n = big;
};
static int bwd(const spo_norm_desc *d, const Back &b = {}) {
    return spo_norm_bwd(d, b.mean, b.rstd, b.dy, b.dy_dtype, b.dy_stride, b.dx, b.dx_dtype, b.dw, b.db, b.dw_dtype, b.accumulate, b.w, b.n, nullptr);
}

static void norms() {
    EXPECT(fwd(nullptr), SPO_ENULL);
    EXPECT(bwd(nullptr), SPO_ENULL);
    EXPECT(spo_norm_bwd_workspace_bytes(nullptr), 0);
    const spo_norm_desc good = norm_desc();
    EXPECT(spo_norm_bwd_workspace_bytes(&good) > 0, 1);
    const auto with = [&](auto change) {
        spo_norm_desc d = good;
        change(d);
        EXPECT(spo_norm_bwd_workspace_bytes(&d), 0);
        const int rc = fwd(&d);
        EXPECT(bwd(&d), rc);
        return rc;
    };
    EXPECT(with([](auto &d) { d.struct_size -= 8; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.kind = 2; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.kind = -1; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.x_dtype = 2; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.y_dtype = -1; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.w_dtype = 7; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.rows = -1; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.rows = int64_t(1) << 31; }), SPO_ERANGE);
    EXPECT(with([](auto &d) { d.rows = large; }), SPO_ERANGE);
    EXPECT(with([](auto &d) { d.cols = 0; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.cols = 65537; }), SPO_ERANGE);
    EXPECT(with([](auto &d) { d.cols = large; }), SPO_ERANGE);
    EXPECT(with([](auto &d) { d.eps = -1e-6f; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.eps = NAN; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.x_stride = 99; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.x_stride = -100; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.x_stride = large; }), SPO_ERANGE);
    EXPECT(with([](auto &d) { d.x = off1; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.x_dtype = SPO_FP32, d.x = off2; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.weight = off2; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.bias = off2; }), SPO_EINVAL);
    spo_norm_desc d = good;
    d.x = nullptr;
    EXPECT(fwd(&d), SPO_ENULL);
    EXPECT(bwd(&d), SPO_ENULL);
    EXPECT(fwd(&good, nullptr), SPO_ENULL);
    EXPECT(fwd(&good, off1), SPO_EINVAL);
    EXPECT(fwd(&good, f, 99), SPO_EINVAL);
    EXPECT(fwd(&good, f, -1), SPO_EINVAL);
    EXPECT(fwd(&good, f, large), SPO_ERANGE);
    d = good;
    d.rows = 0;
    d.x = nullptr;
    EXPECT(fwd(&d, nullptr), SPO_OK);                                        // nothing to do
    const auto back = [&](auto change) {
        Back b;
        change(b);
        return bwd(&good, b);
    };
    EXPECT(back([](Back &b) { b.mean = nullptr; }), SPO_ENULL);
    EXPECT(back([](Back &b) { b.rstd = nullptr; }), SPO_ENULL);
    EXPECT(back([](Back &b) { b.dy = nullptr; }), SPO_ENULL);
    EXPECT(back([](Back &b) { b.dy_dtype = 3; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.dx_dtype = 3; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.dw_dtype = 3; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.dw_dtype = SPO_BF16, b.accumulate = 1; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.dy_stride = 99; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.dy_stride = -1; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.dy_stride = large; }), SPO_ERANGE);
    EXPECT(back([](Back &b) { b.dy = off1; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.dx = off1; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.dw = off2; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.db = off2; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.w = nullptr; }), SPO_EWORKSPACE);
    EXPECT(back([](Back &b) { b.w = odd; }), SPO_EINVAL);
    EXPECT(back([](Back &b) { b.n = 255; }), SPO_EWORKSPACE);
    EXPECT(back([](Back &b) { b.n = spo_norm_bwd_workspace_bytes(nullptr); }), SPO_EWORKSPACE);
    EXPECT(back([](Back &b) { b.dx = b.dw = b.db = nullptr, b.w = nullptr; }), SPO_OK);   // nothing asked for
}

static spo_adamw_tensor tensor() {
    spo_adamw_tensor t{};
    t.param = t.m = t.v = f;
    t.grad = f;
    t.m_scale = t.v_scale = codes;
    t.n = 1000;
    t.weight_decay = 0.1;
    t.param_dtype = SPO_FP32;
    t.grad_dtype = SPO_BF16;
    return t;
}
struct Step {
    double lr = 1e-3;
    const float *lr_device = nullptr;
    double beta1 = 0.9, beta2 = 0.999, eps = 1e-8;
    int64_t step = 1;
    int64_t *step_device = nullptr;
    const float *norm = nullptr;
    double most = 1.0;
    int rounding = SPO_ROUND_NEAREST;
    void *w = nullptr;
    size_t n = 0;
};
static int update(const spo_adamw_desc *d, const Step &s = {}) {
    return spo_adamw_update(d, s.lr, s.lr_device, s.beta1, s.beta2, s.eps, s.step, s.step_device, s.norm, s.most, s.rounding, s.w, s.n, nullptr);
}

static void steps() {
    EXPECT(update(nullptr), SPO_ENULL);
    EXPECT(spo_grad_norm(nullptr, f, ws, big, nullptr), SPO_ENULL);
    EXPECT(spo_grad_norm_workspace_bytes(nullptr), 0);
    spo_adamw_tensor of[3] = {tensor(), tensor(), tensor()};
    spo_adamw_desc d{};
    d.struct_size = sizeof d;
    d.state_bits = 32;
    d.count = 3;
    d.tensors = of;
    const spo_adamw_desc good = d;
    const auto with = [&](auto change) {
        spo_adamw_desc e = good;
        change(e);
        const int rc = update(&e);
        EXPECT(spo_grad_norm(&e, f, ws, big, nullptr), rc);
        return rc;
    };
    EXPECT(with([](auto &e) { e.struct_size = 8; }), SPO_EINVAL);
    EXPECT(with([](auto &e) { e.state_bits = 16; }), SPO_EINVAL);
    EXPECT(with([](auto &e) { e.count = -1; }), SPO_EINVAL);
    EXPECT(with([](auto &e) { e.count = large; }), SPO_ERANGE);
    EXPECT(with([](auto &e) { e.tensors = nullptr; }), SPO_ENULL);
    // a tensor's own: the middle one's
    const auto tensors = [&](int bits, auto change) {
        of[1] = tensor();
        change(of[1]);
        d.state_bits = bits;
        const int rc = update(&d);
        of[1] = tensor();
        return rc;
    };
    for (int bits : {32, 8}) {
        EXPECT(tensors(bits, [](auto &t) { t.n = -1; }), SPO_EINVAL);
        EXPECT(tensors(bits, [](auto &t) { t.n = (int64_t(1) << 35) + 1; }), SPO_ERANGE);
        EXPECT(tensors(bits, [](auto &t) { t.param = nullptr; }), SPO_ENULL);
        EXPECT(tensors(bits, [](auto &t) { t.grad = nullptr; }), SPO_ENULL);
        EXPECT(tensors(bits, [](auto &t) { t.m = nullptr; }), SPO_ENULL);
        EXPECT(tensors(bits, [](auto &t) { t.v = nullptr; }), SPO_ENULL);
        EXPECT(tensors(bits, [](auto &t) { t.param_dtype = 5; }), SPO_EINVAL);
        EXPECT(tensors(bits, [](auto &t) { t.grad_dtype = -2; }), SPO_EINVAL);
        EXPECT(tensors(bits, [](auto &t) { t.weight_decay = -0.1; }), SPO_EINVAL);
        EXPECT(tensors(bits, [](auto &t) { t.weight_decay = NAN; }), SPO_EINVAL);
        EXPECT(tensors(bits, [](auto &t) { t.param = off2; }), SPO_EINVAL);
        EXPECT(tensors(bits, [](auto &t) { t.grad = off1; }), SPO_EINVAL);
        EXPECT(tensors(bits, [](auto &t) { t.copy = off1; }), SPO_EINVAL);
        EXPECT(tensors(bits, [](auto &t) { t.copy = f, t.param_dtype = SPO_BF16; }), SPO_EINVAL);
    }
    EXPECT(tensors(32, [](auto &t) { t.m = off2; }), SPO_EINVAL);
    EXPECT(tensors(32, [](auto &t) { t.v = off1; }), SPO_EINVAL);
    EXPECT(tensors(8, [](auto &t) { t.m_scale = nullptr; }), SPO_ENULL);
    EXPECT(tensors(8, [](auto &t) { t.v_scale = nullptr; }), SPO_ENULL);
    const auto step = [&](auto change) {
        Step s;
        change(s);
        return update(&good, s);
    };
    EXPECT(step([](Step &s) { s.lr = -1.0; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.lr = NAN; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.beta1 = 1.0; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.beta1 = -0.1; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.beta2 = 1.0; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.beta2 = NAN; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.eps = -1e-8; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.step = 0; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.norm = f, s.most = -1.0; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.norm = f, s.most = NAN; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.rounding = 2; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.lr_device = f; }), SPO_EWORKSPACE);
    EXPECT(step([](Step &s) { s.step_device = reinterpret_cast<int64_t *>(f); }), SPO_EWORKSPACE);
    EXPECT(step([](Step &s) { s.lr_device = f, s.w = ws, s.n = 8; }), SPO_EWORKSPACE);
    EXPECT(step([](Step &s) { s.lr_device = f, s.w = odd, s.n = big; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.lr_device = static_cast<float *>(off2), s.w = ws, s.n = big; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.step_device = reinterpret_cast<int64_t *>(uintptr_t(4100)), s.w = ws, s.n = big; }), SPO_EINVAL);
    EXPECT(step([](Step &s) { s.norm = static_cast<float *>(off2); }), SPO_EINVAL);
    EXPECT(spo_grad_norm(&good, nullptr, ws, big, nullptr), SPO_ENULL);
    EXPECT(spo_grad_norm(&good, f, nullptr, 0, nullptr), SPO_EWORKSPACE);
    EXPECT(spo_grad_norm(&good, f, ws, 64, nullptr), SPO_EWORKSPACE);
    EXPECT(spo_grad_norm(&good, f, odd, big, nullptr), SPO_EINVAL);
    EXPECT(spo_grad_norm(&good, static_cast<float *>(off2), ws, big, nullptr), SPO_EINVAL);
    d = good;
    d.count = 0;
    d.tensors = nullptr;
    EXPECT(update(&d), SPO_OK);                                               // nothing to do
    for (auto &t : of) t = spo_adamw_tensor{};                                // tensors without elements
    EXPECT(update(&good), SPO_OK);
    size_t last = 0;
    for (int64_t n = 0; n < 2000; n += 7) {
        d.count = n;
        const size_t bytes = spo_grad_norm_workspace_bytes(&d);
        EXPECT(bytes >= last && bytes > 0, 1);
        last = bytes;
    }
    EXPECT(spo_adamw_update_workspace_bytes() > 0, 1);
    EXPECT(spo_adamw_state_values(codes, codes, codes, codes, -1, f, f, SPO_FP32, nullptr), SPO_EINVAL);
    EXPECT(spo_adamw_state_values(codes, codes, codes, codes, large, f, f, SPO_FP32, nullptr), SPO_ERANGE);
    EXPECT(spo_adamw_state_values(codes, codes, codes, codes, 5, f, f, 4, nullptr), SPO_EINVAL);
    EXPECT(spo_adamw_state_values(nullptr, codes, codes, codes, 5, f, f, SPO_FP32, nullptr), SPO_ENULL);
    EXPECT(spo_adamw_state_values(codes, codes, codes, nullptr, 5, f, f, SPO_FP32, nullptr), SPO_ENULL);
    EXPECT(spo_adamw_state_values(codes, codes, codes, codes, 5, off2, f, SPO_FP32, nullptr), SPO_EINVAL);
    EXPECT(spo_adamw_state_values(codes, codes, codes, codes, 0, f, f, SPO_FP32, nullptr), SPO_OK);
    EXPECT(spo_adamw_state_values(nullptr, nullptr, nullptr, nullptr, 5, nullptr, nullptr, SPO_FP32, nullptr), SPO_OK);
}

int main() {
    norms();
    steps();
    if (failures) return 1;
    std::puts("normalisation and step host-side sanitizer run ok");
    return 0;
}
