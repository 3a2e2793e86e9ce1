// Calls the entry points of token scores and of orthogonalised updates with arguments that the host-side checks must refuse
// (and the queries with valid ones), in a build whose HOST code carries AddressSanitizer and UndefinedBehaviorSanitizer.  No
// kernel is launched and no GPU is needed.  Built and run by tests/test_score_update_cpu.py.
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
static int32_t *ids = reinterpret_cast<int32_t *>(uintptr_t(8192));
static void *ws = reinterpret_cast<void *>(uintptr_t(1) << 20);
static void *odd = reinterpret_cast<void *>((uintptr_t(1) << 20) + 8);
static const size_t big = size_t(1) << 50;

static spo_logprob_desc logits_desc() {
    spo_logprob_desc d{};
    d.struct_size = sizeof d;
    d.dtype = SPO_FP32;
    d.T = 10;
    d.V = 1000;
    d.logits = f;
    d.target = ids;
    return d;
}
static spo_logprob_desc head_desc() {
    spo_logprob_desc d = logits_desc();
    d.dtype = SPO_BF16;
    d.logits = nullptr;
    d.hidden = d.W = f;
    d.H = 128;
    return d;
}
static int fwd(const spo_logprob_desc &d, float *logp = f, float *lse = f, int32_t *top = ids, float *top_logp = f, void *w = ws, size_t n = big) {
    return spo_logprob_fwd(&d, logp, lse, f, top, top_logp, w, n, nullptr);
}
static int bwd(const spo_logprob_desc &d, const float *lse = f, const float *entropy = f, const float *dl = f, const float *de = f,
               const int32_t *top = nullptr, const float *dt = nullptr, int hidden_type = SPO_BF16, int W_type = SPO_FP32, int accumulate = 0,
               void *d_logits = f, int64_t chunk = 0, void *w = ws, size_t n = big) {
    return spo_logprob_bwd(&d, lse, entropy, dl, de, top, dt, f, hidden_type, f, W_type, accumulate, d_logits, chunk, w, n, nullptr);
}

static void scores() {
    EXPECT(spo_logprob_fwd(nullptr, f, f, f, ids, f, ws, big, nullptr), SPO_ENULL);
    EXPECT(spo_logprob_fwd_workspace_bytes(nullptr), 0);
    EXPECT(spo_logprob_bwd_workspace_bytes(nullptr, 0), 0);
    for (int form = 0; form < 2; ++form) {
        const spo_logprob_desc good = form ? head_desc() : logits_desc();
        EXPECT(spo_logprob_fwd_workspace_bytes(&good) > 0, 1);
        EXPECT(spo_logprob_bwd_workspace_bytes(&good, 0) > 0, 1);
        EXPECT(spo_logprob_bwd_workspace_bytes(&good, -1), 0);
        auto with = [&](auto change) {
            spo_logprob_desc d = good;
            change(d);
            EXPECT(spo_logprob_fwd_workspace_bytes(&d), 0);
            EXPECT(spo_logprob_bwd_workspace_bytes(&d, 0), 0);
            const int rc = fwd(d);
            EXPECT(bwd(d), rc);
            return rc;
        };
        EXPECT(with([](auto &d) { d.struct_size -= 8; }), SPO_EINVAL);
        EXPECT(with([](auto &d) { d.dtype = 7; }), SPO_EINVAL);
        EXPECT(with([](auto &d) { d.T = -1; }), SPO_EINVAL);
        EXPECT(with([](auto &d) { d.T = int64_t(1) << 31; }), SPO_ERANGE);
        EXPECT(with([](auto &d) { d.V = 0; }), SPO_EINVAL);
        EXPECT(with([](auto &d) { d.V = int64_t(1) << 31; }), SPO_ERANGE);
        EXPECT(with([](auto &d) { d.top_k = -1; }), SPO_EINVAL);
        EXPECT(with([](auto &d) { d.top_k = 65; }), SPO_ERANGE);
        EXPECT(with([](auto &d) { d.V = 20, d.top_k = 21; }), SPO_EINVAL);
        EXPECT(fwd(good, nullptr), SPO_ENULL);                                     // a target, and no place for its log-prob
        EXPECT(fwd(good, f, nullptr), SPO_ENULL);
        EXPECT(fwd(good, f, f, ids, f, nullptr, 0), SPO_EWORKSPACE);
        EXPECT(fwd(good, f, f, ids, f, odd), SPO_EINVAL);
        EXPECT(fwd(good, f, f, ids, f, ws, 16), SPO_EWORKSPACE);
        EXPECT(bwd(good, nullptr), SPO_ENULL);
        EXPECT(bwd(good, f, nullptr), SPO_ENULL);                                  // d_entropy without the entropy
        EXPECT(bwd(good, f, f, f, f, nullptr, f), SPO_ENULL);                      // d_top_logp without the ids
        EXPECT(bwd(good, f, f, f, f, ids, f), SPO_EINVAL);                         // and of a descriptor without alternatives
        EXPECT(bwd(good, f, f, f, f, nullptr, nullptr, 1, 0, 0, f, -1), SPO_EINVAL);
        spo_logprob_desc no_target = good;
        no_target.target = nullptr;
        EXPECT(bwd(no_target), SPO_ENULL);
    }
    spo_logprob_desc d = logits_desc();
    d.top_k = 5;
    EXPECT(fwd(d, f, f, nullptr), SPO_ENULL);
    EXPECT(fwd(d, f, f, ids, nullptr), SPO_ENULL);
    d = logits_desc();
    d.logits_stride = d.V - 1;
    EXPECT(fwd(d), SPO_EINVAL);
    d.logits_stride = -5;
    EXPECT(fwd(d), SPO_EINVAL);
    d = logits_desc();
    d.logits = reinterpret_cast<const char *>(f) + 2;
    EXPECT(fwd(d), SPO_EINVAL);
    d = logits_desc();
    EXPECT(bwd(d, f, f, f, f, nullptr, nullptr, 1, 0, 0, nullptr), SPO_ENULL);
    EXPECT(bwd(d, f, f, f, f, nullptr, nullptr, 1, 0, 0, reinterpret_cast<char *>(f) + 2), SPO_EINVAL);
    d.T = 0;                                                                       // nothing to do, and nothing is done
    EXPECT(bwd(d, nullptr, nullptr, nullptr, nullptr), SPO_OK);

    d = head_desc();
    d.H = 100;
    EXPECT(fwd(d), SPO_EUNSUPPORTED);
    d.H = 0;
    EXPECT(fwd(d), SPO_EINVAL);
    d.H = 65536 + 64;
    EXPECT(fwd(d), SPO_ERANGE);
    d = head_desc();
    d.top_k = 3;
    EXPECT(fwd(d), SPO_EUNSUPPORTED);
    d = head_desc();
    d.w_layout = 9;
    EXPECT(fwd(d), SPO_EINVAL);
    d = head_desc();
    d.hidden = nullptr;
    EXPECT(fwd(d), SPO_ENULL);
    d = head_desc();
    d.W = reinterpret_cast<const char *>(f) + 2;
    EXPECT(fwd(d), SPO_EINVAL);
    d = head_desc();
    EXPECT(bwd(d, f, f, f, f, nullptr, nullptr, 7), SPO_EINVAL);
    EXPECT(bwd(d, f, f, f, f, nullptr, nullptr, SPO_BF16, 7), SPO_EINVAL);
    EXPECT(bwd(d, f, f, f, f, nullptr, nullptr, SPO_BF16, SPO_BF16, 1), SPO_EINVAL);  // sums in bf16
    EXPECT(bwd(d, f, f, f, f, nullptr, nullptr, 1, 0, 0, nullptr, 0, nullptr, 0), SPO_EWORKSPACE);
    EXPECT(bwd(d, f, f, f, f, nullptr, nullptr, 1, 0, 0, nullptr, 0, odd), SPO_EINVAL);
    EXPECT(bwd(d, f, f, f, f, nullptr, nullptr, 1, 0, 0, nullptr, 0, ws, 16), SPO_EWORKSPACE);
    d.dtype = SPO_FP32;
    EXPECT(bwd(d), SPO_EUNSUPPORTED);
}

static spo_orth_desc orth_desc() {
    spo_orth_desc d{};
    d.struct_size = sizeof d;
    d.batch = 2;
    d.rows = 100;
    d.cols = 300;
    d.steps = 5;
    d.a = 3.4445f, d.b = -4.775f, d.c = 2.0315f;
    d.eps = 1e-7f;
    return d;
}
static int orth(const spo_orth_desc &d, const void *G = f, int g_type = SPO_FP32, int64_t stride = 0, int64_t step = 0, void *out = f,
                int out_type = SPO_FP32, void *w = ws, size_t n = big) {
    return spo_orthogonalize(&d, G, g_type, stride, step, out, out_type, w, n, nullptr);
}
static int muon(const spo_orth_desc &d, void *W = f, int w_type = SPO_FP32, float *m = f, const void *g = f, int g_type = SPO_FP32, float mu = 0.9f,
                float lr = 0.1f, float decay = 0.0f, float scale = 1.0f, void *w = ws, size_t n = big) {
    return spo_muon_update(&d, W, w_type, m, g, g_type, mu, 1, lr, decay, scale, w, n, nullptr);
}

static void updates() {
    EXPECT(spo_orthogonalize(nullptr, f, 0, 0, 0, f, 0, ws, big, nullptr), SPO_ENULL);
    EXPECT(spo_orthogonalize_workspace_bytes(nullptr), 0);
    const spo_orth_desc good = orth_desc();
    EXPECT(spo_orthogonalize_workspace_bytes(&good) > 0, 1);
    auto with = [&](auto change) {
        spo_orth_desc d = good;
        change(d);
        EXPECT(spo_orthogonalize_workspace_bytes(&d), 0);
        const int rc = orth(d);
        EXPECT(muon(d), rc);
        return rc;
    };
    EXPECT(with([](auto &d) { d.struct_size += 8; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.batch = 0; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.rows = 0; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.cols = -4; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.steps = -1; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.products = 2; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.eps = -1.0f; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.eps = NAN; }), SPO_EINVAL);
    EXPECT(with([](auto &d) { d.batch = 65536; }), SPO_ERANGE);
    EXPECT(with([](auto &d) { d.rows = 65537; }), SPO_ERANGE);
    EXPECT(with([](auto &d) { d.cols = 65537; }), SPO_ERANGE);
    EXPECT(with([](auto &d) { d.steps = 65; }), SPO_ERANGE);
    spo_orth_desc most = good;  // sizes in 64 bits
    most.batch = 65535;
    most.rows = most.cols = 65536;
    EXPECT(spo_orthogonalize_workspace_bytes(&most) > (size_t(1) << 50), 1);

    void *between = reinterpret_cast<char *>(f) + 1, *half = reinterpret_cast<char *>(f) + 2;
    EXPECT(orth(good, nullptr), SPO_ENULL);
    EXPECT(orth(good, f, SPO_FP32, 0, 0, nullptr), SPO_ENULL);
    EXPECT(orth(good, f, 5), SPO_EINVAL);
    EXPECT(orth(good, f, SPO_FP32, 0, 0, f, 5), SPO_EINVAL);
    EXPECT(orth(good, between, SPO_BF16), SPO_EINVAL);
    EXPECT(orth(good, f, SPO_FP32, 0, 0, half), SPO_EINVAL);
    EXPECT(orth(good, f, SPO_FP32, 299), SPO_EINVAL);
    EXPECT(orth(good, f, SPO_FP32, -300), SPO_EINVAL);
    EXPECT(orth(good, f, SPO_FP32, 0, -1), SPO_EINVAL);
    EXPECT(orth(good, f, SPO_FP32, 0, 0, f, SPO_FP32, nullptr, 0), SPO_EWORKSPACE);
    EXPECT(orth(good, f, SPO_FP32, 0, 0, f, SPO_FP32, odd), SPO_EINVAL);
    EXPECT(orth(good, f, SPO_FP32, 0, 0, f, SPO_FP32, ws, 16), SPO_EWORKSPACE);
    EXPECT(muon(good, nullptr), SPO_ENULL);
    EXPECT(muon(good, f, SPO_FP32, nullptr), SPO_ENULL);
    EXPECT(muon(good, f, SPO_FP32, f, nullptr), SPO_ENULL);
    EXPECT(muon(good, f, 5), SPO_EINVAL);
    EXPECT(muon(good, f, SPO_FP32, f, f, 5), SPO_EINVAL);
    EXPECT(muon(good, half, SPO_FP32), SPO_EINVAL);
    EXPECT(muon(good, f, SPO_FP32, static_cast<float *>(half)), SPO_EINVAL);
    for (float mu : {-0.1f, 1.0f, NAN}) EXPECT(muon(good, f, SPO_FP32, f, f, SPO_FP32, mu), SPO_EINVAL);
    for (float v : {-1.0f, NAN}) {
        EXPECT(muon(good, f, SPO_FP32, f, f, SPO_FP32, 0.9f, v), SPO_EINVAL);
        EXPECT(muon(good, f, SPO_FP32, f, f, SPO_FP32, 0.9f, 0.1f, v), SPO_EINVAL);
    }
    EXPECT(muon(good, f, SPO_FP32, f, f, SPO_FP32, 0.9f, 0.1f, 0.0f, NAN), SPO_EINVAL);
    EXPECT(muon(good, f, SPO_FP32, f, f, SPO_FP32, 0.9f, 0.1f, 0.0f, 1.0f, nullptr, 0), SPO_EWORKSPACE);
    EXPECT(muon(good, f, SPO_FP32, f, f, SPO_FP32, 0.9f, 0.1f, 0.0f, 1.0f, ws, 16), SPO_EWORKSPACE);
}

int main() {
    scores();
    updates();
    if (failures) return 1;
    std::puts("score and update host-side sanitizer run ok");
    return 0;
}
