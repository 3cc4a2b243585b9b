// The gated block and the calls on 4-bit weights over the runtime of driver.cpp, which
// launches nothing (tests/test_glu_host_runtime.py).  Usage: glu_driver CHECK; exit
// status 0 = every expectation of that check held.
#define main other_checks
#include "driver.cpp"
#undef main

namespace fake {
hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
}

extern "C" hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) {
    *s = fake::capture;
    return hipSuccess;
}

static uint32_t *const kU = (uint32_t *)kV;

static int glu(int64_t n, int64_t d, int64_t f, int prec, void *st) {
    return exemplar_glu(kV, n, d, kV, kV, f, kF, kF, prec, EXEMCL_SILU, kV, kV, kV, st);
}
static int grad(int64_t n, int64_t d, int64_t f, int prec, int act, bool bias, void *st) {
    return exemplar_glu_backward(kV, kV, kV, kV, kV, kV, n, d, f, prec, act, kV, kV, kV, bias ? kF : nullptr, bias ? kF : nullptr, st);
}

// Temporary memory that a capture allocates belongs to its graph: calls that need some
// refuse a capturing stream and queue nothing, the others are captured.
static void check_capture() {
    for (const bool warm : {false, true}) {
        const std::string at = warm ? "with a kept block" : "without one";
        void *st = fresh_stream();
        if (warm) expect(grad(500, 300, 200, EXEMCL_BF16, 0, true, st) == EXEMCL_OK, "gradient");
        fake::launches.clear();
        fake::allocs.clear();
        fake::capture = hipStreamCaptureStatusActive;
        expect(grad(500, 300, 200, EXEMCL_BF16, 0, true, st) == EXEMCL_EINVAL, "gradient refuses", at);
        expect(glu(2000, 300, 2000, EXEMCL_BF16, st) == EXEMCL_EINVAL, "rows to lay out", at);
        expect(glu(2000, 304, 2000, EXEMCL_FP32, st) == EXEMCL_EINVAL, "parts to lay out", at);
        expect(fake::launches.empty() && fake::allocs.empty(), "nothing queued", at);
        expect(glu(500, 304, 200, EXEMCL_FP16, st) == EXEMCL_OK, "whole rows", at);
        expect(glu(64, 301, 200, EXEMCL_FP32, st) == EXEMCL_OK && glu(1, 301, 200, EXEMCL_BF16, st) == EXEMCL_OK, "few rows", at);
        expect(exemplar_w4_product(kV, 500, 301, EXEMCL_FP32, kV, kU, 70, 64, kF, kV, st) == EXEMCL_OK, "4-bit product", at);
        expect(exemplar_w4_glu(kV, 5000, 301, EXEMCL_FP16, kV, kU, kV, kU, 7000, 32, kF, kF, EXEMCL_GELU, kV, st) == EXEMCL_OK, "4-bit block", at);
        expect(fake::allocs.empty() && fake::launches.size() == 5, "captured", at);
        fake::capture = hipStreamCaptureStatusNone;
    }
}

// Launches of any size keep within the grids' 32 bits and the LDS that is announced
// (driver.cpp checks each), or are refused.
static void check_glu_grids() {
    const int64_t rows[] = {1, 16, 17, 64, 65, 1000, int64_t(1) << 20, (int64_t(1) << 31) - 1};
    const int64_t cols[] = {1, 7, 128, 3001, 1 << 14, 1 << 20};
    for (int prec = 0; prec < 3; ++prec)
        for (int64_t n : rows)
            for (int64_t d : cols)
                for (int64_t f : cols) {
                    const std::string at = std::to_string(n) + " x " + std::to_string(d) + " x " + std::to_string(f);
                    if ((double)n * (double)std::max(d, f) > 1e11 || (double)d * (double)f > 1e11) continue;  // of no memory
                    expect(glu(n, d, f, prec, fresh_stream()) == EXEMCL_OK, "block", at);
                    expect(grad(n, d, f, prec, 0, true, fresh_stream()) == EXEMCL_OK, "gradient", at);
                    for (int group : {32, 64, 128}) {
                        expect(exemplar_w4_product(kV, n, d, prec, kV, kU, f, group, kF, kV, fresh_stream()) == EXEMCL_OK, "product", at);
                        expect(exemplar_w4_glu(kV, n, d, prec, kV, kU, kV, kU, f, group, kF, kF, 0, kV, fresh_stream()) == EXEMCL_OK, "4-bit block", at);
                        expect(exemplar_w4_quantize(kV, n, d, prec, group, kV, kU, fresh_stream()) == EXEMCL_OK, "rounding", at);
                        expect(exemplar_w4_dequantize(kV, kU, n, d, group, prec, kV, fresh_stream()) == EXEMCL_OK, "and back", at);
                    }
                }
}

// A limit that leaves no room for partial sums: the products run undivided.
static void check_glu_limits() {
    const int64_t n = 16000, d = 128, f = 512;
    void *st = fresh_stream();
    fake::launches.clear();
    expect(grad(n, d, f, EXEMCL_BF16, 0, false, st) == EXEMCL_OK, "gradient");
    const size_t divided = fake::launches.size();
    const size_t left = fake::pool_left;
    fake::pool_left = (size_t)(2 * n * f * 2 + (1 << 16));
    fake::launches.clear();
    expect(grad(n, d, f, EXEMCL_BF16, 0, false, fresh_stream()) == EXEMCL_OK, "without partial sums");
    expect(fake::launches.size() < divided, "not divided");
    fake::pool_left = 1 << 16;
    fake::launches.clear();
    expect(grad(n, d, f, EXEMCL_BF16, 0, false, fresh_stream()) == EXEMCL_ENOMEM && fake::launches.empty(), "no memory");
    fake::pool_left = left;
}

// Calls read from the standard input, a line each: the kernels that each launches,
// with their workgroups.
static void print_kernels_of_calls() {
    char what[16];
    long long n, d, f, prec, e;
    while (scanf("%15s %lld %lld %lld %lld %lld", what, &n, &d, &f, &prec, &e) == 6) {
        const std::string call = what;
        void *st = fresh_stream();
        fake::launches.clear();
        int rc = -1;
        if (call == "glu") rc = glu(n, d, f, (int)prec, st);
        if (call == "grad") rc = grad(n, d, f, (int)prec, (int)e, true, st);
        if (call == "w4") rc = exemplar_w4_product(kV, n, d, (int)prec, kV, kU, f, (int)e, kF, kV, st);
        if (call == "w4_glu") rc = exemplar_w4_glu(kV, n, d, (int)prec, kV, kU, kV, kU, f, (int)e, kF, kF, 0, kV, st);
        if (call == "quantize") rc = exemplar_w4_quantize(kV, n, d, (int)prec, (int)e, kV, kU, st);
        if (call == "dequantize") rc = exemplar_w4_dequantize(kV, kU, n, d, (int)e, (int)prec, kV, st);
        if (call == "empty") rc = exemplar_glu_backward(kV, kV, kV, kV, kV, kV, 0, d, f, (int)prec, 0, kV, kV, kV, kF, kF, st);
        expect(rc == EXEMCL_OK, "a call", call);
        for (const auto &x : fake::launches) printf("%s:%u ", x.name.c_str(), x.grid.x * x.grid.y);
        printf("\n");
    }
}

int main(int argc, char **argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "capture") check_capture();
    else if (what == "grids") check_glu_grids();
    else if (what == "limits") check_glu_limits();
    else if (what == "calls") print_kernels_of_calls();
    else if (what == "all") for (const auto &x : fake::kernels()) printf("%s\n", x.second.c_str());
    else expect(false, "no such check", what);
    if (failures) fprintf(stderr, "%d checks failed\n", failures);
    else printf("%s: checks passed\n", what.c_str());
    return failures ? 1 : 0;
}
