// The calls on microscaled rows over the runtime of driver.cpp, which launches
// nothing (tests/test_mx_host_runtime.py).  Usage: mx_driver CHECK; exit status 0
// = every expectation of that check held.
#define main other_checks
#include "driver.cpp"
#undef main

namespace fake {
hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
hipError_t capture_error = hipSuccess;
}  // namespace fake

extern "C" hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) {
    *s = fake::capture;
    if (fake::capture_error != hipSuccess) fake::last = fake::capture_error;
    return fake::capture_error;
}

static int eval(int64_t n, int64_t d, int64_t l, int64_t k, void *st) {
    return exemplar_mx_eval(kV, kV, n, d, kI, l, k, kF, st);
}
static int grad(float *dweight, void *st) {
    return exemplar_rmsnorm_backward(kV, kV, kV, kF, nullptr, 500, 300, EXEMCL_BF16, kV, dweight, st);
}

// Temporary memory that a capture allocates belongs to its graph, and what a
// stream keeps may be released while a graph still uses it: calls that need some
// refuse a capturing stream, whether or not a block is kept for it, and queue
// nothing.  Calls that need none are captured.
static void check_capture() {
    for (const bool warm : {false, true}) {
        const std::string at = warm ? "with a kept block" : "without one";
        void *st = fresh_stream();
        if (warm) {
            expect(eval(5000, 300, 40, 3, st) == EXEMCL_OK, "eval");
            expect(grad(kF, st) == EXEMCL_OK, "gradient");
        }
        for (const auto status : {hipStreamCaptureStatusActive, hipStreamCaptureStatusInvalidated}) {
            fake::launches.clear();
            fake::allocs.clear();
            fake::capture = status;
            expect(eval(5000, 300, 40, 3, st) == EXEMCL_EINVAL, "eval refuses", at);
            expect(eval(5000, 2500, 40, 3, st) == EXEMCL_EINVAL, "eval of long rows refuses", at);
            expect(grad(kF, st) == EXEMCL_EINVAL, "gradient refuses", at);
            expect(fake::launches.empty() && fake::allocs.empty(), "nothing queued", at);
            expect(eval(5000, 300, 0, 3, st) == EXEMCL_OK && eval(5000, 300, 40, 0, st) == EXEMCL_OK, "no temporary memory", at);
            expect(grad(nullptr, st) == EXEMCL_OK, "no dweight, no temporary memory", at);
            expect(exemplar_mx_product(kV, kV, 5, EXEMCL_MXFP8, kV, kV, 900, 500, kF, EXEMCL_FP32, kF, st) == EXEMCL_OK, "product", at);
            expect(fake::allocs.empty() && fake::launches.size() == 3, "captured", at);
            fake::capture = hipStreamCaptureStatusNone;
        }
        fake::capture_error = hipErrorStreamCaptureImplicit;  // the null stream while another captures
        fake::launches.clear();
        expect(eval(5000, 300, 40, 3, st) == EXEMCL_EDEVICE && grad(kF, st) == EXEMCL_EDEVICE, "cannot be told", at);
        expect(fake::launches.empty() && fake::last == hipSuccess, "nothing queued, no error left", at);
        fake::capture_error = hipSuccess;
        expect(eval(5000, 300, 40, 3, st) == EXEMCL_OK && grad(kF, st) == EXEMCL_OK, "after the capture", at);
    }
}

// Sets of any size, as exemplar_eval takes them: the count of members is 64 bits,
// and the tiles of one group of 16 sets bound it through their memory alone.
static void check_members() {
    for (int64_t d : {20, 300, 1536, 2048, 2500})
        for (int64_t k : {int64_t(1) << 24, (int64_t(1) << 24) + 1, int64_t(40000000), int64_t(1) << 28})
            for (int64_t l : {1, 40, 100}) {
                const std::string at = "d " + std::to_string(d) + " k " + std::to_string(k) + " l " + std::to_string(l);
                expect(eval(1000, d, l, k, fresh_stream()) == EXEMCL_OK, "members", at);
                const size_t left = fake::pool_left;
                fake::pool_left = size_t(1) << 20;
                expect(eval(1000, d, l, k, fresh_stream()) == EXEMCL_ENOMEM, "no memory for one group", at);
                fake::pool_left = left;
            }
}

// Calls read from the standard input, a line each: the kernels that each launches,
// with their workgroups.
static void print_kernels_of_calls() {
    char what[16];
    long long a, b, c, d, e;
    while (scanf("%15s %lld %lld %lld %lld %lld", what, &a, &b, &c, &d, &e) == 6) {
        const std::string call = what;
        void *st = fresh_stream();
        fake::launches.clear();
        int rc = -1;
        if (call == "product")  // m n d format precision
            rc = exemplar_mx_product(kV, kV, a, (int)d, kV, kV, b, c, nullptr, (int)e, kF, st);
        if (call == "sets")  // n d l k
            rc = exemplar_mx_eval(kV, kV, a, b, kI, c, d, kF, st);
        if (call == "gradient")  // n d precision
            rc = exemplar_rmsnorm_backward(kV, kV, kV, kF, nullptr, a, b, (int)c, kV, kF, st);
        if (call == "norm")  // n d precision format
            rc = exemplar_rmsnorm(kV, kV, kV, a, b, (int)c, 1e-6f, (int)d, kV, kV, kV, kF, st);
        if (call == "quantize")  // n d precision format
            rc = exemplar_mx_quantize(kV, a, b, (int)c, (int)d, kV, kV, st);
        if (call == "dequantize")  // n d precision format
            rc = exemplar_mx_dequantize(kV, kV, a, b, (int)d, (int)c, kV, st);
        expect(rc == EXEMCL_OK, "a call", call);
        for (const auto &x : fake::launches) printf("%s:%u ", x.name.c_str(), x.grid.x * x.grid.y);
        printf("\n");
    }
}

// Every kernel in the library.
static void print_all_kernels() {
    for (const auto &x : fake::kernels()) printf("%s\n", x.second.c_str());
}

int main(int argc, char **argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "capture") check_capture();
    else if (what == "members") check_members();
    else if (what == "calls") print_kernels_of_calls();
    else if (what == "all") print_all_kernels();
    else expect(false, "no such check", what);
    if (failures) fprintf(stderr, "%d checks failed\n", failures);
    else printf("%s: checks passed\n", what.c_str());
    return failures ? 1 : 0;
}
