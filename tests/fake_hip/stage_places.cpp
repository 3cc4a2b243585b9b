// Which values threads lay out for the tiled products (csrc/glu_stage.hpp), on the host
// (tests/test_glu_places_host.py).  Usage: stage_places; exit status 0 = all held.
#include <stdio.h>

#include <algorithm>
#include <vector>

#include "glu_stage.hpp"

using namespace exemcl;

static int failures = 0;
static void expect(bool ok, const char *what, long long at) {
    if (!ok && ++failures <= 20) fprintf(stderr, "FAILED: %s (%lld)\n", what, at);
}

// Every eight values of every job once, and nothing for workgroups past the jobs'.
static void check_all(const std::vector<DenseStageJob> &jobs) {
    StageJobs s{};
    const int64_t blocks = stage_jobs(jobs.data(), (int)jobs.size(), &s);
    std::vector<std::vector<int>> seen;
    for (const auto &j : jobs) seen.emplace_back((size_t)(j.n * ((j.d + 7) / 8)), 0);
    for (int64_t b = 0; b < blocks + 5; ++b)
        for (int t = 0; t < kStageThreads; ++t) {
            const StagePlace p = stage_place(s, b, t);
            if (p.job < 0) continue;
            expect(b < blocks && p.job < (int)jobs.size(), "a job that there is", b);
            const DenseStageJob &j = jobs[(size_t)p.job];
            expect(p.ld == (j.d + 7) / 8 * 8 && p.row >= 0 && p.row < j.n && p.c >= 0 && p.c < j.d && p.c % 8 == 0, "inside", b);
            ++seen[(size_t)p.job][(size_t)(p.row * (p.ld / 8) + p.c / 8)];
        }
    for (const auto &job : seen)
        expect(std::all_of(job.begin(), job.end(), [](int n) { return n == 1; }), "each once", (long long)job.size());
}

// Counts of workgroups that a grid rounds up to whole rows of 2^20: its last ones have no
// job, whether one, two or three are set.
static void check_padding() {
    const DenseStageJob large{nullptr, (int64_t(1) << 31) - 1, 1 << 20, nullptr}, small{nullptr, 3, 5, nullptr};
    for (int count = 1; count <= 3; ++count) {
        const DenseStageJob jobs[3] = {count == 1 ? large : small, count == 2 ? large : small, large};
        StageJobs s{};
        const int64_t blocks = stage_jobs(jobs, count, &s), row = int64_t(1) << 20, end = (blocks + row - 1) / row * row;
        for (int64_t b : {blocks, blocks + 1, (blocks + end) / 2, end - 1, end})
            for (int t : {0, 1, 255}) expect(stage_place(s, b, t).job == -1, "padding", count);
        const StagePlace last = stage_place(s, blocks - 1, 0);
        expect(last.job == count - 1 && last.row < jobs[count - 1].n, "the last workgroup", count);
    }
}

int main() {
    check_all({{nullptr, 7, 13, nullptr}});
    check_all({{nullptr, 100, 1, nullptr}, {nullptr, 33, 301, nullptr}});
    check_all({{nullptr, 257, 8, nullptr}, {nullptr, 1, 4099, nullptr}, {nullptr, 64, 32, nullptr}});
    check_padding();
    if (failures) fprintf(stderr, "%d checks failed\n", failures);
    else printf("checks passed\n");
    return failures ? 1 : 0;
}
