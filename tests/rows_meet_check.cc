// Common elements of two sets of rows (csrc/rows_meet.h) against a map of all their bytes. Argument "spans": the spans from first to last are
// compared instead, which must fail.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "rows_meet.h"

int main(int argc, char** argv) {
    const bool spans = argc > 1 && !strcmp(argv[1], "spans");
    srand(3);
    int failures = 0, meet = 0, trials = 200000;
    for (int t = 0; t < trials; ++t) {
        const int64_t aw = 1 + rand() % 6, bw = t % 2 ? aw : 1 + rand() % 6, most = aw > bw ? aw : bw;
        const int64_t rows = 1 + rand() % 4, groups = 1 + rand() % 4;
        const int64_t pitch = most + (rand() % 2 ? rand() % 9 : 0), apart = most + (rows - 1) * pitch + (rand() % 2 ? rand() % 9 : 0);
        const int64_t inner = most + (rows - 1) * pitch + (groups - 1) * apart;
        const int64_t d = rand() % (2 * inner + 9) - inner - 4, base = 2 * inner + 20;
        std::vector<char> map(4 * inner + 60);
        bool have = false;
        for (int set = 0; set < 2; ++set)
            for (int64_t i = 0; i < groups; ++i)
                for (int64_t j = 0; j < rows; ++j)
                    for (int64_t e = 0; e < (set ? bw : aw); ++e) {
                        char& c = map[base + (set ? d : 0) + i * apart + j * pitch + e];
                        if (set) have |= c != 0;
                        else c = 1;
                    }
        const int64_t span = inner - most;
        bool got = spans ? d < span + aw && -d < span + bw : sage::groups_meet(d, apart, groups, pitch, rows, aw, bw);
        if (!spans && groups == 1) got = sage::rows_meet(d, pitch, rows, aw, bw);
        meet += have;
        if (got != have && ++failures <= 5) printf("%d x %d rows, d %d: %d, not %d\n", (int)groups, (int)rows, (int)d, (int)got, (int)have);
    }
    if (meet < trials / 10 || meet > trials * 9 / 10) ++failures, printf("meeting in %d of %d\n", meet, trials);
    if (failures) printf("%d failures\n", failures);
    else printf("rows_meet_check ok\n");
    return failures ? 1 : 0;
}
