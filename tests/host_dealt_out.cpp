// dealt_out of csrc/decode.hpp: every task once, runs together on one die.
#include "decode.hpp"

#include <cstdio>

int main() {
    uint64_t r = 1;
    auto random = [&](int most) {
        r = r * 6364136223846793005ull + 1442695040888963407ull;
        return 1 + (int)((r >> 33) % (uint64_t)most);
    };
    for (int t = 0; t < 4000; ++t) {
        const int n = random(t % 2 ? 5000 : 200), run = random(t % 3 ? 40 : 700);
        std::vector<int> die(n, -1);
        for (int b = 0; b < n; ++b) {
            const int id = evospec::dealt_out(b, n, run);
            if (id < 0 || id >= n || die[id] >= 0) return printf("%d of %d, runs of %d: task %d\n", b, n, run, id), 1;
            die[id] = b & 7;
        }
        const int whole = n / (8 * run) * (8 * run);
        for (int i = 0; i < whole; ++i)
            if (die[i] != die[i / run * run]) return printf("task %d of %d: run of %d on two dies\n", i, n, run), 1;
    }
    // the largest grid
    const int n = (1 << 24) - 1024;
    for (int run : {1, 16, 1000, n / 8})
        for (int b : {0, 1, n / 2, n - 2, n - 1})
            if (evospec::dealt_out(b, n, run) < 0 || evospec::dealt_out(b, n, run) >= n) return puts("out of range"), 1;
    puts("ok");
}
