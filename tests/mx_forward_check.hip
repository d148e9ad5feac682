// Host check of the 4-bit layer's forward launches (paper_2106_05373_amd/csrc/mx_layer_layout.h): each of
// them stays below 2^32 work-items, whatever the layer and the rows.
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include "mx_layer_layout.h"

using namespace bcpnn;

static int failures = 0;
#define CHECK(cond, what)                                                                        \
    do {                                                                                         \
        if (!(cond) && ++failures <= 20)                                                         \
            printf("%s: %dx%d -> %dx%d, %lld rows\n", what, g.in_hcu, g.in_mcu, g.out_hcu,       \
                   g.out_mcu, (long long)rows);                                                  \
    } while (0)

static Geometry layer(int in_hcu, int in_mcu, int out_hcu, int out_mcu) {
    return Geometry{in_hcu, in_mcu, out_hcu, out_mcu, (int64_t)in_hcu * in_mcu, (int64_t)out_hcu * out_mcu};
}

static void check_launches(const Geometry& g, int64_t kg) {
    const int64_t most = mx_launch_rows(g);
    for (int64_t rows : {most, most - 1, most - 31, (int64_t)1}) {
        CHECK(most >= 2 * kMxRows && most % kMxRows == 0, "row blocks of a launch");
        const ForwardShape f = mx_forward_shape(g, kg, rows);
        CHECK(mx_row_blocks(rows) * g.out_hcu * 64 * f.waves < 1ll << 32, "work-items");
        if (mx_rows_in_lds(g, rows))
            CHECK((rows + kMxTileRows - 1) / kMxTileRows * 64 * kMxWaves < 1ll << 32, "work-items of rows in LDS");
    }
}

int main() {
    for (int out_mcu : {1, 2, 10, 32, 33, 100, 128, 129, 256, 257, 300, 512, 513, 1000, 1024})
        for (int out_hcu : {1, 2, 15, 16, 17, 30, 100, 1023, 4096, 32513, 1 << 17, 1 << 21, (1 << 21) + 1, 1 << 22})
            for (int in_mcu : {1, 2, 4})
                for (int64_t kg : {1, 2, 11, 48})
                    if ((int64_t)out_hcu * out_mcu <= 1 << 22) check_launches(layer(16, in_mcu, out_hcu, out_mcu), kg);
    printf("%d failures\n", failures);
    return failures ? 1 : 0;
}
