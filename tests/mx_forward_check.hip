// Host check of the 4-bit layer's forward pass (paper_2106_05373_amd/csrc/mx_layer_layout.h): each launch
// stays below 2^32 work-items, and the accesses of its kernels, followed lane by lane through the index
// functions that they share with this file, lie inside their buffers: the inputs and the transposed ones, the
// units, the packed weights and scales, the biases, the LDS and the results.  Of a launch the first and last
// row blocks and hidden HCUs are followed, of a hidden HCU all units.
#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <vector>

#include "mx_layer_layout.h"

using namespace bcpnn;

static int failures = 0;
static int64_t accesses = 0;
static const char* form = "";
struct Layer {
    Geometry g;
    int32_t max_batch;
    std::vector<int32_t> active;         // active input HCUs of each hidden HCU
    int32_t most;                        // units of the largest
    int64_t kg;
};
#define CHECK(cond, what)                                                                                    \
    do {                                                                                                     \
        ++accesses;                                                                                          \
        if (!(cond) && ++failures <= 20)                                                                     \
            printf("%s (%s): %dx%d -> %dx%d, %d units, %lld rows\n", what, form, g.in_hcu, g.in_mcu, g.out_hcu, \
                   g.out_mcu, most, (long long)rows);                                                        \
    } while (0)

static Geometry geometry(int in_hcu, int in_mcu, int out_hcu, int out_mcu) {
    return Geometry{in_hcu, in_mcu, out_hcu, out_mcu, (int64_t)in_hcu * in_mcu, (int64_t)out_hcu * out_mcu};
}

static void check_launches(const Geometry& g, int64_t kg) {
    const int64_t most_rows = mx_launch_rows(g);
    const int most = (int)(kg * kMxGroup);
    for (int64_t rows : {most_rows, most_rows - 1, most_rows - 31, (int64_t)1}) {
        CHECK(most_rows >= 2 * kMxRows && most_rows % kMxRows == 0, "row blocks of a launch");
        const ForwardShape f = mx_forward_shape(g, kg, rows);
        CHECK(mx_row_blocks(rows) * g.out_hcu * 64 * f.waves < 1ll << 32, "work-items");
        if (mx_rows_in_lds(g, rows))
            CHECK((rows + kMxTileRows - 1) / kMxTileRows * 64 * kMxWaves < 1ll << 32, "work-items of rows in LDS");
    }
}

// The k-th entry of a hidden HCU's units: its active HCUs are the last ones, so that the last input is read.
struct Units {
    std::vector<int32_t> list;
    int k_total, in_mcu;
    Units(const Geometry& g, int active) : list(active), k_total(active * g.in_mcu), in_mcu(g.in_mcu) {
        for (int i = 0; i < active; ++i) list[i] = g.in_hcu - active + i;
    }
    uint32_t operator[](int k) const { return mx_active_unit(list.data(), k, k_total, in_mcu); }
};

static std::vector<int64_t> ends(int64_t n) {
    std::vector<int64_t> v{0};
    if (n > 2) v.push_back(n / 2);
    if (n > 1) v.push_back(n - 1);
    return v;
}

// forward_kernel over `rows` rows: x [rows][n_in] (vec > 0), or [n_in][stride] (vec = 0).
static void check_forward(const Layer& L, int64_t rows, int vec, int64_t stride) {
    const Geometry& g = L.g;
    const int most = L.most;
    const ForwardShape f = mx_forward_shape(g, L.kg, rows);
    const int M = g.out_mcu, tiles = (M + 31) / 32, kg = (int)L.kg, n_waves = f.waves;
    const int64_t lds = (int64_t)mx_forward_lds(f, M), inputs = 4 * (vec ? rows * g.n_in : g.n_in * stride);
    const int64_t groups_held = (int64_t)g.out_hcu * tiles * kg;
    CHECK(lds <= kMxForwardLds && n_waves <= kMxWaves, "launch");
    const InputSteps in = mx_input_steps(vec == 0, g.n_in, (int32_t)stride);
    for (int64_t rb : ends(mx_row_blocks(rows)))
        for (int64_t h64 : ends(g.out_hcu)) {
            const int h = (int)h64;
            const int64_t row0 = rb * kMxRows;
            const Units units(g, L.active[h]);
            const int64_t base = 4 * mx_input_base(vec == 0, row0, g.n_in);
            const int chunk = f.steps * kMxStep;
            for (int k0 = 0; k0 < units.k_total; k0 += chunk) {
                const int live = std::min(chunk, units.k_total - k0), groups = (live + kMxGroup - 1) / kMxGroup;
                CHECK((4 * groups - 1) * 1024 + 63 * 16 + 16 <= f.steps * kMxStepCodes, "codes in LDS");
                CHECK(f.steps * kMxStepCodes + (groups - 1) * kMxGroupScales + 4 * 63 + 3 < lds, "scales in LDS");
                for (int st = 0; st < 4 * groups; ++st) {
                    CHECK(k0 + st * kMxStep + 63 < kg * kMxGroup, "units");
                    const int step = vec ? vec : 1;
                    for (int half = 0; half < 2; ++half) {
                        if (st * kMxStep + 32 * half >= live) continue;
                        for (int i = 0; i < 32; i += step) {
                            const uint32_t u = units[k0 + st * kMxStep + 32 * half + i];
                            for (int lane_row : {0, 1, 15, 30, 31}) {
                                const uint32_t r = mx_live_row(lane_row, rows - row0);
                                const int64_t exact = (int64_t)u * in.unit + (int64_t)r * in.row;
                                CHECK((uint32_t)(u * in.unit + r * in.row) == exact, "offset beyond 32 bits");
                                CHECK(base + exact + 4 * step <= inputs, "inputs");
                                CHECK((base + exact) % (4 * step) == 0, "alignment of inputs");
                                CHECK(vec ? (base + exact) / 4 == (row0 + r) * g.n_in + u
                                          : (base + exact) / 4 == u * stride + row0 + r, "another input");
                            }
                        }
                    }
                }
                for (int wave = 0; wave < n_waves; ++wave) {
                    const int part = f.parts > 1 ? wave / tiles : 0, tile0 = f.parts > 1 ? wave % tiles : wave;
                    if (part >= f.parts || tile0 >= tiles) continue;
                    for (int q = part; q < groups; q += f.parts)
                        for (int t = 0; t < f.tiles; ++t) {
                            if (f.tiles > 1 && tile0 + t * n_waves >= tiles) continue;
                            const int64_t at = mx_weight_group(h, tiles, tile0 + t * n_waves, kg, k0 / kMxGroup + q);
                            CHECK(at >= 0 && at < groups_held, "weights");
                        }
                }
            }
            const int pitch = mx_support_pitch(M);
            for (int part : {0, f.parts - 1})
                for (int c : {0, M - 1}) {
                    CHECK(4 * (int64_t)mx_support_at(part, 31, pitch, c) + 4 <= lds, "supports in LDS");
                    CHECK(4 * (int64_t)(mx_support_at(part, 31, pitch, c / 4 * 4) + 4) <= lds, "quads in LDS");
                }
            for (int r : {0, 31})
                if (row0 + r < rows)
                    CHECK((row0 + r) * g.n_out + (int64_t)h * M + M <= rows * g.n_out, "results");
        }
}

// forward_rows_kernel over `rows` rows.
static void check_rows(const Layer& L, int64_t rows, int vec) {
    const Geometry& g = L.g;
    const int most = L.most, kg = (int)L.kg, rbs = (g.out_mcu + 31) / 32;
    const int64_t pitch = mx_input_pitch(g.n_in), lds = kMxTileRows * pitch * 4;
    const int64_t groups_held = (int64_t)g.out_hcu * rbs * kg;
    CHECK(lds <= kMxRowsLds && kMxTileRows == kMxWaves && g.out_mcu <= 16 * 8, "launch");
    CHECK(pitch >= g.n_in && pitch % 4 == 0, "pitch");
    for (int64_t b : ends((rows + kMxTileRows - 1) / kMxTileRows)) {
        const int64_t row0 = b * kMxTileRows;
        const int live = (int)std::min<int64_t>(kMxTileRows, rows - row0);
        for (int wave = 0; wave < live; ++wave) {
            const int step = g.n_in % 4 == 0 ? 4 : 1;
            const int64_t last = (g.n_in - 1) / step * step;
            CHECK((row0 + wave) * g.n_in + last + step <= rows * g.n_in, "inputs");
            CHECK(((row0 + wave) * g.n_in) % step == 0, "alignment of inputs");
            CHECK(wave * pitch + last + step <= lds / 4, "inputs in LDS");
        }
        for (int64_t h64 : ends(g.out_hcu)) {
            const int h = (int)h64;
            const Units units(g, L.active[h]);
            for (int k0 = 0; k0 < units.k_total; k0 += 128)
                for (int quarter = 0; quarter < 4; ++quarter) {
                    const int at = k0 + 32 * quarter;
                    CHECK(at % 4 == 0 && at + 32 <= kg * kMxGroup, "units");
                    for (int c0 = 0; c0 < 16; ++c0) {
                        for (int t = 0; t < 8; ++t) {
                            const int64_t grp = mx_weight_group(h, rbs, mx_rows_block(t, rbs), kg, k0 / kMxGroup);
                            const int step = mx_rows_step(k0, quarter), lane = mx_rows_lane(c0, quarter, t);
                            CHECK(grp >= 0 && grp < groups_held, "weights");
                            CHECK(step >= 0 && step < 4 && lane >= 0 && lane < 64, "lanes of the weights");
                            if (16 * t + c0 < g.out_mcu)
                                CHECK(32 * mx_rows_block(t, rbs) + lane % 32 == 16 * t + c0 &&
                                          k0 / kMxGroup * kMxGroup + 64 * step + 32 * (lane / 32) == at, "another weight");
                        }
                        const uint32_t r = mx_live_row(c0, live);
                        CHECK((int)r < live, "rows in LDS");
                        for (int i = 0; i < 32; i += vec) {
                            const uint32_t u = units[at + i];
                            CHECK(u % vec == 0 && r * pitch + u + vec <= (r + 1) * pitch && u + vec <= g.n_in,
                                  "a gather past its row");
                        }
                    }
                }
            CHECK((int64_t)h * g.out_mcu + std::min(16 * 7 + 15, g.out_mcu - 1) < g.n_out, "biases");
            for (int r = 0; r < live; ++r)
                CHECK((row0 + r) * g.n_out + (int64_t)(h + 1) * g.out_mcu <= rows * g.n_out, "results");
        }
    }
}

// Every form over `rows` rows, whichever a launch would choose.
static void check(const Layer& L, int64_t rows) {
    const Geometry& g = L.g;
    const int most = L.most, vec = mx_gather_width(g.in_mcu);
    for (int k : {0, L.active[0] * g.in_mcu - 1})
        CHECK(k < most && (k + 1 <= L.kg * kMxGroup), "units of a hidden HCU");
    form = "direct";
    if (rows <= mx_launch_rows(g)) check_forward(L, rows, vec, 0);
    const int64_t turned = mx_forward_turned_rows(g, L.max_batch);
    form = "transposed";
    if (turned > 0) {
        CHECK(turned * g.n_in * 4 <= 64ll << 20 && turned % 64 == 0, "the transposition's workspace");
        for (int64_t r : {(int64_t)0, (rows - 1) / turned * turned}) {     // the first piece and the last
            const int64_t n = std::min(turned, rows - r);
            CHECK((g.n_in - 1) * turned + n <= turned * g.n_in, "transposed rows");
            CHECK((g.n_in + 63) / 64 * ((n + 63) / 64) * 256 < 1ll << 32, "work-items of the transposition");
            check_forward(L, n, 0, turned);
        }
    }
    form = "rows in LDS";
    if (mx_rows_in_lds(g, rows)) check_rows(L, rows, vec);
}

// Hidden HCUs of unequal receptive fields: `active` inputs, down to one.
static Layer layer(int in_hcu, int in_mcu, int out_hcu, int out_mcu, int active, int32_t max_batch) {
    Layer L{geometry(in_hcu, in_mcu, out_hcu, out_mcu), max_batch, {}, 0, 0};
    for (int h = 0; h < out_hcu; ++h)
        L.active.push_back(h == 0 || active < 3 ? active : h == out_hcu - 1 ? 1 : active - h % (active / 2 + 1));
    L.most = active * in_mcu;
    L.kg = mx_groups(L.most);
    return L;
}

int main() {
    for (int out_mcu : {1, 2, 10, 32, 33, 100, 128, 129, 256, 257, 300, 512, 513, 1000, 1024})
        for (int out_hcu : {1, 2, 15, 16, 17, 30, 100, 1023, 4096, 32513, 1 << 17, 1 << 21, (1 << 21) + 1, 1 << 22})
            for (int in_mcu : {1, 2, 4})
                for (int64_t kg : {1, 2, 11, 48})
                    if ((int64_t)out_hcu * out_mcu <= 1 << 22)
                        check_launches(geometry(16, in_mcu, out_hcu, out_mcu), kg);

    // the image layers, a ragged one, a readout, a wide one and a shard of the large image layer
    struct Case { int in_hcu, in_mcu, out_hcu, out_mcu, active; std::vector<int> rows; };
    const Case cases[] = {
        {784, 2, 30, 100, 78, {1, 16, 128, 512, 1024, 2048, 3200, 8192, 8209}},
        {27648, 2, 100, 100, 1382, {1, 8, 16, 32, 64, 128, 256, 300}},
        {500, 3, 17, 70, 167, {1, 75, 512, 4096, 4097}},
        {30, 100, 1, 10, 30, {1, 128, 1024}},
        {2000, 2, 10, 1000, 600, {1, 128, 1024}},
        {27648, 2, 13, 100, 1382, {32, 256}},
        // limits: N_in = 65535 * 64, the most active units, the widest hidden HCU, the widest rows in LDS
        {32767, 128, 2, 33, 96, {1, 33}},
        {49152, 85, 1, 16, 144, {5}},
        {6144, 2, 3, 1024, 6144, {1, 40}},
        {2396, 1, 16, 128, 2396, {3200, 3217}},
        {599, 4, 16, 1, 599, {3201}},
        {1198, 2, 17, 33, 9, {4096}},
        {1, 1, 1, 1, 1, {1, 5000}},
        {3, 1, 16, 2, 3, {3200, 5000}},
    };
    for (const Case& c : cases)
        for (int max_batch : {1, 64, 8209})
            for (int rows : c.rows) check(layer(c.in_hcu, c.in_mcu, c.out_hcu, c.out_mcu, c.active, max_batch), rows);
    for (int in_hcu : {1, 2, 7, 129, 700})
        for (int in_mcu : {1, 2, 3, 4, 6, 10, 25})
            for (int out_mcu : {1, 8, 31, 32, 33, 97, 128, 129, 300, 513})
                for (int out_hcu : {1, 16, 40})
                    for (int active : {1, 2, 5, 64, 127, 500})
                        for (int rows : {1, 31, 33, 100, 3205})
                            if (active <= in_hcu && active * in_mcu <= 12288)
                                check(layer(in_hcu, in_mcu, out_hcu, out_mcu, active, 100), rows);
    printf("%d failures in %lld accesses\n", failures, (long long)accesses);
    return failures ? 1 : 0;
}
