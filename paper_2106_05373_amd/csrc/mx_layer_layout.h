// How the 4-bit layer's forward pass is laid out (host and device).
#pragma once

#include <algorithm>

#include "bcpnn_internal.h"
#include "mx_format.h"

namespace bcpnn {

// Input unit of a hidden HCU's k-th active one, `list` holding its ascending active input HCUs.  Past
// the last (k_total = active HCUs * in_mcu) the first unit of the first active HCU: what is read there
// does not count, but it is read, `vec` units at a time (a divisor of in_mcu), from a k that is a
// multiple of vec, and all of them have to be inputs.
__host__ __device__ inline uint32_t mx_active_unit(const int32_t* list, int k, int k_total, int in_mcu) {
    const int i = k < k_total ? k : 0;
    return (uint32_t)(list[i / in_mcu] * in_mcu + i % in_mcu);
}

// Units that a lane reads at once.
inline int mx_gather_width(int in_mcu) { return in_mcu % 4 == 0 ? 4 : in_mcu % 2 == 0 ? 2 : 1; }

// Waves of a workgroup and how many column tiles of 32 each takes, in how many parts they share the groups,
// and how many steps of 64 units are quantised at a time.
struct ForwardShape { int waves, tiles, parts, steps; };

constexpr int kMxStepCodes = 1024;
constexpr int kMxWaves = 16;
// Floats of a row of supports in LDS: whole quads, and rows 4 apart lie 32 banks apart.
__host__ __device__ inline int mx_support_pitch(int out_mcu) { return (out_mcu + 7) / 16 * 16 + 8; }
// Most dynamic LDS of a launch: 1024 columns' supports.
constexpr int kMxForwardLds = 4 * kMxRows * 1032;

// A wave per column tile of 32 at least (two tiles from 17 on, and from 9 on where there are more
// workgroups of 16 waves than CUs: two then share a CU; 2000 rows of 784 x 2 -> 40 x 300 units 81 -> 64
// us).  Many workgroups fill the chip with the least of them, 16 steps at a time, so that one's reads pass
// under another's products; few take up to 16 waves, which share the groups too, and all steps at once.
inline ForwardShape mx_forward_shape(const Geometry& g, int64_t kg, int64_t rows) {
    const int tiles = (int)mx_row_blocks(g.out_mcu);
    const int64_t wgs = mx_row_blocks(rows) * g.out_hcu;
    ForwardShape f{tiles <= 4 ? 4 : tiles <= 8 ? 8 : kMxWaves, tiles <= 16 ? 1 : 2, 1, 16};
    if (tiles > 8 && tiles <= 16 && wgs > 256) {
        f.waves = 8;
        f.tiles = 2;
    } else if (wgs <= 512) {
        while (f.waves < kMxWaves && 4 * kg > f.waves) f.waves *= 2;
        f.steps = 64;
    }
    f.steps = (int)std::min<int64_t>(f.steps, 4 * kg);
    f.parts = (int)std::max<int64_t>(1, std::min<int64_t>(f.waves / tiles, kg));
    return f;
}

// Rows that a launch takes, whole row blocks: it stays below 2^32 work-items.  (A launch of so many
// workgroups has the least waves for its column tiles; N_out <= 2^22 leaves room for two row blocks at least.)
inline int64_t mx_launch_rows(const Geometry& g) {
    const int64_t tiles = mx_row_blocks(g.out_mcu), waves = tiles <= 4 ? 4 : tiles <= 16 ? 8 : kMxWaves;
    return ((1ll << 32) - 1) / (64 * waves) / g.out_hcu * kMxRows;
}

// The form for many rows of a narrow layer (forward_rows_kernel): 16 rows of the inputs in LDS.
constexpr int kMxTileRows = 16;
constexpr int kMxRowsLds = 150 * 1024;
// Floats of such a row: whole quads, and rows lie 4 banks apart.
__host__ __device__ inline int64_t mx_input_pitch(int64_t n_in) { return n_in + ((4 - n_in) & 63); }
// Whether a launch takes it: the rows fit, one wave's tiles cover a hidden HCU, and row tiles and hidden
// HCUs fill most of the chip.  Measured (us, this form / the other): MNIST shape, 8192 rows 67 / 101, 4096
// rows 34 / 50, 2048 rows 36 / 32.9; 500 x 3 -> 17 x 70 units, 4096 rows 33.6 / 50; 784 x 2 -> 30 HCUs of 2, 16
// and 128 units, 3200 rows 19.5 / 34.8, 20.9 / 33.7 and 32.4 / 44.8; 40 x 4 -> 100 x 2, 3200 rows 38 / 51.
inline bool mx_rows_in_lds(const Geometry& g, int64_t rows) {
    return kMxTileRows * mx_input_pitch(g.n_in) * 4 <= kMxRowsLds && mx_row_blocks(g.out_mcu) <= 4 &&
           g.out_hcu >= kMxWaves && rows >= 200 * kMxTileRows;
}

// ---- Indices of the forward kernels, which the host's check follows ----

// Where the inputs of a workgroup's first row begin (in floats), and the bytes from row to row and from unit
// to unit: 32-bit offsets from there, x [rows][n_in] or, transposed, [n_in][stride].
struct InputSteps { uint32_t row, unit; };
__host__ __device__ inline int64_t mx_input_base(bool turned, int64_t row0, int64_t n_in) {
    return turned ? row0 : row0 * n_in;
}
__host__ __device__ inline InputSteps mx_input_steps(bool turned, int64_t n_in, int32_t stride) {
    return turned ? InputSteps{4u, 4u * (uint32_t)stride} : InputSteps{4u * (uint32_t)n_in, 4u};
}
// The row that a lane reads: its own, or the last of the rows that there are.
__host__ __device__ inline uint32_t mx_live_row(int row, int64_t rows_left) {
    return (uint32_t)(row < rows_left ? row : rows_left - 1);
}
// Group of the packed weights: `tiles` row blocks of kg groups for each hidden HCU.
__host__ __device__ inline int64_t mx_weight_group(int h, int tiles, int64_t tile, int kg, int grp) {
    return ((int64_t)h * tiles + tile) * kg + grp;
}
// Support of a row and a column in LDS, each part's in a place of its own.
__host__ __device__ inline int mx_support_at(int part, int row, int pitch, int c) {
    return part * (kMxRows * pitch) + row * pitch + c;
}
// Of forward_rows_kernel, whose lane takes a block of 16 rows or columns and 32 of 128 units (a quarter of
// the wave each): row block, step of the group at k0 and lane of the weights of column tile t.
__host__ __device__ inline int mx_rows_block(int t, int row_blocks) {
    return t / 2 < row_blocks ? t / 2 : row_blocks - 1;
}
__host__ __device__ inline int mx_rows_step(int k0, int quarter) { return k0 / kMxStep % 4 + quarter / 2; }
__host__ __device__ inline int mx_rows_lane(int c0, int quarter, int t) { return 32 * (quarter & 1) + c0 + 16 * (t & 1); }

// Rows of the transposed input: as many as a batch has, within 64 MiB.
inline int64_t mx_forward_turned_rows(const Geometry& g, int32_t max_batch) {
    const int64_t fit = (64ll << 20) / 4 / g.n_in / 64 * 64;
    return std::min<int64_t>(fit, ((int64_t)max_batch + 63) / 64 * 64);
}

// Codes and scales of a chunk; afterwards the parts' supports.
inline size_t mx_forward_lds(const ForwardShape& f, int out_mcu) {
    const size_t chunk = (size_t)f.steps * (kMxStepCodes + kMxStep);
    return std::max(chunk, sizeof(float) * f.parts * kMxRows * mx_support_pitch(out_mcu));
}

}  // namespace bcpnn
