// Forward pass of a layer on 4-bit weights: for every hidden HCU the active inputs are gathered and
// quantised (blocks of 32 along the ascending active units), multiplied with the MX weights of that
// HCU, and the supports go through the softmax or the argmax, in one launch (two where the inputs are
// transposed first).
//
// The matrix instructions are the least of it (an STL-shaped batch of 256 has 14 GFLOP, 3 us of them):
// the bound is the gather, since every (row, hidden HCU) pair reads inputs of its own, and in fp32, a
// block's scale depending on its values.  Three forms, by what the gather costs (transposes,
// mx_rows_in_lds): directly, a line per lane and load; from the transposed inputs, whole lines; from
// LDS.  Four batches in turn, activities and supports: MNIST shape, 1 row 6.0 us, 128 rows 8.8, 8192 rows 78
// (196 MB of stores; 64 where the same batch comes again, partly from the caches); STL shape, 1 row 12.8, 256
// rows 82 (283 MB of gathered inputs and 141 MB of weights from L2; 71).
#include <algorithm>

#include "bcpnn_internal.h"
#include "device_common.h"
#include "mx_format.h"
#include "mx_layer_layout.h"

namespace bcpnn {
namespace {

// The active input units of every hidden HCU in ascending order, [out_hcu][256 kg], and their number.
__global__ void __launch_bounds__(kMxGroup)
units_kernel(Geometry g, ActiveLists act, uint32_t kg, int32_t* __restrict__ units, int32_t* __restrict__ n_units) {
    const int h = blockIdx.x / kg, k = (blockIdx.x % kg) * kMxGroup + threadIdx.x;
    const int k_total = act.count[h] * g.in_mcu;
    units[(int64_t)h * kg * kMxGroup + k] =
        (int32_t)mx_active_unit(act.list + (int64_t)h * act.stride, k, k_total, g.in_mcu);
    if (k == 0) n_units[h] = k_total;
}

// Weights of the active blocks in the MX layout: per hidden HCU an operand [out_mcu][k], k counting
// its ascending active units, with the row blocks and groups of the largest one.
__global__ void __launch_bounds__(256)
pack_kernel(Geometry g, const float* __restrict__ w, ActiveUnits act, uint32_t rbs, uint8_t* __restrict__ codes,
            uint8_t* __restrict__ scales) {
    const int lane = threadIdx.x & 63, step = threadIdx.x >> 6;
    const uint32_t grp = blockIdx.x % act.kg, rb = blockIdx.x / act.kg % rbs, h = blockIdx.x / act.kg / rbs;
    const int m = rb * kMxRows + (lane & 31);
    const int k_total = act.count[h];
    const int k0 = grp * kMxGroup + step * kMxStep + 32 * (lane >> 5);
    const int32_t* units = act.units + (int64_t)h * act.kg * kMxGroup + k0;
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i)
        v[i] = k0 + i < k_total && m < g.out_mcu ? w[units[i] * g.n_out + (int64_t)h * g.out_mcu + m] : 0.0f;
    uint32_t byte;
    const mx_codes c = mx_block(v, byte);
    reinterpret_cast<mx_codes*>(codes + (int64_t)blockIdx.x * kMxGroupCodes)[threadIdx.x] = c;
    scales[(int64_t)blockIdx.x * kMxGroupScales + 4 * lane + step] = (uint8_t)byte;
}

// x [B][n] -> xt [n][stride]: the rows of one unit side by side.
__global__ void __launch_bounds__(256)
transpose_kernel(const float* __restrict__ x, int32_t B, int64_t n, uint32_t unit_tiles, float* __restrict__ xt,
                 int32_t stride) {
    __shared__ float tile[64][65];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t u0 = (int64_t)(blockIdx.x % unit_tiles) * 64;
    const int32_t r0 = (int32_t)(blockIdx.x / unit_tiles) * 64;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = 4 * i + wave;
        if (r0 + r < B && u0 + lane < n) tile[r][lane] = x[(int64_t)(r0 + r) * n + u0 + lane];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int u = 4 * i + wave;
        if (r0 + lane < B && u0 + u < n) xt[(u0 + u) * stride + r0 + lane] = tile[lane][u];
    }
}

// A row's M columns from LDS, times `scale`, by 16 lanes (l is this one), 4 columns each at a time (global
// memory takes them at any alignment of a float).
__device__ __forceinline__ void store_row(float* __restrict__ out, const float* d, int M, int l, float scale) {
    for (int c = 4 * l; c < M; c += 64) {
        const mx_quad v = *reinterpret_cast<const mx_quad*>(d + c) * scale;
        if (c + 4 <= M) {
            __builtin_memcpy(out + c, &v, sizeof v);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (c + e < M) out[c + e] = v[e];
        }
    }
}

// A workgroup takes 32 rows and one hidden HCU.  Quantising: a wave takes every n_waves-th step of
// the chunk, a lane the block of its row and half, as the matrix instruction will read it, so the
// block's largest value needs no other lane.  Products: wave w takes column tile w % tiles (and
// w + n_waves) and, where there are more waves than tiles, its share of the groups; its first weights
// are requested before the inputs.
//
// kVec > 0: x is [B][n_in] and a lane reads its own row, kVec units at a time (a divisor of in_mcu):
// every lane another line.  kVec = 0: x is [n_in][stride], so a load covers the rows of two units, two
// whole lines.
template <int kTiles, int kVec>
__global__ void __launch_bounds__(1024)
forward_kernel(Geometry g, ForwardShape shape, const float* __restrict__ x, int32_t stride, int32_t B,
               const uint8_t* __restrict__ codes, const uint32_t* __restrict__ scales,
               const float* __restrict__ bias, ActiveUnits act, float gain, float* __restrict__ y,
               float* __restrict__ s, int32_t* __restrict__ winner) {
    extern __shared__ __align__(16) uint8_t lds[];
    mx_codes* la = reinterpret_cast<mx_codes*>(lds);                       // [step][lane]
    uint8_t* lsa = lds + shape.steps * kMxStepCodes;                       // [group][lane][step]
    const int tid = threadIdx.x, lane = tid & 63, n_waves = shape.waves, chunk = shape.steps * kMxStep;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.x % g.out_hcu;
    const int64_t row0 = (int64_t)(blockIdx.x / g.out_hcu) * kMxRows;
    const int M = g.out_mcu, tiles = (M + 31) / 32;
    const int parts = shape.parts, part = parts > 1 ? wave / tiles : 0, tile0 = parts > 1 ? wave % tiles : wave;
    const int kg = act.kg, k_total = act.count[h];
    const int half = lane >> 5;
    // x as this workgroup's base, the same for all lanes, and 32-bit offsets in bytes: a lane's row
    // (past the last row: that one) and a unit
    const char* base = reinterpret_cast<const char*>(x + mx_input_base(kVec == 0, row0, g.n_in));
    const InputSteps in = mx_input_steps(kVec == 0, g.n_in, stride);
    const uint32_t my_row = mx_live_row(lane & 31, B - row0) * in.row;
    const int32_t* units = act.units + (int64_t)h * kg * kMxGroup;

    mx_acc acc[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = 0.0f;
    struct Weights { mx_codes c[4]; uint32_t s; };
    auto load_w = [&](Weights& w, int t, int grp) __attribute__((always_inline)) {
        const int64_t at = mx_weight_group(h, tiles, (int64_t)tile0 + t * n_waves, kg, grp);
        w.s = scales[at * 64 + lane];
#pragma unroll
        for (int st = 0; st < 4; ++st)
            w.c[st] = reinterpret_cast<const mx_codes*>(codes + at * kMxGroupCodes)[64 * st + lane];
    };
    const bool works = part < parts && tile0 < tiles;

    for (int k0 = 0; k0 < k_total; k0 += chunk) {
        const int live = min(chunk, k_total - k0);
        const int groups = (live + kMxGroup - 1) / kMxGroup;
        Weights first;                                       // of this wave's first group of the chunk
        if (kTiles == 1 && works && part < groups) load_w(first, 0, k0 / kMxGroup + part);
        if (k0 > 0) __syncthreads();                         // the last chunk's reads are done
        for (int st = wave; st < 4 * groups; st += n_waves) {
            const int at = st * kMxStep + 32 * half;
            float v[32];
            if (at < live) {
                constexpr int kStep = kVec ? kVec : 1;
                typedef float vec __attribute__((ext_vector_type(kStep)));
                const int32_t* u = units + k0 + st * kMxStep;    // (the wave's: scalar loads)
#pragma unroll
                for (int i = 0; i < 32; i += kStep) {
                    const uint32_t lo = (uint32_t)u[i] * in.unit, hi = (uint32_t)u[32 + i] * in.unit;
                    const vec q = *reinterpret_cast<const vec*>(base + ((half ? hi : lo) + my_row));
#pragma unroll
                    for (int e = 0; e < kStep; ++e) v[i + e] = q[e];
                }
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = at + i < live ? v[i] : 0.0f;
            uint32_t byte;
            la[st * 64 + lane] = mx_block(v, byte);
            lsa[(st >> 2) * kMxGroupScales + 4 * lane + (st & 3)] = (uint8_t)byte;
        }
        __syncthreads();
        if (!works) continue;
        for (int q = part; q < groups; q += parts) {
            const uint32_t sa = reinterpret_cast<const uint32_t*>(lsa)[q * 64 + lane];
            const mx_codes* ca = la + q * 256 + lane;
            auto block = [&](mx_acc& c, const Weights& w) __attribute__((always_inline)) {
                c = mx_mfma<0>(ca[0], w.c[0], c, sa, w.s);
                c = mx_mfma<1>(ca[64], w.c[1], c, sa, w.s);
                c = mx_mfma<2>(ca[128], w.c[2], c, sa, w.s);
                c = mx_mfma<3>(ca[192], w.c[3], c, sa, w.s);
            };
            if constexpr (kTiles == 1) {                     // (the next group's weights on their way)
                const Weights w = first;
                if (q + parts < groups) load_w(first, 0, k0 / kMxGroup + q + parts);
                block(acc[0], w);
            } else {
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
                    if (tile0 + t * n_waves < tiles) {
                        Weights w;
                        load_w(w, t, k0 / kMxGroup + q);
                        block(acc[t], w);
                    }
            }
        }
    }

    // supports to LDS, each part's sums in a place of their own (the first with the bias)
    float* sup = reinterpret_cast<float*>(lds);
    const int pitch = mx_support_pitch(M);
    __syncthreads();
    if (works) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int c = (tile0 + t * n_waves) * kMxRows + (lane & 31);
            if (c >= M) continue;
            const float b = part == 0 ? bias[(int64_t)h * M + c] : 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) sup[mx_support_at(part, mx_row(e, half), pitch, c)] = acc[t][e] + b;
        }
    }
    __syncthreads();
    // 16 lanes per row, 4 columns at a time: the parts in order, then the softmax or the argmax
    for (int r = tid >> 4; r < kMxRows; r += 4 * n_waves) {
        const int64_t row = row0 + r;
        if (row >= B) continue;                              // uniform over the 16 lanes
        const int l = tid & 15;
        float* d = sup + mx_support_at(0, r, pitch, 0);
        const int64_t o = row * g.n_out + (int64_t)h * M;
        float top = -INFINITY;                               // (a NaN takes no part)
        int at = 0x7fffffff;
        for (int c = 4 * l; c < M; c += 64) {
            mx_quad v = *reinterpret_cast<mx_quad*>(d + c);
            if (parts > 1) {
                for (int p = 1; p < parts; ++p) v += *reinterpret_cast<mx_quad*>(sup + mx_support_at(p, r, pitch, c));
                *reinterpret_cast<mx_quad*>(d + c) = v;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < M && v[e] > top) { top = v[e]; at = c + e; }
        }
        if (s) store_row(s + o, d, M, l, 1.0f);
        if (!winner) {
            const float mx = row16_max(top);
            float sum = 0.0f;
            for (int c = 4 * l; c < M; c += 64) {
                mx_quad v = *reinterpret_cast<mx_quad*>(d + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = expf(gain * (v[e] - mx));
                    if (c + e < M) sum += v[e];
                }
                *reinterpret_cast<mx_quad*>(d + c) = v;
            }
            const float inv = 1.0f / row16_sum(sum);
            store_row(y + o, d, M, l, inv);
        } else {
            for (int off = 8; off > 0; off >>= 1) {
                const float ov = __shfl_xor(top, off, 64);
                const int oi = __shfl_xor(at, off, 64);
                if (ov > top || (ov == top && oi < at)) { top = ov; at = oi; }
            }
            if (l == 0) winner[row * g.out_hcu + h] = at == 0x7fffffff ? 0 : at;
        }
    }
}

// Many rows of a layer whose inputs are few: a workgroup holds 16 rows of them in LDS, read once, and
// its waves take the hidden HCUs in turn, alone from the gather to the softmax: the block that a lane
// quantises is its operand of the matrix instruction (16 x 16 over 128 units, so that every lane has
// one), and the supports stay in registers, a row's in 16 lanes.
template <int kVec>
__global__ void __launch_bounds__(64 * kMxWaves)
forward_rows_kernel(Geometry g, const float* __restrict__ x, int32_t B, const uint8_t* __restrict__ codes,
                    const uint32_t* __restrict__ scales, const float* __restrict__ bias, ActiveUnits act, float gain,
                    float* __restrict__ y, float* __restrict__ s, int32_t* __restrict__ winner) {
    extern __shared__ __align__(16) uint8_t lds[];
    constexpr int kTiles = 8;                                // of 16 columns
    float* xs = reinterpret_cast<float*>(lds);
    const int tid = threadIdx.x, lane = tid & 63, c0 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row0 = (int64_t)blockIdx.x * kMxTileRows;
    const int rows = (int)min((int64_t)kMxTileRows, B - row0), n_in = (int)g.n_in;
    const int pitch = (int)mx_input_pitch(n_in), M = g.out_mcu, rbs = (M + 31) / 32;
    if (wave < rows) {                                       // a wave loads a row
        const float* src = x + (row0 + wave) * n_in;
        if (n_in % 4 == 0) {
            for (int c = 4 * lane; c < n_in; c += 256)
                *reinterpret_cast<mx_quad*>(xs + wave * pitch + c) = *reinterpret_cast<const mx_quad*>(src + c);
        } else {
            for (int c = lane; c < n_in; c += 64) xs[wave * pitch + c] = src[c];
        }
    }
    __syncthreads();
    const float* mine = xs + (int)mx_live_row(c0, rows) * pitch;
    for (int h = wave; h < g.out_hcu; h += kMxWaves) {
        const int k_total = act.count[h], kg = act.kg;
        const int32_t* units = act.units + (int64_t)h * kg * kMxGroup;
        mx_acc16 acc[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) acc[t] = mx_acc16{0.0f, 0.0f, 0.0f, 0.0f};
        for (int k0 = 0; k0 < k_total; k0 += 128) {
            const int step = mx_rows_step(k0, quarter);
            mx_codes w[kTiles];
            uint32_t ws[kTiles];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const int64_t at = mx_weight_group(h, rbs, mx_rows_block(t, rbs), kg, k0 / kMxGroup);
                const int l = mx_rows_lane(c0, quarter, t);
                w[t] = reinterpret_cast<const mx_codes*>(codes + at * kMxGroupCodes)[64 * step + l];
                ws[t] = scales[at * 64 + l] >> (8 * step);
            }
            const int at = k0 + 32 * quarter;
            typedef float vec __attribute__((ext_vector_type(kVec)));
            const int4* u = reinterpret_cast<const int4*>(units + at);
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                const int4 q4 = u[i / 4];
                const int q[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
                for (int j = 0; j < 4; j += kVec) {
                    const vec r = *reinterpret_cast<const vec*>(mine + q[j]);
#pragma unroll
                    for (int e = 0; e < kVec; ++e) v[i + j + e] = at + i + j + e < k_total ? r[e] : 0.0f;
                }
            }
            uint32_t byte;
            const mx_codes a = mx_block(v, byte);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) acc[t] = mx_mfma16(a, w[t], acc[t], byte, ws[t]);
        }
        // a lane has rows 4 quarter + e of columns 16 t + c0
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
            if (16 * t + c0 < M) {
                const float b = bias[(int64_t)h * M + 16 * t + c0];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][e] += b;
            }
        const int64_t o = (row0 + 4 * quarter) * g.n_out + (int64_t)h * M + c0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool live = 4 * quarter + e < rows;
            float top = -INFINITY;                           // (a NaN takes no part)
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
                if (16 * t + c0 < M) {
                    top = fmaxf(top, acc[t][e]);
                    if (s && live) s[o + e * g.n_out + 16 * t] = acc[t][e];
                }
            top = row16_max(top);
            if (!winner) {
                float sum = 0.0f;
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
                    if (16 * t + c0 < M) {
                        acc[t][e] = expf(gain * (acc[t][e] - top));
                        sum += acc[t][e];
                    }
                const float inv = 1.0f / row16_sum(sum);
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
                    if (live && 16 * t + c0 < M) y[o + e * g.n_out + 16 * t] = acc[t][e] * inv;
            } else {
                int at = 0x7fffffff;                         // the first of the largest
#pragma unroll
                for (int t = kTiles - 1; t >= 0; --t)
                    if (16 * t + c0 < M && acc[t][e] == top && top > -INFINITY) at = 16 * t + c0;
                for (int off = 8; off > 0; off >>= 1) at = min(at, __shfl_xor(at, off, 64));
                if (live && c0 == 0)
                    winner[(row0 + 4 * quarter + e) * g.out_hcu + h] = at == 0x7fffffff ? 0 : at;
            }
        }
    }
}

}  // namespace

hipError_t launch_mx_units(hipStream_t stream, const Geometry& g, const ActiveLists& lists, const ActiveUnits& act) {
    units_kernel<<<dim3((uint32_t)(g.out_hcu * act.kg)), kMxGroup, 0, stream>>>(g, lists, (uint32_t)act.kg, act.units,
                                                                               act.count);
    return hipGetLastError();
}

hipError_t launch_mx_pack(hipStream_t stream, const Geometry& g, const float* w, const ActiveUnits& act, void* codes,
                          void* scales) {
    const uint32_t rbs = (uint32_t)mx_row_blocks(g.out_mcu);
    pack_kernel<<<dim3((uint32_t)(g.out_hcu * rbs * act.kg)), 256, 0, stream>>>(g, w, act, rbs, (uint8_t*)codes,
                                                                               (uint8_t*)scales);
    return hipGetLastError();
}

namespace {

using ForwardKernel = void (*)(Geometry, ForwardShape, const float*, int32_t, int32_t, const uint8_t*,
                               const uint32_t*, const float*, ActiveUnits, float, float*, float*, int32_t*);

// By tiles per wave (1, 2) and kVec (0, 1, 2, 4).
ForwardKernel forward_for(int tiles, int vec) {
    static const ForwardKernel table[2][4] = {
        {forward_kernel<1, 0>, forward_kernel<1, 1>, forward_kernel<1, 2>, forward_kernel<1, 4>},
        {forward_kernel<2, 0>, forward_kernel<2, 1>, forward_kernel<2, 2>, forward_kernel<2, 4>}};
    return table[tiles - 1][vec == 4 ? 3 : vec];
}

// Whether B rows are transposed first.  A round of a workgroup per CU gathers k units of up to 32 rows
// directly in what its loads cost or, where each meets another line, its lines (2700 and 1230 rows of
// them per us); transposing takes a launch, 8 bytes per input value and then reads whole lines.
// Measured, directly / transposed (us): STL shape, 8 rows 18.7 / 20.4, 16 rows 26.6 / 20.8, 256 rows 229
// / 73; MNIST shape, 2048 rows 34.7 / 36.7, 8192 rows 109 / 103; 4000 -> 10 x 1000 units, 128 rows 44.6 /
// 37.7; 3000 -> 10 units, 128 rows 13.0 / 16.9.
bool transposes(const Geometry& g, int64_t k, int64_t B, int vec) {
    const double rounds = (double)((mx_row_blocks(B) * g.out_hcu + 255) / 256);
    const double loads = (double)k / vec, lines = std::min(loads, g.n_in / 32.0);
    const double direct = rounds * std::min<int64_t>(B, kMxRows) * std::max(loads / 2700.0, lines / 1230.0);
    return direct > 4.0 + 8.0 * B * g.n_in / 5e6 + rounds * k * 0.0015;
}

}  // namespace

hipError_t mx_forward_prepare() {
    hipError_t e = hipSuccess;
    for (const void* kernel : {(const void*)forward_rows_kernel<1>, (const void*)forward_rows_kernel<2>,
                               (const void*)forward_rows_kernel<4>})
        if (e == hipSuccess)
            e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kMxRowsLds);
    for (int tiles : {1, 2})
        for (int vec : {0, 1, 2, 4})
            if (e == hipSuccess)
                e = hipFuncSetAttribute((const void*)forward_for(tiles, vec),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, kMxForwardLds);
    return e;
}

namespace {

// Rows that one launch of each kernel takes (mx_launch_rows).
hipError_t forward_part(hipStream_t stream, const Geometry& g, const float* x, int32_t B, const void* codes,
                        const void* scales, const float* bias, const ActiveUnits& act, float gain, float* turned,
                        int64_t turned_rows, float* y, float* s, int32_t* winner) {
    const int vec = mx_gather_width(g.in_mcu);
    if (mx_rows_in_lds(g, B)) {
        auto* kernel = vec == 4   ? &forward_rows_kernel<4>
                       : vec == 2 ? &forward_rows_kernel<2>
                                  : &forward_rows_kernel<1>;
        kernel<<<dim3((uint32_t)((B + kMxTileRows - 1) / kMxTileRows)), 64 * kMxWaves,
                 kMxTileRows * mx_input_pitch(g.n_in) * 4, stream>>>(g, x, B, (const uint8_t*)codes,
                                                                    (const uint32_t*)scales, bias, act, gain, y, s,
                                                                    winner);
        return hipGetLastError();
    }
    const bool turn = turned_rows > 0 && transposes(g, act.most, std::min<int64_t>(B, turned_rows), vec);
    const int64_t rows = turn ? turned_rows : B;
    for (int64_t r = 0; r < B; r += rows) {
        const int32_t n = (int32_t)std::min<int64_t>(rows, B - r);
        const float* xr = x + r * g.n_in;
        if (turn) {
            const uint32_t unit_tiles = (uint32_t)((g.n_in + 63) / 64);
            transpose_kernel<<<dim3(unit_tiles * (uint32_t)((n + 63) / 64)), 256, 0, stream>>>(
                xr, n, g.n_in, unit_tiles, turned, (int32_t)turned_rows);
            xr = turned;
        }
        const dim3 grid((uint32_t)(mx_row_blocks(n) * g.out_hcu));
        const ForwardShape f = mx_forward_shape(g, act.kg, n);
        forward_for(f.tiles, turn ? 0 : vec)<<<grid, 64 * f.waves, mx_forward_lds(f, g.out_mcu), stream>>>(
            g, f, xr, (int32_t)turned_rows, n, (const uint8_t*)codes, (const uint32_t*)scales, bias, act, gain,
            y ? y + r * g.n_out : nullptr, s ? s + r * g.n_out : nullptr, winner ? winner + r * g.out_hcu : nullptr);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_mx_forward(hipStream_t stream, const Geometry& g, const float* x, int32_t B, const void* codes,
                             const void* scales, const float* bias, const ActiveUnits& act, float gain, float* turned,
                             int64_t turned_rows, float* y, float* s, int32_t* winner) {
    const int64_t most = mx_launch_rows(g);
    for (int64_t r = 0; r < B; r += most) {
        const hipError_t e = forward_part(stream, g, x + r * g.n_in, (int32_t)std::min<int64_t>(most, B - r), codes,
                                          scales, bias, act, gain, turned, turned_rows, y ? y + r * g.n_out : nullptr,
                                          s ? s + r * g.n_out : nullptr, winner ? winner + r * g.out_hcu : nullptr);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace bcpnn
