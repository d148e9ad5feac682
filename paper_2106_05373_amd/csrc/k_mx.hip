// Quantisation of matrices to the MX layout (mx_format.h) and reading them back.
//
// Per block of 32 values v: s = max(floor(log2 max|v|) - 2, -126), code = RNE(v / 2^s) among the 4-bit
// values, saturating.  Both are bound by memory, 4 + 17 / 32 bytes per fp32 value: 8192 x 10000 by row 71 us, by
// column 71, both ways from one read 81 (5.1 TB/s; 304 when the values went through LDS).
#include <algorithm>

#include "bcpnn_internal.h"
#include "device_common.h"
#include "mx_format.h"

namespace bcpnn {
namespace {

// Values col .. col + 3 of a row of `cols`, zero past its end: one load (global memory takes it at any
// alignment of the elements).
template <typename T>
__device__ __forceinline__ void load4(const T* __restrict__ row, int64_t col, int64_t cols, float (&v)[4]) {
    if (col + 4 <= cols) {
        T r[4];
        __builtin_memcpy(r, row + col, sizeof r);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)r[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = col + i < cols ? (float)row[col + i] : 0.0f;
    }
}

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, kCtrl, 0xf, 0xf, false));
}
// Largest of the 8 lanes of each eighth of a wave: pairs, quads, then the mirrored quad.
__device__ __forceinline__ uint32_t max_of_8(uint32_t v) {
    return dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v)));
}

constexpr int kThreads = 256;

// A workgroup takes 32 rows x 256 columns, one group of a row block of the by-row operand and one
// block of 256 rows of the by-column one, so that rows are read and codes written as whole lines.  A
// wave reads 8 rows, 4 columns per lane.  By row (kRows) the 8 lanes of a block find its largest value
// and the codes are turned around in LDS.  By column (kCols) a lane has 8 of the 32 values of its 4
// columns: their largest goes through LDS to the other waves, then their 8 codes, one word.
template <typename T, bool kRows, bool kCols>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const T* __restrict__ src, int64_t rows, int64_t cols, int64_t ld, uint32_t slabs,
                uint8_t* __restrict__ row_codes, uint32_t* __restrict__ row_scales, uint32_t row_kg,
                uint8_t* __restrict__ col_codes, uint8_t* __restrict__ col_scales, uint32_t col_kg) {
    __shared__ __align__(16) uint8_t lc[kRows ? kMxGroupCodes : 16];
    __shared__ __align__(16) uint8_t ls[kRows ? kMxGroupScales : 16];
    __shared__ __align__(16) mx_codes tops[4][kCols ? 64 : 1];
    __shared__ __align__(16) mx_codes words[4][kCols ? 64 : 1];
    __shared__ uint32_t bytes[kCols ? 64 : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // the slabs of one group of columns in turn, on one XCD: the scales that they write share lines
    const uint32_t id = (uint32_t)xcd_linear_index(blockIdx.x, gridDim.x);
    const int64_t g = id / slabs, slab = id % slabs;
    const int64_t col = g * kMxGroup + 4 * lane;
    float v[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = slab * kMxRows + 8 * wave + i;
        if (row < rows) {
            load4(src + row * ld, col, cols, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = 0.0f;
        }
    }
    if constexpr (kCols) {
        mx_codes top;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t t = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) t = max(t, mx_magnitude(v[i][j]));
            top[j] = (int)t;
        }
        tops[wave][lane] = top;
    }
    if constexpr (kRows) {
        const int step = lane >> 4, half = (lane >> 3) & 1, part = lane & 7;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t top = max(max(mx_magnitude(v[i][0]), mx_magnitude(v[i][1])),
                               max(mx_magnitude(v[i][2]), mx_magnitude(v[i][3])));
            const uint32_t byte = mx_scale_byte(max_of_8(top));
            const float s = mx_scale(byte);
            const uint32_t c = mx_pack<1>(mx_pack<0>(0u, v[i][0], v[i][1], s), v[i][2], v[i][3], s);
            const int l = 32 * half + 8 * wave + i;
            *reinterpret_cast<uint16_t*>(lc + 1024 * step + 16 * l + 2 * part) = (uint16_t)c;
            if (part == 0) ls[4 * l + step] = (uint8_t)byte;
        }
    }
    __syncthreads();
    if constexpr (kRows) {
        if (slab < mx_row_blocks(rows)) {
            const int64_t at = slab * row_kg + g;
            reinterpret_cast<mx_codes*>(row_codes + at * kMxGroupCodes)[tid] =
                reinterpret_cast<const mx_codes*>(lc)[tid];
            if (tid < 64) row_scales[at * 64 + tid] = reinterpret_cast<const uint32_t*>(ls)[tid];
        }
    }
    if constexpr (kCols) {
        mx_codes word;
        uint32_t all = 0;
        const mx_codes t0 = tops[0][lane], t1 = tops[1][lane], t2 = tops[2][lane], t3 = tops[3][lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t byte = mx_scale_byte((uint32_t)max(max(t0[j], t1[j]), max(t2[j], t3[j])));
            const float s = mx_scale(byte);
            uint32_t w = mx_pack<0>(0u, v[0][j], v[1][j], s);
            w = mx_pack<1>(w, v[2][j], v[3][j], s);
            w = mx_pack<2>(w, v[4][j], v[5][j], s);
            word[j] = (int)mx_pack<3>(w, v[6][j], v[7][j], s);
            all |= byte << (8 * j);
        }
        words[wave][lane] = word;
        if (wave == 0) bytes[lane] = all;
        __syncthreads();
        const int64_t crb = (g * kMxGroup + tid) / kMxRows;  // row block of the by-column operand
        if (crb < mx_row_blocks(cols)) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(words) + tid;
            const int step = (int)(slab >> 1) & 3, l = 32 * (int)(slab & 1) + (tid & 31);
            const int64_t at = crb * col_kg + slab / 8;
            reinterpret_cast<mx_codes*>(col_codes + at * kMxGroupCodes + 1024 * step)[l] =
                mx_codes{(int)w[0], (int)w[256], (int)w[512], (int)w[768]};
            col_scales[at * kMxGroupScales + 4 * l + step] = reinterpret_cast<const uint8_t*>(bytes)[tid];
        }
    }
}

// Outputs from here on are stored past the caches, which they would only turn over: 8192 x 10000 fp32 (328
// MB) 96 -> 62 us; 4096 x 10000 (164 MB) 31.9 and 31.6 us.
constexpr int64_t kStreamBytes = 128ll << 20;

// Back to numbers: a workgroup takes one group of a row block; a lane writes 16 bytes of a row, kC columns,
// so that a wave's store covers one or two rows of the group.  (Global memory takes
// it at any alignment of the elements: rows of 10001 bf16 values 41 us against 113 by elements.)
template <typename T>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(MxOperand m, int64_t rows, int64_t cols, T* __restrict__ dst, int64_t ld, bool stream) {
    constexpr int kC = 16 / sizeof(T), kLanes = kMxGroup / kC, kRowsPer = 64 / kLanes;
    __shared__ __align__(16) uint8_t lc[kMxGroupCodes];
    __shared__ __align__(16) uint8_t ls[kMxGroupScales];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t rb = blockIdx.x / m.kg, g = blockIdx.x % m.kg;
    reinterpret_cast<mx_codes*>(lc)[tid] =
        reinterpret_cast<const mx_codes*>(m.codes + (int64_t)blockIdx.x * kMxGroupCodes)[tid];
    if (tid < 64) reinterpret_cast<uint32_t*>(ls)[tid] = m.scales[(int64_t)blockIdx.x * 64 + tid];
    __syncthreads();
    auto scale = [&](int l, int step) __attribute__((always_inline)) {
        const uint32_t byte = ls[4 * l + step];
        return byte == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(byte ? byte << 23 : 0x00400000u);
    };
    const int c0 = kC * (lane % kLanes), step = c0 / kMxStep, half = c0 / 32 % 2;
    const int64_t col = g * kMxGroup + c0;
#pragma unroll
    for (int i = 0; i < 8; i += kRowsPer) {
        const int r = 8 * wave + i + lane / kLanes, l = 32 * half + r;
        const int64_t row = rb * kMxRows + r;
        const uint8_t* code = lc + 1024 * step + 16 * l + c0 % 32 / 2;
        const float s = scale(l, step);
        T v[kC];
#pragma unroll
        for (int j = 0; j < kC; j += 4) {
            const uint32_t c = *reinterpret_cast<const uint16_t*>(code + j / 2);
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
            const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
            v[j] = (T)(lo[0] * s);
            v[j + 1] = (T)(lo[1] * s);
            v[j + 2] = (T)(hi[0] * s);
            v[j + 3] = (T)(hi[1] * s);
        }
        if (row >= rows) continue;
        T* out = dst + row * ld + col;
        if (col + kC <= cols) {
            typedef int at_elements __attribute__((ext_vector_type(4), aligned(2)));
            at_elements words;
            __builtin_memcpy(&words, v, sizeof words);
            at_elements* p = reinterpret_cast<at_elements*>(out);
            if (stream) __builtin_nontemporal_store(words, p);
            else *p = words;
        } else {
#pragma unroll
            for (int j = 0; j < kC; ++j)
                if (col + j < cols) out[j] = v[j];
        }
    }
}

template <typename T>
hipError_t quantize(hipStream_t stream, const T* src, int64_t rows, int64_t cols, int64_t ld, void* by_row,
                    void* by_col) {
    const int64_t rrb = mx_row_blocks(rows), rkg = mx_groups(cols);
    const int64_t crb = mx_row_blocks(cols), ckg = mx_groups(rows);
    uint8_t* rc = static_cast<uint8_t*>(by_row);
    uint32_t* rs = reinterpret_cast<uint32_t*>(rc + rrb * rkg * kMxGroupCodes);
    uint8_t* cc = static_cast<uint8_t*>(by_col);
    uint8_t* cs = cc + crb * ckg * kMxGroupCodes;
    const uint32_t slabs = (uint32_t)(by_col ? 8 * ckg : rrb);
    auto launch = [&](auto* kernel) {
        kernel<<<dim3((uint32_t)(rkg * slabs)), kThreads, 0, stream>>>(src, rows, cols, ld, slabs, rc, rs,
                                                                      (uint32_t)rkg, cc, cs, (uint32_t)ckg);
        return hipGetLastError();
    };
    return !by_col  ? launch(quantize_kernel<T, true, false>)
           : by_row ? launch(quantize_kernel<T, true, true>)
                    : launch(quantize_kernel<T, false, true>);
}

template <typename T>
hipError_t dequantize(hipStream_t stream, const void* mx, int64_t rows, int64_t cols, T* dst, int64_t ld) {
    const MxOperand m = mx_operand(mx, rows, cols);
    const dim3 grid((uint32_t)(mx_row_blocks(rows) * m.kg));
    const bool past = rows * cols * (int64_t)sizeof(T) > kStreamBytes;
    dequantize_kernel<T><<<grid, kThreads, 0, stream>>>(m, rows, cols, dst, ld, past);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(hipStream_t stream, const void* src, int32_t dtype, int64_t rows, int64_t cols,
                              int64_t ld, void* by_row, void* by_col) {
    switch (dtype) {
        case BCPNN_F16: return quantize(stream, (const _Float16*)src, rows, cols, ld, by_row, by_col);
        case BCPNN_BF16: return quantize(stream, (const __bf16*)src, rows, cols, ld, by_row, by_col);
        default: return quantize(stream, (const float*)src, rows, cols, ld, by_row, by_col);
    }
}

hipError_t launch_mx_dequantize(hipStream_t stream, const void* mx, int64_t rows, int64_t cols, void* dst,
                                int32_t dtype, int64_t ld) {
    switch (dtype) {
        case BCPNN_F16: return dequantize(stream, mx, rows, cols, (_Float16*)dst, ld);
        case BCPNN_BF16: return dequantize(stream, mx, rows, cols, (__bf16*)dst, ld);
        default: return dequantize(stream, mx, rows, cols, (float*)dst, ld);
    }
}

int64_t mx_quantize_workgroups(int64_t rows, int64_t cols, bool by_col) {
    return mx_groups(cols) * (by_col ? 8 * mx_groups(rows) : mx_row_blocks(rows));
}

}  // namespace bcpnn
