// Product of two MX operands: C = alpha A B^T + beta C + bias, A [M][K], B [N][K] (mx_format.h).
#include <algorithm>
#include <type_traits>

#include "bcpnn_internal.h"
#include "device_common.h"
#include "mx_format.h"

namespace bcpnn {
namespace {

template <typename T>
struct Epilogue {
    float alpha, beta;
    const float* bias;
    T* c;
    int64_t ld, m, n;

    __device__ __forceinline__ float bias_at(int64_t col) const { return bias && col < n ? bias[col] : 0.0f; }
    __device__ __forceinline__ void store(int64_t row, int64_t col, float acc, float b) const {
        if (row >= m || col >= n) return;
        float v = fmaf(alpha, acc, b);
        T* p = c + row * ld + col;
        if (beta != 0.0f) v = fmaf(beta, (float)*p, v);
        *p = (T)v;
    }
    // Four columns with their biases (global memory takes them at any alignment of the elements).
    __device__ __forceinline__ void store4(int64_t row, int64_t col, mx_quad acc, mx_quad b) const {
        if (col + 4 > n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) store(row, col + j, acc[j], b[j]);
            return;
        }
        if (row >= m) return;
        T* p = c + row * ld + col;
        T o[4];
        if (beta != 0.0f) __builtin_memcpy(o, p, sizeof o);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v = fmaf(alpha, acc[j], b[j]);
            if (beta != 0.0f) v = fmaf(beta, (float)o[j], v);
            o[j] = (T)v;
        }
        __builtin_memcpy(p, o, sizeof o);
    }
};

typedef void __attribute__((address_space(3))) lds_void;

// Shape of a tile: kWM x kWN waves of kTM x kTN blocks of 32 x 32.
template <int kWM_, int kWN_, int kTM_, int kTN_>
struct Tile {
    static constexpr int kWM = kWM_, kWN = kWN_, kTM = kTM_, kTN = kTN_;
    static constexpr int kM = kWM * kTM, kN = kWN * kTN;     // row blocks of A and of B
    static constexpr int kWaves = kWM * kWN, kThreads = 64 * kWaves;
    static constexpr int kPer = (kM + kN) / kWaves;          // row blocks that a wave loads
    static_assert((kM + kN) % kWaves == 0, "whole row blocks per wave");
};

// Bound by the loads into LDS and the matrix instructions, which overlap in part only (below): 8192 x 8192 x
// 10000 takes 312 us with bf16 results (4.3 PFLOP/s; a loop of the instruction alone reaches 6.6), 355 with
// fp32.  With one tile per workgroup and bf16 results it took 329, without the loads 282, the matrix
// instructions alone 260, the loads alone 202 (29 bytes per cycle and CU).
// 2 x 4 waves of 4 x 2 blocks (128 accumulators a wave, two waves per SIMD) rather than 2 x 2 of 4 x 4:
// those read a third less LDS, but spill around the loop (377 us against 458 when first measured).
//
// Both operands go through LDS in halves of a group, 128 columns (global_load_lds: 1 KiB of codes or
// 256 bytes of scales per instruction, in the order the waves read them).  Four halves are held, in
// separate arrays, so that the reads of one do not wait for the loads into the others: one being
// multiplied and up to three on their way.  That is so at one barrier in four: ahead of the other three,
// of an odd last group's and of a tile's first the compiler waits for every load in flight
// (s_waitcnt vmcnt(0) beside the fence of LDS in its listing), so that three half steps in four wait for the
// loads that the one before requested.
template <typename T, typename S>
__global__ void __launch_bounds__(S::kThreads)
product_tile_kernel(MxOperand a, MxOperand b, uint32_t m_tiles, uint32_t n_tiles, int64_t m_blocks,
                    int64_t n_blocks, Epilogue<T> ep) {
    constexpr int kTM = S::kTM, kTN = S::kTN, kPer = S::kPer, kSlots = S::kM + S::kN, kHalf = kMxGroupCodes / 2;
    __shared__ __align__(16) uint8_t half0[kSlots * kHalf];
    __shared__ __align__(16) uint8_t half1[kSlots * kHalf];
    __shared__ __align__(16) uint8_t half2[kSlots * kHalf];
    __shared__ __align__(16) uint8_t half3[kSlots * kHalf];
    __shared__ __align__(16) uint8_t scales0[kSlots * kMxGroupScales];
    __shared__ __align__(16) uint8_t scales1[kSlots * kMxGroupScales];
    uint8_t* const ring[4] = {half0, half1, half2, half3};
    uint8_t* const ring_scales[2] = {scales0, scales1};
    constexpr int kCols = 32 * kTN, kStride = kCols + 8, kLanes = kCols / 4;
    __shared__ __align__(16) float turn[S::kWaves][8 * kStride];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t kg = a.kg, tiles = (int64_t)m_tiles * n_tiles;
    // First blocks of a tile's rows and columns.  Neighbouring tiles share an XCD's L2: each takes a run
    // of tiles, in strips of kStrip tile rows.
    auto blocks_of = [&](int64_t tile, int64_t& mb, int64_t& nb) __attribute__((always_inline)) {
        constexpr uint32_t kStrip = 8;
        const uint32_t id = (uint32_t)xcd_linear_index(tile, tiles);
        const uint32_t strip = id / (kStrip * n_tiles), high = min(kStrip, m_tiles - strip * kStrip);
        const uint32_t in_strip = id - strip * kStrip * n_tiles;
        mb = S::kM * (int64_t)(strip * kStrip + in_strip % high);
        nb = S::kN * (int64_t)(in_strip / high);
    };
    // (addresses as a wave's base in scalar registers and a lane's 32-bit offset)
    const uint32_t lane4 = 4 * lane, lane16 = 16 * lane;
    const uint8_t *src[kPer], *scl[kPer];
    auto sources = [&](int64_t mb, int64_t nb) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int slot = wave * kPer + j;
            const MxOperand& o = slot < S::kM ? a : b;
            const int64_t block = slot < S::kM ? min(mb + slot, m_blocks - 1)
                                               : min(nb + slot - S::kM, n_blocks - 1);
            const int64_t at = block * kg;
            src[j] = o.codes + at * kMxGroupCodes;
            scl[j] = reinterpret_cast<const uint8_t*>(o.scales) + at * kMxGroupScales;
        }
    };
    // Half q % 2 of group g into the ring's place q, with the group's scales before its first half.
    auto request = [&](auto place, int64_t g) __attribute__((always_inline)) {
        constexpr int q = decltype(place)::value;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int slot = wave * kPer + j;
            if constexpr (q % 2 == 0)
                __builtin_amdgcn_global_load_lds(
                    (const void*)(scl[j] + g * kMxGroupScales + lane4),
                    (lds_void*)(ring_scales[q / 2] + slot * kMxGroupScales), 4, 0, 0);
#pragma unroll
            for (int st = 0; st < 2; ++st)
                __builtin_amdgcn_global_load_lds(
                    (const void*)(src[j] + g * kMxGroupCodes + (q % 2) * kHalf + 1024 * st + lane16),
                    (lds_void*)(ring[q] + slot * kHalf + 1024 * st), 16, 0, 0);
        }
    };
    const int ma = (wave / S::kWN) * kTM, na = (wave % S::kWN) * kTN;   // this wave's blocks of the tile
    auto read_scales = [&](const uint8_t* from, uint32_t (&x)[kTM], uint32_t (&y)[kTN])
                           __attribute__((always_inline)) {
        const uint32_t* sc = reinterpret_cast<const uint32_t*>(from) + lane;
#pragma unroll
        for (int j = 0; j < kTM; ++j) x[j] = sc[64 * (ma + j)];
#pragma unroll
        for (int j = 0; j < kTN; ++j) y[j] = sc[64 * (S::kM + na + j)];
    };
    mx_acc acc[kTM][kTN];
    auto read = [&](const uint8_t* half, int st, mx_codes (&ca)[kTM], mx_codes (&cb)[kTN])
                    __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kTM; ++j)
            ca[j] = reinterpret_cast<const mx_codes*>(half + (ma + j) * kHalf + 1024 * st)[lane];
#pragma unroll
        for (int j = 0; j < kTN; ++j)
            cb[j] = reinterpret_cast<const mx_codes*>(half + (S::kM + na + j) * kHalf + 1024 * st)[lane];
    };
    auto step = [&](auto st, const mx_codes (&ca)[kTM], const mx_codes (&cb)[kTN], const uint32_t (&x)[kTM],
                    const uint32_t (&y)[kTN]) __attribute__((always_inline)) {
        constexpr int kStep = decltype(st)::value;
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int j = 0; j < kTN; ++j) acc[i][j] = mx_mfma<kStep>(ca[i], cb[j], acc[i][j], x[i], y[j]);
        // the reads of the next step, and in a half's second step the loads of a later one, one by one
        // among the products (in a burst they hold the wave back: 8192 x 8192 x 10000 355 -> 332 us)
#pragma unroll
        for (int q = 0; q < kTM + kTN; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if constexpr (kStep % 2 == 1) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
    };
    // One half (two steps), the first of which the wave has read.  The barrier stands between the steps:
    // by then every wave has read the whole half, so its place can be filled again (with the same half of
    // the group after next), and the loads of the next half have arrived (those of the two after it need
    // not have: kLater; the compiler's own wait leaves them in flight at place 0 only), so its first step is
    // read under the products of this one's second.
    mx_codes ca[2][kTM], cb[2][kTN];
    uint32_t sa[2][kTM], sb[2][kTN];
    auto multiply = [&](auto place, int64_t g) __attribute__((always_inline)) {
        constexpr int q = decltype(place)::value, o = q / 2, first = 2 * (q % 2);
        constexpr int kLater = 5 * kPer;                     // loads of two halves, one with scales
        // (of a SIMD's two waves the one that is ahead goes first: 332 -> 322 us)
        __builtin_amdgcn_s_setprio(q & 1);
        read(ring[q], 1, ca[1], cb[1]);
        step(std::integral_constant<int, first>{}, ca[0], cb[0], sa[o], sb[o]);
        // s_waitcnt vmcnt(kLater), no wait on the other counters
        __builtin_amdgcn_s_waitcnt((kLater & 15) | ((kLater >> 4) << 14) | 0x0f70);
        lds_barrier();
        request(place, g);
        read(ring[(q + 1) % 4], 0, ca[0], cb[0]);
        if constexpr (q % 2 == 1) read_scales(ring_scales[1 - o], sa[1 - o], sb[1 - o]);
        step(std::integral_constant<int, first + 1>{}, ca[1], cb[1], sa[o], sb[o]);
    };
    constexpr std::integral_constant<int, 0> p0{};
    constexpr std::integral_constant<int, 1> p1{};
    constexpr std::integral_constant<int, 2> p2{};
    constexpr std::integral_constant<int, 3> p3{};
    const int64_t last = kg - 1, second = min((int64_t)1, last);
    auto request_first = [&]() __attribute__((always_inline)) {
        // (past the last group the last one again, rather than a branch)
        request(p0, 0);
        request(p1, 0);
        request(p2, second);
        request(p3, second);
    };
    // A workgroup takes a tile after another.  The next one's first halves are requested before this one's
    // results are turned around and stored (7 us of a 256 x 256 tile's 80 when all CUs store at once), and
    // arrive under that.  The stores themselves do not pass under the next tile's products: store4 may read C,
    // so that the compiler waits for all memory operations ahead of each of them, beta or not.
    int64_t mb, nb;
    blocks_of(blockIdx.x, mb, nb);
    if (kg > 0) {
        sources(mb, nb);
        request_first();
    }
    for (int64_t tile = blockIdx.x;;) {
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int j = 0; j < kTN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
        if (kg > 0) {
            __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0): the first halves are there
            lds_barrier();
            read(half0, 0, ca[0], cb[0]);
            read_scales(scales0, sa[0], sb[0]);
            for (int64_t g = 0; g + 1 < kg; g += 2) {
                const int64_t g2 = min(g + 2, last), g3 = min(g + 3, last);
                multiply(p0, g2);
                multiply(p1, g2);
                multiply(p2, g3);
                multiply(p3, g3);
            }
            if (kg & 1) {
                multiply(p0, last);
                multiply(p1, last);
            }
            __syncthreads();                                 // nothing is on its way into the ring, or read
        }
        const int64_t row0 = (mb + ma) * kMxRows, col = (nb + na) * kMxRows + 4 * (lane % kLanes);
        mx_quad bias;                                        // of the columns that this lane stores
#pragma unroll
        for (int j = 0; j < 4; ++j) bias[j] = ep.bias_at(col + j);
        tile += gridDim.x;
        const bool more = tile < tiles;
        if (more) {
            blocks_of(tile, mb, nb);
            if (kg > 0) {
                sources(mb, nb);
                request_first();
            }
        }
        // A lane holds single columns of many rows: each wave turns 8 rows at a time around in LDS of its
        // own, so that it stores 4 columns per lane, whole lines per row.  (Rows 4 apart lie 32 banks apart.)
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int j = 0; j < kTN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        turn[wave][(4 * (lane >> 5) + e) * kStride + 32 * j + (lane & 31)] = acc[i][j][4 * q + e];
                wave_lds_fence();
#pragma unroll
                for (int r0 = 0; r0 < 8; r0 += 64 / kLanes) {
                    const int r = r0 + lane / kLanes;
                    const float* from = &turn[wave][r * kStride + 4 * (lane % kLanes)];
                    ep.store4(row0 + 32 * i + 8 * q + r, col, *reinterpret_cast<const mx_quad*>(from), bias);
                }
                wave_lds_fence();
            }
        if (!more) break;
    }
}

template <typename S, typename T>
hipError_t product_tiles(hipStream_t stream, const MxOperand& a, const MxOperand& b, const Epilogue<T>& ep) {
    const int64_t mb = mx_row_blocks(ep.m), nb = mx_row_blocks(ep.n);
    const int64_t mt = (mb + S::kM - 1) / S::kM, nt = (nb + S::kN - 1) / S::kN;
    // the large tiles one per CU, each workgroup several of them; the others, of which a CU holds several,
    // one per workgroup
    int64_t wgs = mt * nt;
    if (S::kM == 8) {
        int dev = 0, cus = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
        if (e != hipSuccess) return e;
        wgs = std::min<int64_t>(wgs, std::max(8, cus / 8 * 8));   // (whole rounds of XCDs: a run each)
    }
    product_tile_kernel<T, S><<<dim3((uint32_t)wgs), S::kThreads, 0, stream>>>(a, b, (uint32_t)mt, (uint32_t)nt,
                                                                                    mb, nb, ep);
    return hipGetLastError();
}

// Few rows of A: the weights' bytes bound it (1 x 10000 x 55296: 58 us, 5.0 TB/s; 315 by tiles), so a
// workgroup streams one row block of B straight into registers, a group per wave at a time and the next
// one in flight, against kM row blocks of A (rows past the last are not read).  The waves take the
// groups in turn, and where the row blocks of B are too few to fill the chip, `splits` workgroups share
// them (blockIdx.z); the sums are added in a fixed order, the waves' through LDS, the splits' through
// `parts` by finish_kernel.
template <typename T, int kM, int kWaves>
__global__ void __launch_bounds__(64 * kWaves)
product_rows_kernel(MxOperand a, MxOperand b, int64_t groups, Epilogue<T> ep, float* __restrict__ parts) {
    __shared__ float sums[kWaves][1024];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t nb = blockIdx.x, mb = (int64_t)blockIdx.y * kM;
    const int64_t m_live = ep.m - mb * kMxRows;              // rows from this workgroup's first on
    const int64_t g_end = min(a.kg, (int64_t)(blockIdx.z + 1) * groups);
    int64_t g = (int64_t)blockIdx.z * groups + wave;
    struct Group { mx_codes c[4]; uint32_t s; };
    auto load_b = [&](Group& r, int64_t at) __attribute__((always_inline)) {
        const int64_t bt = nb * b.kg + at;
        r.s = b.scales[bt * 64 + lane];
#pragma unroll
        for (int st = 0; st < 4; ++st)
            r.c[st] = reinterpret_cast<const mx_codes*>(b.codes + bt * kMxGroupCodes)[64 * st + lane];
    };
    auto load_a = [&](Group& r, int i, int64_t at) __attribute__((always_inline)) {
        r.s = 0;
#pragma unroll
        for (int st = 0; st < 4; ++st) r.c[st] = mx_codes{0, 0, 0, 0};
        if (i * kMxRows + (lane & 31) < m_live) {
            const int64_t ar = (mb + i) * a.kg + at;
            r.s = a.scales[ar * 64 + lane];
#pragma unroll
            for (int st = 0; st < 4; ++st)
                r.c[st] = reinterpret_cast<const mx_codes*>(a.codes + ar * kMxGroupCodes)[64 * st + lane];
        }
    };
    mx_acc acc[kM];
#pragma unroll
    for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
    auto block = [&](mx_acc& c, const Group& x, const Group& y) __attribute__((always_inline)) {
        c = mx_mfma<0>(x.c[0], y.c[0], c, x.s, y.s);
        c = mx_mfma<1>(x.c[1], y.c[1], c, x.s, y.s);
        c = mx_mfma<2>(x.c[2], y.c[2], c, x.s, y.s);
        c = mx_mfma<3>(x.c[3], y.c[3], c, x.s, y.s);
    };
    // (one block of A is requested with its B; more of them, which come from the caches, when needed)
    struct Pair { Group b, a; };
    auto load = [&](Pair& r, int64_t at) __attribute__((always_inline)) {
        load_b(r.b, at);
        if constexpr (kM == 1) load_a(r.a, 0, at);
    };
    auto multiply = [&](const Pair& r, int64_t at) __attribute__((always_inline)) {
        if constexpr (kM == 1) {
            block(acc[0], r.a, r.b);
        } else {
#pragma unroll
            for (int i = 0; i < kM; ++i) {
                Group x;
                load_a(x, i, at);
                block(acc[i], x, r.b);
            }
        }
    };
    if (g < g_end) {
        Pair r0, r1;
        load(r0, g);
        while (true) {
            if (g + kWaves >= g_end) { multiply(r0, g); break; }
            load(r1, g + kWaves);
            multiply(r0, g);
            g += 2 * kWaves;
            if (g >= g_end) { multiply(r1, g - kWaves); break; }
            load(r0, g);
            multiply(r1, g - kWaves);
        }
    }
#pragma unroll
    for (int i = 0; i < kM; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (i * kMxRows + mx_row(e, 0) < m_live) sums[wave][64 * e + lane] = acc[i][e];
        __syncthreads();
#pragma unroll
        for (int e0 = 0; e0 < 16; e0 += kWaves) {
            const int e = e0 + wave;
            const int64_t row = (mb + i) * kMxRows + mx_row(e, lane >> 5), col = nb * kMxRows + (lane & 31);
            if (row >= ep.m || col >= ep.n) continue;
            float v = sums[0][64 * e + lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v += sums[w][64 * e + lane];
            if (parts)
                parts[((int64_t)blockIdx.z * ep.m + row) * ep.n + col] = v;
            else
                ep.store(row, col, v, ep.bias_at(col));
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
finish_kernel(const float* __restrict__ parts, int splits, Epilogue<T> ep) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = ep.m * ep.n;
    if (i >= n) return;
    float v = parts[i];
    for (int s = 1; s < splits; ++s) v += parts[s * n + i];
    ep.store(i / ep.n, i % ep.n, v, ep.bias_at(i % ep.n));
}

// How a product is laid out.
struct Plan {
    int tile;                        // row blocks of a tile's side, 0: product_rows
    int waves, m_blocks, splits;     // of product_rows
    int64_t groups;                  // per split
};

// Measured (us, tiles of 256 / 128 / 64 rows, product_rows; n tiles of each):
//   3000 x 3000 x 3000    30.9 / 35.0 / 35.7 / 79    (144 / 576 / 2209): the widest tile that gives half
//   512 x 10000 x 3000    28.0 / 20.3 / 22.9 / 47    (80 / 316 / 1256)   of the CUs work
//   2048 x 2048 x 2048    22.4 / 13.9 / 12.9 / 31    (64 / 256 / 1024): two of the second kind per CU
//   256 x 3000 x 1568     20.5 / 10.9 / 6.2 / 6.1    (12 / 48 / 188)
//   512 x 1024 x 4096     28.5 / 14.5 / 8.7 / 5.4    (8 / 32 / 128): below that the columns are shared out
// Up to 128 rows the bytes of B are most of the work, and a tile's chain of groups is longer:
//   128 x 10000 x 10000   - / 37.8 / 29.0 / 24.3;  128 x 10000 x 3000   - / 13.4 / 9.1 / 12.6
Plan plan(int64_t m, int64_t n, int64_t k) {
    const int64_t mb = mx_row_blocks(m), nb = mx_row_blocks(n), kg = mx_groups(k);
    Plan p{0, 4, 1, 1, kg};
    auto tiles = [&](int64_t t) { return ((mb + t - 1) / t) * ((nb + t - 1) / t); };
    if ((mb > 4 || (mb > 2 && kg <= 16)) && tiles(2) >= 192) {
        p.tile = tiles(8) >= 128 ? 8 : tiles(4) >= 300 ? 4 : 2;
        return p;
    }
    // two row blocks of A per workgroup where B's alone fill the chip (four: 128 x 10000 x 10000 28.2 us
    // against 24.3)
    if (mb > 1 && nb * ((mb + 1) / 2) >= 256) p.m_blocks = 2;
    p.waves = kg < 16 ? 4 : p.m_blocks == 1 ? 16 : 8;
    const int64_t wgs = std::max<int64_t>(1, nb * ((mb + p.m_blocks - 1) / p.m_blocks));
    // as many splits as fill the chip, each wave keeping two groups (1 x 1000 x 55296: four groups 9.6 us,
    // two 8.0, one 7.8; 128 x 128 x 50000: 8.7, 7.8, 8.9)
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({256 / wgs, kg / (2 * p.waves), 64}));
    p.groups = (kg + p.splits - 1) / p.splits;
    return p;
}

template <typename T, int kM, int kWaves>
hipError_t product_rows(hipStream_t stream, const MxOperand& a, const MxOperand& b, const Plan& p,
                        const Epilogue<T>& ep, float* work) {
    const int64_t mb = mx_row_blocks(ep.m), nb = mx_row_blocks(ep.n);
    const dim3 grid((uint32_t)nb, (uint32_t)((mb + kM - 1) / kM), (uint32_t)p.splits);
    product_rows_kernel<T, kM, kWaves><<<grid, 64 * kWaves, 0, stream>>>(a, b, p.groups, ep,
                                                                        p.splits > 1 ? work : nullptr);
    if (p.splits > 1)
        finish_kernel<T><<<dim3((uint32_t)((ep.m * ep.n + 255) / 256)), 256, 0, stream>>>(work, p.splits, ep);
    return hipGetLastError();
}

template <typename T>
hipError_t product(hipStream_t stream, const MxOperand& a, const MxOperand& b, int64_t k, const Epilogue<T>& ep,
                   float* work) {
    const Plan p = plan(ep.m, ep.n, k);
    switch (p.tile) {
        case 8: return product_tiles<Tile<2, 4, 4, 2>>(stream, a, b, ep);
        case 4: return product_tiles<Tile<2, 2, 2, 2>>(stream, a, b, ep);
        case 2: return product_tiles<Tile<2, 2, 1, 1>>(stream, a, b, ep);
    }
    if (p.waves > 4) {
        if (p.m_blocks == 1) return product_rows<T, 1, 16>(stream, a, b, p, ep, work);
        return product_rows<T, 2, 8>(stream, a, b, p, ep, work);
    }
    if (p.m_blocks == 1) return product_rows<T, 1, 4>(stream, a, b, p, ep, work);
    return product_rows<T, 2, 4>(stream, a, b, p, ep, work);
}

}  // namespace

hipError_t launch_mx_product(hipStream_t stream, const void* a, const void* b, int64_t m, int64_t n, int64_t k,
                             float alpha, float beta, const float* bias, void* c, int32_t dtype, int64_t ld,
                             void* work) {
    const MxOperand ao = mx_operand(a, m, k), bo = mx_operand(b, n, k);
    float* w = static_cast<float*>(work);
    switch (dtype) {
        case BCPNN_F16:
            return product(stream, ao, bo, k, Epilogue<_Float16>{alpha, beta, bias, (_Float16*)c, ld, m, n}, w);
        case BCPNN_BF16:
            return product(stream, ao, bo, k, Epilogue<__bf16>{alpha, beta, bias, (__bf16*)c, ld, m, n}, w);
        default:
            return product(stream, ao, bo, k, Epilogue<float>{alpha, beta, bias, (float*)c, ld, m, n}, w);
    }
}

int64_t mx_product_work_items(int64_t m, int64_t n, int64_t k) {
    const Plan p = plan(m, n, k);
    const int64_t mb = mx_row_blocks(m), nb = mx_row_blocks(n);
    if (p.tile) return ((mb + p.tile - 1) / p.tile) * ((nb + p.tile - 1) / p.tile) * (p.tile == 8 ? 512 : 256);
    const int64_t rows = nb * ((mb + p.m_blocks - 1) / p.m_blocks) * p.splits * p.waves * 64;
    return p.splits > 1 ? std::max(rows, m * n) : rows;
}

int64_t mx_product_work_bytes(int64_t m, int64_t n, int64_t k) {
    const Plan p = plan(m, n, k);
    return p.tile || p.splits == 1 ? 0 : (int64_t)sizeof(float) * p.splits * m * n;
}

}  // namespace bcpnn
