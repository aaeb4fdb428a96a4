// MXFP4: rows of bf16 <-> 4-bit E2M1 codes with one E8M0 scale per 32 consecutive elements of a row.
//     amax = largest magnitude of the block (the 15 non-sign bits as an integer: NaN > Inf > finite)
//     s    = 255 (NaN) if amax is Inf or NaN, else max(exponent field of amax - 2, 0)
//     code = e2m1_rne(x * 2^(127 - s)), 6 at most in magnitude;  the code stands for its E2M1 value times 2^(s - 127)
// The factor is a power of two, so the product is exact (or so small that the code is 0 either way): the code is the
// E2M1 value nearest to x / 2^(s - 127), and no fp32 rounding can move an element over a border.
//
// Codes: row-major, two per byte, the even element in the low nibble.  Scales: in the order the block-scaled MMA wants them
// in tensor memory.  tcgen05.cp.32x128b.warpx4 writes 32 rows of 16 bytes into four columns; the MMA takes row r's scales
// of 128 consecutive k from lane r % 32, column r / 32.  So a tile of 128 rows x 128 k is 512 bytes, row r's four scales at
// (r % 32) * 16 + (r / 32) * 4, and the tiles of a row tile follow one another along k.
//
// What bounds both kernels is memory: 2 + 17/32 bytes per element.  A lane takes one block of 32 (64 bytes in flight per thread, 2048
// threads per SM; dequantising 16 bytes and, with 34 registers, 1536), four lanes a piece of 128 elements, whose four scales are one 4-byte store; the L2 puts the tiles together.  A
// warp's pieces run on over the rows' ends, or, with offsets, stay in one row, which finds its group itself.  16384 x 10240: 66 us,
// 6.4 TB/s, the rate of a copy; 16384 x 3840 26.4 us; 77 x 3840 1.6; 64 rows in 64 groups 2.2.  Warps that stay in one row without
// offsets too: 10927 x 128 4.2 us (now 1.7), 16384 x 1088 10.7 (7.7), 16384 x 1536 11.0 (10.0), the same from K = 3840 on.  Blocks of 128
// rows x 256 elements per CTA, which write whole scale tiles, were no faster on large matrices and slower on all others: 2.3 us on 77
// rows, 6.7 on the 64 groups, 15.2 on 4096 rows in 64 groups (8.0 now).  Both kernels load their block before they look for the row's
// group, whose search takes several dependent loads, and find it in 32 bits: both in turn, 16384 x 3840 54.3 -> 51.2 us, 1337 x 3840 7.2
// -> 6.3, 77 x 3840 3.25 -> 3.0; 4096 rows in 64 groups 8.7 -> 8.0.
//
#pragma once

#include "ptx.cuh"

namespace lynx {

constexpr int MX_TILE_ROWS = 128, MX_CHUNK_BYTES = 512;
constexpr int MX_WARPS = 4, MX_WARP_K = 1024;
constexpr uint32_t MX_ONE = 127, MX_NAN = 255;

// How the rows are cut into row tiles of 128.  offsets == nullptr: `groups` groups of `group_rows` rows each, every group
// starts a tile.  Else group g holds the rows [offsets[g], offsets[g + 1]) and starts at tile offsets[g] / 128 + g, which leaves
// room for the ceil(rows / 128) tiles of the groups before it, whatever their sizes, without a sum over them.
struct MxRows {
    int64_t M;
    const int32_t* offsets;
    int groups;
    int64_t group_rows;
};

__host__ __device__ inline int64_t mx_row_tiles(int64_t M, int groups, bool ragged) {
    if (ragged) return M / MX_TILE_ROWS + groups;
    return groups * ((M / groups + MX_TILE_ROWS - 1) / MX_TILE_ROWS);
}

__device__ __forceinline__ int64_t mx_clamp_row(int32_t v, int64_t M) { return v < 0 ? 0 : (v > M ? M : v); }

// The last of the groups with `starts(g)`, which holds for the first group (or is taken to) and up to some other: 32 candidates
// at a time.  Called by whole warps.
template <class F>
__device__ __forceinline__ int mx_last_group(int groups, int lane, F starts) {
    int g = 0, span = groups;  // it is one of g .. g + span - 1
    while (span > 1) {
        const int step = (span + 31) / 32, c = g + lane * step;
        const uint32_t votes = __ballot_sync(0xffffffffu, c < g + span && starts(c));
        const int hit = votes ? 31 - __clz(votes) : 0, left = span - hit * step;
        g += hit * step;
        span = left < step ? left : step;
    }
    return g;
}

// Row -> its row tile and its place there; false: it belongs to no group.  Called by whole warps.  (M <= 2^30, so 32 bits do.)
__device__ __forceinline__ bool mx_row_place(const MxRows& R, uint32_t row, int lane, uint32_t& tile, uint32_t& in_tile) {
    uint32_t in_group;
    if (R.offsets == nullptr) {
        const uint32_t per = (uint32_t)R.group_rows, g = per == (uint32_t)R.M ? 0 : row / per;
        in_group = row - g * per;
        tile = g * ((per + MX_TILE_ROWS - 1) / MX_TILE_ROWS);
    } else {
        auto first = [&](int g) { return (uint32_t)mx_clamp_row(R.offsets[g], R.M); };
        const int g = mx_last_group(R.groups, lane, [&](int c) { return first(c) <= row; });
        const uint32_t start = first(g);
        if (row < start || row >= first(g + 1)) return false;
        in_group = row - start;
        tile = start / MX_TILE_ROWS + g;
    }
    tile += in_group / MX_TILE_ROWS;
    in_tile = in_group % MX_TILE_ROWS;
    return true;
}

// eight fp32 -> eight E2M1 codes (round to nearest even, 6 at most), element i in bits 4 i
__device__ __forceinline__ uint32_t cvt_e2m1x8(const float (&v)[8]) {
    uint32_t d;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(d)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return d;
}

// One block of 32 bf16 (16 words) -> four words of codes; returns the scale byte.
__device__ __forceinline__ uint32_t mx_quantize_block(const uint32_t (&x)[16], uint32_t (&codes)[4]) {
    uint32_t m = x[0] & 0x7FFF7FFFu;
#pragma unroll
    for (int i = 1; i < 16; ++i) m = vmax_u16x2(m, x[i] & 0x7FFF7FFFu);
    const uint32_t amax = max(m & 0xFFFFu, m >> 16);
    const uint32_t e = amax >> 7;
    if (e == 255) {
#pragma unroll
        for (int i = 0; i < 4; ++i) codes[i] = 0;
        return MX_NAN;
    }
    const uint32_t s = e < 2 ? 0 : e - 2;
    const float f = __uint_as_float((254 - s) << 23);  // 2^(127 - s)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_lo_f(x[4 * i + j]) * f;
            v[2 * j + 1] = bf16_hi_f(x[4 * i + j]) * f;
        }
        codes[i] = cvt_e2m1x8(v);
    }
    return s;
}

// The block of a lane.  Without offsets four lanes take 128 elements of a row, and a warp eight such pieces in a row, over the rows'
// ends; with offsets a warp stays in one row, for whose group it searches together.
struct MxBlock {
    int64_t row, k;  // row >= M: none
};
__host__ __device__ inline int64_t mx_units(int64_t M, int64_t K, bool ragged) {  // warps
    return ragged ? M * ((K + MX_WARP_K - 1) / MX_WARP_K) : (M * ((K + 127) / 128) + 7) / 8;
}
// pieces: of a row, 128 elements without offsets and MX_WARP_K with them
__device__ __forceinline__ MxBlock mx_block(const MxRows& R, int pieces, int lane) {
    const int64_t warp = (int64_t)blockIdx.x * MX_WARPS + (threadIdx.x >> 5);
    const bool ragged = R.offsets != nullptr;
    const int64_t piece = ragged ? warp : warp * 8 + (lane >> 2);
    const int64_t row = warp >> 28 ? piece / pieces : (uint32_t)piece / (uint32_t)pieces, in_row = piece - row * pieces;
    return MxBlock{row, ragged ? in_row * MX_WARP_K + 32 * lane : in_row * 128 + 32 * (lane & 3)};
}
// Offset of its scale byte; false: the row is of no group.
__device__ __forceinline__ bool mx_scale_offset(const MxRows& R, int64_t K, const MxBlock& b, int lane, int64_t& offset) {
    uint32_t tile, in_tile;
    if (!mx_row_place(R, (uint32_t)b.row, lane, tile, in_tile)) return false;
    offset = ((int64_t)tile * ((K + 127) >> 7) + (b.k >> 7)) * MX_CHUNK_BYTES + (in_tile & 31) * 16 + (in_tile >> 5) * 4 + (lane & 3);
    return true;
}

__global__ void __launch_bounds__(MX_WARPS * 32)
quantize_mxfp4_kernel(const uint16_t* X, MxRows R, int64_t K, int64_t ldx, uint8_t* codes, uint8_t* scales, int pieces) {
    griddep_wait();
    // A dependent launch reads nothing of this kernel's before its own wait; what it may read before (weights, offsets) was there
    // before this kernel's wait ended.
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    const MxBlock p = mx_block(R, pieces, lane);
    const bool there = p.row < R.M && p.k < K;
    uint32_t x[16], c[4];
    if (there) {  // (before the row's group is known: its search takes several dependent loads)
        const uint16_t* src = X + p.row * ldx + p.k;
        ldg256_stream(src, *reinterpret_cast<uint32_t(*)[8]>(&x[0]));
        ldg256_stream(src + 16, *reinterpret_cast<uint32_t(*)[8]>(&x[8]));
    }
    int64_t scale;
    if (R.offsets != nullptr && p.row >= R.M) return;  // (the whole warp)
    if (!mx_scale_offset(R, K, p, lane, scale)) return;
    uint32_t s = MX_ONE;  // behind K: 1
    if (there) {
        s = mx_quantize_block(x, c);
        stg128(codes + p.row * (K / 2) + p.k / 2, c[0], c[1], c[2], c[3]);
    }
    s <<= 8 * (lane & 3);  // four lanes' bytes to a word: one row of a scale tile
    s |= __shfl_xor_sync(0xffffffffu, s, 1);
    s |= __shfl_xor_sync(0xffffffffu, s, 2);
    if ((lane & 3) == 0 && there) *reinterpret_cast<uint32_t*>(scales + scale) = s;
}

// Four codes (16 bits) -> four bf16 E2M1 values in two words.  The magnitudes' bf16 bytes are looked up by permutation.
__device__ __forceinline__ void mx_decode4(uint32_t c, uint32_t& w0, uint32_t& w1) {
    const uint32_t sel = c & 0x7777u;
    const uint32_t hi = prmt(0x3F3F3F00u, 0x40404040u, sel);  // 0, .5, 1, 1.5 | 2, 3, 4, 6
    const uint32_t lo = prmt(0xC0800000u, 0xC0804000u, sel);
    w0 = prmt(lo, hi, 0x5140) | (c & 0x8u) << 12 | (c & 0x80u) << 24;
    w1 = prmt(lo, hi, 0x7362) | (c & 0x800u) << 4 | (c & 0x8000u) << 16;
}

__global__ void __launch_bounds__(MX_WARPS * 32)
dequantize_mxfp4_kernel(const uint8_t* codes, const uint8_t* scales, MxRows R, int64_t K, uint16_t* X, int64_t ldx, int pieces) {
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const MxBlock p = mx_block(R, pieces, lane);
    if (p.row >= R.M) return;
    uint4 c = make_uint4(0, 0, 0, 0);
    if (p.k < K) c = *reinterpret_cast<const uint4*>(codes + p.row * (K / 2) + p.k / 2);
    int64_t scale;
    if (!mx_scale_offset(R, K, p, lane, scale) || p.k >= K) return;
    const uint32_t s = scales[scale];
    // 2^(s - 127); s = 0 is the subnormal 2^-127, s = 255 a NaN
    const float f = s == MX_NAN ? __uint_as_float(0x7FC00000u) : (s == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23));
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t o[16];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t a, b;
            mx_decode4(w[j] >> (16 * h), a, b);
            o[4 * j + 2 * h] = pack_bf16x2(bf16_lo_f(a) * f, bf16_hi_f(a) * f);
            o[4 * j + 2 * h + 1] = pack_bf16x2(bf16_lo_f(b) * f, bf16_hi_f(b) * f);
        }
    uint16_t* dst = X + p.row * ldx + p.k;
    stg256(dst, *reinterpret_cast<const uint32_t(*)[8]>(&o[0]));
    stg256(dst + 16, *reinterpret_cast<const uint32_t(*)[8]>(&o[8]));
}

}  // namespace lynx
