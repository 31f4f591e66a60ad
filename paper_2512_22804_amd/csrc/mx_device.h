// Device-side building blocks of the microscaled 4-bit operands (gfx950 only).
//
// Arithmetic contract (bit-identical codes and scales):
//   amax   = largest magnitude of the block, compared as bit patterns, so that an infinity or a NaN wins;
//   byte   = biased exponent of the scale 2^e: from the binary32 exponent of amax (scale_byte below);
//   |x| 2^-e is exact in binary32 unless it is far below the grid's smallest step, where it rounds to code 0;
//   code   = nearest grid value, ties to the even code (hardware conversion), or the stochastic rule of mor_mx.h.
#pragma once
#include "mor_device.h"

namespace mor {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kMxNan = 255u;

// E8M0 byte of a block from the binary32 bits of its amax.  For a normal amax of biased exponent E the floor rule's exponent is
// E - 127 - 2, stored with a bias of 127; subnormals and the smallest normals clamp to 2^-127 (byte 0).
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits, bool ceil_rule) {
    if (amax_bits == 0u) return 127u;
    if (amax_bits >= 0x7F800000u) return kMxNan;
    int e = (int)(amax_bits >> 23) - 2;
    if (ceil_rule && (amax_bits & 0x7FFFFFu) > 0x400000u) ++e;      // amax > 1.5 * 2^(e+2) = 6 * 2^e
    return (uint32_t)max(e, 0);
}

// Philox 4 x 32 (J. Salmon, M. Moraes, R. Dror, D. Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011) with seven
// rounds, the fewest for which the authors report that every statistical test passes; ten cost 1.4 times as much.
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
__device__ __forceinline__ u32x4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = xor3((uint32_t)(p1 >> 32), c1, k0);
        c1 = (uint32_t)p1;
        c2 = xor3((uint32_t)(p0 >> 32), c3, k1);
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// Stochastic code of one magnitude, not yet less kStochasticBase and not yet with its sign: v = element in binary32, shift = 23 - e, r = 16
// random bits.  From 1 on a grid value has one mantissa bit, so y = |v| 2^-e rounds up where the 22 bits behind it, plus r 2^6,
// carry: bit 22 of y's pattern on is the code (plus a constant).  Below 1 the same holds of y 2^23 as a whole number, whose
// steps are those of the binade below 2.  Whole numbers throughout: floor(y / step + r / 65536) without a rounding of its own.
//
// The constant makes the two agree at 1, y 2^23 = 2^23 in either form; below it the pattern is the smaller of the two and both lie
// below 2^23's, above it the pattern is the smaller too and both lie above: the one wanted is the median of all three.
constexpr uint32_t kStochasticBase = 2 * (127 - 1) + 2 * 23;
template <int HALF>                                                         // of `random`: r
__device__ __forceinline__ uint32_t mx_code_stochastic(float v, int shift, uint32_t random) {
    const float y = __builtin_amdgcn_ldexpf(__builtin_fabsf(v), shift);     // y 2^23
    const uint32_t whole = (uint32_t)y + (kStochasticBase << 22);
    const uint32_t w = __float_as_uint(__builtin_amdgcn_fmed3f(__uint_as_float(whole), y, 0x1p23f));
    uint32_t sum;                                                           // w + (r << 6)
    if (HALF == 0) asm("v_mad_u32_u16 %0, %1, 64, %2" : "=v"(sum) : "v"(random), "v"(w));
    else asm("v_mad_u32_u16 %0, %1, 64, %2 op_sel:[1,0,0,0]" : "=v"(sum) : "v"(random), "v"(w));
    return min(sum >> 22, kStochasticBase + 7u);
}

__device__ __forceinline__ bf16x2 bf16_pair(uint32_t word) { return __builtin_bit_cast(bf16x2, word); }

// Eight elements to eight codes (element 0 in the lowest nibble).  Values as packed BF16 pairs or in binary32.
__device__ __forceinline__ uint32_t mx_codes8_nearest(const u32x4& v, uint32_t byte) {
    const float s = __uint_as_float(byte << 23);                    // the conversion reads the exponent field alone
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, bf16_pair(v[0]), s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, bf16_pair(v[1]), s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, bf16_pair(v[2]), s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, bf16_pair(v[3]), s, 3);
    return byte == kMxNan ? 0u : c;
}
__device__ __forceinline__ uint32_t mx_codes8_nearest(const float (&v)[8], uint32_t byte) {
    const float s = __uint_as_float(byte << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    return byte == kMxNan ? 0u : c;
}
__device__ __forceinline__ uint32_t mx_codes8_stochastic(const float (&v)[8], uint32_t byte, const u32x4& random) {
    const int shift = 23 + 127 - (int)byte;
    uint32_t c = 0u - kStochasticBase * 0x11111111u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c += mx_code_stochastic<0>(v[2 * j], shift, random[j]) << (8 * j);
        c += mx_code_stochastic<1>(v[2 * j + 1], shift, random[j]) << (8 * j + 4);
    }
    // the signs: the highest bytes of the even elements and of the odd ones, side by side
    uint32_t high[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
        high[j] = __builtin_amdgcn_perm(__float_as_uint(v[2 + j]), __float_as_uint(v[j]), 0x0C0C0703u) |
                  __builtin_amdgcn_perm(__float_as_uint(v[6 + j]), __float_as_uint(v[4 + j]), 0x07030C0Cu);
    const uint32_t sign = (high[0] >> 4 & 0x08080808u) | (high[1] & 0x80808080u);
    return byte == kMxNan ? 0u : c | sign;
}
__device__ __forceinline__ void widen8(const u32x4& raw, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(raw[j] << 16);
        v[2 * j + 1] = __uint_as_float(raw[j] & 0xFFFF0000u);
    }
}

// The XCDs take the workgroups in turn: tile of workgroup `b` of `n`, such that each XCD has a run of neighbouring ones.  Lines that two
// tiles share then meet in one L2, whole when they leave it (de-quantisation of 14336 x 4096: 27.7 us in the workgroups' own order,
// 21.3 so; of 18432 x 4104, whose rows end inside lines, 44.7 and 28.2).
__device__ __forceinline__ uint32_t tile_of(uint32_t b, uint32_t n) {
    const uint32_t x = b % 8;
    return x * (n / 8) + min(x, n % 8) + b / 8;
}

// Eight elements of a BF16 row from column c on; the last ones of a row may be missing and read as zeros.  Rows may start at any
// element: the wide accesses need no more than the elements' own alignment.  At the end of a row its last eight elements are loaded
// and then moved down.  Two functions, so that all of a lane's loads are on their way before the first is moved (columns of 1685 x
// 1358, in tiles of 128 rows: 9.1 us when each load was waited for, 4.8 so).
typedef u32x4 u32x4_anywhere __attribute__((aligned(2)));
typedef u32x2 u32x2_anywhere __attribute__((aligned(2)));
typedef uint32_t u32_anywhere __attribute__((aligned(2)));
template <bool STREAM = false>
__device__ __forceinline__ u32x4 load8_start(const uint16_t* row, int64_t c, int64_t cols) {
    if (cols >= 8) {
        const u32x4_anywhere* p = reinterpret_cast<const u32x4_anywhere*>(row + min(c, cols - 8));
        return STREAM ? __builtin_nontemporal_load(p) : *p;
    }
    u32x4 v{0u, 0u, 0u, 0u};
    for (int j = 0; j < 8; ++j)
        if (c + j < cols) v[j >> 1] |= (uint32_t)row[c + j] << (16 * (j & 1));
    return v;
}
__device__ __forceinline__ u32x4 load8_end(const u32x4& v, int64_t c, int64_t cols) {
    if (c + 8 <= cols || cols < 8) return v;
    const int bits = 16 * (int)(c + 8 - cols);          // 16 .. 112
    const uint64_t low = ((uint64_t)v[1] << 32) | v[0], high = ((uint64_t)v[3] << 32) | v[2];
    const uint64_t first = bits >= 64 ? high >> (bits - 64) : (low >> bits) | (high << (64 - bits)), second = bits >= 64 ? 0u : high >> bits;
    return u32x4{(uint32_t)first, (uint32_t)(first >> 32), (uint32_t)second, (uint32_t)(second >> 32)};
}
template <bool STREAM = false>
__device__ __forceinline__ u32x4 load8(const uint16_t* row, int64_t c, int64_t cols) { return load8_end(load8_start<STREAM>(row, c, cols), c, cols); }
template <bool STREAM = false>
__device__ __forceinline__ void store8(uint16_t* row, int64_t c, int64_t cols, const u32x4& v) {
    if (c + 8 <= cols) {
        u32x4_anywhere* p = reinterpret_cast<u32x4_anywhere*>(row + c);
        if (STREAM) __builtin_nontemporal_store(v, p);
        else *p = v;
        return;
    }
    const int n = (int)(cols - c);
    if (n & 4) *reinterpret_cast<u32x2_anywhere*>(row + c) = u32x2{v[0], v[1]};
    const uint32_t third = n & 4 ? v[2] : v[0], fourth = n & 4 ? v[3] : v[1];
    if (n & 2) *reinterpret_cast<u32_anywhere*>(row + c + (n & 4)) = third;
    if (n & 1) row[c + n - 1] = (uint16_t)(n & 2 ? fourth : third);
}
// Nearest BF16 value, ties to even; a NaN becomes the quiet NaN of its sign.
__device__ __forceinline__ uint32_t bf16_of(float v) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0u | ((u >> 16) & 0x8000u);
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

}  // namespace mor
