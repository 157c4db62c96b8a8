// Device-side pieces of the 8-bit integer path (w8_linear.hip, w8_moe.hip): the row quantizer and the blocked
// layout that weights and dense activations have.
//
// Blocked layout of an int8 matrix [R x K]: blocks of 16 rows by 64 columns, 1024 bytes each, block (r/16, k/64) at
// ((r/16) * kb + k/64) * 1024 with kb = 2 ceil(K/128).  Inside a block the 16-byte piece of row r%16 and columns
// 16c .. 16c+15 lies at c*256 + (r%16)*16, which is where lane c*16 + r%16 of a wave holds it as an operand of
// v_mfma_i32_16x16x64_i8: a fragment is one contiguous 1-KB load, and staged in LDS as it is, both that operand and
// the halves of a v_mfma_i32_32x32x32_i8 operand are read without bank conflicts.
#pragma once

#include "milo_device.h"

namespace milo {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* LdsDst;
// A pointer that was read from memory (an expert table's) says nothing about its address space, and a load through it would count as an
// LDS operation too: fragments go through these.
typedef const __attribute__((address_space(1))) u32x4* GlobalFrag;
__device__ __forceinline__ GlobalFrag global_frag(const void* p) { return (GlobalFrag)(uintptr_t)p; }
__device__ __forceinline__ const __attribute__((address_space(1))) float* global_float(const void* p) { return (const __attribute__((address_space(1))) float*)(uintptr_t)p; }

// Columns are padded to whole chunks of 128 (zeros), rows to whole blocks of 16.
__host__ __device__ inline int64_t w8_kblocks(int64_t K) { return (K + 127) / 128 * 2; }
__host__ __device__ inline int64_t w8_rblocks(int64_t R) { return (R + 15) / 16; }
__host__ __device__ inline int64_t w8_code_bytes(int64_t R, int64_t K) { return w8_rblocks(R) * w8_kblocks(K) * 1024; }

// ---------------------------------------------------------------------------------------------
// Quantizing a row: s = fp32(top / 127), code = round-half-even(x / s) of the exact quotient.
struct RowStep {
    float s, inv, lim;      // scale; 1 / s, or 0 for a row whose codes are all zero; what twice a remainder is compared with: s, or infinity for such a row
};
// `top_bits`: largest magnitude of the row as the bits of an fp32 number (an infinity or a NaN, whose bits are the
// largest, marks the row).  A row with such a value gets the scale NaN, so that everything computed from it is NaN;
// one whose scale is zero or subnormal gets the scale zero.
__device__ __forceinline__ RowStep row_step(uint32_t top_bits) {
    RowStep r;
    r.s = __uint_as_float(top_bits) / 127.0f;
    r.inv = 0.0f;
    r.lim = __uint_as_float(0x7f800000u);
    if (top_bits >= 0x7f800000u) {
        r.s = __uint_as_float(0x7fc00000u);
    } else if (r.s < 0x1p-126f) {
        r.s = 0.0f;
    } else {
        r.inv = 1.0f / r.s;
        r.lim = r.s;
    }
    return r;
}
// The product with 1/s is off by at most two units in the last place of a number below 2^7, so its rounding is the code or a neighbour
// of it.  x - c s is a multiple of half a unit in the last place of s (of a whole one in the lowest binade) and at most about s/2, hence exact
// in fp32, and comparing its double with s settles the code, ties included, without a division.  (s/2 need not be a number: 2^-126 is the
// smallest scale, and half of an odd one below 2^-125 has no fp32.)
__device__ __forceinline__ int row_code(float x, const RowStep& r) {
    const float c = rintf(x * r.inv), d = fmaf(-c, r.s, x), far = 2.0f * fabsf(d);
    const int q = (int)c, away = d > 0.0f ? 1 : -1;
    const bool other = (far > r.lim) | ((far == r.lim) & ((q & 1) != 0));
    return r.inv > 0.0f ? q + (other ? away : 0) : 0;
}
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
    return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)d << 24;
}
// The low bytes of four words.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return lo | hi;
}
constexpr float kRoundMagic = 12582912.0f;      // 1.5 * 2^23: a sum with it has the nearest whole number in its low bits, half to even
// 16 codes.  The rounding of the product is the code unless the remainder is half a step or more, which a tie or
// a quotient within 2^-17 of one does: only then the elements go one by one.
__device__ __forceinline__ u32x4 row_codes16(const float (&v)[16], const RowStep& r) {
    uint32_t b[16];
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float t = fmaf(v[i], r.inv, kRoundMagic);
        b[i] = __float_as_uint(t);
        far = fmaxf(far, fabsf(fmaf(-(t - kRoundMagic), r.s, v[i])));
    }
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = low_bytes(b[4 * i], b[4 * i + 1], b[4 * i + 2], b[4 * i + 3]);
    if (2.0f * far >= r.lim) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = pack4(row_code(v[4 * i], r), row_code(v[4 * i + 1], r), row_code(v[4 * i + 2], r), row_code(v[4 * i + 3], r));
    }
    return o;
}
// Four codes, by the same rule.
__device__ __forceinline__ uint32_t row_codes4(const float (&v)[4], const RowStep& r) {
    uint32_t b[4];
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float t = fmaf(v[i], r.inv, kRoundMagic);
        b[i] = __float_as_uint(t);
        far = fmaxf(far, fabsf(fmaf(-(t - kRoundMagic), r.s, v[i])));
    }
    if (2.0f * far >= r.lim) return pack4(row_code(v[0], r), row_code(v[1], r), row_code(v[2], r), row_code(v[3], r));
    return low_bytes(b[0], b[1], b[2], b[3]);
}

// Element types of what is quantized.
enum W8In { W8_F32 = 0, W8_F16 = 1, W8_BF16 = 2 };
template <int IN> struct W8Raw { uint32_t w[IN == W8_F32 ? 16 : 8]; };      // 16 elements as loaded

// Elements [k, k + 16) of a row of K, zeros beyond it.  The row may start at any element's address: whole pieces are
// copied by the widest loads (which need no alignment here), the last one element by element.
template <int IN>
__device__ __forceinline__ W8Raw<IN> load16(const void* row, int64_t k, int64_t K) {
    constexpr int SZ = IN == W8_F32 ? 4 : 2;
    W8Raw<IN> r;
    const char* p = reinterpret_cast<const char*>(row) + k * SZ;
    if (k + 16 <= K) {
        __builtin_memcpy(&r, p, 16 * SZ);
    } else {
#pragma unroll
        for (int i = 0; i < 4 * SZ; ++i) r.w[i] = 0u;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k + i < K) {
                if constexpr (SZ == 4) r.w[i] = reinterpret_cast<const uint32_t*>(p)[i];
                else r.w[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i & 1));
            }
    }
    return r;
}
template <int IN>
__device__ __forceinline__ float raw_value(const W8Raw<IN>& r, int i) {
    if constexpr (IN == W8_F32) return __uint_as_float(r.w[i]);
    else if constexpr (IN == W8_F16) return (float)f16_bits((r.w[i >> 1] >> (16 * (i & 1))) & 0xffffu);
    else return __uint_as_float(i & 1 ? r.w[i >> 1] & 0xffff0000u : r.w[i >> 1] << 16);
}
template <int IN>
__device__ __forceinline__ void raw_values(const W8Raw<IN>& r, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = raw_value<IN>(r, i);
}
// Largest magnitude so far: of 16-bit elements in both halves of a word, as their bits without the sign (whose order is that of the
// magnitudes, infinities and NaN on top), of fp32 as its bits.  top_bits() turns it into fp32 bits.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int IN>
__device__ __forceinline__ uint32_t raw_top(const W8Raw<IN>& r, uint32_t top) {
    if constexpr (IN == W8_F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t b = r.w[i] & 0x7fffffffu;
            top = b > top ? b : top;
        }
        return top;
    } else {
        u16x2 t = __builtin_bit_cast(u16x2, top);
#pragma unroll
        for (int i = 0; i < 8; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, r.w[i] & 0x7fff7fffu));
        return __builtin_bit_cast(uint32_t, t);
    }
}
template <int IN>
__device__ __forceinline__ uint32_t top_bits(uint32_t top) {
    if constexpr (IN == W8_F32) return top;
    const uint32_t lo = top & 0xffffu, hi = top >> 16, most = lo > hi ? lo : hi;
    if constexpr (IN == W8_F16) return __float_as_uint((float)f16_bits(most)) & 0x7fffffffu;
    else return most << 16;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const uint32_t o = __shfl_xor(v, d, 64);
        v = o > v ? o : v;
    }
    return v;
}

// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ i32x4 mfma16_i8(u32x4 a, u32x4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}
__device__ __forceinline__ i32x16 mfma32_i8(u32x4 a, u32x4 b, i32x16 c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// fp32 -> 16-bit output, rounded to nearest even.
template <bool BF>
__device__ __forceinline__ uint16_t out_bits(float v) {
    if constexpr (BF) {
        return __builtin_bit_cast(uint16_t, (__bf16)v);
    } else {
        return __builtin_bit_cast(uint16_t, (f16)v);
    }
}
// Four consecutive outputs at element `at` of `out`, of which those below `left` exist; `vec`: the rows keep 8-byte alignment.
template <bool BF>
__device__ __forceinline__ void store4(uint16_t* out, const float (&v)[4], int left, bool vec) {
    uint16_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = out_bits<BF>(v[i]);
    if (vec && left >= 4) {
        *reinterpret_cast<u32x2*>(out) = u32x2{b[0] | (uint32_t)b[1] << 16, b[2] | (uint32_t)b[3] << 16};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) out[i] = b[i];
    }
}

__device__ __forceinline__ float silu_times(float a, float b) { return a / (1.0f + expf(-a)) * b; }

}  // namespace milo
