// What the kernels around a projection in 8 bits share: eight consecutive elements of a row to a lane, codes and scales.
//
// A value is code * 2^(s - 127), code in e4m3 (largest 448 = 1.75 * 2^8), s one byte for 128 consecutive elements
// of a row.  s is the smallest that lets the largest finite magnitude fit, so x * 2^(127 - s) is exact and a code
// is rounded once (to nearest, ties to even); a value loses bits only below the smallest normal code, 2^-6: that is
// 2^-14.8 to 2^-13.8 of its block's largest, whose code is above 224.
#pragma once
#include "common.h"

namespace dlcx {

constexpr int kBlockLen = 128;  // elements that share a scale

struct Bf16x8 { uint32_t w[4]; };
// At any address that the element's type allows: the hardware takes 16 bytes from anywhere.
struct __attribute__((packed, aligned(2))) Loose16 { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) Loose16f { float f[4]; };

struct TypeBf16 {
    typedef uint16_t elem;
    static constexpr int size = 2;
    static __device__ __forceinline__ float get(elem e) { return __uint_as_float((uint32_t)e << 16); }
    // to nearest, ties to even; NaN stays NaN
    static __device__ __forceinline__ elem put(float x) {
        const uint32_t u = __float_as_uint(x);
        const uint32_t r = (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
        return (elem)((u & 0x7fffffffu) > 0x7f800000u ? (u >> 16) | 0x40u : r);
    }
};
struct TypeF32 {
    typedef float elem;
    static constexpr int size = 4;
    static __device__ __forceinline__ float get(elem e) { return e; }
    static __device__ __forceinline__ elem put(float x) { return x; }
};

// two fp32 values to bf16 in one register (one instruction; to nearest, ties to even)
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    const v2 p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}

// Eight elements from p on, of which `count` are there (the others: 0).  ENDS: rows may end within the eight; where
// their length is a multiple of eight, the code for that is left out (its registers would be there all the time).
template <typename T, bool ENDS = true>
__device__ __forceinline__ void load8(const typename T::elem *p, int count, float (&v)[8]) {
    if (ENDS ? count >= 8 : count > 0) {
        if constexpr (T::size == 2) {
            const Loose16 a = *reinterpret_cast<const Loose16 *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(a.w[i] << 16);
                v[2 * i + 1] = __uint_as_float(a.w[i] & 0xffff0000u);
            }
        } else {
            const Loose16f a = reinterpret_cast<const Loose16f *>(p)[0], b = reinterpret_cast<const Loose16f *>(p)[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = a.f[i];
                v[4 + i] = b.f[i];
            }
        }
    } else if (ENDS && count > 0) {  // (all of them asked for at once: one wait, not eight)
        typename T::elem e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = p[min(i, count - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? T::get(e[i]) : 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
}
// The same as it lies in memory, for later: `load` asks for it and `settle` makes it what is meant, where the row (of at
// least eight elements) ends within the eight: then its last eight are asked for, by the same instruction as everywhere, and
// moved down by `settle`.  So nothing is waited for before everything is asked for.
template <typename T>
struct Raw8 {
    uint32_t w[2 * T::size];
    __device__ __forceinline__ void load(const typename T::elem *p) {
#pragma unroll
        for (int h = 0; h < T::size / 2; ++h) {
            const Loose16 a = reinterpret_cast<const Loose16 *>(p)[h];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[4 * h + i] = a.w[i];
        }
    }
    template <bool ENDS>
    __device__ __forceinline__ void load(const typename T::elem *p, int count) {
        if (count > 0) {
            load(ENDS ? p + min(count - 8, 0) : p);
        } else {
#pragma unroll
            for (int i = 0; i < 2 * T::size; ++i) w[i] = 0;
        }
    }
    template <bool ENDS>
    __device__ __forceinline__ void settle(int count) {
        if (ENDS && count > 0 && count < 8) {
            const int by = 8 - count;
            if constexpr (T::size == 2) {
                if (by & 4) w[0] = w[2], w[1] = w[3], w[2] = w[3] = 0;
                if (by & 2) w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = 0;
                if (by & 1) {
#pragma unroll
                    for (int i = 0; i < 3; ++i) w[i] = w[i] >> 16 | w[i + 1] << 16;
                    w[3] >>= 16;
                }
            } else {
#pragma unroll
                for (int d = 4; d > 0; d >>= 1)
                    if (by & d)
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = i + d < 8 ? w[i + d] : 0u;
            }
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (T::size == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
};
template <typename T, bool ENDS = true>
__device__ __forceinline__ void store8(typename T::elem *p, int count, const float (&v)[8]) {
    if (ENDS ? count >= 8 : count > 0) {
        if constexpr (T::size == 2) {
            Loose16 a;
#pragma unroll
            for (int i = 0; i < 4; ++i) a.w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<Loose16 *>(p) = a;
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Loose16f a;
#pragma unroll
                for (int i = 0; i < 4; ++i) a.f[i] = v[4 * h + i];
                reinterpret_cast<Loose16f *>(p)[h] = a;
            }
        }
    } else if constexpr (ENDS) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = T::put(v[i]);
    }
}
// What a value is once it is stored.
template <typename T>
__device__ __forceinline__ void round8(float (&v)[8]) {
    if constexpr (T::size == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = pack_bf16(v[2 * i], v[2 * i + 1]);
            v[2 * i] = __uint_as_float(w << 16);
            v[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
}

// |x| where that is finite, else 0: an infinity or a NaN takes no part in its block's scale.  As bits, whose order is
// that of the magnitudes.
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t a = __float_as_uint(x) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}
__device__ __forceinline__ uint32_t finite_max8(const float (&v)[8]) {
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, finite_bits(v[i]));
    return a;
}
// the largest of a row of 16 lanes, in all of them (row_ror)
__device__ __forceinline__ uint32_t max16(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, true));
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, true));
}
// The scale's byte for a block whose largest magnitude has these bits: a = f 2^e with 1 <= f < 2 takes 2^(e - 8) up to
// f = 1.75, else 2^(e - 7); no less than 2^-127, and 2^0 for a block of zeros.  (Adding 2^22 - ... carries into the
// exponent where the fraction passes 0x600000, that is f > 1.75; magnitudes below 2^-119 all take the smallest.)
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest) {
    const int e = (int)((largest + 0x1fffffu) >> 23) - 8;
    return largest == 0 ? 127u : (uint32_t)max(e, 0);
}
// 2^(127 - s): what a value is multiplied by before it becomes a code (s <= 247, so this is a normal number)
__device__ __forceinline__ float scale_inverse(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// 2^(s - 127); s = 0 is the only one below the normal range, 255 is NaN
constexpr uint32_t kScaleNan = 255;
__device__ __forceinline__ float scale_value(uint32_t s) {
    return __uint_as_float(s == kScaleNan ? 0x7fc00000u : s ? s << 23 : 0x400000u);
}

__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inverse) {
    int w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * inverse, v[4 * h + 1] * inverse, 0, false);
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * inverse, v[4 * h + 3] * inverse, w[h], true);
    }
    return make_uint2((uint32_t)w[0], (uint32_t)w[1]);
}

// ---- on the host ----
inline int64_t code_pitch(int64_t cols) { return (cols + 127) / 128 * 128; }
inline int64_t scale_pitch(int64_t cols) { return (cols + 511) / 512 * 4; }
constexpr int64_t kMaxSide = 1 << 24;        // rows or columns
constexpr int64_t kMostGroups = 1 << 23;     // workgroups of a launch (2^32 threads are too many); the rest in their loops
constexpr int64_t kMaxRowStride = 1 << 29;   // elements or bytes between rows
inline bool off_by(const void *p, unsigned to) { return ((uintptr_t)p & (to - 1)) != 0; }
// DLCX_OK for a matrix in 8 bits that is laid out as the header says
int check_fp8(const dlcx_fp8 *a);
// a row-major matrix of DLCX_F32 or DLCX_BF16
inline bool bad_rows(const void *p, int64_t ld, int64_t cols, int dtype) {
    return !p || off_by(p, dtype == DLCX_BF16 ? 2 : 4) || ld < cols || ld > kMaxRowStride;
}

}  // namespace dlcx
