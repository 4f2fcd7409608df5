// One optimizer step over many tensors at once (InnerOpt of Alg. 2; AdamW in Appendix A.3), the
// gradients' global norm before it, and the 8-bit form of the moments.
//
// All of them are streams over the tensors' elements, bound by HBM.  A launch covers every tensor
// of a table: the elements are cut into blocks of kBlock, a tensor's last block may be shorter, and
// table.start holds each tensor's first block, so a workgroup finds its tensor by searching there.
//
// Measured: AdamW with fp32 moments 5.4 TB/s (26.5 M fp32 elements in 140 tensors 146 us; 50 M with bf16
// gradients 262 us), with 8-bit moments 5.6 TB/s (856 M bf16 elements 1.54 ms), where a copy of 2 GiB reaches
// 4.9; the norm of 856 M bf16 gradients 252 + 5 us, 6.7 TB/s, of 26.5 M fp32 ones 21 + 4 us.
#include <math.h>

#include "common.h"

namespace dlcx {

constexpr int kThreads = 256;
constexpr int kVec = 8;                       // consecutive elements of a thread
constexpr int kStep = kThreads * kVec;        // elements of a workgroup's step
constexpr int kBlock = 2 * kStep;             // elements of a block
constexpr int kStateGroup = 128;              // elements that share a scale: 16 lanes
constexpr int kNormGroups = 2048;             // most workgroups (and partial sums) of the norm
constexpr int kTablePart = 32;                // tensors passed to one launch of the table's kernel
constexpr int kComplete = 1, kHas32 = 2, kHas8 = 4;  // of a table's `steps`
constexpr float kTopM = 127.f, kTopV = 255.f;

// What `memory` of a table holds.
struct TableView {
    double *partial;      // kNormGroups sums of the norm
    int32_t *start;       // count + 1: first block of each tensor, then the number of blocks
    dlcx_tensor *tensor;  // count
};
static size_t table_start_bytes(int count) { return a256x((size_t)(count + 1) * sizeof(int32_t)); }
static TableView table_view(void *memory, int count) {
    char *p = (char *)memory;
    TableView v;
    v.partial = (double *)p;
    v.start = (int32_t *)(p + kNormGroups * sizeof(double));
    v.tensor = (dlcx_tensor *)((char *)v.start + table_start_bytes(count));
    return v;
}

struct TablePart {
    int n, at, last;  // tensors here, their place, is this the last part?
    int32_t start[kTablePart + 1];
    dlcx_tensor tensor[kTablePart];
};

// The table travels as kernel arguments, so that nothing of the host's is read after the call.
__global__ __launch_bounds__(64) void tensor_table_kernel(TablePart part, TableView v) {
    const int i = threadIdx.x;
    if (i < part.n) {
        v.start[part.at + i] = part.start[i];
        v.tensor[part.at + i] = part.tensor[i];
    }
    if (part.last && i == 0) v.start[part.at + part.n] = part.start[part.n];
}

// The last tensor whose first block is at most `block` (one of no elements shares its start with the
// next one, so it is never found).  64 lanes look at 64 places at a time: two trips to memory up to
// 4096 tensors.
__device__ __forceinline__ int find_tensor(const int32_t *__restrict__ start, int count, int block) {
    const int lane = threadIdx.x & 63;
    int lo = 0, len = count;
    while (len > 1) {
        const int stride = (len + 63) / 64;
        const int at = lane * stride;
        const bool le = at < len && start[lo + at] <= block;
        const int k = __popcll(__ballot(le)) - 1;
        lo += k * stride;
        len = min(stride, len - k * stride);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

typedef float ad_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t ad_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t ad_u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 ad_bf16x2 __attribute__((ext_vector_type(2)));
typedef float ad_f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const ad_f32x2 x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, ad_bf16x2));
}

// Where a thread's elements begin: `first`, the workgroup's, is the same in all lanes, so that an access takes its
// address from scalar registers and one 32-bit offset.  A pointer read from the table is not known to be one
// to global memory unless it is said.
#define AD_GLOBAL __attribute__((address_space(1)))
template <class T>
__device__ __forceinline__ AD_GLOBAL T *elements(const void *base, int64_t first) {
    AD_GLOBAL char *p = (AD_GLOBAL char *)base + first * (int64_t)sizeof(T);
    return (AD_GLOBAL T *)(p + threadIdx.x * (kVec * (unsigned)sizeof(T)));
}

// A thread's elements as they lie in memory: all of them, or the `left` (less than 8; less or equal 0: none) that are
// inside the tensor and zeros.  All loads of a step come before what is made of any of them, in one branch
// each for whole and for part, so that none waits for another.
template <int DT>
struct Raw {
    uint32_t w[DT == DLCX_F32 ? kVec : kVec / 2];
};
// STREAM: past the caches' order of use.  Against plain loads: 8-bit moments 1.56 (1.60) ms; a norm of bf16 gradients,
// 1.7 GB 257 (303) us, 200 MB 34.9 (39.1); but of fp32 ones, which take twice the bytes a step, 1 GB 171 (169),
// 300 MB that are read again 53 (47); and 32-bit moments, whose 12 or 14 bytes an element are read and written at
// the same places, 155 (148) and 278 (264) us, so these two are plain.  Stores: all streamed, 1.56 (1.64) ms and
// 278 (282) us.
template <class T, bool STREAM>
__device__ __forceinline__ T load_vector(AD_GLOBAL const T *p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(p);
    return *p;
}
template <int DT, bool STREAM = true>
__device__ __forceinline__ Raw<DT> load_whole(const void *base, int64_t first) {
    Raw<DT> x;
    if constexpr (DT == DLCX_F32) {
        AD_GLOBAL const ad_u32x4 *p = (AD_GLOBAL const ad_u32x4 *)elements<const float>(base, first);
        const ad_u32x4 a = load_vector<ad_u32x4, STREAM>(p), b = load_vector<ad_u32x4, STREAM>(p + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.w[i] = a[i], x.w[4 + i] = b[i];
    } else {
        AD_GLOBAL const ad_u32x4 *p = (AD_GLOBAL const ad_u32x4 *)elements<const uint16_t>(base, first);
        const ad_u32x4 a = load_vector<ad_u32x4, STREAM>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.w[i] = a[i];
    }
    return x;
}
template <int DT>
__device__ __forceinline__ Raw<DT> load_part(const void *base, int64_t first, int left) {
    Raw<DT> x;
    if constexpr (DT == DLCX_F32) {
        AD_GLOBAL const uint32_t *p = elements<const uint32_t>(base, first);
#pragma unroll
        for (int i = 0; i < kVec; ++i) x.w[i] = i < left ? p[i] : 0u;
    } else {
        AD_GLOBAL const uint16_t *p = elements<const uint16_t>(base, first);
#pragma unroll
        for (int i = 0; i < kVec; i += 2)
            x.w[i / 2] = (i < left ? p[i] : 0u) | (i + 1 < left ? (uint32_t)p[i + 1] << 16 : 0u);
    }
    return x;
}
template <int DT>
__device__ __forceinline__ void unpack(const Raw<DT> &r, float (&x)[kVec]) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        if constexpr (DT == DLCX_F32)
            x[i] = __uint_as_float(r.w[i]);
        else
            x[i] = __uint_as_float(i & 1 ? r.w[i / 2] & 0xFFFF0000u : r.w[i / 2] << 16);
    }
}
template <int DT>
__device__ __forceinline__ void store_floats(void *base, int64_t first, int left, const float (&x)[kVec]) {
    uint32_t b[4];
    if constexpr (DT != DLCX_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    }
    AD_GLOBAL float *f = elements<float>(base, first);
    AD_GLOBAL uint16_t *h = elements<uint16_t>(base, first);
    if (left >= kVec) {
        if constexpr (DT == DLCX_F32) {
            AD_GLOBAL ad_f32x4 *p = (AD_GLOBAL ad_f32x4 *)f;
            const ad_f32x4 lo = {x[0], x[1], x[2], x[3]}, hi = {x[4], x[5], x[6], x[7]};
            __builtin_nontemporal_store(lo, p);
            __builtin_nontemporal_store(hi, p + 1);
        } else {
            const ad_u32x4 w = {b[0], b[1], b[2], b[3]};
            __builtin_nontemporal_store(w, (AD_GLOBAL ad_u32x4 *)h);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < left) {
                if constexpr (DT == DLCX_F32)
                    f[i] = x[i];
                else
                    h[i] = (uint16_t)(b[i / 2] >> (16 * (i & 1)));
            }
    }
}
__device__ __forceinline__ ad_u32x2 load_whole_codes(const void *base, int64_t first) {
    return __builtin_nontemporal_load((AD_GLOBAL const ad_u32x2 *)elements<const uint8_t>(base, first));
}
__device__ __forceinline__ ad_u32x2 load_part_codes(const void *base, int64_t first, int left) {
    AD_GLOBAL const uint8_t *p = elements<const uint8_t>(base, first);
    ad_u32x2 w = {0u, 0u};
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < left) w[i / 4] |= (uint32_t)p[i] << (8 * (i & 3));
    return w;
}
__device__ __forceinline__ void store_codes(void *base, int64_t first, int left, ad_u32x2 w) {
    AD_GLOBAL uint8_t *p = elements<uint8_t>(base, first);
    if (left >= kVec) {
        __builtin_nontemporal_store(w, (AD_GLOBAL ad_u32x2 *)p);
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < left) p[i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
}

// ---- 8-bit moments ------------------------------------------------------------------------------
// The square of the code times the scale: half a code off is a relative error of 1 / (2 c) of the root, 1 / c of
// the value, so values down to 6e-5 of a group's largest m (2.5e-10 of its largest v) keep a code of their
// own, where a linear code ends at 8e-3 (4e-3).
__device__ __forceinline__ float decode_m(uint32_t w, int i, float scale) {
    const float c = (float)(int8_t)(w >> (8 * i));
    return c * fabsf(c) * scale;
}
__device__ __forceinline__ float decode_v(uint32_t w, int i, float scale) {
    const float c = (float)((w >> (8 * i)) & 0xFFu);
    const float s = c * c * scale;
    return s * s;
}
// The largest of the 16 lanes of a row; of bit patterns of non-negative floats, where a NaN is larger than
// any number, so that a group with a NaN gets a NaN for a scale and does not lose it.
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, true));
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, true));
}
// Scale of a group and what its values are multiplied with before the root: a group whose largest value is
// below 2^-100 gives scale 0 and codes 0, as the quantiser of the payloads does.
__device__ __forceinline__ float group_scale(float amax, float top, float *inv) {
    const bool none = amax < 0x1p-100f;
    const float scale = none ? 0.f : amax * (1.f / (top * top));
    *inv = none ? 0.f : __builtin_amdgcn_rcpf(scale);
    return scale;
}
// The code of x >= 0 is the integer next to sqrt(x / scale), both operations rounded correctly, where x of a
// second moment is a correctly rounded root itself.  With IEEE quotients and roots throughout the step was bound
// by its arithmetic (4.2 TB/s; it still is, at 64 vector instructions an element).  So a code is taken from a product and the hardware's roots and reciprocals (1 unit in the
// last place), together off by 1e-4 codes at most, and only where that lies within 1.25e-4 of the middle between
// two codes is it decided by the definition: one code in 4000, hardly ever two of a thread's sixteen.
__device__ __forceinline__ float near_root(float x, float inv) { return __builtin_amdgcn_sqrtf(x * inv); }
__device__ __forceinline__ float from_middle(float root) { return fabsf(__builtin_amdgcn_fractf(root) - 0.5f); }
__device__ __forceinline__ float exact_code(float x, float scale) { return rintf(sqrtf(x / scale)); }
constexpr float kUndecided = 1.25e-4f;
// (the conversion rounds to the nearest, to even codes from the middle)
__device__ __forceinline__ void put_m(ad_u32x2 &w, int i, float root, float m) {
    w[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(copysignf(fminf(root, kTopM), m) + 128.f, i & 3, w[i / 4]);
}
__device__ __forceinline__ void put_v(ad_u32x2 &w, int i, float root, float v) {
    w[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(v > 0.f ? fmaxf(root, 1.f) : 0.f, i & 3, w[i / 4]);
}
// Below this a group's largest v may have company whose hardware root is flushed to zero and whose code is not 1.
constexpr float kTinyV = 0x1p-89f;
// m below 2^60, v below 2^100 (bit patterns; a NaN is above) and eps between 2^-50 and 2^100.
constexpr uint32_t kPlainM = (127u + 60) << 23, kPlainV = (127u + 100) << 23;
constexpr float kPlainEpsLow = 0x1p-50f, kPlainEpsHigh = 0x1p100f;

// a x + b y with every operation rounded: what the codes of the moments hang on is then the same wherever
// the formula is evaluated.
__device__ __forceinline__ float weighted_sum(float x, float a, float y, float b) {
#pragma clang fp contract(off)
    const float ax = a * x, by = b * y;
    return ax + by;
}

template <int PDT, int GDT, int BITS>
__device__ __forceinline__ void adamw_elements(const dlcx_tensor &t, const AdamwStep &s, float gs,
                                               float decay, float rate, int64_t first, int left) {
    float p[kVec], g[kVec], m[kVec], v[kVec];
    float m_scale = 0.f, v_scale = 0.f;
    ad_u32x2 mc = {0u, 0u}, vc = {0u, 0u};
    const unsigned mine = threadIdx.x / (kStateGroup / kVec);
    AD_GLOBAL float *const m_scales = (AD_GLOBAL float *)t.m_scale + first / kStateGroup;
    AD_GLOBAL float *const v_scales = (AD_GLOBAL float *)t.v_scale + first / kStateGroup;
    Raw<PDT> rp;
    Raw<GDT> rg;
    Raw<DLCX_F32> rm, rv;
    if (left >= kVec) {
        if constexpr (BITS == 8) {
            mc = load_whole_codes(t.m, first);
            vc = load_whole_codes(t.v, first);
            m_scale = m_scales[mine];
            v_scale = v_scales[mine];
        } else {
            rm = load_whole<DLCX_F32, BITS == 8>(t.m, first);
            rv = load_whole<DLCX_F32, BITS == 8>(t.v, first);
        }
        rp = load_whole<PDT, BITS == 8>(t.param, first);
        rg = load_whole<GDT, BITS == 8>(t.grad, first);
    } else {
        if constexpr (BITS == 8) {
            mc = load_part_codes(t.m, first, left);
            vc = load_part_codes(t.v, first, left);
            m_scale = left > 0 ? m_scales[mine] : 0.f;
            v_scale = left > 0 ? v_scales[mine] : 0.f;
        } else {
            rm = load_part<DLCX_F32>(t.m, first, left);
            rv = load_part<DLCX_F32>(t.v, first, left);
        }
        rp = load_part<PDT>(t.param, first, left);
        rg = load_part<GDT>(t.grad, first, left);
    }
    unpack(rp, p);
    unpack(rg, g);
    if constexpr (BITS == 32) {
        unpack(rm, m);
        unpack(rv, v);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            m[i] = decode_m(mc[i / 4], i & 3, m_scale);
            v[i] = decode_v(vc[i / 4], i & 3, v_scale);
        }
    }
    float root[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const float gi = g[i] * gs;
        m[i] = weighted_sum(m[i], s.beta1, gi, s.one_minus_beta1);
        v[i] = weighted_sum(v[i], s.beta2, gi * gi, s.one_minus_beta2);
        if constexpr (BITS == 32) p[i] = p[i] * decay - rate * (m[i] / (sqrtf(v[i]) * s.inv_sqrt_bc2 + s.eps));
    }
    if constexpr (BITS == 8) {
        uint32_t am = 0, av = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            am = max(am, __float_as_uint(m[i]) & 0x7FFFFFFFu);
            av = max(av, __float_as_uint(v[i]));  // (v >= 0 or a NaN, whose sign makes it the larger)
        }
        // Root and quotient are the hardware's approximations with one correction each: at most 1e-4 units in the last
        // place beyond the half of a correct rounding, 1.54 ms for 856 M elements where IEEE roots and quotients take
        // 1.82 and approximations alone 1.43.  No step of them leaves fp32's range below these limits; beyond, IEEE.
        if (am < kPlainM && av < kPlainV && s.eps >= kPlainEpsLow && s.eps <= kPlainEpsHigh) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float y = __builtin_amdgcn_rsqf(__uint_as_float(max(__float_as_uint(v[i]), 0x00800000u)));
                const float near = v[i] * y;
                root[i] = fmaf(0.5f * y, fmaf(-near, near, v[i]), near);
                const float d = root[i] * s.inv_sqrt_bc2 + s.eps, inv = __builtin_amdgcn_rcpf(d), q = m[i] * inv;
                p[i] = p[i] * decay - rate * fmaf(inv, fmaf(-q, d, m[i]), q);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                root[i] = sqrtf(v[i]);
                p[i] = p[i] * decay - rate * (m[i] / (root[i] * s.inv_sqrt_bc2 + s.eps));
            }
        }
        float m_inv, v_inv;
        const float v_max = __uint_as_float(row_max(av));
        m_scale = group_scale(__uint_as_float(row_max(am)), kTopM, &m_inv);
        v_scale = group_scale(sqrtf(v_max), kTopV, &v_inv);
        float m_closest = 1.f, v_closest = 1.f;
        mc = vc = ad_u32x2{0u, 0u};
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float cm = near_root(fabsf(m[i]), m_inv), cv = near_root(root[i], v_inv);
            m_closest = fminf(m_closest, from_middle(cm));
            v_closest = fminf(v_closest, from_middle(cv));
            put_m(mc, i, cm, m[i]);
            put_v(vc, i, cv, v[i]);
        }
        if (m_closest < kUndecided) {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (from_middle(near_root(fabsf(m[i]), m_inv)) < kUndecided)
                    put_m(mc, i, m_scale > 0.f ? exact_code(fabsf(m[i]), m_scale) : 0.f, m[i]);
        }
        const bool tiny = v_max < kTinyV;
        if (v_closest < kUndecided || tiny) {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (from_middle(near_root(root[i], v_inv)) < kUndecided || tiny)
                    put_v(vc, i, v_scale > 0.f ? exact_code(sqrtf(v[i]), v_scale) : 0.f, v[i]);
        }
        mc ^= 0x80808080u;
        if (left > 0) {
            store_codes(t.m, first, left, mc);
            store_codes(t.v, first, left, vc);
            if (threadIdx.x % (kStateGroup / kVec) == 0) {
                m_scales[mine] = m_scale;
                v_scales[mine] = v_scale;
            }
        }
    } else {
        store_floats<DLCX_F32>(t.m, first, left, m);
        store_floats<DLCX_F32>(t.v, first, left, v);
    }
    store_floats<PDT>(t.param, first, left, p);
    if (PDT == DLCX_F32 && t.copy != nullptr) store_floats<DLCX_BF16>(t.copy, first, left, p);
}

// A workgroup has 1 / PARTS of a block: with 32-bit moments one step, 264 us for the 50 M elements against 274 with
// two, one after the other; with 8-bit ones two, 1.56 ms against 1.61, since what every thread does before its
// first element is worth the arithmetic of one.  A table with both kinds takes two launches.
constexpr int kParts32 = 2, kParts8 = 1;
template <int BITS, int PARTS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(TableView tv, int count, int64_t blocks,
                                                         AdamwStep s) {
    float gs = s.grad_scale;
    if (s.norm != nullptr) {
        const float norm = *s.norm;
        if (!(fabsf(norm) < __builtin_inff())) return;
        if (norm > s.max_norm) gs *= s.max_norm / norm;
    }
    const int64_t part = (int64_t)blockIdx.x + (int64_t)blockIdx.y * gridDim.x, block = part / PARTS;
    if (block >= blocks) return;
    const int which = find_tensor(tv.start, count, (int)block);
    const dlcx_tensor t = tv.tensor[which];
    if ((t.state_bits == 8) != (BITS == 8)) return;
    const float decay = (float)(1.0 - s.lr * (double)t.lr_scale * (double)t.weight_decay);
    const float rate = (float)(s.lr_bc1 * (double)t.lr_scale);
    int64_t first = (block - tv.start[which]) * kBlock + (int)(part % PARTS) * (kBlock / PARTS);
#pragma unroll 1
    for (int u = 0; u < kBlock / kStep / PARTS; ++u, first += kStep) {
        const int64_t rest = t.numel - first;
        const int left = (rest > kStep ? kStep : (int)rest) - (int)threadIdx.x * kVec;
        if (t.param_dtype == DLCX_F32) {
            if (t.grad_dtype == DLCX_F32)
                adamw_elements<DLCX_F32, DLCX_F32, BITS>(t, s, gs, decay, rate, first, left);
            else
                adamw_elements<DLCX_F32, DLCX_BF16, BITS>(t, s, gs, decay, rate, first, left);
        } else {
            if (t.grad_dtype == DLCX_F32)
                adamw_elements<DLCX_BF16, DLCX_F32, BITS>(t, s, gs, decay, rate, first, left);
            else
                adamw_elements<DLCX_BF16, DLCX_BF16, BITS>(t, s, gs, decay, rate, first, left);
        }
    }
}

// ---- global norm --------------------------------------------------------------------------------
// fp64 throughout: a square of fp32 has room there at any size, and the order of the sum no weight.
template <int DT>
__device__ __forceinline__ double sum_squares(const void *grad, int64_t first, int64_t numel, double acc) {
    constexpr int kSteps = kBlock / kStep;
    Raw<DT> r[kSteps];
    if (numel - first >= kBlock) {
#pragma unroll
        for (int u = 0; u < kSteps; ++u) r[u] = load_whole<DT, DT != DLCX_F32>(grad, first + u * kStep);
    } else {
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            r[u] = load_part<DT>(grad, first + u * kStep, (int)(numel - first) - u * kStep - (int)threadIdx.x * kVec);
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        float x[kVec];
        unpack(r[u], x);
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc = fma((double)x[i], (double)x[i], acc);
    }
    return acc;
}

__device__ __forceinline__ double workgroup_sum(double x, double *lds) {
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    x = lds[0] + lds[1] + lds[2] + lds[3];
    __syncthreads();
    return x;
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(TableView tv, int count, int64_t blocks) {
    __shared__ double lds[kThreads / 64];
    const int64_t lo = blocks * blockIdx.x / gridDim.x, hi = blocks * (blockIdx.x + 1) / gridDim.x;
    double acc = 0.0;
    int which = lo < hi ? find_tensor(tv.start, count, (int)lo) : 0;
    for (int64_t b = lo; b < hi; ++b) {
        while (b >= tv.start[which + 1]) ++which;
        const dlcx_tensor &t = tv.tensor[which];
        const int64_t first = (b - tv.start[which]) * kBlock;
        acc = t.grad_dtype == DLCX_F32 ? sum_squares<DLCX_F32>(t.grad, first, t.numel, acc)
                                       : sum_squares<DLCX_BF16>(t.grad, first, t.numel, acc);
    }
    acc = workgroup_sum(acc, lds);
    if (threadIdx.x == 0) tv.partial[blockIdx.x] = acc;
}
__global__ __launch_bounds__(kThreads) void norm_finish_kernel(const double *__restrict__ partial, int n,
                                                               double scale, float *out) {
    __shared__ double lds[kThreads / 64];
    double x[kNormGroups / kThreads], acc = 0.0;
#pragma unroll
    for (int u = 0; u < kNormGroups / kThreads; ++u) x[u] = partial[min(u * kThreads + (int)threadIdx.x, n - 1)];
#pragma unroll
    for (int u = 0; u < kNormGroups / kThreads; ++u) acc += u * kThreads + (int)threadIdx.x < n ? x[u] : 0.0;
    acc = workgroup_sum(acc, lds);
    if (threadIdx.x == 0) *out = (float)(scale * sqrt(acc));
}

template <int SECOND, int DT>
__global__ __launch_bounds__(kThreads) void state_decode_kernel(const void *codes, const float *scales,
                                                                int64_t numel, void *out) {
    const int64_t first = (int64_t)blockIdx.x * kStep, rest = numel - first;
    const int left = (rest > kStep ? kStep : (int)rest) - (int)threadIdx.x * kVec;
    if (left <= 0) return;
    const ad_u32x2 w = left >= kVec ? load_whole_codes(codes, first) : load_part_codes(codes, first, left);
    const float scale = (scales + first / kStateGroup)[threadIdx.x / (kStateGroup / kVec)];
    float x[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        x[i] = SECOND ? decode_v(w[i / 4], i & 3, scale) : decode_m(w[i / 4], i & 3, scale);
    store_floats<DT>(out, first, left, x);
}

// ---- launches -----------------------------------------------------------------------------------
int launch_tensor_table(const dlcx_tensor *t, int count, void *memory, dlcx_table *table,
                        hipStream_t st) {
    const TableView v = table_view(memory, count);
    int64_t blocks = 0;
    int steps = kComplete;
    bool complete = true;
    for (int i = 0; i < count; ++i) {
        blocks += ceil_div(t[i].numel, kBlock);
        if (blocks > 0x7FFFFFFF) return DLCX_EINVAL;
        if (t[i].numel == 0) continue;
        if (t[i].param == nullptr) complete = false;
        steps |= t[i].state_bits == 8 ? kHas8 : kHas32;
    }
    table->memory = memory;
    table->blocks = blocks;
    table->count = count;
    table->steps = complete ? steps : 0;
    TablePart part;
    int64_t at = 0;
    for (int i = 0; i < count; i += kTablePart) {
        part.at = i;
        part.n = count - i < kTablePart ? count - i : kTablePart;
        part.last = i + part.n == count;
        for (int k = 0; k < part.n; ++k) {
            part.start[k] = (int32_t)at;
            part.tensor[k] = t[i + k];
            at += ceil_div(t[i + k].numel, kBlock);
        }
        part.start[part.n] = (int32_t)at;
        Timed timed(KID_TENSOR_TABLE, st);
        tensor_table_kernel<<<1, 64, 0, st>>>(part, v);
        const int rc = check_launch("tensor_table");
        if (rc != DLCX_OK) return rc;
    }
    return DLCX_OK;
}

int launch_grad_norm(const dlcx_table &table, double grad_scale, float *norm_out, hipStream_t st) {
    const unsigned groups =
        (unsigned)(table.blocks < 1 ? 1 : table.blocks < kNormGroups ? table.blocks : kNormGroups);
    Timed timed(KID_GRAD_NORM, st);
    const TableView tv = table_view(table.memory, table.count);
    grad_norm_kernel<<<groups, kThreads, 0, st>>>(tv, table.count, table.blocks);
    norm_finish_kernel<<<1, kThreads, 0, st>>>(tv.partial, (int)groups, grad_scale, norm_out);
    return check_launch("grad_norm");
}

template <int BITS, int PARTS>
static void launch_adamw_bits(const dlcx_table &table, const AdamwStep &step, hipStream_t st) {
    const int64_t parts = table.blocks * PARTS, gx = parts < (1 << 20) ? parts : (1 << 20);
    adamw_kernel<BITS, PARTS><<<dim3((unsigned)gx, (unsigned)ceil_div(parts, gx)), kThreads, 0, st>>>(
        table_view(table.memory, table.count), table.count, table.blocks, step);
}
int launch_adamw(const dlcx_table &table, const AdamwStep &step, hipStream_t st) {
    if (table.blocks == 0) return DLCX_OK;
    Timed timed(KID_ADAMW, st);
    if (table.steps & kHas32) launch_adamw_bits<32, kParts32>(table, step, st);
    if (table.steps & kHas8) launch_adamw_bits<8, kParts8>(table, step, st);
    return check_launch("adamw");
}

int launch_state_decode(int second, const void *codes, const float *scales, int64_t numel, void *out,
                        int out_dtype, hipStream_t st) {
    const unsigned groups = (unsigned)ceil_div(numel, kStep);
    Timed timed(KID_STATE_DECODE, st);
    if (second) {
        if (out_dtype == DLCX_F32)
            state_decode_kernel<1, DLCX_F32><<<groups, kThreads, 0, st>>>(codes, scales, numel, out);
        else
            state_decode_kernel<1, DLCX_BF16><<<groups, kThreads, 0, st>>>(codes, scales, numel, out);
    } else {
        if (out_dtype == DLCX_F32)
            state_decode_kernel<0, DLCX_F32><<<groups, kThreads, 0, st>>>(codes, scales, numel, out);
        else
            state_decode_kernel<0, DLCX_BF16><<<groups, kThreads, 0, st>>>(codes, scales, numel, out);
    }
    return check_launch("state_decode");
}

}  // namespace dlcx

using namespace dlcx;

// ---- entry points ---------------------------------------------------------------------------------
extern "C" {

size_t dlcx_tensor_table_bytes(int32_t count) {
    if (count < 1 || count > DLCX_MAX_TENSORS) return 0;
    return kNormGroups * sizeof(double) + table_start_bytes(count) +
           a256x((size_t)count * sizeof(dlcx_tensor));
}

static int check_tensor(const dlcx_tensor &t) {
    if (t.numel < 0 || t.numel > (int64_t)0x7FFFFFFF * kBlock || t.reserved != 0) return DLCX_EINVAL;
    if (t.grad_dtype != DLCX_F32 && t.grad_dtype != DLCX_BF16) return DLCX_EINVAL;
    if (t.numel == 0) return DLCX_OK;
    if (!t.grad || !aligned16(t.grad)) return DLCX_EINVAL;
    if (!t.param) return DLCX_OK;  // for the norm alone
    if (t.param_dtype != DLCX_F32 && t.param_dtype != DLCX_BF16) return DLCX_EINVAL;
    if (t.state_bits != 32 && t.state_bits != 8) return DLCX_EINVAL;
    if (!t.m || !t.v || !aligned16(t.param) || !aligned16(t.m) || !aligned16(t.v)) return DLCX_EINVAL;
    if (t.state_bits == 8 && (!t.m_scale || !t.v_scale || ((uintptr_t)t.m_scale & 3) || ((uintptr_t)t.v_scale & 3)))
        return DLCX_EINVAL;
    if (t.copy && (t.param_dtype != DLCX_F32 || !aligned16(t.copy))) return DLCX_EINVAL;
    if (!isfinite(t.lr_scale) || !isfinite(t.weight_decay)) return DLCX_EINVAL;
    return DLCX_OK;
}

int dlcx_tensor_table(const dlcx_tensor *tensors_host, int32_t count, void *memory,
                      dlcx_table *table_out_host, void *stream) {
    if (!tensors_host || !table_out_host || count < 1 || count > DLCX_MAX_TENSORS) return DLCX_EINVAL;
    if (!memory || ((uintptr_t)memory & 255)) return DLCX_EINVAL;
    for (int i = 0; i < count; ++i) {
        const int rc = check_tensor(tensors_host[i]);
        if (rc != DLCX_OK) return rc;
    }
    return launch_tensor_table(tensors_host, count, memory, table_out_host, as_stream(stream));
}

static int check_table(const dlcx_table *t) {
    if (!t || !t->memory || t->count < 1 || t->count > DLCX_MAX_TENSORS || t->blocks < 0) return DLCX_EINVAL;
    return DLCX_OK;
}

int dlcx_grad_norm(const dlcx_table *table_host, double grad_scale, float *norm_out, void *stream) {
    const int rc = check_table(table_host);
    if (rc != DLCX_OK) return rc;
    if (!norm_out || ((uintptr_t)norm_out & 3) || !(grad_scale >= 0) || !isfinite(grad_scale)) return DLCX_EINVAL;
    return launch_grad_norm(*table_host, grad_scale, norm_out, as_stream(stream));
}

int dlcx_adamw(const dlcx_table *table_host, double lr, double beta1, double beta2, double eps,
               int64_t step, double grad_scale, const float *norm, double max_norm, void *stream) {
    const int rc = check_table(table_host);
    if (rc != DLCX_OK) return rc;
    if (!table_host->steps || step < 1) return DLCX_EINVAL;
    if (!isfinite(lr) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1)) return DLCX_EINVAL;
    // (as the step has them, in fp32: an eps that is zero there divides zeros by zeros, a scale that is infinite zeros too)
    if (!((float)eps > 0) || !isfinite((float)eps) || !(grad_scale >= 0) || !isfinite((float)grad_scale)) return DLCX_EINVAL;
    if (!isfinite((float)lr)) return DLCX_EINVAL;
    if (norm && (((uintptr_t)norm & 3) || !(max_norm > 0))) return DLCX_EINVAL;
    AdamwStep s;
    s.beta1 = (float)beta1;
    s.one_minus_beta1 = (float)(1.0 - beta1);
    s.beta2 = (float)beta2;
    s.one_minus_beta2 = (float)(1.0 - beta2);
    s.eps = (float)eps;
    s.inv_sqrt_bc2 = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    s.lr = lr;
    s.lr_bc1 = lr / (1.0 - pow(beta1, (double)step));
    s.grad_scale = (float)grad_scale;
    s.max_norm = (float)max_norm;
    s.norm = norm;
    return launch_adamw(*table_host, s, as_stream(stream));
}

int dlcx_state_decode(int second, const void *codes, const float *scales, int64_t numel, void *out,
                      int out_dtype, void *stream) {
    if (numel < 0 || (second != 0 && second != 1)) return DLCX_EINVAL;
    if (out_dtype != DLCX_F32 && out_dtype != DLCX_BF16) return DLCX_EINVAL;
    if (numel == 0) return DLCX_OK;
    if (!codes || !scales || !out || !aligned16(codes) || !aligned16(out) || ((uintptr_t)scales & 3))
        return DLCX_EINVAL;
    if (numel > (int64_t)0x7FFFFF * kStep) return DLCX_EINVAL;
    return launch_state_decode(second, codes, scales, numel, out, out_dtype, as_stream(stream));
}

}  // extern "C"
