// One optimizer step over many tensors at once (InnerOpt of Alg. 2; AdamW in Appendix A.3), the
// gradients' global norm before it, and the 8-bit form of the moments.
//
// All of them are streams over the tensors' elements, bound by HBM.  A launch covers every tensor
// of a table: the elements are cut into blocks of kBlock, a tensor's last block may be shorter, and
// table.start holds each tensor's first block, so a workgroup finds its tensor by searching there.
//
// Measured: AdamW with fp32 moments 5.0 TB/s (26.5 M fp32 elements in 140 tensors 160 us; 50 M with bf16
// gradients 290 us), with 8-bit moments 4.8 TB/s (856 M bf16 elements 1.79 ms), where a copy of 2 GiB reaches
// 4.9; the norm of 856 M bf16 gradients 252 us, 6.8 TB/s, of 26.5 M fp32 ones 24 + 3 us.
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

// Eight elements from `e` on, of which `left` (1 .. 8; less or equal 0: none) are inside the tensor.
template <int DT>
__device__ __forceinline__ void load_floats(const void *base, int64_t e, int left, float (&x)[kVec]) {
    if (left >= kVec) {
        if constexpr (DT == DLCX_F32) {
            const ad_f32x4 *p = reinterpret_cast<const ad_f32x4 *>((const float *)base + e);
            const ad_f32x4 a = __builtin_nontemporal_load(p), b = __builtin_nontemporal_load(p + 1);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
        } else {
            const ad_u32x4 a = __builtin_nontemporal_load(
                reinterpret_cast<const ad_u32x4 *>((const uint16_t *)base + e));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(a[i] << 16);
                x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            x[i] = 0.f;
            if (i < left)
                x[i] = DT == DLCX_F32 ? ((const float *)base)[e + i]
                                      : __uint_as_float((uint32_t)((const uint16_t *)base)[e + i] << 16);
        }
    }
}
template <int DT>
__device__ __forceinline__ void store_floats(void *base, int64_t e, int left, const float (&x)[kVec]) {
    uint32_t b[4];
    if constexpr (DT != DLCX_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    }
    if (left >= kVec) {
        if constexpr (DT == DLCX_F32) {
            ad_f32x4 *p = reinterpret_cast<ad_f32x4 *>((float *)base + e);
            const ad_f32x4 lo = {x[0], x[1], x[2], x[3]}, hi = {x[4], x[5], x[6], x[7]};
            __builtin_nontemporal_store(lo, p);
            __builtin_nontemporal_store(hi, p + 1);
        } else {
            const ad_u32x4 w = {b[0], b[1], b[2], b[3]};
            __builtin_nontemporal_store(w, reinterpret_cast<ad_u32x4 *>((uint16_t *)base + e));
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < left) {
                if constexpr (DT == DLCX_F32)
                    ((float *)base)[e + i] = x[i];
                else
                    ((uint16_t *)base)[e + i] = (uint16_t)(b[i / 2] >> (16 * (i & 1)));
            }
    }
}
__device__ __forceinline__ ad_u32x2 load_codes(const void *base, int64_t e, int left) {
    if (left >= kVec)
        return __builtin_nontemporal_load(reinterpret_cast<const ad_u32x2 *>((const uint8_t *)base + e));
    ad_u32x2 w = {0u, 0u};
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < left) w[i / 4] |= (uint32_t)((const uint8_t *)base)[e + i] << (8 * (i & 3));
    return w;
}
__device__ __forceinline__ void store_codes(void *base, int64_t e, int left, ad_u32x2 w) {
    if (left >= kVec) {
        __builtin_nontemporal_store(w, reinterpret_cast<ad_u32x2 *>((uint8_t *)base + e));
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < left) ((uint8_t *)base)[e + i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
}

// ---- 8-bit moments ------------------------------------------------------------------------------
// The square of the code times the scale: half a code off is a relative error of 1 / (2 c) of the root, 1 / c of
// the value, so values down to 6e-5 of a group's largest m (2.5e-10 of its largest v) keep a code of their
// own, where a linear code ends at 8e-3 (4e-3).
__device__ __forceinline__ float decode_m(uint32_t w, int i, float scale) {
    const float c = (float)(((w ^ 0x80808080u) >> (8 * i)) & 0xFFu) - 128.f;
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
    *inv = none ? 0.f : top * top / amax;
    return none ? 0.f : amax * (1.f / (top * top));
}
// The code of x >= 0 is the integer next to sqrt(x / scale), both operations rounded correctly, where x of a
// second moment is a correctly rounded root itself.  With IEEE quotients and roots throughout the step
// was bound by arithmetic (4.2 TB/s, now 4.8); so a code is taken from a product and the
// hardware's roots (1 unit in the last place), together off by less than 8e-5 codes, and where one of a
// thread's lies within 1e-4 of the middle between two codes, all of them are decided by the definition.
__device__ __forceinline__ float near_root(float x, float inv) { return __builtin_amdgcn_sqrtf(x * inv); }
__device__ __forceinline__ float from_middle(float root) { return fabsf(__builtin_amdgcn_fractf(root) - 0.5f); }
__device__ __forceinline__ float exact_code(float x, float scale) { return rintf(sqrtf(x / scale)); }
// Below this a group's largest v may have company whose hardware root is flushed to zero and whose code is not 1.
constexpr float kTinyV = 0x1p-89f;

// a x + b y with every operation rounded: what the codes of the moments hang on is then the same wherever
// the formula is evaluated.
__device__ __forceinline__ float weighted_sum(float x, float a, float y, float b) {
#pragma clang fp contract(off)
    const float ax = a * x, by = b * y;
    return ax + by;
}

template <int PDT, int GDT, int BITS>
__device__ __forceinline__ void adamw_elements(const dlcx_tensor &t, const AdamwStep &s, float gs,
                                               float decay, float rate, int64_t e, int left) {
    float p[kVec], g[kVec], m[kVec], v[kVec];
    float m_scale = 0.f, v_scale = 0.f;
    ad_u32x2 mc = {0u, 0u}, vc = {0u, 0u};
    const int64_t group = e / kStateGroup;
    if (BITS == 8 && left > 0) {
        mc = load_codes(t.m, e, left);
        vc = load_codes(t.v, e, left);
        m_scale = t.m_scale[group];
        v_scale = t.v_scale[group];
    }
    load_floats<PDT>(t.param, e, left, p);
    load_floats<GDT>(t.grad, e, left, g);
    if constexpr (BITS == 32) {
        load_floats<DLCX_F32>(t.m, e, left, m);
        load_floats<DLCX_F32>(t.v, e, left, v);
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
        if constexpr (BITS == 32) {
            p[i] = p[i] * decay - rate * (m[i] / (sqrtf(v[i]) * s.inv_sqrt_bc2 + s.eps));
        } else {
            // (a v that the hardware's root would flush counts as the smallest one that it does not)
            root[i] = __builtin_amdgcn_sqrtf(fmaxf(v[i], 0x1p-126f));
            p[i] = p[i] * decay - rate * (m[i] * __builtin_amdgcn_rcpf(root[i] * s.inv_sqrt_bc2 + s.eps));
        }
    }
    if constexpr (BITS == 8) {
        uint32_t am = 0, av = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            am = max(am, __float_as_uint(m[i]) & 0x7FFFFFFFu);
            av = max(av, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        }
        float m_inv, v_inv;
        const float v_max = __uint_as_float(row_max(av));
        m_scale = group_scale(__uint_as_float(row_max(am)), kTopM, &m_inv);
        v_scale = group_scale(sqrtf(v_max), kTopV, &v_inv);
        float cm[kVec], cv[kVec], closest = v_max < kTinyV ? 0.f : 1.f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            cm[i] = near_root(fabsf(m[i]), m_inv);
            cv[i] = near_root(root[i], v_inv);
            closest = fminf(closest, fminf(from_middle(cm[i]), from_middle(cv[i])));
        }
        if (closest < 1e-4f) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                cm[i] = m_scale > 0.f ? exact_code(fabsf(m[i]), m_scale) : 0.f;
                cv[i] = v_scale > 0.f ? exact_code(sqrtf(v[i]), v_scale) : 0.f;
            }
        }
        mc = vc = ad_u32x2{0u, 0u};
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float c = copysignf(fminf(cm[i], kTopM), m[i]) + 128.f;
            mc[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(rintf(c), i & 3, mc[i / 4]);
            vc[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(rintf(v[i] > 0.f ? fmaxf(cv[i], 1.f) : 0.f), i & 3, vc[i / 4]);
        }
        mc ^= 0x80808080u;
        if (left > 0) {
            store_codes(t.m, e, left, mc);
            store_codes(t.v, e, left, vc);
            if (threadIdx.x % (kStateGroup / kVec) == 0) {
                t.m_scale[group] = m_scale;
                t.v_scale[group] = v_scale;
            }
        }
    } else {
        store_floats<DLCX_F32>(t.m, e, left, m);
        store_floats<DLCX_F32>(t.v, e, left, v);
    }
    store_floats<PDT>(t.param, e, left, p);
    if (PDT == DLCX_F32 && t.copy != nullptr) store_floats<DLCX_BF16>(t.copy, e, left, p);
}

__global__ __launch_bounds__(kThreads) void adamw_kernel(TableView tv, int count, int64_t blocks,
                                                         AdamwStep s) {
    float gs = s.grad_scale;
    if (s.norm != nullptr) {
        const float norm = *s.norm;
        if (!(fabsf(norm) < __builtin_inff())) return;
        if (norm > s.max_norm) gs *= s.max_norm / norm;
    }
    const int64_t block = (int64_t)blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (block >= blocks) return;
    const int which = find_tensor(tv.start, count, (int)block);
    const dlcx_tensor t = tv.tensor[which];
    const float decay = (float)(1.0 - s.lr * (double)t.lr_scale * (double)t.weight_decay);
    const float rate = (float)(s.lr_bc1 * (double)t.lr_scale);
    const int64_t first = (block - tv.start[which]) * kBlock, numel = t.numel;
    const int kind = t.param_dtype + 2 * t.grad_dtype + (t.state_bits == 8 ? 4 : 0);
#define DLCX_ADAMW_KIND(P, G, B)                                                               \
    for (int u = 0; u < kBlock / kStep; ++u) {                                                 \
        const int64_t e = first + u * kStep + threadIdx.x * kVec;                              \
        const int64_t rest = numel - e;                                                        \
        adamw_elements<P, G, B>(t, s, gs, decay, rate, e, rest > kVec ? kVec : (int)rest);     \
    }                                                                                          \
    break
    switch (kind) {
    case 0: DLCX_ADAMW_KIND(DLCX_F32, DLCX_F32, 32);
    case 1: DLCX_ADAMW_KIND(DLCX_BF16, DLCX_F32, 32);
    case 2: DLCX_ADAMW_KIND(DLCX_F32, DLCX_BF16, 32);
    case 3: DLCX_ADAMW_KIND(DLCX_BF16, DLCX_BF16, 32);
    case 4: DLCX_ADAMW_KIND(DLCX_F32, DLCX_F32, 8);
    case 5: DLCX_ADAMW_KIND(DLCX_BF16, DLCX_F32, 8);
    case 6: DLCX_ADAMW_KIND(DLCX_F32, DLCX_BF16, 8);
    default: DLCX_ADAMW_KIND(DLCX_BF16, DLCX_BF16, 8);
    }
#undef DLCX_ADAMW_KIND
}

// ---- global norm --------------------------------------------------------------------------------
// fp64 throughout: a square of fp32 has room there at any size, and the order of the sum no weight.
template <int DT>
__device__ __forceinline__ double sum_squares(const void *grad, int64_t first, int64_t numel, double acc) {
    float x[kBlock / kStep][kVec];
#pragma unroll
    for (int u = 0; u < kBlock / kStep; ++u) {
        const int64_t e = first + u * kStep + threadIdx.x * kVec, rest = numel - e;
        load_floats<DT>(grad, e, rest > kVec ? kVec : (int)(rest < 0 ? 0 : rest), x[u]);
    }
#pragma unroll
    for (int u = 0; u < kBlock / kStep; ++u)
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc = fma((double)x[u][i], (double)x[u][i], acc);
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
    const int64_t e = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kVec, rest = numel - e;
    if (rest <= 0) return;
    const int left = rest > kVec ? kVec : (int)rest;
    const ad_u32x2 w = load_codes(codes, e, left);
    const float scale = scales[e / kStateGroup];
    float x[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        x[i] = SECOND ? decode_v(w[i / 4], i & 3, scale) : decode_m(w[i / 4], i & 3, scale);
    store_floats<DT>(out, e, left, x);
}

// ---- launches -----------------------------------------------------------------------------------
int launch_tensor_table(const dlcx_tensor *t, int count, void *memory, dlcx_table *table,
                        hipStream_t st) {
    const TableView v = table_view(memory, count);
    int64_t blocks = 0;
    int steps = 1;
    for (int i = 0; i < count; ++i) {
        blocks += ceil_div(t[i].numel, kBlock);
        if (blocks > 0x7FFFFFFF) return DLCX_EINVAL;
        if (t[i].numel > 0 && t[i].param == nullptr) steps = 0;
    }
    table->memory = memory;
    table->blocks = blocks;
    table->count = count;
    table->steps = steps;
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

int launch_adamw(const dlcx_table &table, const AdamwStep &step, hipStream_t st) {
    if (table.blocks == 0) return DLCX_OK;
    const int64_t gx = table.blocks < (1 << 20) ? table.blocks : (1 << 20);
    Timed timed(KID_ADAMW, st);
    adamw_kernel<<<dim3((unsigned)gx, (unsigned)ceil_div(table.blocks, gx)), kThreads, 0, st>>>(
        table_view(table.memory, table.count), table.count, table.blocks, step);
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
    if (t.numel < 0 || t.reserved != 0) return DLCX_EINVAL;
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
    if (!(eps > 0) || !isfinite(eps) || !(grad_scale >= 0) || !isfinite(grad_scale)) return DLCX_EINVAL;
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
    if (ceil_div(numel, kStep) > 0x7FFFFF) return DLCX_EINVAL;
    return launch_state_decode(second, codes, scales, numel, out, out_dtype, as_stream(stream));
}

}  // extern "C"
