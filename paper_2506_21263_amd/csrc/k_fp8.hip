// A matrix to 8 bits with a power of two for every 128 elements of a row, and back.
//
// Both are streams, bound by HBM.  The quantiser takes tiles of 128 x 128: a lane holds 8 x 8 elements, sixteen
// lanes a row's 128 columns, so a row's largest is found among a row of lanes and a column's among the sixteen
// such rows of the workgroup; both layouts come from one reading of x.
// 16384 x 8192 of bf16 to both layouts: 129 us (4.2 TB/s; 537 MB, half of them written in two places), along the rows alone 86
// (4.7 TB/s), decoded 71 (5.7 TB/s); 28672 x 8192 of fp32 in squares, both ways, 281 (5.0 TB/s).
#include "eight.h"

namespace dlcx {

int check_fp8(const dlcx_fp8 *a) {
    if (!a || a->rows < 0 || a->rows > kMaxSide || a->cols < 0 || a->cols > kMaxSide) return DLCX_EINVAL;
    if (a->rows == 0 || a->cols == 0) return DLCX_OK;
    if (!a->codes || off_by(a->codes, 16) || !a->scales || off_by(a->scales, 4)) return DLCX_EINVAL;
    if (a->ld < code_pitch(a->cols) || a->ld % 16 || a->ld > kMaxRowStride) return DLCX_EINVAL;
    if (a->ldscale < scale_pitch(a->cols) || a->ldscale % 4 || a->ldscale > kMaxRowStride) return DLCX_EINVAL;
    return DLCX_OK;
}

struct QuantArgs {
    const void *x;
    int64_t ldx;
    int rows, cols, row_tiles, col_tiles;
    uint8_t *codes, *scales, *codes_t, *scales_t;
    int64_t ld, lds, ld_t, lds_t;
};

// The largest of the four lanes 16 apart, in all of them.
__device__ __forceinline__ uint32_t max_over_rows(uint32_t x) {
    x = max(x, (uint32_t)__shfl_xor((int)x, 16, 64));
    return max(x, (uint32_t)__shfl_xor((int)x, 32, 64));
}

// ROWS: codes along the rows; COLS: the transpose's; SQUARE: one scale for the tile.  Each XCD has a contiguous range of
// tiles, along the rows, so that the bytes of a line of scales meet in one L2.
// In LDS the transpose's 128 rows of 128 bytes have their 16-byte pieces at piece ^ (row / 8 & 7) and change places with
// the next row in the upper half, so that the lanes that write at once (rows eight apart) use all banks.
template <typename T, bool ROWS, bool COLS, bool SQUARE, bool ENDS>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t s_max[4 * 128];
    __shared__ __attribute__((aligned(16))) uint8_t s_t[COLS ? 128 * 128 : 16];
    const int tid = threadIdx.x, lane16 = tid & 15, part = tid >> 4, wave = tid >> 6;
    const int64_t total = (int64_t)a.row_tiles * a.col_tiles, share = (total + 7) / 8;
    for (int64_t id = blockIdx.x; id < share * 8; id += gridDim.x) {
        const int64_t tile = (id & 7) * share + (id >> 3);
        if (tile >= total) continue;
        const int tr = (int)(tile / a.col_tiles), tc = (int)(tile % a.col_tiles);
        const int row0 = tr * 128 + part * 8, col0 = tc * 128 + lane16 * 8;
        const int there = a.cols - col0;
        Raw8<T> raw[8];
        const typename T::elem *x = (const typename T::elem *)a.x + (int64_t)row0 * a.ldx + col0;
        if (!ENDS || a.cols >= 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[i].template load<ENDS>(x + i * a.ldx, row0 + i < a.rows ? there : 0);
            if constexpr (ENDS) {
#pragma unroll
                for (int i = 0; i < 8; ++i) raw[i].template settle<ENDS>(row0 + i < a.rows ? there : 0);
            }
        } else {  // (rows of fewer than eight elements)
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {
                float v[8];
                load8<T>(x + i * a.ldx, row0 + i < a.rows ? there : 0, v);
                Raw8<T> r;
#pragma unroll
                for (int k = 0; k < 2 * T::size; ++k)
                    r.w[k] = T::size == 4 ? __float_as_uint(v[k]) : __float_as_uint(v[2 * k & 7]) >> 16 | (__float_as_uint(v[2 * k + 1 & 7]) & 0xffff0000u);
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int k = 0; k < 2 * T::size; ++k) raw[n].w[k] = n == i ? r.w[k] : raw[n].w[k];
            }
        }
        // Elements stay packed between their uses: left to itself, the compiler keeps all of them unpacked, in 190 registers.
        auto packed = [&] {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int k = 0; k < 2 * T::size; ++k) asm volatile("" : "+v"(raw[i].w[k]));
        };
        auto row = [&](int i, float(&v)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = raw[i][j];
        };
        uint32_t shared = 0;
        if constexpr (SQUARE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v[8];
                row(i, v);
                shared = max(shared, finite_max8(v));
            }
            shared = max_over_rows(max16(shared));
            if ((tid & 63) == 0) s_max[wave] = shared;
            __syncthreads();
            shared = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
        }
        uint32_t top[8];  // of the columns
        if constexpr (COLS && !SQUARE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                top[j] = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) top[j] = max(top[j], finite_bits(raw[i][j]));
                top[j] = max_over_rows(top[j]);
            }
            if ((tid & 63) < 16) {
                uint4 *to = reinterpret_cast<uint4 *>(s_max + wave * 128 + lane16 * 8);
                to[0] = make_uint4(top[0], top[1], top[2], top[3]);
                to[1] = make_uint4(top[4], top[5], top[6], top[7]);
            }
        }
        if constexpr (ROWS) {
            packed();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v[8];
                row(i, v);
                const uint32_t s = scale_byte(SQUARE ? shared : max16(finite_max8(v)));
                const uint2 c = codes8(v, scale_inverse(s));
                if (row0 + i < a.rows) {
                    *reinterpret_cast<uint2 *>(a.codes + (int64_t)(row0 + i) * a.ld + col0) = c;
                    if (lane16 == 0) a.scales[(int64_t)(row0 + i) * a.lds + tc] = (uint8_t)s;
                }
            }
        }
        if constexpr (COLS) {
            packed();
            if constexpr (!SQUARE) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) top[j] = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint4 lo = *reinterpret_cast<const uint4 *>(s_max + k * 128 + lane16 * 8);
                    const uint4 hi = *reinterpret_cast<const uint4 *>(s_max + k * 128 + lane16 * 8 + 4);
                    const uint32_t m[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                    for (int j = 0; j < 8; ++j) top[j] = max(top[j], m[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t s = scale_byte(SQUARE ? shared : top[j]);
                float u[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = raw[i][j];
                const int c = lane16 * 8 + j;
                *reinterpret_cast<uint2 *>(s_t + (c ^ (lane16 >> 3)) * 128 + ((part >> 1) ^ (lane16 & 7)) * 16 + (part & 1) * 8) = codes8(u, scale_inverse(s));
                if (part == 0 && col0 + j < a.cols) a.scales_t[(int64_t)(col0 + j) * a.lds_t + tr] = (uint8_t)s;
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = k * 32 + (tid >> 3);
                const uint4 w = *reinterpret_cast<const uint4 *>(s_t + (c ^ (c >> 6)) * 128 + ((tid & 7) ^ (c >> 3 & 7)) * 16);
                if (tc * 128 + c < a.cols)
                    *reinterpret_cast<uint4 *>(a.codes_t + (int64_t)(tc * 128 + c) * a.ld_t + tr * 128 + (tid & 7) * 16) = w;
            }
        }
        if constexpr (COLS || SQUARE) __syncthreads();
    }
}

template <typename T, bool ROWS, bool COLS, bool SQUARE>
static void run_quantize(const QuantArgs &a, hipStream_t st) {
    const int64_t ids = ceil_div((int64_t)a.row_tiles * a.col_tiles, 8) * 8;
    const dim3 grid((unsigned)(ids < kMostGroups ? ids : kMostGroups));
    if (a.cols % 8) quantize_kernel<T, ROWS, COLS, SQUARE, true><<<grid, 256, 0, st>>>(a);
    else quantize_kernel<T, ROWS, COLS, SQUARE, false><<<grid, 256, 0, st>>>(a);
}
template <typename T>
static int launch_quantize8(const QuantArgs &a, bool rows, bool cols, bool square, hipStream_t st) {
    Timed timed(KID_FP8_QUANTIZE, st);
    if (square) {
        if (rows && cols) run_quantize<T, true, true, true>(a, st);
        else if (rows) run_quantize<T, true, false, true>(a, st);
        else run_quantize<T, false, true, true>(a, st);
    } else {
        if (rows && cols) run_quantize<T, true, true, false>(a, st);
        else if (rows) run_quantize<T, true, false, false>(a, st);
        else run_quantize<T, false, true, false>(a, st);
    }
    return check_launch("fp8_quantize");
}

struct DecodeArgs {
    const uint8_t *codes, *scales;
    int64_t ld, lds;
    void *out;
    int64_t ldo;
    int rows, cols, groups;  // groups: of 8 columns in a row
};

template <typename T>
__global__ __launch_bounds__(256) void decode_kernel(DecodeArgs a) {
    const int64_t total = (int64_t)a.rows * a.groups;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        const int64_t row = at / a.groups;
        const int g = (int)(at - row * a.groups);
        const uint2 c = *reinterpret_cast<const uint2 *>(a.codes + row * a.ld + g * 8);
        const float s = scale_value(a.scales[row * a.lds + g / 16]);
        typedef float v2 __attribute__((ext_vector_type(2)));
        const uint32_t w[2] = {c.x, c.y};
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const v2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
            v[4 * h] = lo[0] * s;
            v[4 * h + 1] = lo[1] * s;
            v[4 * h + 2] = hi[0] * s;
            v[4 * h + 3] = hi[1] * s;
        }
        store8<T>((typename T::elem *)a.out + row * a.ldo + g * 8, a.cols - g * 8, v);
    }
}

}  // namespace dlcx

using namespace dlcx;

extern "C" {

int64_t dlcx_fp8_code_pitch(int64_t cols) { return cols < 0 || cols > kMaxSide ? 0 : code_pitch(cols); }
int64_t dlcx_fp8_scale_pitch(int64_t cols) { return cols < 0 || cols > kMaxSide ? 0 : scale_pitch(cols); }

int dlcx_fp8_quantize(int64_t rows, int64_t cols, const void *x, int64_t ldx, int dtype, int square, const dlcx_fp8 *out,
                      const dlcx_fp8 *out_t, void *stream) {
    if (rows < 0 || rows > kMaxSide || cols < 0 || cols > kMaxSide) return DLCX_EINVAL;
    if ((dtype != DLCX_F32 && dtype != DLCX_BF16) || square < 0 || square > 1 || (!out && !out_t)) return DLCX_EINVAL;
    if (out && (check_fp8(out) != DLCX_OK || out->rows != rows || out->cols != cols)) return DLCX_EINVAL;
    if (out_t && (check_fp8(out_t) != DLCX_OK || out_t->rows != cols || out_t->cols != rows)) return DLCX_EINVAL;
    if (rows == 0 || cols == 0) return DLCX_OK;
    if (bad_rows(x, ldx, cols, dtype)) return DLCX_EINVAL;
    QuantArgs a = {};
    a.x = x;
    a.ldx = ldx;
    a.rows = (int)rows;
    a.cols = (int)cols;
    a.row_tiles = (int)ceil_div(rows, 128);
    a.col_tiles = (int)ceil_div(cols, 128);
    if (out) {
        a.codes = (uint8_t *)out->codes;
        a.scales = (uint8_t *)out->scales;
        a.ld = out->ld;
        a.lds = out->ldscale;
    }
    if (out_t) {
        a.codes_t = (uint8_t *)out_t->codes;
        a.scales_t = (uint8_t *)out_t->scales;
        a.ld_t = out_t->ld;
        a.lds_t = out_t->ldscale;
    }
    return dtype == DLCX_BF16 ? launch_quantize8<TypeBf16>(a, out, out_t, square, as_stream(stream))
                              : launch_quantize8<TypeF32>(a, out, out_t, square, as_stream(stream));
}

int dlcx_fp8_decode(const dlcx_fp8 *a, void *out, int64_t ldo, int out_dtype, void *stream) {
    if (check_fp8(a) != DLCX_OK || (out_dtype != DLCX_F32 && out_dtype != DLCX_BF16)) return DLCX_EINVAL;
    if (a->rows == 0 || a->cols == 0) return DLCX_OK;
    if (bad_rows(out, ldo, a->cols, out_dtype)) return DLCX_EINVAL;
    const DecodeArgs d = {(const uint8_t *)a->codes, (const uint8_t *)a->scales, a->ld, a->ldscale, out, ldo, (int)a->rows,
                          (int)a->cols, (int)ceil_div(a->cols, 8)};
    const int64_t blocks = ceil_div((int64_t)d.rows * d.groups, 256);
    const dim3 grid((unsigned)(blocks < kMostGroups ? blocks : kMostGroups));
    Timed timed(KID_FP8_DECODE, as_stream(stream));
    if (out_dtype == DLCX_BF16) decode_kernel<TypeBf16><<<grid, 256, 0, as_stream(stream)>>>(d);
    else decode_kernel<TypeF32><<<grid, 256, 0, as_stream(stream)>>>(d);
    return check_launch("fp8_decode");
}

}  // extern "C"
