// y = y_in + x w^T for two matrices in 8 bits with a power of two for every 128 elements of a row.
//
// bf16 results: CDNA4's scaled matrix instruction multiplies 16 x 128 by 128 x 16 codes and applies a power of two to
// each operand's rows by itself, so sums of blocks with different scales stay in one fp32 accumulator and no vector
// instruction is spent on scales.  It adds eight products at a time after cutting each at 2^-13 of the largest of
// them (measured; the sums of eight are added in fp32): 1.5e-5 of a result of normal inputs, where rounding to bf16
// costs 1.7e-3.
// fp32 results: that would be most of the error, so the codes are widened to bf16 (exact: four significant bits),
// whose instruction keeps all of a product; a block's sum is scaled by an exponent's addition and added in fp32.
//
// w is the instructions' first operand and x the second: a lane then has four consecutive outputs of one row.
#include "eight.h"

namespace dlcx {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct ProductArgs {
    const uint8_t *x, *xs, *w, *ws;
    const void *y_in;
    void *y;
    float *part;  // splits x rows x m, or NULL: one split, which writes y
    int64_t ldx, ldxs, ldw, ldws, ldi, ldo;
    int rows, m, blocks;  // blocks: of 128 along the sum
    int per_split;        // of them, a multiple of 4
    int row_tiles, col_tiles;
};

// 16 bytes to a lane from global memory to LDS: lane l's at lds + 16 l.
__device__ __forceinline__ void load_lds16(const uint8_t *from, uint8_t *lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}

__device__ __forceinline__ i32x8 join(const i32x4 &a, const i32x4 &b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// Eight codes to bf16.
__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// c + the block's sum, whose scales' bytes add up to e
__device__ __forceinline__ f32x4 add_scaled(const f32x4 &c, const f32x4 &sum, const int (&ew)[4], int ex) {
    f32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = c[i] + __builtin_amdgcn_ldexpf(sum[i], ew[i] + ex - 254);
    return r;
}

template <int S>
__device__ __forceinline__ f32x4 scaled_mma(const i32x8 &a, const i32x8 &b, const f32x4 &c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, S, sa, S, sb);
}

// Four consecutive outputs of a row.
template <typename T>
__device__ __forceinline__ void put4(const ProductArgs &a, int64_t row, int64_t col, f32x4 v) {
    typedef typename T::elem elem;
    const int there = (int)min((int64_t)4, a.m - col);
    if (a.y_in) {
        const elem *p = (const elem *)a.y_in + row * a.ldi + col;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < there) v[i] += T::get(p[i]);
    }
    elem *p = (elem *)a.y + row * a.ldo + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < there) p[i] = T::put(v[i]);
}

// 128 x 128 outputs to a workgroup of four wavefronts, 64 x 64 to each.  Tiles of 128 rows x 128 bytes, twice, straight
// to LDS; the 16-byte pieces of a row lie at piece ^ (row & 7), so that eight rows' same piece lies in all banks.
// Rows past the end are read as the last one and not written.
template <typename T>
__global__ __launch_bounds__(256, 2) void product_kernel(ProductArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t s_tile[2][2][128 * 128];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row0 = (int64_t)(blockIdx.x % a.row_tiles) * 128, col0 = (int64_t)(blockIdx.x / a.row_tiles) * 128;
    const int split = blockIdx.y, first = split * a.per_split, last = min(first + a.per_split, a.blocks);
    const uint8_t *from[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = wave * 32 + i * 8 + (lane >> 3), piece = (lane & 7) ^ (r & 7);
        from[0][i] = a.w + min(col0 + r, (int64_t)a.m - 1) * a.ldw + piece * 16;
        from[1][i] = a.x + min(row0 + r, (int64_t)a.rows - 1) * a.ldx + piece * 16;
    }
    auto fetch = [&](int buf, int block) {
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int i = 0; i < 4; ++i) load_lds16(from[o][i] + (int64_t)block * 128, &s_tile[buf][o][(wave * 32 + i * 8) * 128]);
    };
    const int r16 = lane & 15, g = lane >> 4, wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    constexpr bool kWide = T::size == 4;      // fp32 results
    constexpr int kScaleRows = kWide ? 4 : 1;  // of w, to a lane: its outputs' or its operand's
    const uint8_t *sw[4][kScaleRows], *sx[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int e = 0; e < kScaleRows; ++e)
            sw[i][e] = a.ws + min(col0 + wm + i * 16 + (kWide ? g * 4 + e : r16), (int64_t)a.m - 1) * a.ldws;
        sx[i] = a.xs + min(row0 + wn + i * 16 + r16, (int64_t)a.rows - 1) * a.ldxs;
    }
    f32x4 acc[4][4] = {};
    int scale_w[4][kScaleRows], scale_x[4];
    auto step = [&](int buf, auto s) {
        i32x8 fw[4], fx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int rw = wm + i * 16 + r16, rx = wn + i * 16 + r16;
            const uint8_t *pw = &s_tile[buf][0][rw * 128], *px = &s_tile[buf][1][rx * 128];
            fw[i] = join(*(const i32x4 *)(pw + ((g ^ (rw & 7)) * 16)), *(const i32x4 *)(pw + (((g + 4) ^ (rw & 7)) * 16)));
            fx[i] = join(*(const i32x4 *)(px + ((g ^ (rx & 7)) * 16)), *(const i32x4 *)(px + (((g + 4) ^ (rx & 7)) * 16)));
        }
        constexpr int S = decltype(s)::value;
        if constexpr (kWide) {
            f32x4 sum[4][4] = {};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                bf16x8 bw[4], bx[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    bw[i] = widen(fw[i][2 * k], fw[i][2 * k + 1]);
                    bx[i] = widen(fx[i][2 * k], fx[i][2 * k + 1]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[i], bx[j], sum[i][j], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int ew[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) ew[e] = (scale_w[i][e] >> (8 * S)) & 255;
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = add_scaled(acc[i][j], sum[i][j], ew, (scale_x[j] >> (8 * S)) & 255);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = scaled_mma<S>(fw[i], fx[j], acc[i][j], scale_w[i][0], scale_x[j]);
        }
    };
    if (first < last) fetch(0, first);
    for (int block = first; block < last; block += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int e = 0; e < kScaleRows; ++e) scale_w[i][e] = *(const int *)(sw[i][e] + block);
            scale_x[i] = *(const int *)(sx[i] + block);
        }
        unrolled<4>([&](auto s) {
            constexpr int S = decltype(s)::value;
            if (block + S < last) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the tile is there ...
                __syncthreads();                                  // ... all of it, and the other one has been read
                if (block + S + 1 < last) fetch((S + 1) & 1, block + S + 1);
                step(S & 1, s);
            }
        });
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t row = row0 + wn + j * 16 + r16;
        if (row >= a.rows) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t col = col0 + wm + i * 16 + g * 4;
            if (col >= a.m) continue;
            if (a.part) {
                float *p = a.part + ((int64_t)split * a.rows + row) * a.m + col;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < a.m) p[e] = acc[i][j][e];
            } else {
                put4<T>(a, row, col, acc[i][j]);
            }
        }
    }
}

// y from the splits' sums, added in order.
template <typename T>
__global__ __launch_bounds__(256) void product_sum_kernel(ProductArgs a, int splits) {
    const int64_t quads = (a.m + 3) / 4, total = quads * a.rows;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        const int64_t row = at / quads, col = (at - row * quads) * 4;
        f32x4 v = {};
        for (int s = 0; s < splits; ++s) {
            const float *p = a.part + ((int64_t)s * a.rows + row) * a.m + col;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < a.m) v[e] += p[e];
        }
        put4<T>(a, row, col, v);
    }
}

struct ProductPlan {
    int splits, per_split;
};
// The sum is split where the tiles do not fill the GPU.
static ProductPlan product_plan(int64_t rows, int64_t m, int64_t n) {
    const int64_t tiles = ceil_div(rows, 128) * ceil_div(m, 128), blocks = ceil_div(n, 128);
    int64_t splits = 1;
    if (tiles < 512 && tiles > 0) splits = ceil_div(512, tiles);
    if (splits > blocks / 4) splits = blocks / 4;
    if (splits < 1) splits = 1;
    const int64_t per = (ceil_div(blocks, splits) + 3) / 4 * 4;
    return {(int)(blocks ? ceil_div(blocks, per) : 1), (int)per};
}

template <typename T>
static int launch_product(ProductArgs a, const ProductPlan &plan, hipStream_t st) {
    {
        Timed timed(KID_FP8_PRODUCT, st);
        product_kernel<T><<<dim3((unsigned)(a.row_tiles * (int64_t)a.col_tiles), plan.splits), 256, 0, st>>>(a);
        const int rc = check_launch("fp8_product");
        if (rc != DLCX_OK || plan.splits == 1) return rc;
    }
    const int64_t groups = ceil_div(ceil_div(a.m, 4) * a.rows, 256);
    Timed timed(KID_FP8_PRODUCT_SUM, st);
    product_sum_kernel<T><<<dim3((unsigned)(groups < kMostGroups ? groups : kMostGroups)), 256, 0, st>>>(a, plan.splits);
    return check_launch("fp8_product_sum");
}

}  // namespace dlcx

using namespace dlcx;

extern "C" {

static bool bad_product(int64_t rows, int64_t m, int64_t n) {
    return rows < 0 || rows > kMaxSide || m < 0 || m > kMaxSide || n < 0 || n > kMaxSide;
}

size_t dlcx_fp8_product_workspace_bytes(int64_t rows, int64_t m, int64_t n) {
    if (bad_product(rows, m, n)) return 0;
    size_t most = 0;  // of fewer rows, too: these may be split further
    for (int64_t tiles = 1; tiles <= ceil_div(rows, 128) && tiles <= 512; ++tiles) {
        const int64_t r = tiles * 128 < rows ? tiles * 128 : rows;
        const ProductPlan plan = product_plan(r, m, n);
        const size_t need = plan.splits > 1 ? (size_t)plan.splits * r * m * sizeof(float) : 0;
        if (need > most) most = need;
    }
    return a256x(most) + 256;
}

int dlcx_fp8_product(const dlcx_fp8 *x, const dlcx_fp8 *w, const void *y_in, int64_t ldy_in, void *y_out, int64_t ldy_out,
                     int dtype, void *workspace, void *stream) {
    if (check_fp8(x) != DLCX_OK || check_fp8(w) != DLCX_OK || x->cols != w->cols) return DLCX_EINVAL;
    if (dtype != DLCX_F32 && dtype != DLCX_BF16) return DLCX_EINVAL;
    if (x->rows == 0 || w->rows == 0) return DLCX_OK;
    if (bad_rows(y_out, ldy_out, w->rows, dtype) || (y_in && bad_rows(y_in, ldy_in, w->rows, dtype))) return DLCX_EINVAL;
    if ((y_in == y_out && ldy_in != ldy_out) || !workspace || off_by(workspace, 256)) return DLCX_EINVAL;
    const ProductPlan plan = product_plan(x->rows, w->rows, x->cols);
    ProductArgs a = {(const uint8_t *)x->codes, (const uint8_t *)x->scales, (const uint8_t *)w->codes, (const uint8_t *)w->scales,
                     y_in, y_out, plan.splits > 1 ? (float *)workspace : nullptr, x->ld, x->ldscale, w->ld, w->ldscale,
                     ldy_in, ldy_out, (int)x->rows, (int)w->rows, (int)ceil_div(x->cols, 128), plan.per_split,
                     (int)ceil_div(x->rows, 128), (int)ceil_div(w->rows, 128)};
    if ((int64_t)a.row_tiles * a.col_tiles >= kMostGroups) return DLCX_EUNSUPPORTED;
    return dtype == DLCX_BF16 ? launch_product<TypeBf16>(a, plan, as_stream(stream)) : launch_product<TypeF32>(a, plan, as_stream(stream));
}

}  // extern "C"
