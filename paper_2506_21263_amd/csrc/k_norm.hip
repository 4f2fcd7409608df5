// Root-mean-square norm of the rows of a matrix, with the residual's addition before it and an output in 8 bits
// behind it, and its gradient.
//
//   s = x + residual (as it is stored) ;  rstd = 1 / sqrt(mean s^2 + eps) ;  y = s rstd w
//   dx = dx_in + rstd (g - h mean(g h)),  g = dy w,  h = s rstd ;  dw = sum over rows of dy h
//
// Streams over the rows, bound by HBM.  Up to 8192 columns (and, where n is a multiple of eight, 16384, of bf16 32768;
// gradients of bf16 16384) a row is read once and held in the registers of its workgroup (a wavefront for short rows); longer
// rows, and rows of fewer than eight elements, are read twice.  Sums are fp32, in an order that hangs on n and, for dw, on
// the number of rows.
// 4133 x 8192 bf16 with residual, to 8 bits: 50 us (237 MB, 4.7 TB/s), gradient of 16384 x 8192 with residual 190 + 5 us
// (5.6 TB/s); fp32 with residual, 6000 x 6000, 113 us each way (5.1 TB/s), 6000 x 5999 126 and 117.
#include <algorithm>

#include "eight.h"

namespace dlcx {

struct NormArgs {
    const void *x, *residual, *weight;
    void *sum, *y;
    uint8_t *codes, *scales;
    float *rstd;
    int64_t ldx, ldr, ldsum, ldy, ld8, lds;
    int rows, n;
    float eps;
};

// The sum over the LANES lanes of a row's group, in all of them: LANES = 64, or a workgroup.
template <int LANES>
__device__ __forceinline__ float sum_lanes(float x, float *s_part) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int k = 0; k < LANES / 64; ++k) x += s_part[k];
    }
    return x;
}

// Codes from n on are zeros (in v they are NaN where rstd is not finite).
template <bool ENDS>
__device__ __forceinline__ void put_eight(const NormArgs &a, int64_t row, int col, const float (&v)[8], int lane) {
    const uint32_t s = scale_byte(max16(finite_max8(v)));
    uint2 c = codes8(v, scale_inverse(s));
    const int there = a.n - col;
    if (ENDS ? there < 8 : there <= 0) {
        const uint64_t keep = ENDS && there > 0 ? (1ull << (8 * there)) - 1 : 0;
        c.x &= (uint32_t)keep;
        c.y &= (uint32_t)(keep >> 32);
    }
    if (col < (a.n + 127) / 128 * 128) {
        *reinterpret_cast<uint2 *>(a.codes + row * a.ld8 + col) = c;
        if ((lane & 15) == 0) a.scales[row * a.lds + col / 128] = (uint8_t)s;
    }
}

// Floats between the parts of dw.
__host__ __device__ __forceinline__ int64_t part_pitch(int64_t n) { return (n + 7) / 8 * 8; }

// LANES to a row, each with CH times 8 elements of it; the next row is asked for before this one's sum is formed.
template <typename T, int LANES, int CH, bool ENDS>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_kernel(NormArgs a) {
    typedef typename T::elem elem;
    __shared__ float s_part[2][16];
    constexpr int kRows = LANES < 256 ? 256 / LANES : 1;
    const int lane = threadIdx.x % LANES;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    if (row >= a.rows) return;  // (a wavefront of its own: rows share workgroups only where no barrier is met)
    Raw8<T> w[CH], x[CH], r[CH];
    auto load = [&](Raw8<T>(&to)[CH], const void *p, int64_t at) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * LANES + lane) * 8;
            if (c < CH / 2) to[c].load((const elem *)p + at + col);  // (n is more than LANES * 4 * CH)
            else to[c].template load<ENDS>((const elem *)p + at + col, a.n - col);
        }
    };
    auto settle = [&](Raw8<T>(&x)[CH]) {
#pragma unroll
        for (int c = CH / 2; c < CH; ++c) x[c].template settle<ENDS>(a.n - (c * LANES + lane) * 8);
    };
    load(x, a.x, row * a.ldx);
    if (a.residual) load(r, a.residual, row * a.ldr);
    load(w, a.weight, 0);
    settle(w);
    for (int turn = 0;; turn ^= 1) {
        const int64_t next = row + stride;
        settle(x);
        if (a.residual) settle(r);
        float v[CH][8];
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * LANES + lane) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = x[c][i];
            if (a.residual) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] += r[c][i];
                round8<T>(v[c]);
                store8<T, ENDS>((elem *)a.sum + row * a.ldsum + col, a.n - col, v[c]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) ss += v[c][i] * v[c][i];
        }
        if (next < a.rows) {
            load(x, a.x, next * a.ldx);
            if (a.residual) load(r, a.residual, next * a.ldr);
        }
        ss = sum_lanes<LANES>(ss, s_part[turn]);
        const float rstd = 1.f / sqrtf(ss / (float)a.n + a.eps);
        if (a.rstd && lane == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * LANES + lane) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * rstd * w[c][i];
            if (a.y) store8<T, ENDS>((elem *)a.y + row * a.ldy + col, a.n - col, v[c]);
            if (a.codes) put_eight<ENDS>(a, row, col, v[c], lane);
        }
        if (next >= a.rows) break;
        row = next;
    }
}

// Rows of any length: read twice, the sum (where there is a residual) from where it was written by the same lane.
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
    typedef typename T::elem elem;
    __shared__ float s_part[16];
    const int lane = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const elem *x = (const elem *)a.x + row * a.ldx;
        elem *sum = (elem *)a.sum + row * a.ldsum;
        float ss = 0.f;
        for (int64_t col = lane * 8; col < a.n; col += 8192) {
            const int there = (int)min((int64_t)8, a.n - col);
            float v[8], r[8];
            load8<T>(x + col, there, v);
            if (a.residual) {
                load8<T>((const elem *)a.residual + row * a.ldr + col, there, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += r[i];
                round8<T>(v);
                store8<T>(sum + col, there, v);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) ss += v[i] * v[i];
        }
        ss = sum_lanes<1024>(ss, s_part);
        const float rstd = 1.f / sqrtf(ss / (float)a.n + a.eps);
        if (a.rstd && lane == 0) a.rstd[row] = rstd;
        const int64_t end = a.codes ? ((int64_t)a.n + 127) / 128 * 128 : a.n;  // (whole rows of 16 lanes)
        for (int64_t col = lane * 8; col < end; col += 8192) {
            const int there = (int)min((int64_t)8, a.n - col);
            float v[8], w[8];
            if (a.residual) load8<T>(sum + col, there, v);
            else load8<T>(x + col, there, v);
            load8<T>((const elem *)a.weight + col, there, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = v[i] * rstd * w[i];
            if (a.y) store8<T>((elem *)a.y + row * a.ldy + col, there, v);
            if (a.codes) put_eight<true>(a, row, (int)col, v, lane);
        }
        __syncthreads();
    }
}

constexpr int kMostLong = 1 << 20;  // workgroups of 1024 threads in a launch: 2^32 threads are too many

template <typename T, bool ENDS>
static void run_norm(const NormArgs &a, hipStream_t st) {
    // Workgroups: no more than the GPU holds at once, and rows shared out evenly.
    auto grid = [&a](int per, int most) { return dim3((unsigned)ceil_div(a.rows, per * ceil_div(a.rows, (int64_t)per * most))); };
    if (ENDS && a.n < 8) norm_long_kernel<T><<<grid(1, kMostLong), 1024, 0, st>>>(a);
    else if (a.n <= 512) norm_kernel<T, 64, 1, ENDS><<<grid(4, 2048), 256, 0, st>>>(a);
    else if (a.n <= 2048) norm_kernel<T, 256, 1, ENDS><<<grid(1, 2048), 256, 0, st>>>(a);
    else if (a.n <= 4096) norm_kernel<T, 256, 2, ENDS><<<grid(1, 1280), 256, 0, st>>>(a);
    else if (a.n <= 8192) norm_kernel<T, 512, 2, ENDS><<<grid(1, 768), 512, 0, st>>>(a);
    else if (!ENDS && a.n <= 16384) norm_kernel<T, 1024, 2, false><<<grid(1, 256), 1024, 0, st>>>(a);
    else if (T::size == 2 && !ENDS && a.n <= 32768) norm_kernel<TypeBf16, 1024, 4, false><<<grid(1, 256), 1024, 0, st>>>(a);
    else norm_long_kernel<T><<<grid(1, kMostLong), 1024, 0, st>>>(a);
}
template <typename T>
static int launch_norm(const NormArgs &a, hipStream_t st) {
    Timed timed(KID_RMS_NORM, st);
    if (a.n % 8) run_norm<T, true>(a, st);
    else run_norm<T, false>(a, st);
    return check_launch("rms_norm");
}

// ---- the gradient --------------------------------------------------------------------------------------
// A workgroup takes every gridDim'th row and keeps its part of dw in registers; the parts are added by a second
// kernel, in order.
struct NormGradArgs {
    const void *x, *weight, *dy, *dx_in;
    const float *rstd;
    void *dx;
    float *part, *dw, *dot;  // parts x n ; n ; rows (long rows)
    int64_t ldx, lddy, ldi, ldo;
    int rows, n, parts;
};

// Eight elements of a part of dw; a part that is all of it goes where it belongs.
__device__ __forceinline__ void put_part(const NormGradArgs &a, int part, int64_t col, const float (&dw)[8]) {
    if (a.parts == 1) {
        store8<TypeF32>(a.dw + col, (int)(a.n - col), dw);
        return;
    }
    float *p = a.part + (int64_t)part * part_pitch(a.n) + col;
    *reinterpret_cast<float4 *>(p) = make_float4(dw[0], dw[1], dw[2], dw[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(dw[4], dw[5], dw[6], dw[7]);
}

// A row's x and dy (and, where there are registers for it, dx_in) are asked for while the row before is worked on, so that
// neither the sum nor its barrier is waited for with nothing on its way; they stay packed until they are used.  Short rows
// have a wavefront each, whose parts of dw are added in LDS.
template <typename T, int LANES, int CH, bool ENDS>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_grad_kernel(NormGradArgs a) {
    typedef typename T::elem elem;
    constexpr int kRows = LANES < 256 ? 256 / LANES : 1;
    constexpr bool kAhead = CH == 1;
    __shared__ float s_part[2][16];
    __shared__ __attribute__((aligned(16))) float s_dw[kRows > 1 ? kRows * LANES * 8 : 4];
    const int lane = threadIdx.x % LANES;
    Raw8<T> w[CH], x[CH], dy[CH], r[CH];
    float dw[CH][8], rstd = 0.f;
    auto load = [&](Raw8<T>(&to)[CH], const void *p, int64_t at) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * LANES + lane) * 8;
            if (c < CH / 2) to[c].load((const elem *)p + at + col);  // (n is more than LANES * 4 * CH)
            else to[c].template load<ENDS>((const elem *)p + at + col, a.n - col);
        }
    };
    auto settle = [&](Raw8<T>(&x)[CH]) {
#pragma unroll
        for (int c = CH / 2; c < CH; ++c) x[c].template settle<ENDS>(a.n - (c * LANES + lane) * 8);
    };
    load(w, a.weight, 0);
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    if (row < a.rows) {
        load(x, a.x, row * a.ldx);
        load(dy, a.dy, row * a.lddy);
        if (kAhead && a.dx_in) load(r, a.dx_in, row * a.ldi);
        rstd = a.rstd[row];
    }
    settle(w);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = 0.f;
    for (int turn = 0; row < a.rows; turn ^= 1) {
        const int64_t next = row + stride;
        Raw8<T> nx[CH], ndy[CH], nr[CH];
        float nrstd = 0.f;
        if (!kAhead && a.dx_in) load(r, a.dx_in, row * a.ldi);
        if (next < a.rows) {
            load(nx, a.x, next * a.ldx);
            load(ndy, a.dy, next * a.lddy);
            if (kAhead && a.dx_in) load(nr, a.dx_in, next * a.ldi);
            nrstd = a.rstd[next];
        }
        settle(x);
        settle(dy);
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float h = x[c][i] * rstd;
                dw[c][i] += dy[c][i] * h;
                dot += dy[c][i] * w[c][i] * h;
            }
        dot = sum_lanes<LANES>(dot, s_part[turn]) / (float)a.n;  // (two places, so one barrier a row)
        if (a.dx_in) settle(r);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * LANES + lane) * 8;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = rstd * (dy[c][i] * w[c][i] - x[c][i] * rstd * dot);
                if (a.dx_in) v[i] += r[c][i];
            }
            store8<T, ENDS>((elem *)a.dx + row * a.ldo + col, a.n - col, v);
            x[c] = nx[c];
            dy[c] = ndy[c];
            if constexpr (kAhead) r[c] = nr[c];
        }
        row = next;
        rstd = nrstd;
    }
    if constexpr (kRows > 1) {
        const int wave = threadIdx.x / LANES;
#pragma unroll
        for (int i = 0; i < 8; ++i) s_dw[(wave * 8 + i) * LANES + lane] = dw[0][i];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < kRows; ++k) t += s_dw[(k * 8 + i) * LANES + lane];
            dw[0][i] = t;
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * LANES + lane) * 8;
        if (col < a.n) put_part(a, blockIdx.x, col, dw[c]);
    }
}

// Long rows: first mean(g h) of each ...
template <typename T>
__global__ __launch_bounds__(1024) void norm_dot_kernel(NormGradArgs a) {
    typedef typename T::elem elem;
    __shared__ float s_part[16];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float rstd = a.rstd[row];
        float dot = 0.f;
        for (int64_t col = threadIdx.x * 8; col < a.n; col += 8192) {
            const int there = (int)min((int64_t)8, a.n - col);
            float x[8], g[8], w[8];
            load8<T>((const elem *)a.x + row * a.ldx + col, there, x);
            load8<T>((const elem *)a.dy + row * a.lddy + col, there, g);
            load8<T>((const elem *)a.weight + col, there, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) dot += g[i] * w[i] * (x[i] * rstd);
        }
        dot = sum_lanes<1024>(dot, s_part) / (float)a.n;
        if (threadIdx.x == 0) a.dot[row] = dot;
        __syncthreads();
    }
}
// ... then columns: a workgroup has 2048 of them and every parts'th row.
template <typename T>
__global__ __launch_bounds__(256) void norm_grad_long_kernel(NormGradArgs a) {
    typedef typename T::elem elem;
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    const int there = (int)max((int64_t)0, min((int64_t)8, a.n - col));
    if (there == 0) return;
    float w[8], dw[8] = {};
    load8<T>((const elem *)a.weight + col, there, w);
    for (int64_t row = blockIdx.y; row < a.rows; row += a.parts) {
        const float rstd = a.rstd[row], dot = a.dot[row];
        float h[8], g[8], r[8] = {};
        load8<T>((const elem *)a.x + row * a.ldx + col, there, h);
        load8<T>((const elem *)a.dy + row * a.lddy + col, there, g);
        if (a.dx_in) load8<T>((const elem *)a.dx_in + row * a.ldi + col, there, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] *= rstd;
            dw[i] += g[i] * h[i];
            r[i] += rstd * (g[i] * w[i] - h[i] * dot);
        }
        store8<T>((elem *)a.dx + row * a.ldo + col, there, r);
    }
    put_part(a, blockIdx.y, col, dw);
}

// dw from its parts: 32 columns to a workgroup, 32 shares of the parts to them, eight parts at a time.
constexpr int kSumCols = 32;
__global__ __launch_bounds__(256) void norm_sum_kernel(const float *__restrict__ part, int parts, int n, float *__restrict__ dw) {
    __shared__ float4 s[32][9];
    const int c = threadIdx.x & 7, share = threadIdx.x >> 3;
    const int64_t col = (int64_t)blockIdx.x * kSumCols + c * 4, pitch = part_pitch(n);
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < n)
        for (int p = share; p < parts; p += 256) {
            float4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const float4 *>(part + min(p + 32 * k, parts - 1) * pitch + col);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool on = p + 32 * k < parts;
                t.x += on ? v[k].x : 0.f;
                t.y += on ? v[k].y : 0.f;
                t.z += on ? v[k].z : 0.f;
                t.w += on ? v[k].w : 0.f;
            }
        }
    s[share][c] = t;
    __syncthreads();
    if (share < 4) {  // (a component to each)
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) sum += reinterpret_cast<const float *>(&s[k][c])[share];
        if (col + share < n) dw[col + share] = sum;
    }
}

// Workgroups of the gradient, each with a part of dw: no more than the GPU holds at once, and rows shared out evenly.  Few
// rows are one's, which saves the second launch: a turn takes 0.7 us (8192 columns: 1.2), the launch 2 and the host 3.
static int64_t most_norm_parts(int64_t n) { return n <= 2048 ? 1024 : n <= 4096 ? 768 : n <= 8192 ? 512 : 256; }
static int norm_parts(int64_t rows, int64_t n) {
    const int64_t units = n >= 8 && n <= 512 ? ceil_div(rows, 4) : rows;  // (four rows to a workgroup)
    if (units <= (n <= 512 ? 4 : n <= 2048 ? 3 : n <= 8192 ? 2 : 1)) return units ? 1 : 0;
    const int64_t turns = ceil_div(units, most_norm_parts(n));
    return turns ? (int)ceil_div(units, turns) : 0;
}

template <typename T>
static void long_norm_grad(const NormGradArgs &a, hipStream_t st) {
    norm_dot_kernel<T><<<dim3((unsigned)(a.rows < kMostLong ? a.rows : kMostLong)), 1024, 0, st>>>(a);
    norm_grad_long_kernel<T><<<dim3((unsigned)ceil_div(a.n, 2048), (unsigned)a.parts), 256, 0, st>>>(a);
}
template <typename T, bool ENDS>
static void run_norm_grad(const NormGradArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)a.parts);
    if (ENDS && a.n < 8) long_norm_grad<T>(a, st);
    else if (a.n <= 512) norm_grad_kernel<T, 64, 1, ENDS><<<grid, 256, 0, st>>>(a);
    else if (a.n <= 2048) norm_grad_kernel<T, 256, 1, ENDS><<<grid, 256, 0, st>>>(a);
    else if (a.n <= 4096) norm_grad_kernel<T, 256, 2, ENDS><<<grid, 256, 0, st>>>(a);
    else if (a.n <= 8192) norm_grad_kernel<T, 512, 2, ENDS><<<grid, 512, 0, st>>>(a);
    else if (T::size == 2 && !ENDS && a.n <= 16384) norm_grad_kernel<TypeBf16, 1024, 2, false><<<grid, 1024, 0, st>>>(a);
    else long_norm_grad<T>(a, st);
}
template <typename T>
static int launch_norm_grad(const NormGradArgs &a, hipStream_t st) {
    {
        Timed timed(KID_RMS_NORM_GRAD, st);
        if (a.n % 8) run_norm_grad<T, true>(a, st);
        else run_norm_grad<T, false>(a, st);
        const int rc = check_launch("rms_norm_backward");
        if (rc != DLCX_OK || a.parts == 1) return rc;
    }
    Timed timed(KID_RMS_NORM_SUM, st);
    norm_sum_kernel<<<dim3((unsigned)ceil_div(a.n, kSumCols)), 256, 0, st>>>(a.part, a.parts, a.n, a.dw);
    return check_launch("rms_norm_sum");
}

}  // namespace dlcx

using namespace dlcx;

extern "C" {

static int check_norm(int64_t rows, int64_t n, int dtype) {
    if (rows < 0 || rows > kMaxSide || n < 1 || n > kMaxSide) return DLCX_EINVAL;
    return dtype == DLCX_F32 || dtype == DLCX_BF16 ? DLCX_OK : DLCX_EINVAL;
}

int dlcx_rms_norm(int64_t rows, int64_t n, int dtype, const void *x, int64_t ldx, const void *residual, int64_t ldr,
                  const void *weight, float eps, void *sum_out, int64_t ldsum, void *y_out, int64_t ldy,
                  const dlcx_fp8 *y8_out, float *rstd_out, void *stream) {
    if (check_norm(rows, n, dtype) != DLCX_OK || !(eps >= 0.f) || eps > 1e30f) return DLCX_EINVAL;
    if (y8_out && (check_fp8(y8_out) != DLCX_OK || y8_out->rows != rows || y8_out->cols != n)) return DLCX_EINVAL;
    if (rows == 0) return DLCX_OK;  // (tensors without elements have no address)
    if ((residual != nullptr) != (sum_out != nullptr) || (!y_out && !y8_out)) return DLCX_EINVAL;
    if (bad_rows(x, ldx, n, dtype) || !weight || off_by(weight, dtype == DLCX_BF16 ? 2 : 4) || off_by(rstd_out, 4)) return DLCX_EINVAL;
    if (residual && (bad_rows(residual, ldr, n, dtype) || bad_rows(sum_out, ldsum, n, dtype))) return DLCX_EINVAL;
    if (y_out && bad_rows(y_out, ldy, n, dtype)) return DLCX_EINVAL;
    if ((sum_out == x && sum_out && ldsum != ldx) || (sum_out == residual && sum_out && ldsum != ldr)) return DLCX_EINVAL;
    NormArgs a = {x, residual, weight, sum_out, y_out, nullptr, nullptr, rstd_out, ldx, ldr, ldsum, ldy, 0, 0, (int)rows, (int)n, eps};
    if (y8_out) {
        a.codes = (uint8_t *)y8_out->codes;
        a.scales = (uint8_t *)y8_out->scales;
        a.ld8 = y8_out->ld;
        a.lds = y8_out->ldscale;
    }
    return dtype == DLCX_BF16 ? launch_norm<TypeBf16>(a, as_stream(stream)) : launch_norm<TypeF32>(a, as_stream(stream));
}

size_t dlcx_rms_norm_workspace_bytes(int64_t rows, int64_t n) {
    if (check_norm(rows, n, DLCX_F32) != DLCX_OK) return 0;
    const int64_t parts = std::min(rows, most_norm_parts(n));  // (no fewer than of fewer rows)
    return a256x((size_t)parts * part_pitch(n) * sizeof(float)) + a256x(n > 8192 || n < 8 ? (size_t)rows * sizeof(float) : 0) + 256;
}

int dlcx_rms_norm_backward(int64_t rows, int64_t n, int dtype, const void *x, int64_t ldx, const void *weight,
                           const float *rstd, const void *dy, int64_t lddy, const void *dx_in, int64_t lddx_in,
                           void *dx_out, int64_t lddx_out, float *dw_out, void *workspace, void *stream) {
    if (check_norm(rows, n, dtype) != DLCX_OK) return DLCX_EINVAL;
    if (!dw_out || off_by(dw_out, 4) || !workspace || off_by(workspace, 256)) return DLCX_EINVAL;
    if (rows > 0) {
        if (bad_rows(x, ldx, n, dtype) || bad_rows(dy, lddy, n, dtype) || bad_rows(dx_out, lddx_out, n, dtype)) return DLCX_EINVAL;
        if (dx_in && bad_rows(dx_in, lddx_in, n, dtype)) return DLCX_EINVAL;
        if (!weight || off_by(weight, dtype == DLCX_BF16 ? 2 : 4) || !rstd || off_by(rstd, 4)) return DLCX_EINVAL;
        if ((dx_in == dx_out && lddx_in != lddx_out) || (dy == dx_out && lddy != lddx_out) || (x == dx_out && ldx != lddx_out))
            return DLCX_EINVAL;
    }
    NormGradArgs a = {x, weight, dy, dx_in, rstd, dx_out, (float *)workspace, dw_out, nullptr, ldx, lddy, lddx_in, lddx_out,
                      (int)rows, (int)n, norm_parts(rows, n)};
    a.dot = (float *)((char *)workspace + a256x((size_t)a.parts * part_pitch(n) * sizeof(float)));
    if (rows == 0) {
        Timed timed(KID_RMS_NORM_SUM, as_stream(stream));
        norm_sum_kernel<<<dim3((unsigned)ceil_div(n, kSumCols)), 256, 0, as_stream(stream)>>>(a.part, 0, a.n, dw_out);
        return check_launch("rms_norm_sum");
    }
    return dtype == DLCX_BF16 ? launch_norm_grad<TypeBf16>(a, as_stream(stream)) : launch_norm_grad<TypeF32>(a, as_stream(stream));
}

}  // extern "C"
