// Dropout whose mask is computed where it is needed and never stored: y = y_in + x mask / (1 - p).
//
// Element i of the matrix (counted along the rows, whatever their strides) takes 16 bits of the Philox 4x32 block
// cipher with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): key = seed,
// counter = (i / 8, offset), the eight halves of the block from the lowest one up.  So the same call on the gradient
// has the same mask, and any launch shape gives the same bits.  Sixteen bits an element: p is rounded to a multiple
// of 2^-16, and what is kept is divided by 1 minus that multiple, so that the expectation is exact.  A stream with
// integer products beside it: 40 of them, quarter rate, for eight elements.  16384 x 8192 of bf16, added: 138 us, 5.8 TB/s.
#include "eight.h"

namespace dlcx {

struct DropArgs {
    const void *x, *y_in;
    void *y;
    const uint64_t *more;
    uint64_t seed, offset;
    int64_t ldx, ldi, ldo, rows, cols, groups;
    uint32_t threshold;  // dropped below
    float scale;
};

__device__ __forceinline__ uint4 philox(uint64_t counter, uint64_t offset, uint64_t seed) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// FLAT: no gaps between rows.  Else the eight elements of a group may lie in several rows.
template <typename T, bool FLAT>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs a) {
    typedef typename T::elem elem;
    const uint64_t offset = a.offset + (a.more ? *a.more : 0);
    const int64_t total = a.rows * a.cols;
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < a.groups; g += (int64_t)gridDim.x * 256) {
        const int there = (int)min((int64_t)8, total - g * 8);
        int64_t row = 0, col = g * 8;
        if constexpr (!FLAT) {
            row = col / a.cols;
            col -= row * a.cols;
        }
        const bool whole = FLAT || col + there <= a.cols;  // in one row
        float v[8], y[8] = {};
        if (whole) {
            load8<T>((const elem *)a.x + row * a.ldx + col, there, v);
            if (a.y_in) load8<T>((const elem *)a.y_in + row * a.ldi + col, there, y);
        } else {
            int64_t r = row, c = col;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = 0.f;
                if (i < there) {
                    v[i] = T::get(((const elem *)a.x)[r * a.ldx + c]);
                    if (a.y_in) y[i] = T::get(((const elem *)a.y_in)[r * a.ldi + c]);
                }
                if (++c == a.cols) c = 0, ++r;
            }
        }
        const uint4 w = philox((uint64_t)g, offset, a.seed);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = i & 1 ? word[i / 2] >> 16 : word[i / 2] & 0xffffu;
            y[i] = bits >= a.threshold ? y[i] + v[i] * a.scale : y[i];  // (a NaN that is dropped is gone)
        }
        if (whole) {
            store8<T>((elem *)a.y + row * a.ldo + col, there, y);
        } else {
            int64_t r = row, c = col;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i < there) ((elem *)a.y)[r * a.ldo + c] = T::put(y[i]);
                if (++c == a.cols) c = 0, ++r;
            }
        }
    }
}

template <typename T>
static int launch_dropout(const DropArgs &a, bool flat, hipStream_t st) {
    const int64_t blocks = ceil_div(a.groups, 256);
    const dim3 grid((unsigned)(blocks < kMostGroups ? blocks : kMostGroups));
    Timed timed(KID_DROPOUT, st);
    if (flat) dropout_kernel<T, true><<<grid, 256, 0, st>>>(a);
    else dropout_kernel<T, false><<<grid, 256, 0, st>>>(a);
    return check_launch("dropout");
}

}  // namespace dlcx

using namespace dlcx;

extern "C" int dlcx_dropout(int64_t rows, int64_t cols, int dtype, const void *x, int64_t ldx, const void *y_in,
                            int64_t ldy_in, void *y_out, int64_t ldy_out, double p, uint64_t seed, uint64_t offset,
                            const uint64_t *offset_more, void *stream) {
    if (rows < 0 || rows > kMaxSide || cols < 0 || cols > kMaxSide || (dtype != DLCX_F32 && dtype != DLCX_BF16)) return DLCX_EINVAL;
    if (!(p >= 0.0 && p < 1.0) || off_by(offset_more, 8)) return DLCX_EINVAL;
    const uint32_t threshold = (uint32_t)__builtin_nearbyint(p * 65536.0);
    if (threshold > 65535) return DLCX_EINVAL;  // nothing would be left
    if (rows == 0 || cols == 0) return DLCX_OK;
    if (bad_rows(x, ldx, cols, dtype) || bad_rows(y_out, ldy_out, cols, dtype)) return DLCX_EINVAL;
    if (y_in && bad_rows(y_in, ldy_in, cols, dtype)) return DLCX_EINVAL;
    if ((x == y_out && ldx != ldy_out) || (y_in == y_out && ldy_in != ldy_out)) return DLCX_EINVAL;
    const DropArgs a = {x, y_in, y_out, offset_more, seed, offset, ldx, ldy_in, ldy_out, rows, cols, ceil_div(rows * cols, 8),
                        threshold, (float)(65536.0 / (65536.0 - threshold))};
    const bool flat = rows == 1 || (ldx == cols && ldy_out == cols && (!y_in || ldy_in == cols));
    return dtype == DLCX_BF16 ? launch_dropout<TypeBf16>(a, flat, as_stream(stream))
                              : launch_dropout<TypeF32>(a, flat, as_stream(stream));
}
