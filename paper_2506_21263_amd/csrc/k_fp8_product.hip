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
#include <algorithm>

#include "eight.h"

namespace dlcx {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
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

// Eight codes to bf16, times a power of two.
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float scale = 1.f) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Where all scales of a quad are from 2^-63 to 2^64, they are applied as the codes are widened (bf16 has the exponents of
// fp32, so that is exact, too) and blocks add up in one accumulator.  The smallest product is then 2^-144, and the matrix
// cores keep what is below fp32's normal range, down to its last bit of 2^-149.  `outside` collects the quad's dwords: bit 7 of a byte from 64 to 191 differs from bit 6.
__device__ __forceinline__ uint32_t outside(int scales) { return ~((uint32_t)scales ^ (uint32_t)scales << 1) & 0x80808080u; }
// true for the whole wavefront if none of the first `count` blocks' scales is outside
__device__ __forceinline__ bool all_inside(uint32_t collected, int count) {
    const uint32_t valid = count >= 4 ? 0xffffffffu : (1u << 8 * count) - 1u;
    return __ballot((collected & valid) != 0) == 0;
}
template <int S>
__device__ __forceinline__ float scale_of(int scales) { return __uint_as_float(((uint32_t)scales >> (8 * S) & 255u) << 23); }
// c + the block's sum, whose scales' bytes are ew and ex (the scaled instruction takes 255 for NaN by itself)
__device__ __forceinline__ f32x4 add_scaled(const f32x4 &c, const f32x4 &sum, const int (&ew)[4], int ex) {
    f32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float scaled = __builtin_amdgcn_ldexpf(sum[i], ew[i] + ex - 254);
        r[i] = c[i] + (max(ew[i], ex) == (int)kScaleNan ? __builtin_nanf("") : scaled);
    }
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
    struct __attribute__((packed, aligned(T::size))) Four { elem e[4]; };
    const int there = (int)min((int64_t)4, a.m - col);
    const elem *in = (const elem *)a.y_in + row * a.ldi + col;
    elem *out = (elem *)a.y + row * a.ldo + col;
    if (there == 4) {
        if (a.y_in) {
            const Four f = *(const Four *)in;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += T::get(f.e[i]);
        }
        Four f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f.e[i] = T::put(v[i]);
        *(Four *)out = f;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < there) out[i] = T::put(a.y_in ? v[i] + T::get(in[i]) : v[i]);
}
// Partial sums of a split, rows padded to a multiple of four.
__device__ __forceinline__ int64_t part_pitch(int m) { return (m + 3) / 4 * 4; }
__device__ __forceinline__ void put_part(const ProductArgs &a, int64_t split, int64_t row, int64_t col, const f32x4 &v) {
    *(f32x4 *)(a.part + (split * a.rows + row) * part_pitch(a.m) + col) = v;
}

struct TilePlace {
    int row, col;
};
// The tile of workgroup `id`.  Consecutive ones go to different XCDs: each XCD gets a contiguous range of tiles, in
// groups of `group` rows of tiles, whose operands its L2 holds.
__device__ __forceinline__ TilePlace tile_place(int id, int row_tiles, int col_tiles, int group) {
    const int total = row_tiles * col_tiles, share = total / 8, more = total % 8, xcd = id & 7;
    const int t = xcd * share + min(xcd, more) + (id >> 3);
    const int per = group * col_tiles, first = t / per * group, rows = min(group, row_tiles - first), in = t % per;
    return {__builtin_amdgcn_readfirstlane(first + in % rows), __builtin_amdgcn_readfirstlane(in / rows)};
}

// A wavefront's 64 x 16 FN outputs and one block of 128: lane r16 has row r16 of each 16 of w's (from pw) and x's (from px) in
// LDS, pieces of 16 bytes at p0 and p1; S: the byte of their scales.
template <int S, int FN>
__device__ __forceinline__ void multiply_scaled(const uint8_t *pw, const uint8_t *px, int p0, int p1, const int (&scale_w)[4],
                                                const int (&scale_x)[FN], f32x4 (&acc)[4][FN]) {
    i32x8 fw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) fw[i] = join(*(const i32x4 *)(pw + i * 2048 + p0), *(const i32x4 *)(pw + i * 2048 + p1));
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const i32x8 fx = join(*(const i32x4 *)(px + j * 2048 + p0), *(const i32x4 *)(px + j * 2048 + p1));
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = scaled_mma<S>(fw[i], fx, acc[i][j], scale_w[i], scale_x[j]);
    }
}
// The same of widened codes, scaled as they are widened.  TIGHT: half of them at a time (two wavefronts to a SIMD have no
// registers for more).  Two conversions (128 rows; three: 64) of four cycles come to a matrix instruction of sixteen, 3.3 vector
// instructions with all others, and the two hardly overlap: 8192 x 8192 x 4096 takes 577 us (0.95 PFLOP/s) in tiles of 128 rows,
// 46 % of a SIMD's cycles matrix instructions and 38 % others; 659 us in tiles of 64.
template <int S, int FN, bool TIGHT = false>
__device__ __forceinline__ void multiply_widened(const uint8_t *pw, const uint8_t *px, int p0, int p1, const int (&scale_w)[4],
                                                 const int (&scale_x)[FN], f32x4 (&acc)[4][FN]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = h ? p1 : p0;
        bf16x8 bw[4][2];
        if (TIGHT) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const i32x4 f = *(const i32x4 *)(pw + i * 2048 + at);
            bw[i][0] = widen(f[0], f[1], scale_of<S>(scale_w[i]));
            bw[i][1] = widen(f[2], f[3], scale_of<S>(scale_w[i]));
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const i32x4 f = *(const i32x4 *)(px + j * 2048 + at);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bf16x8 bx = widen(f[2 * k], f[2 * k + 1], scale_of<S>(scale_x[j]));
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[i][k], bx, acc[i][j], 0, 0, 0);
            }
        }
    }
    if (!TIGHT) {
        __builtin_amdgcn_sched_group_barrier(0x100, 8 + 2 * FN, 0);  // all reads, the first half of w widened, ...
        __builtin_amdgcn_sched_group_barrier(0x002, 28, 0);
#pragma unroll
        for (int k = 0; k < 16 * FN; ++k) {  // ... and the rest between the products
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
        }
    }
}
// The same of scales that bf16 does not hold: a block's sum is scaled.
template <int S, int FN>
__device__ __forceinline__ void multiply_apart(const uint8_t *pw, const uint8_t *px, int p0, int p1, const int (&scale_w)[4],
                                               const int (&scale_x)[FN], f32x4 (&acc)[4][FN]) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        asm volatile("" ::: "memory");  // (else x's columns stay in registers from one i to the next)
        const i32x8 fw = join(*(const i32x4 *)(pw + i * 2048 + p0), *(const i32x4 *)(pw + i * 2048 + p1));
        int ew[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) ew[e] = (__shfl(scale_w[i], g * 4 + e, 64) >> (8 * S)) & 255;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const i32x8 fx = join(*(const i32x4 *)(px + j * 2048 + p0), *(const i32x4 *)(px + j * 2048 + p1));
            f32x4 sum = {};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(fw[2 * k], fw[2 * k + 1]), widen(fx[2 * k], fx[2 * k + 1]), sum, 0, 0, 0);
            acc[i][j] = add_scaled(acc[i][j], sum, ew, (scale_x[j] >> (8 * S)) & 255);
        }
    }
}

// ---- tiles --------------------------------------------------------------------------------------------
// 128 columns x 32 FN rows of outputs to a workgroup of four wavefronts, 64 x 16 FN to each.  128 bytes of the tile's
// rows at a time, twice, straight to LDS; the 16-byte pieces of a row lie at piece ^ (row & 7), so that what is read at
// once lies in all banks.  Rows past the end are read as the last one and not written.
template <typename T, int FN>
__global__ __launch_bounds__(256, 2) void product_kernel(ProductArgs a) {
    constexpr int kRows = 32 * FN, kStage = (128 + kRows) * 128, kFetchX = kRows / 32;
    constexpr bool kWiden = T::size == 4;  // fp32 results
    // (Widened, two workgroups to a compute unit are 3 - 5 % faster than the three that would fit: 2048^3 26.0 us, not 27.0.)
    __shared__ __attribute__((aligned(16))) uint8_t s_tile[kWiden && 2 * kStage < 56 * 1024 ? 56 * 1024 : 2 * kStage];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const TilePlace place = tile_place(blockIdx.x, a.row_tiles, a.col_tiles, 8);
    const int64_t row0 = (int64_t)place.row * kRows, col0 = (int64_t)place.col * 128;
    const int split = blockIdx.y, first = split * a.per_split, last = min(first + a.per_split, a.blocks);
    const uint8_t *from_w[4], *from_x[kFetchX];
    const int piece = (lane & 7) ^ (lane >> 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) from_w[i] = a.w + min(col0 + wave * 32 + i * 8 + (lane >> 3), (int64_t)a.m - 1) * a.ldw + piece * 16;
#pragma unroll
    for (int i = 0; i < kFetchX; ++i)
        from_x[i] = a.x + min(row0 + (wave * kFetchX + i) * 8 + (lane >> 3), (int64_t)a.rows - 1) * a.ldx + piece * 16;
    auto fetch = [&](int buf, int block) {
        uint8_t *to = s_tile + buf * kStage;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_lds16(from_w[i] + (int64_t)block * 128, to + (wave * 4 + i) * 1024);
#pragma unroll
        for (int i = 0; i < kFetchX; ++i) load_lds16(from_x[i] + (int64_t)block * 128, to + 128 * 128 + (wave * kFetchX + i) * 1024);
    };
    const int r16 = lane & 15, g = lane >> 4, wm = (wave & 1) * 64, wn = (wave >> 1) * 16 * FN;
    const uint8_t *sw[4], *sx[FN];
#pragma unroll
    for (int i = 0; i < 4; ++i) sw[i] = a.ws + min(col0 + wm + i * 16 + r16, (int64_t)a.m - 1) * a.ldws;
#pragma unroll
    for (int j = 0; j < FN; ++j) sx[j] = a.xs + min(row0 + wn + j * 16 + r16, (int64_t)a.rows - 1) * a.ldxs;
    const int p0 = (g ^ (lane & 7)) * 16, p1 = ((g + 4) ^ (lane & 7)) * 16;
    f32x4 acc[4][FN] = {};
    int scale_w[4], scale_x[FN], next_w[4], next_x[FN];
    auto fetch_scales = [&](int block) {
#pragma unroll
        for (int i = 0; i < 4; ++i) next_w[i] = *(const int *)(sw[i] + block);
#pragma unroll
        for (int j = 0; j < FN; ++j) next_x[j] = *(const int *)(sx[j] + block);
    };
    bool inside = false;
    auto step = [&](int buf, auto s) {
        constexpr int S = decltype(s)::value;
        const uint8_t *pw = s_tile + buf * kStage + (wm + r16) * 128, *px = s_tile + buf * kStage + (128 + wn + r16) * 128;
        if constexpr (kWiden) {
            if (inside) multiply_widened<S, FN, FN == 4>(pw, px, p0, p1, scale_w, scale_x, acc);
            else multiply_apart<S, FN>(pw, px, p0, p1, scale_w, scale_x, acc);
        } else {
            multiply_scaled<S, FN>(pw, px, p0, p1, scale_w, scale_x, acc);
        }
    };
    if (first < last) {
        fetch_scales(first);
        fetch(0, first);
    }
    for (int block = first; block < last; block += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) scale_w[i] = next_w[i];
#pragma unroll
        for (int j = 0; j < FN; ++j) scale_x[j] = next_x[j];
        if constexpr (kWiden) {
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) bad |= outside(scale_w[i]);
#pragma unroll
            for (int j = 0; j < FN; ++j) bad |= outside(scale_x[j]);
            inside = all_inside(bad, last - block);
        }
        unrolled<4>([&](auto s) {
            constexpr int S = decltype(s)::value;
            if (block + S < last) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the tile is there ...
                __syncthreads();                                  // ... all of it, and the other one has been read
                if (block + S + 1 < last) fetch((S + 1) & 1, block + S + 1);
                if (S == 0 && block + 4 < last) fetch_scales(block + 4);
                step(S & 1, s);
            }
        });
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t row = row0 + wn + j * 16 + r16;
        if (row >= a.rows) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t col = col0 + wm + i * 16 + g * 4;
            if (col >= a.m) continue;
            if (a.part) put_part(a, split, row, col, acc[i][j]);
            else put4<T>(a, row, col, acc[i][j]);
        }
    }
}

// ---- large products with bf16 results -----------------------------------------------------------------
// 256 x 256 outputs to a workgroup of four wavefronts, one to a SIMD, 128 x 128 to each in 32 x 32 x 64 products: the
// accumulators take 256 of its registers, a half stage's operands 64 and the next half's 64 more.  A stage is 512 rows
// of 128 bytes, straight to LDS, two of them; a row's 16-byte pieces lie at piece ^ (row / 2 & 7), so that the sixteen
// lanes that read at once hit all banks.  One barrier a stage, in its middle: from there on its operands are in
// registers, so its place is fetched anew while the second half is multiplied, and the next stage is there to be read.
// Scales go through LDS, too (four stages' to a dword), so that not every lane that needs one asks the cache for it.  Results leave through LDS as whole lines.  Edge tiles are moved inside the matrix and write
// only what is theirs, so no address is checked.
// 16384 x 8192 x 8192: 0.87 ms, 2.5 PFLOP/s (1.44 ms with 128 x 128 tiles): matrix cores are at work 62 % of the cycles, 13 %
// of a wavefront's are waits, and the clock is at 1.8 GHz; 8192^3 0.41 - 0.44 ms.  Added to y_in, which comes 8 bytes a lane: 0.93.
constexpr int kWideTile = 256, kWideStage = 512 * 128, kWideLds = 2 * kWideStage + 2 * 2048;

typedef __attribute__((address_space(3))) uint8_t lds_byte;
template <typename V>
__device__ __forceinline__ V lds_read(uint32_t at) { return *(const __attribute__((address_space(3))) V *)(uintptr_t)at; }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void *p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, -1, 0x00020000);
}
// 16 or 4 bytes to a lane from a buffer to LDS, lane after lane.
__device__ __forceinline__ void fetch_lds16(__amdgpu_buffer_rsrc_t from, uint8_t *to, uint32_t lane_at, uint32_t at) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)(lds_byte *)to, 16, lane_at, at, 0, 0);
}
__device__ __forceinline__ void fetch_lds4(__amdgpu_buffer_rsrc_t from, uint8_t *to, uint32_t lane_at, uint32_t at) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)(lds_byte *)to, 4, lane_at, at, 0, 0);
}

template <bool ADD>
__global__ __launch_bounds__(256, 1) void product_wide_kernel(ProductArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t s_wide[];
    uint8_t *const s_scale = s_wide + 2 * kWideStage;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const TilePlace place = tile_place(blockIdx.x, a.row_tiles, a.col_tiles, 4);
    const int row0 = min(place.row * kWideTile, a.rows - kWideTile), col0 = min(place.col * kWideTile, a.m - kWideTile);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte *)s_wide;
    const auto from_w = buffer_at(a.w + col0 * a.ldw), from_x = buffer_at(a.x + row0 * a.ldx);
    const bool of_w = wave < 2;  // whose scales this wavefront fetches, 128 rows
    const auto from_s = buffer_at(of_w ? a.ws + col0 * a.ldws : a.xs + row0 * a.ldxs);
    const uint32_t pitch_s = (uint32_t)(of_w ? a.ldws : a.ldxs), lane_s = ((wave & 1) * 128 + lane) * pitch_s;
    uint32_t lane_w[2], lane_x[2];  // 64 rows of either operand to a wavefront, eight to a load
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        const uint32_t r = wave * 64 + o * 8 + (lane >> 3), piece = ((lane & 7) ^ (o * 4 + (lane >> 4))) * 16;
        lane_w[o] = r * (uint32_t)a.ldw + piece;
        lane_x[o] = r * (uint32_t)a.ldx + piece;
    }
    const uint32_t w16 = (uint32_t)a.ldw * 16, x16 = (uint32_t)a.ldx * 16;
    auto fetch = [&](int buf, int block, int i) {
        uint8_t *to = s_wide + buf * kWideStage + (wave * 8 + (i & 7)) * 1024;
        if (i < 8) fetch_lds16(from_w, to, lane_w[i & 1], block * 128 + (i >> 1) * w16);
        else fetch_lds16(from_x, to + 256 * 128, lane_x[i & 1], block * 128 + ((i - 8) >> 1) * x16);
    };
    auto fetch_scales = [&](int buf, int block, int i) {
        fetch_lds4(from_s, s_scale + buf * 2048 + (wave * 2 + i) * 256, lane_s, block + i * 64 * pitch_s);
    };
    const int r32 = lane & 31, g = lane >> 5, wm = (wave & 1) * 128, wn = (wave >> 1) * 128;
    uint32_t at_w[2][2][2], at_x[2][2][2];  // buffer, half, piece
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const uint32_t piece = ((4 * h + 2 * g + p) ^ ((r32 >> 1) & 7)) * 16;
                at_w[b][h][p] = lds0 + b * kWideStage + (wm + r32) * 128 + piece;
                at_x[b][h][p] = lds0 + b * kWideStage + (256 + wn + r32) * 128 + piece;
                asm volatile("" : "+v"(at_w[b][h][p]), "+v"(at_x[b][h][p]));  // (kept, with offsets in the reads)
            }
    uint32_t at_sw = lds0 + 2 * kWideStage + (wm + r32) * 4, at_sx = lds0 + 2 * kWideStage + (256 + wn + r32) * 4;
    asm volatile("" : "+v"(at_sw), "+v"(at_sx));
    auto read_w = [&](int b, int h, int i) { return join(lds_read<i32x4>(at_w[b][h][0] + i * 4096), lds_read<i32x4>(at_w[b][h][1] + i * 4096)); };
    auto read_x = [&](int b, int h, int i) { return join(lds_read<i32x4>(at_x[b][h][0] + i * 4096), lds_read<i32x4>(at_x[b][h][1] + i * 4096)); };

    const int last = a.blocks - 1;
    f32x16 acc[4][4] = {};
    int scale_w[4], scale_x[4], next_w[4], next_x[4];
    i32x8 fw[2][4], fx[2][4];
    fetch_scales(0, 0, 0);
    fetch_scales(0, 0, 1);
#pragma unroll
    for (int i = 0; i < 16; ++i) fetch(0, 0, i);
#pragma unroll
    for (int i = 0; i < 16; ++i) fetch(1, min(1, last), i);
    asm volatile("s_waitcnt vmcnt(16)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        fw[0][i] = read_w(0, 0, i);
        fx[0][i] = read_x(0, 0, i);
        scale_w[i] = next_w[i] = lds_read<int>(at_sw + i * 128);
        scale_x[i] = next_x[i] = lds_read<int>(at_sx + i * 128);
    }
    // Four matrix instructions' worth of issue between reads and fetches is given, not found: the compiler would put
    // them all in front.  (masks: 8 matrix, 0x100 LDS reads, 0x20 loads)
    auto step = [&](auto s, int block, int scales) {
        constexpr int S = decltype(s)::value, B = S & 1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fx[1][i] = read_x(B, 1, i);
            fw[1][i] = read_w(B, 1, i);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw[0][i], fx[0][j], acc[i][j], 0, 0, S, scale_w[i], S, scale_x[j]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            __builtin_amdgcn_sched_group_barrier(8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(8, 8, 0);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        const int next = min(block + S + 2, last);  // (past the last one it comes again, and is not used)
        if constexpr (S == 0) {
            fetch_scales(scales ^ 1, min(block + 4, last & ~3), 0);
            fetch_scales(scales ^ 1, min(block + 4, last & ~3), 1);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fx[0][i] = read_x(B ^ 1, 0, i);
            fw[0][i] = read_w(B ^ 1, 0, i);
        }
        if constexpr (S == 3) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                next_w[i] = lds_read<int>(at_sw + (scales ^ 1) * 2048 + i * 128);
                next_x[i] = lds_read<int>(at_sx + (scales ^ 1) * 2048 + i * 128);
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) fetch(B, next, i);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw[1][i], fx[1][j], acc[i][j], 0, 0, S, scale_w[i], S, scale_x[j]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            __builtin_amdgcn_sched_group_barrier(8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            __builtin_amdgcn_sched_group_barrier(8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x20, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(8, 4, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    int block = 0, scales = 0;
    for (; block + 4 <= a.blocks; block += 4, scales ^= 1) {
        unrolled<4>([&](auto s) { step(s, block, scales); });
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            scale_w[i] = next_w[i];
            scale_x[i] = next_x[i];
        }
    }
    if (block < a.blocks) step(std::integral_constant<int, 0>(), block, scales);
    if (block + 1 < a.blocks) step(std::integral_constant<int, 1>(), block, scales);
    if (block + 2 < a.blocks) step(std::integral_constant<int, 2>(), block, scales);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");  // no stage is on its way or read any more

    // A wavefront's 128 rows of x by 128 columns, rows of 256 bytes in its own quarter of the stages.
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const uint32_t mine = lds0 + wave * 32768;
    const int keep_row = place.row * kWideTile, keep_col = place.col * kWideTile;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = j * 32 + r32, piece = i * 4 + q;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
                if constexpr (ADD) {
                    const uint16_t *p = (const uint16_t *)a.y_in + (int64_t)(row0 + wn + r) * a.ldi + col0 + wm + piece * 8 + g * 4;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += TypeBf16::get(p[e]);
                }
                *(__attribute__((address_space(3))) u32x2 *)(uintptr_t)(mine + r * 256 + ((piece ^ (r32 & 15)) * 16) + g * 8) =
                    u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 8
    for (int k = 0; k < 32; ++k) {
        const int r = k * 4 + (lane >> 4), piece = lane & 15, row = row0 + wn + r, col = col0 + wm + piece * 8;
        const i32x4 v = lds_read<i32x4>(mine + r * 256 + ((piece ^ (r & 15)) * 16));
        uint16_t *to = (uint16_t *)a.y + (int64_t)row * a.ldo + col;
        if (row >= keep_row && col >= keep_col) {
            Loose16 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w.w[e] = (uint32_t)v[e];
            *reinterpret_cast<Loose16 *>(to) = w;
        } else if (row >= keep_row) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e >= keep_col) to[e] = (uint16_t)((uint32_t)v[e / 2] >> (16 * (e & 1)));
        }
    }
}

// ---- few rows -------------------------------------------------------------------------------------------
// w is read once and straight into registers; what bounds this is HBM, or the launch.  Sixteen rows of w to a
// wavefront; the sum is cut into quads of four blocks (whose scales are one dword), two of them on their way.
//
// A lane's part of a 16 x 128 operand: 16 bytes at 16 g and 16 at 64 + 16 g of its row (the order of a sum's terms
// is free, as long as both operands have it).
struct Quad {
    i32x4 lo[4], hi[4];
    int scale;
};
// Blocks `block` .. `block` + 3 of a row, none past the last one (which comes again, and is not used).
__device__ __forceinline__ void load_quad(Quad &q, const uint8_t *row, const uint8_t *scales, int block, int last) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint8_t *p = row + (int64_t)min(block + k, last) * 128;
        q.lo[k] = *(const i32x4 *)p;
        q.hi[k] = *(const i32x4 *)(p + 64);
    }
    q.scale = *(const int *)(scales + block);
}

// acc + w x^T for one block of 128; S: the byte of the scales.  ew: the scales of the lane's four outputs' rows (fp32).
template <typename T, int S>
__device__ __forceinline__ f32x4 block_product(const i32x8 &w, const i32x8 &x, const f32x4 &acc, int sw, int sx, const int (&ew)[4]) {
    if constexpr (T::size == 2) {
        return scaled_mma<S>(w, x, acc, sw, sx);
    } else {
        f32x4 sum = {};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w[2 * k], w[2 * k + 1]), widen(x[2 * k], x[2 * k + 1]), sum, 0, 0, 0);
        int e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = (ew[i] >> (8 * S)) & 255;
        return add_scaled(acc, sum, e, (sx >> (8 * S)) & 255);
    }
}

// Up to 16 rows of x (a lane whose row is not there has the last one's, and writes nothing).  Where m alone does not
// fill the GPU, KW wavefronts of a workgroup take every KW'th quad and their sums are added through LDS, in order.
// 1 row of 28672 x 8192: 45 - 48 us (5.0 TB/s); 16 rows: 64 - 66; fp32 results 47 - 50 and 65.
template <typename T, int KW>
__global__ __launch_bounds__(256, 2) void product_few_kernel(ProductArgs a) {
    constexpr int WR = 4 / KW;
    __shared__ f32x4 s_sum[KW > 1 ? 4 * 64 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4, kw = wave % KW, xrow = min(r16, a.rows - 1);
    const int64_t col0 = ((int64_t)blockIdx.x * WR + wave / KW) * 16, wrow = min(col0 + r16, (int64_t)a.m - 1);
    const uint8_t *w = a.w + wrow * a.ldw + g * 16, *ws = a.ws + wrow * a.ldws;
    const uint8_t *x = a.x + xrow * a.ldx + g * 16, *xs = a.xs + xrow * a.ldxs;
    const int last = a.blocks - 1;
    f32x4 acc = {};
    Quad qw[2], qx[2];
    auto load = [&](auto at, int block) {
        load_quad(qw[decltype(at)::value], w, ws, block, last);
        load_quad(qx[decltype(at)::value], x, xs, block, last);
    };
    auto multiply = [&](auto at, int block) {
        constexpr int A = decltype(at)::value;
        int ew[4] = {};
        if constexpr (T::size == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) ew[e] = __shfl(qw[A].scale, g * 4 + e, 64);
        }
        unrolled<4>([&](auto k) {
            constexpr int K = decltype(k)::value;
            if (block + K <= last)
                acc = block_product<T, K>(join(qw[A].lo[K], qw[A].hi[K]), join(qx[A].lo[K], qx[A].hi[K]), acc, qw[A].scale, qx[A].scale, ew);
        });
    };
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> odd{};
    int block = kw * 4;
    if (block <= last) {
        load(even, block);
        for (;;) {
            if (block + KW * 4 > last) {
                multiply(even, block);
                break;
            }
            load(odd, block + KW * 4);
            multiply(even, block);
            block += KW * 4;
            if (block + KW * 4 > last) {
                multiply(odd, block);
                break;
            }
            load(even, block + KW * 4);
            multiply(odd, block);
            block += KW * 4;
        }
    }
    if constexpr (KW > 1) {
        s_sum[threadIdx.x] = acc;
        __syncthreads();
        if (kw > 0) return;
        acc = f32x4{};
#pragma unroll
        for (int k = 0; k < KW; ++k) acc += s_sum[(wave + k) * 64 + lane];
    }
    const int64_t col = col0 + g * 4;
    if (r16 < a.rows && col < a.m) put4<T>(a, r16, col, acc);
}

// Tiles of 128 columns x 32 FN rows, one workgroup to a compute unit: 17 .. 128 rows, and as many tiles of 128 as there are
// compute units.  Few rows are bound by the reading of w, so what counts is how much of it is on its way: a ring of as many
// stages as LDS holds (128 bytes of each row, straight to LDS; pieces at piece ^ (row & 7)), all but one of them in flight,
// 64 KB of w to a compute unit beside 96 rows.  (Twice as much, in registers and with a barrier only every four blocks,
// measured the same.)  28672 x 8192, by 224 of the 256 compute units: 17 rows 59 us (4.0 TB/s of w), and 3 to 5 us for every 32
// rows more, which come again for each 128 columns: 64 rows 64, 96 rows 70 (3.4 TB/s of w; 63 % of the cycles waits, 15 % matrix
// instructions), 128 rows 71.  Where rows of w are 8320 bytes apart, not 8192, 96 rows take 66.  fp32 results, 128 rows: 98.
// Scales come four stages to a dword, two dwords ahead, 256 rows (w's, then x's) to a load of the workgroup.
template <typename T, int FN>
struct SomeShape {
    static constexpr int kRows = 32 * FN, kStage = (128 + kRows) * 128, kRing = 152 * 1024 / kStage;
    static constexpr int kLds = kRing * kStage + 4 * 1024;
};
template <typename T, int FN>
__global__ __launch_bounds__(256, 1) void product_some_kernel(ProductArgs a) {
    typedef SomeShape<T, FN> Shape;
    constexpr int kStage = Shape::kStage, kRing = Shape::kRing;
    constexpr bool kWiden = T::size == 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t s_ring[];
    uint8_t *const s_scale = s_ring + kRing * kStage;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const TilePlace place = tile_place(blockIdx.x, a.row_tiles, a.col_tiles, 8);
    const int64_t row0 = (int64_t)place.row * Shape::kRows, col0 = (int64_t)place.col * 128;
    const int split = blockIdx.y, first = split * a.per_split, last = min(first + a.per_split, a.blocks);
    const int piece = (lane & 7) ^ (lane >> 3);
    const uint8_t *from_w[4], *from_x[FN];
#pragma unroll
    for (int i = 0; i < 4; ++i) from_w[i] = a.w + min(col0 + (wave * 4 + i) * 8 + (lane >> 3), (int64_t)a.m - 1) * a.ldw + piece * 16;
#pragma unroll
    for (int i = 0; i < FN; ++i) from_x[i] = a.x + min(row0 + (wave * FN + i) * 8 + (lane >> 3), (int64_t)a.rows - 1) * a.ldx + piece * 16;
    const uint8_t *from_s = wave < 2 ? a.ws + min(col0 + tid, (int64_t)a.m - 1) * a.ldws : a.xs + min(row0 + tid - 128, (int64_t)a.rows - 1) * a.ldxs;
    // (past the last stage it comes again, and is not used: every wavefront always has the same number under way)
    auto fetch = [&](int slot, int block) {
        const int64_t at = (int64_t)min(block, last - 1) * 128;
        uint8_t *to = s_ring + slot * kStage;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_lds16(from_w[i] + at, to + (wave * 4 + i) * 1024);
#pragma unroll
        for (int i = 0; i < FN; ++i) load_lds16(from_x[i] + at, to + 128 * 128 + (wave * FN + i) * 1024);
    };
    auto fetch_scales = [&](int block) {  // (first is a multiple of four)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from_s + min(block, (last - 1) & ~3)),
                                         (__attribute__((address_space(3))) void *)(s_scale + (block >> 2 & 3) * 1024 + wave * 256), 4, 0, 0);
    };
    fetch_scales(first);
    fetch_scales(first + 4);
#pragma unroll
    for (int k = 0; k < kRing - 1; ++k) fetch(k, first + k);
    const int r16 = lane & 15, g = lane >> 4, wm = (wave & 1) * 64, wn = (wave >> 1) * 16 * FN;
    const int p0 = (g ^ (lane & 7)) * 16, p1 = ((g + 4) ^ (lane & 7)) * 16;
    f32x4 acc[4][FN] = {};
    int scale_w[4], scale_x[FN], slot = 0;
    bool inside = false;
    for (int block = first; block < last; block += 4) {
        unrolled<4>([&](auto s) {
            constexpr int S = decltype(s)::value;
            if (block + S < last) {
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kRing - 2) * (4 + FN)) : "memory");  // this stage is there,
                __syncthreads();                                                              // and the last one has been read
                if constexpr (S == 0) {
                    fetch_scales(block + 8);
                    const int *at = (const int *)(s_scale + (block >> 2 & 3) * 1024);
                    uint32_t bad = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) bad |= outside(scale_w[i] = at[wm + i * 16 + r16]);
#pragma unroll
                    for (int j = 0; j < FN; ++j) bad |= outside(scale_x[j] = at[128 + wn + j * 16 + r16]);
                    if constexpr (kWiden) inside = all_inside(bad, last - block);
                }
                fetch(slot == 0 ? kRing - 1 : slot - 1, block + S + kRing - 1);
                const uint8_t *pw = s_ring + slot * kStage + (wm + r16) * 128, *px = s_ring + slot * kStage + (128 + wn + r16) * 128;
                slot = slot + 1 == kRing ? 0 : slot + 1;
                if constexpr (kWiden) {
                    if (inside) multiply_widened<S, FN>(pw, px, p0, p1, scale_w, scale_x, acc);
                    else multiply_apart<S, FN>(pw, px, p0, p1, scale_w, scale_x, acc);
                } else {
                    multiply_scaled<S, FN>(pw, px, p0, p1, scale_w, scale_x, acc);
                }
            }
        });
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nothing is on its way to LDS that is no longer this workgroup's)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t row = row0 + wn + j * 16 + r16;
        if (row >= a.rows) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t col = col0 + wm + i * 16 + g * 4;
            if (col >= a.m) continue;
            if (a.part) put_part(a, split, row, col, acc[i][j]);
            else put4<T>(a, row, col, acc[i][j]);
        }
    }
}

// y from the splits' sums, added in order, four of them asked for at a time.  (Outputs that are split are fewer than 2^23.)
template <typename T>
__global__ __launch_bounds__(256) void product_sum_kernel(ProductArgs a, int splits) {
    const uint32_t quads = (uint32_t)(a.m + 3) / 4, total = quads * (uint32_t)a.rows;
    for (uint32_t at = blockIdx.x * 256 + threadIdx.x; at < total; at += gridDim.x * 256) {
        f32x4 v = {};
        const f32x4 *p = (const f32x4 *)a.part + at;
        for (int s = 0; s < splits; s += 4) {
            f32x4 u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = p[(int64_t)min(s + k, splits - 1) * total];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s + k < splits) v += u[k];
        }
        const uint32_t row = at / quads;
        put4<T>(a, row, (int64_t)(at - row * quads) * 4, v);
    }
}

enum ProductForm { kFew, kSome, kTiles, kWide };
struct ProductPlan {
    ProductForm form;
    int splits, per_split;  // of the sum, and its blocks in one
    int kw;  // kFew: wavefronts along the sum; others: 32nds of a tile's rows
};
// Which form, and how the sum is split where the outputs alone do not fill the GPU.
static ProductPlan product_plan(int64_t rows, int64_t m, int64_t n, int dtype, int64_t most_stride) {
    const int64_t blocks = ceil_div(n, 128), quads = ceil_div(blocks, 4);
    if (rows <= 16) {
        int kw = 1;
        while (kw < 4 && ceil_div(m, 16) * kw < 4096 && kw * 2 <= quads) kw *= 2;
        return {kFew, 1, 0, kw};
    }
    if (blocks == 0) return {kTiles, 1, 4, 2};  // (the others begin with a fetch)
    // Tiles of 256 x 256 run one to a compute unit: they lose by a last round that is nearly empty.
    const int64_t wide = ceil_div(rows, kWideTile) * ceil_div(m, kWideTile);
    if (dtype == DLCX_BF16 && rows >= kWideTile && m >= kWideTile && wide >= 128 && most_stride <= (1 << 23))  // (256 rows: 32 bits)
        return {kWide, 1, 0, 0};
    const int64_t col_tiles = ceil_div(m, 128);
    if (rows <= 128) {
        // Splits as far as they fill the GPU, by the us that a block, a split and its sums were measured to take.  (100 x 2050 x
        // 4133 fp32: nine splits 16.7, five 20.1; 40 x 700 x 20000 bf16: 20 splits 13.1, and 40 were 4.7 more before sums were read four at a time.)
        const int fn = (int)ceil_div(rows, 32);
        const double block = dtype == DLCX_F32 ? 0.5 + 0.3 * fn : 0.25 + 0.13 * fn, split = 0.25 + 5e-5 * (double)(fn * m);
        ProductPlan best = {kSome, 1, (int)(quads * 4), fn};
        double least = (double)blocks * block;
        const int64_t most = col_tiles < 160 ? 256 / col_tiles : 1;
        for (int64_t per = ceil_div(ceil_div(blocks, most), 4) * 4; per < blocks && (double)per * block < least; per += 4) {
            const int64_t used = ceil_div(blocks, per);
            const double cost = (double)per * block + 2.0 + (double)used * split;
            if (cost >= least) continue;
            least = cost;
            best = {kSome, (int)used, (int)per, fn};
        }
        return best;
    }
    // Tiles of 128 rows or 64, in pairs that share a compute unit, or (bf16) of 128 rows alone on it with a ring of stages;
    // and splits.  The least of what the busiest compute unit takes, as
    // measured in us for a block of a tile, and of writing and adding the splits' sums.  (1024 x 4096 x 4096 bf16: ring 25.8,
    // 128 rows 31.7 and 34.5 in two splits, 64 rows 31.5; 3000 x 700 x 6000: 128 rows in three splits 29.0, ring 35.0; 2050 x
    // 1021 x 4133 fp32: 64 rows 46.6, 44.1, 40.0, 40.2 in one to four splits, 128 rows 37.9 in three.)
    ProductPlan best = {};
    double least = 1e300;
    auto consider = [&](ProductForm form, int fn, int64_t splits, double alone, double paired) {
        const int64_t tiles = ceil_div(rows, 32 * fn) * col_tiles;
        if (splits > 1 && tiles >= 512) return;
        const int64_t per = ceil_div(ceil_div(blocks, splits), 4) * 4, used = ceil_div(blocks, per), busiest = ceil_div(tiles * used, 256);
        double cost = (double)(busiest * std::min(per, blocks)) * (busiest == 1 ? alone : paired);
        const int f32 = dtype == DLCX_F32 ? 1 : 0;  // (the sums' launch reads and writes y, too)
        if (used > 1) cost += 3.0 - f32 + 1e-6 * (double)((used + f32) * ceil_div(rows, 64) * 64 * m);  // (rows of whole tiles: see the workspace)
        if (cost >= least) return;
        least = cost;
        best = {form, (int)used, (int)per, fn};
    };
    for (int64_t splits = 1; splits <= std::max((int64_t)1, std::min(blocks / 4, (int64_t)16)); ++splits) {
        if (dtype == DLCX_BF16) {
            consider(kTiles, 4, splits, 1.0, 0.8);
            consider(kTiles, 2, splits, 0.6, 0.47);
        } else {
            consider(kTiles, 4, splits, 1.6, 1.18);
            consider(kTiles, 2, splits, 0.85, 0.7);
        }
    }
    if (dtype == DLCX_BF16) consider(kSome, 4, 1, 0.77, 0.8);
    return best;
}

template <typename T, int FN>
static int run_some(ProductArgs a, int splits, hipStream_t st) {
    static size_t granted = 0;
    const int lds = SomeShape<T, FN>::kLds;
    const int rc = grant_dynamic_lds((const void *)product_some_kernel<T, FN>, lds, &granted, "fp8_product");
    if (rc != DLCX_OK) return rc;
    a.row_tiles = (int)ceil_div(a.rows, 32 * FN);
    product_some_kernel<T, FN><<<dim3((unsigned)(a.row_tiles * (int64_t)a.col_tiles), splits), 256, lds, st>>>(a);
    return DLCX_OK;
}

template <typename T>
static int launch_product(ProductArgs a, const ProductPlan &plan, hipStream_t st) {
    {
        Timed timed(KID_FP8_PRODUCT, st);
        if (plan.form == kWide) {
            static size_t granted[2] = {0, 0};
            const auto kernel = a.y_in ? product_wide_kernel<true> : product_wide_kernel<false>;
            int rc = grant_dynamic_lds((const void *)kernel, kWideLds, &granted[a.y_in ? 1 : 0], "fp8_product");
            if (rc != DLCX_OK) return rc;
            a.row_tiles = (int)ceil_div(a.rows, kWideTile);
            a.col_tiles = (int)ceil_div(a.m, kWideTile);
            kernel<<<dim3((unsigned)(a.row_tiles * (int64_t)a.col_tiles)), 256, kWideLds, st>>>(a);
        } else if (plan.form == kFew) {
            const dim3 grid((unsigned)ceil_div(a.m, 16 * (4 / plan.kw)));
            if (plan.kw == 1) product_few_kernel<T, 1><<<grid, 256, 0, st>>>(a);
            else if (plan.kw == 2) product_few_kernel<T, 2><<<grid, 256, 0, st>>>(a);
            else product_few_kernel<T, 4><<<grid, 256, 0, st>>>(a);
        } else if (plan.form == kSome) {
            const int rc = plan.kw == 1   ? run_some<T, 1>(a, plan.splits, st)
                           : plan.kw == 2 ? run_some<T, 2>(a, plan.splits, st)
                           : plan.kw == 3 ? run_some<T, 3>(a, plan.splits, st)
                                          : run_some<T, 4>(a, plan.splits, st);
            if (rc != DLCX_OK) return rc;
        } else {
            a.row_tiles = (int)ceil_div(a.rows, 32 * plan.kw);
            const dim3 grid((unsigned)(a.row_tiles * (int64_t)a.col_tiles), plan.splits);
            if (plan.kw == 4) product_kernel<T, 4><<<grid, 256, 0, st>>>(a);
            else product_kernel<T, 2><<<grid, 256, 0, st>>>(a);
        }
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
    size_t most = 0;  // of fewer rows, too: these may be split further (the plan is the same for 32 rows each, above 128 for 64)
    auto look = [&](int64_t r) {
        for (int dtype : {DLCX_F32, DLCX_BF16}) {
            const ProductPlan plan = product_plan(r, m, n, dtype, INT64_MAX);
            if (plan.splits > 1) most = std::max(most, (size_t)plan.splits * r * ceil_div(m, 4) * 16);
        }
    };
    for (int64_t r = 32; r < rows + 32 && r <= 128; r += 32) look(std::min(r, rows));
    for (int64_t r = 192; r < rows + 64 && r <= 65536; r += 64) {
        look(std::min(r, rows));
        if (ceil_div(r, 128) * ceil_div(m, 128) >= 512) break;  // (never split)
    }
    return a256x(most) + 256;
}

int dlcx_fp8_product_plan(int64_t rows, int64_t m, int64_t n, int dtype, int32_t *form, int32_t *tile, int32_t *splits) {
    if (bad_product(rows, m, n) || (dtype != DLCX_F32 && dtype != DLCX_BF16) || !form || !tile || !splits) return DLCX_EINVAL;
    const ProductPlan plan = product_plan(rows, m, n, dtype, 0);
    *form = plan.form;
    *tile = plan.form == kWide ? kWideTile : plan.form == kFew ? plan.kw : 32 * plan.kw;
    *splits = plan.splits;
    return DLCX_OK;
}

int dlcx_fp8_product(const dlcx_fp8 *x, const dlcx_fp8 *w, const void *y_in, int64_t ldy_in, void *y_out, int64_t ldy_out,
                     int dtype, void *workspace, void *stream) {
    if (check_fp8(x) != DLCX_OK || check_fp8(w) != DLCX_OK || x->cols != w->cols) return DLCX_EINVAL;
    if (dtype != DLCX_F32 && dtype != DLCX_BF16) return DLCX_EINVAL;
    if (x->rows == 0 || w->rows == 0) return DLCX_OK;
    if (bad_rows(y_out, ldy_out, w->rows, dtype) || (y_in && bad_rows(y_in, ldy_in, w->rows, dtype))) return DLCX_EINVAL;
    if ((y_in == y_out && ldy_in != ldy_out) || !workspace || off_by(workspace, 256)) return DLCX_EINVAL;
    const int64_t stride = std::max({x->ld, w->ld, x->ldscale, w->ldscale});
    const ProductPlan plan = product_plan(x->rows, w->rows, x->cols, dtype, stride);
    ProductArgs a = {(const uint8_t *)x->codes, (const uint8_t *)x->scales, (const uint8_t *)w->codes, (const uint8_t *)w->scales,
                     y_in, y_out, plan.splits > 1 ? (float *)workspace : nullptr, x->ld, x->ldscale, w->ld, w->ldscale,
                     ldy_in, ldy_out, (int)x->rows, (int)w->rows, (int)ceil_div(x->cols, 128), plan.per_split,
                     (int)ceil_div(x->rows, 128), (int)ceil_div(w->rows, 128)};
    // tiles of 128 x 128, in 2^36 outputs: the form with tiles of 64 rows has twice as many workgroups
    if ((int64_t)a.row_tiles * a.col_tiles >= kMostGroups / 2) return DLCX_EUNSUPPORTED;
    return dtype == DLCX_BF16 ? launch_product<TypeBf16>(a, plan, as_stream(stream)) : launch_product<TypeF32>(a, plan, as_stream(stream));
}

}  // extern "C"
