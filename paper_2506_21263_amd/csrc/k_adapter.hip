// Low-rank adapters of many requests (or of K workers) beside a shared projection, and their
// gradient.  With the rows of one adapter gathered, every product is one of three:
//
//   down  h[t][c] = sum_i x[t][i] F[c][i]           (x, Q) -> h      (dy, P) -> g
//   up    y[t][j] = y_in[t][j] + sum_c h[t][c] F[c][j]   (h, P) -> y      (g, Q) -> dx
//   grad  D[c][j] = sum_t u[t][c] z[t][j]           (h, dy) -> dP    (g, x) -> dQ
//
// A row is 2 to 60 KB and meets r <= 256 columns, so all three are bound by the stream of rows as long
// as the matrix cores are fed from the registers the stream arrives in.
#include "common.h"

namespace dlcx {

// ---- rows grouped by adapter ----------------------------------------------------------------------
// Bucket a < count holds the rows of adapter a, bucket `count` the rows without one.  A launch cuts every
// bucket into tiles of as many rows as fill the GPU; a workgroup finds its tile in the buckets' places.
constexpr int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64;
constexpr int kRouteKept = 1024;  // rows of a wavefront whose buckets stay in LDS from one pass to the next

struct Route {
    int32_t *first;  // count + 2: first place of each bucket in `order`, then the number of rows
    int32_t *order;  // rows: bucket after bucket, in a bucket in the rows' own order
    int count;
    const int32_t *ids;  // not nullptr: no buckets, every row is a tile, in the rows' own order
};
static size_t route_view(int64_t rows, int count, char *base, Route *v) {
    const size_t heads = a256x((size_t)(count + 2) * sizeof(int32_t));
    if (v) *v = {(int32_t *)base, (int32_t *)(base + heads), count, nullptr};
    return heads + a256x((size_t)rows * sizeof(int32_t));
}
static inline int64_t max_tiles(int64_t rows, int count, int size) {
    return rows / size + (rows < count + 1 ? rows : count + 1);
}

// Inclusive prefix sum over a wavefront's lanes.
__device__ __forceinline__ int scan_wave(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
    return x;
}

// A launch has at most 2^32 threads along x: workgroups beyond kGroupsX go on along the dimension that a kernel leaves free.
constexpr int64_t kGroupsX = 1 << 22;
static inline unsigned groups_x(int64_t groups) { return (unsigned)(groups < kGroupsX ? groups : kGroupsX); }
static inline unsigned groups_on(int64_t groups) { return (unsigned)ceil_div(groups, kGroupsX); }

struct Tile {
    int adapter;  // -1: rows without one; -2: there is no such tile
    int at, rows; // places in `order`
    int slab;     // number among the tiles of adapters that have several, -1: the only one
    int block;    // number of its first 16 rows, when all buckets are cut into blocks of 32 and these into two
};
// Tile `index` of the buckets' tiles of up to `size` rows; 64 buckets at a time, the same in every wavefront.
// EVEN: a bucket's tiles have equal numbers of rows, in sixteens; else all but the last have `size`.
template <bool EVEN>
__device__ __forceinline__ Tile find_tile(const Route &r, int size, int index) {
    const int lane = threadIdx.x & 63;
    if (r.ids) {
        const int id = r.ids[index];
        return {id >= 0 && id < r.count ? id : -1, index, 1, -1, 0};
    }
    int tiles = 0, slabs = 0, blocks = 0;
    for (int base = 0; base <= r.count; base += 64) {
        const int b = base + lane;
        const int at = b <= r.count ? r.first[b] : 0, end = b <= r.count ? r.first[b + 1] : 0;
        const int n = (end - at + size - 1) / size, several = n > 1 && b < r.count ? n : 0;
        const int upto = tiles + scan_wave(n), slabs_upto = slabs + scan_wave(several);
        const int n32 = (end - at + 31) / 32, blocks_upto = blocks + scan_wave(n32);
        const uint64_t after = __ballot(upto > index);
        if (after) {
            const int l = __ffsll((unsigned long long)after) - 1;
            const int k = index - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
            const int begin = __builtin_amdgcn_readlane(at, l), stop = __builtin_amdgcn_readlane(end, l);
            const int each = EVEN ? ((stop - begin + 16 * __builtin_amdgcn_readlane(n, l) - 1) /
                                     (16 * __builtin_amdgcn_readlane(n, l))) * 16 : size;
            const int from = begin + k * each;
            if (EVEN && from >= stop) return {-2, 0, 0, -1, 0};
            const int several_l = __builtin_amdgcn_readlane(several, l);
            Tile t;
            t.adapter = base + l < r.count ? base + l : -1;
            t.at = from;
            t.rows = min(each, stop - from);
            t.slab = several_l ? __builtin_amdgcn_readlane(slabs_upto, l) - several_l + k : -1;
            t.block = 2 * (__builtin_amdgcn_readlane(blocks_upto, l) - __builtin_amdgcn_readlane(n32, l)) + k * (each / 16);
            return t;
        }
        tiles = __builtin_amdgcn_readlane(upto, 63);
        slabs = __builtin_amdgcn_readlane(slabs_upto, 63);
        blocks = __builtin_amdgcn_readlane(blocks_upto, 63);
    }
    return {-2, 0, 0, -1, 0};
}

// One workgroup sorts the rows by counting: every wavefront counts its own share, the counts become the
// places where it writes, and the lanes of equal adapters find their order by ballots of the index's
// bits, so the order within an adapter is that of the rows.  It runs alone, so the loops are kept short: the code
// of an unrolled one came from memory for longer than it ran (16384 rows, one adapter after the other, 18 us, now 10).
// One workgroup at any size: rows in any order of 64 adapters take 26 us for 16384, 1.5 ms for 2^20 (one after the other
// 0.4), where the rows themselves, beside 8192 x 8192 in bf16, take 10 ms to read and write.
__global__ __launch_bounds__(kRouteThreads) void adapter_route_kernel(int rows,
                                                                      const int32_t *__restrict__ ids, Route r) {
    extern __shared__ int cursor[];  // kRouteWaves x buckets, then kRouteKept buckets of every wavefront's rows
    __shared__ int sums[kRouteWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, buckets = r.count + 1;
    for (int i = threadIdx.x; i < kRouteWaves * buckets; i += kRouteThreads) cursor[i] = 0;
    const int share = (rows + kRouteThreads - 1) / kRouteThreads * 64;
    const int lo = min(rows, wave * share), hi = min(rows, lo + share);
    const int bits = 32 - __clz(buckets - 1);
    int *mine = cursor + wave * buckets;
    uint16_t *kept = reinterpret_cast<uint16_t *>(cursor + kRouteWaves * buckets) + wave * kRouteKept;
    int run = -1, run_at = 0;  // a bucket whose count (or place) is ahead of the one in LDS
    auto settle = [&](int pass) {
        if (run >= 0 && lane == 0) mine[run] = pass == 0 ? mine[run] + run_at : run_at;
        run = -1;
        wave_sync();
    };
    __syncthreads();
    for (int pass = 0; pass < 2; ++pass) {
        for (int base = lo; base < hi; base += kRouteKept) {
            if (pass == 0 || share > kRouteKept) {
                int id[kRouteKept / 64];
#pragma unroll
                for (int u = 0; u < kRouteKept / 64; ++u) id[u] = ids[min(base + u * 64 + lane, rows - 1)];
#pragma unroll
                for (int u = 0; u < kRouteKept / 64; ++u)
                    kept[u * 64 + lane] = (uint16_t)(id[u] >= 0 && id[u] < r.count ? id[u] : r.count);
                wave_sync();
            }
#pragma unroll 1
            for (int t0 = base; t0 < min(hi, base + kRouteKept); t0 += 64) {
                const int t = t0 + lane, b = kept[t - base], b0 = __builtin_amdgcn_readfirstlane(b);
                uint64_t same = __ballot(t < hi);
                if (__ballot(t < hi && b != b0) == 0) {  // rows of one bucket, as the rows before them or not
                    if (b0 != run) {
                        settle(pass);
                        run = b0;
                        run_at = pass == 0 ? 0 : mine[b0];
                    }
                    if (pass == 1 && t < hi) r.order[run_at + lane] = t;
                    run_at += __popcll(same);
                    continue;
                }
                settle(pass);
#pragma unroll 1
                for (int k = 0; k < bits; ++k) {
                    const uint64_t one = __ballot((b >> k) & 1);
                    same &= (b >> k) & 1 ? one : ~one;
                }
                const int rank = __popcll(same & ((1ull << lane) - 1));
                if (t < hi && pass == 1) r.order[mine[b] + rank] = t;
                wave_sync();
                if (t < hi && rank == 0) mine[b] += __popcll(same);
                wave_sync();
            }
        }
        settle(pass);
        __syncthreads();
        if (pass == 1) return;
        int before = 0;
        for (int base = 0; base < buckets; base += kRouteThreads) {
            const int b = base + (int)threadIdx.x;
            int n = 0;
            if (b < buckets)
                for (int w = 0; w < kRouteWaves; ++w) n += cursor[w * buckets + b];
            const int upto = scan_wave(n);
            if (lane == 63) sums[wave] = upto;
            __syncthreads();
            int at = before + upto - n;
            for (int w = 0; w < kRouteWaves; ++w) {
                at += w < wave ? sums[w] : 0;
                before += sums[w];
            }
            if (b < buckets) {
                r.first[b] = at;
                for (int w = 0; w < kRouteWaves; ++w) {
                    const int c = cursor[w * buckets + b];
                    cursor[w * buckets + b] = at;
                    at += c;
                }
            }
            __syncthreads();
        }
        if (threadIdx.x == 0) r.first[buckets] = rows;
    }
}

// ---- operands -------------------------------------------------------------------------------------
// A block of 16 x 32 (or 32 x 16) of an operand: lane l holds row (column) l % 16 and the 8 reduction
// indices from 8 (l / 16) on.  bf16: one product of 16 x 16 x 32; fp32: eight of 16 x 16 x 4, the j-th with the
// j-th index of every lane, which is a reordering of the same sum.  Element v of the result is
// row 4 (l / 16) + v, column l % 16.
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 ab_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 ab_bf16x2 __attribute__((ext_vector_type(2)));
typedef float ab_f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t ab_u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const ab_f32x2 x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, ab_bf16x2));
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Sixteen bytes at any address that their elements may have: the memory system takes them in one request.
__device__ __forceinline__ ab_u32x4 load_any(const void *p) {
    ab_u32x4 w;
    __builtin_memcpy(&w, p, sizeof w);
    return w;
}

// How rows are read and written: element by element where they begin anywhere, by 16 aligned bytes, or by these and past
// the caches' order of use, for matrices of kStreamed bytes and more that pass by once.  A backward pass beside
// 8192 + 8192 columns at rank 64, plain -> streamed, us: 16384 rows (268 MB a matrix) 350 -> 343 (down 74 -> 70, up 117 ->
// 120, grad 140 -> 132: more of the rows of one product is in the cache for the next), 2000 rows (33 MB) 80 -> 80; 4133 rows
// forward 80 -> 74.  Above 64 columns of a factor down and grad read the rows again for the next 64, plainly: 4133 rows at
// rank 256, streamed -> plain, down 74 -> 62, grad 201 -> 173.
constexpr int kAnywhere = 0, kAligned = 1, kStream = 2;
constexpr int64_t kStreamed = 24000000;
template <bool STREAM>
__device__ __forceinline__ ab_u32x4 load_vector(const void *p) {
    const ab_u32x4 *v = reinterpret_cast<const ab_u32x4 *>(p);
    return STREAM ? __builtin_nontemporal_load(v) : *v;
}
struct Bf16 {
    static constexpr int lane = 8;  // elements of 16 bytes
    typedef uint16_t elem;
    struct Frag {
        ab_u32x4 w;
    };
    static __device__ __forceinline__ Frag zero() { return {ab_u32x4{0u, 0u, 0u, 0u}}; }
    static __device__ __forceinline__ f32x4_t mma(const Frag &a, const Frag &b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ab_bf16x8, a.w),
                                                       __builtin_bit_cast(ab_bf16x8, b.w), c, 0, 0, 0);
    }
    // elements k .. k + 7 of a row of `len`; ALL: all of them are there
    template <bool VEC, bool ALL = false, bool STREAM = false>
    static __device__ __forceinline__ Frag load8(const elem *row, int k, int len) {
        if constexpr (ALL && VEC) return {load_vector<STREAM>(row + k)};
        if constexpr (ALL) return {load_any(row + k)};
        Frag f = zero();
        if constexpr (VEC) {
            if (k < len) f.w = *reinterpret_cast<const ab_u32x4 *>(row + k);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < len) f.w[i / 2] |= (uint32_t)row[k + i] << (16 * (i & 1));
        }
        return f;
    }
    static __device__ __forceinline__ Frag pack(const float (&x)[8]) {
        return {ab_u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])}};
    }
    static __device__ __forceinline__ elem round(float x) { return (uint16_t)pack2(x, x); }
    static __device__ __forceinline__ void drop(Frag &f, int n) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f.w[i / 2] &= i < n ? (i & 1 ? 0x0000FFFFu : 0xFFFF0000u) : 0xFFFFFFFFu;
    }
    static __device__ __forceinline__ float value(elem x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ float at(const Frag &f, int i) {
        return i & 1 ? high_bf16(f.w[i / 2]) : low_bf16(f.w[i / 2]);
    }
    // x as a sum of three bf16 numbers, its 24 bits eight by eight: the sum is x itself.  All three have the sign of x, and
    // what is not finite is that three times; a piece that would be zero is x / 2^32 instead (from 2^-80 on): so x times
    // an infinity is that infinity in every piece, where 0 times it or two of different signs would be a NaN.
    static __device__ __forceinline__ void parts(float x, elem (&e)[3]) {
        const uint32_t bits = __float_as_uint(x), quiet = (bits & 0x007FFFFFu) ? 0x00400000u : 0u;
        const uint32_t small = fabsf(x) >= 0x1p-80f ? __float_as_uint(x * 0x1p-32f) : 0u;
        const bool finite = (bits & 0x7F800000u) != 0x7F800000u;
        float rest = x;
#pragma unroll
        for (int h = 0; h < 3; ++h) {
            uint32_t top = __float_as_uint(rest) & 0xFFFF0000u;
            rest -= __uint_as_float(top);
            if (h > 0 && (top & 0x7FFF0000u) == 0) top = small;
            e[h] = (uint16_t)((finite ? top : bits | quiet) >> 16);
        }
    }
    static __device__ __forceinline__ void split(const float (&x)[8], Frag (&f)[3]) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            elem lo[3], hi[3];
            parts(x[i], lo);
            parts(x[i + 1], hi);
#pragma unroll
            for (int h = 0; h < 3; ++h) f[h].w[i / 2] = lo[h] | (uint32_t)hi[h] << 16;
        }
    }
    static constexpr int pieces = 3;
};
struct F32 {
    static constexpr int lane = 4;
    typedef float elem;
    struct Frag {
        float x[8];
    };
    static __device__ __forceinline__ Frag zero() {
        Frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f.x[i] = 0.f;
        return f;
    }
    static __device__ __forceinline__ f32x4_t mma(const Frag &a, const Frag &b, f32x4_t c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[j], b.x[j], c, 0, 0, 0);
        return c;
    }
    template <bool VEC, bool ALL = false, bool STREAM = false>
    static __device__ __forceinline__ Frag load8(const elem *row, int k, int len) {
        Frag f = zero();
        if (ALL || (VEC && k < len)) {
            const ab_u32x4 a = VEC ? load_vector<STREAM>(row + k) : load_any(row + k);
            const ab_u32x4 b = VEC ? load_vector<STREAM>(row + k + 4) : load_any(row + k + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) f.x[i] = __uint_as_float(a[i]), f.x[4 + i] = __uint_as_float(b[i]);
        } else if (!VEC) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < len) f.x[i] = row[k + i];
        }
        return f;
    }
    static __device__ __forceinline__ Frag pack(const float (&x)[8]) {
        Frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f.x[i] = x[i];
        return f;
    }
    static __device__ __forceinline__ void parts(float x, elem (&e)[1]) { e[0] = x; }
    static __device__ __forceinline__ void split(const float (&x)[8], Frag (&f)[1]) { f[0] = pack(x); }
    static __device__ __forceinline__ elem round(float x) { return x; }
    // the first n elements are zero
    static __device__ __forceinline__ void drop(Frag &f, int n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.x[i] = i < n ? 0.f : f.x[i];
    }
    static __device__ __forceinline__ float value(elem x) { return x; }
    static __device__ __forceinline__ float at(const Frag &f, int i) { return f.x[i]; }
    static constexpr int pieces = 1;
};

// Where a lane's 16 bytes of a row begin that should begin at element j: at the row's last 16 where it ends before
// j + lane, so that no lane waits at a branch.  What it has twice then, or beyond the row, it does not store.
template <typename T>
__device__ __forceinline__ int column_base(int j, int len) {
    return len >= T::lane ? min(j, len - T::lane) : j;
}
template <typename T, int VEC>
__device__ __forceinline__ ab_u32x4 load16(const typename T::elem *row, int base, int len) {
    if constexpr (VEC) return load_vector<VEC == kStream>(row + base);
    if (len >= T::lane) return load_any(row + base);
    ab_u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < T::lane; ++i)
        if (base + i < len) {
            if constexpr (T::lane == 8)
                w[i / 2] |= (uint32_t)row[base + i] << (16 * (i & 1));
            else
                w[i] = __float_as_uint(row[base + i]);
        }
    return w;
}
template <typename T, int VEC>
__device__ __forceinline__ void store16(typename T::elem *row, const ab_u32x4 &w, int base, int j, int len) {
    if (VEC || j + T::lane <= len) {
        if (j >= len) return;
        if constexpr (VEC == kStream) __builtin_nontemporal_store(w, reinterpret_cast<ab_u32x4 *>(row + base));
        else if constexpr (VEC) *reinterpret_cast<ab_u32x4 *>(row + base) = w;
        else __builtin_memcpy(row + base, &w, sizeof w);
        return;
    }
#pragma unroll
    for (int i = 0; i < T::lane; ++i)
        if (base + i >= j && base + i < len) {
            if constexpr (T::lane == 8)
                row[base + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
            else
                row[base + i] = __uint_as_float(w[i]);
        }
}

// Eight rows of 16 bytes each, turned: fragment s holds element s of the eight rows.  Where the rows are
// 8 (l / 16) + 0 .. 7 of a block and lane l has the elements from lane * g(l % 16) on, that is an
// operand block of the columns lane * g(0 .. 15) + s without a word moved between lanes.
__device__ __forceinline__ void turn(const ab_u32x4 (&row)[8], Bf16::Frag (&f)[8]) {
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int p = 0; p < 4; ++p)
            f[s].w[p] = __builtin_amdgcn_perm(row[2 * p + 1][s / 2], row[2 * p][s / 2],
                                              s & 1 ? 0x07060302u : 0x05040100u);
}
__device__ __forceinline__ void turn(const ab_u32x4 (&row)[8], F32::Frag (&f)[4]) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) f[s].x[j] = __uint_as_float(row[j][s]);
}

__device__ __forceinline__ int adapter_rank(int adapter, const int32_t *ranks, int r) {
    return adapter < 0 ? 0 : ranks ? max(0, min(ranks[adapter], r)) : r;
}

// ---- down -------------------------------------------------------------------------------------------
// Row t of a matrix whose rows are `pitch` bytes apart: one multiply-add.
template <typename E>
__device__ __forceinline__ const E *row_at(const void *base, uint32_t t, uint32_t pitch) {
    return (const E *)((const char *)base + (uint64_t)t * pitch);
}

struct DownArgs {
    const void *x;       // rows x len
    uint32_t pitch;
    const void *f;       // count x r x len
    const int32_t *ranks;
    float *out;          // places x r, columns below the adapter's rank; shares of the reduction `stride` floats apart
    int64_t stride;
    int len, r, shares, tiles;
};

// A workgroup has a share of the reduction (its eight wavefronts 256 to 512 bytes of it each), CT x 16 columns and
// up to `size` rows of one adapter.  A wavefront keeps its part of the factor in registers and meets it with 16 rows
// at a time; the eight sums are joined in LDS, in turn in two places, so that one barrier a round is enough.
// With whole rows to a workgroup instead, the factor comes from L2 as often as there are tiles of
// rows, by the same few channels at a time: 91 us for 16384 x 8192 bf16 at rank 64, 88 us for 4133 rows.
// This form: 66 us (4.1 TB/s of rows, and 34 MB of shares) and 22 us.
// In bf16 a load has 256 bytes of each of four rows, neighbouring lanes the same row; the four loads of sixteen rows
// then change places within four lanes, into the layout of the matrix instructions.  With one row to each of 16
// lanes instead (as fp32 rows are read): 79 and 31 us.
constexpr int kDownWaves = 8;
template <typename T>
constexpr int down_steps(int ct) {  // of 32 elements, per wavefront
    return (ct == 4 ? 4 : 8) * T::lane / 8;
}
// Four vectors of 16 bytes in four neighbouring lanes change places: vector s of lane c is vector c of lane s after it.
template <int CTRL>
__device__ __forceinline__ uint32_t quad_dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ void exchange(ab_u32x4 &a, ab_u32x4 &b, bool second, ab_u32x4 a_there, ab_u32x4 b_there) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = second ? b_there[i] : a[i];
        b[i] = second ? b[i] : a_there[i];
    }
}
template <int CTRL>
__device__ __forceinline__ ab_u32x4 quad_dpp4(const ab_u32x4 &x) {
    return ab_u32x4{quad_dpp<CTRL>(x[0]), quad_dpp<CTRL>(x[1]), quad_dpp<CTRL>(x[2]), quad_dpp<CTRL>(x[3])};
}
__device__ __forceinline__ void transpose_quads(Bf16::Frag (&f)[4]) {
    const bool one = threadIdx.x & 1, two = threadIdx.x & 2;
#pragma unroll
    for (int s = 0; s < 4; s += 2) exchange(f[s].w, f[s + 1].w, one, quad_dpp4<0xB1>(f[s].w), quad_dpp4<0xB1>(f[s + 1].w));
#pragma unroll
    for (int s = 0; s < 2; ++s) exchange(f[s].w, f[s + 2].w, two, quad_dpp4<0x4E>(f[s].w), quad_dpp4<0x4E>(f[s + 2].w));
}
template <typename T, int CT, int VEC>
__global__ __launch_bounds__(kDownWaves * 64, CT == 4 && VEC ? 4 : 2) void adapter_down_kernel(DownArgs a, Route route, int size) {
    constexpr int KS = down_steps<T>(CT);
    typedef typename T::Frag Frag;
    typedef typename T::elem elem;
    __shared__ f32x4_t sums[2][kDownWaves][CT][64];
    const uint32_t group = blockIdx.x + blockIdx.z * (uint32_t)kGroupsX;
    const int share = (int)(group % (uint32_t)a.shares), index = (int)(group / (uint32_t)a.shares);
    if (index >= a.tiles) return;
    const Tile tile = find_tile<true>(route, size, index);
    if (tile.adapter < 0) return;
    const int32_t *__restrict__ order = route.order + tile.at;
    const int lane = threadIdx.x & 63, row16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int c0 = blockIdx.y * CT * 16, last = tile.rows - 1;
    const int rank = adapter_rank(tile.adapter, a.ranks, a.r);
    if (c0 >= rank) return;
    const int k0 = (share * kDownWaves + wave) * KS * 32;
    const bool whole = k0 + KS * 32 <= a.len;
    // The lane's elements of step s (with kQuads, after the exchange).  Where a row that is not read by 16 aligned bytes ends before them, its last
    // eight, of which the row's and the factor's are zero as far as another lane has them (shorter rows are read by element).
    constexpr bool kQuads = VEC && T::lane == 8;
    auto at = [&](int s) { return k0 + (kQuads ? s / 4 * 128 + quad * 32 + s % 4 * 8 : s * 32 + quad * 8); };
    auto load = [&](const elem *row, Frag (&f)[KS]) {
        if (whole) {
#pragma unroll
            for (int s = 0; s < KS; ++s) f[s] = T::template load8<VEC != 0, true>(row, at(s), a.len);
        } else if (!VEC && a.len >= 8) {
#pragma unroll
            for (int s = 0; s < KS; ++s) f[s] = T::template load8<VEC != 0, true>(row, min(at(s), a.len - 8), a.len);
        } else {
#pragma unroll
            for (int s = 0; s < KS; ++s) f[s] = T::template load8<VEC != 0, false>(row, at(s), a.len);
        }
    };
    auto index_of = [&](int t0) { return route.ids ? tile.at : order[min(t0 + row16, last)]; };
    auto load_row = [&](int t, Frag (&x)[KS]) {
        if constexpr (kQuads) {
            const int k = k0 + quad * 32 + (lane & 3) * 8;
            const uint32_t n[4] = {quad_dpp<0x00>(t), quad_dpp<0x55>(t), quad_dpp<0xAA>(t), quad_dpp<0xFF>(t)};
            if (whole) {
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    x[s] = T::template load8<true, true, VEC == kStream>(row_at<elem>(a.x, n[s % 4], a.pitch), k + s / 4 * 128, a.len);
            } else {
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    x[s] = T::template load8<VEC != 0, false>(row_at<elem>(a.x, n[s % 4], a.pitch), k + s / 4 * 128, a.len);
            }
        } else {
            load(row_at<elem>(a.x, t, a.pitch), x);
        }
    };
    Frag f[CT][KS];
    auto products = [&](Frag (&x)[KS], int turn) {
        if constexpr (kQuads) {
#pragma unroll
            for (int s = 0; s < KS; s += 4) {
                Frag y[4] = {x[s], x[s + 1], x[s + 2], x[s + 3]};
                transpose_quads(y);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[s + i] = y[i];
            }
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) acc = T::mma(x[s], f[c][s], acc);
            sums[turn][wave][c][lane] = acc;
        }
    };
    float *out = a.out + share * a.stride + (int64_t)tile.at * a.r;
    auto join = [&](int t0, int turn) {
        __syncthreads();
        if (wave >= CT) return;
        f32x4_t acc = sums[turn][0][wave][lane];
#pragma unroll
        for (int w = 1; w < kDownWaves; ++w) acc += sums[turn][w][wave][lane];
        const int col = c0 + wave * 16 + row16;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int t = t0 + quad * 4 + v;
            if (t <= last && col < rank) out[(int64_t)t * a.r + col] = acc[v];
        }
    };
    // Two sets of rows are on their way at any time.  Requests come back in order: the row numbers of a later
    // set go out before the rows of an earlier one, and the sums are stored by place, which needs none.
    Frag x0[KS], x1[KS];
    load_row(index_of(0), x0);
    if (last >= 16) load_row(index_of(16), x1);
    int n0 = index_of(32), n1 = index_of(48);
#pragma unroll
    for (int c = 0; c < CT; ++c)  // columns from the rank on are the last one again: not stored
        load((const elem *)a.f + ((int64_t)tile.adapter * a.r + min(c0 + c * 16 + row16, rank - 1)) * a.len, f[c]);
    const bool twice = !VEC && !whole && a.len >= 8;
    auto drop = [&](Frag (&x)[KS]) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            int n = at(s) - min(at(s), a.len - 8);
            asm volatile("" : "+v"(n));  // (masks formed here and not kept through the loop: 151 registers, not 193)
            T::drop(x[s], n);
        }
    };
    if (twice)
#pragma unroll
        for (int c = 0; c < CT; ++c) drop(f[c]);
    for (int t0 = 0; t0 <= last; t0 += 32) {
        if (twice) drop(x0);
        products(x0, 0);
        const int m0 = n0;
        n0 = index_of(t0 + 64);
        if (t0 + 32 <= last) load_row(m0, x0);
        join(t0, 0);
        if (t0 + 16 > last) break;
        if (twice) drop(x1);
        products(x1, 1);
        const int m1 = n1;
        n1 = index_of(t0 + 80);
        if (t0 + 48 <= last) load_row(m1, x1);
        join(t0 + 16, 1);
    }
}

// ---- operands ---------------------------------------------------------------------------------------
// What the other two products read of h (or g): the sum of its splits, in 32 bits as it is and as two
// operands, so that they are formed once and not by every workgroup that has other columns.  13 us for both of
// 16384 rows at rank 64 (34 MB of shares, 4 of h, 19 of operands).
struct OperandJob {
    const float *splits;  // r columns each, `stride` floats apart
    int64_t stride;
    int n, placed;        // placed: their rows are in the order of the places
    const float *scale_out, *scale_up;  // what `out` and `turned`, and what `up` are multiplied with; nullptr: 1
    float *out;           // rows x r, or nullptr; zero from the adapter's rank on
    void *up;             // [block of 16 rows][step][piece][lane], or nullptr: for the product with the factor
    void *turned;         // [block of 32 rows][16 columns][piece][lane], or nullptr: for the sums over rows
};
struct OperandArgs {
    OperandJob job[2];
    const int32_t *ranks;
    int r, steps;
};
template <typename T>
__global__ __launch_bounds__(256) void adapter_operand_kernel(OperandArgs a, Route route) {
    const Tile tile = find_tile<false>(route, 32, blockIdx.x);
    if (tile.adapter < -1) return;
    const int32_t *__restrict__ order = route.order + tile.at;
    const int rank = adapter_rank(tile.adapter, a.ranks, a.r), cols = a.steps * 32;
    const OperandJob &j = a.job[blockIdx.y];
    const float s_out = j.scale_out && tile.adapter >= 0 ? j.scale_out[tile.adapter] : 1.f;
    const float s_up = j.scale_up && tile.adapter >= 0 ? j.scale_up[tile.adapter] : 1.f;
    const int c = blockIdx.z * 64 + threadIdx.x % 64, quad = threadIdx.x / 64;
    __shared__ float to_up[32][65];
    if (c < cols) {
        int t[8];
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t[i] = quad * 8 + i < tile.rows ? order[quad * 8 + i] : -1;
            x[i] = 0.f;
        }
        const int place = tile.at + quad * 8;
        if (c < rank && t[0] >= 0)
            for (int k = 0; k < j.n; k += 4) {
                float part[4][8];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        part[u][i] = j.splits[min(k + u, j.n - 1) * j.stride +
                                              (int64_t)(t[i] < 0 ? 0 : j.placed ? place + i : t[i]) * a.r + c];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] += k + u < j.n && t[i] >= 0 ? part[u][i] : 0.f;
            }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            to_up[quad * 8 + i][c % 64] = c < rank ? x[i] * s_up : 0.f;
            if (t[i] < 0) continue;
            x[i] = c < rank ? x[i] * s_out : 0.f;
            if (j.out && c < a.r) j.out[(int64_t)t[i] * a.r + c] = x[i];
        }
        if (j.turned) {
            typename T::Frag f[T::pieces];
            T::split(x, f);
#pragma unroll
            for (int h = 0; h < T::pieces; ++h)
                ((typename T::Frag *)j.turned)[(((int64_t)(tile.block / 2) * a.steps * 2 + c / 16) * T::pieces + h) * 64 +
                                               quad * 16 + c % 16] = f[h];
        }
    }
    if (!j.up) return;
    __syncthreads();
    // a thread has a row's eight columns of a step
    const int lane = threadIdx.x % 64, half = threadIdx.x / 64 % 2, step = blockIdx.z * 2 + threadIdx.x / 128;
    if (step >= a.steps) return;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_up[half * 16 + lane % 16][threadIdx.x / 128 * 32 + lane / 16 * 8 + i];
    typename T::Frag f[T::pieces];
    T::split(x, f);
#pragma unroll
    for (int h = 0; h < T::pieces; ++h)
        ((typename T::Frag *)j.up)[(((int64_t)(tile.block + half) * a.steps + step) * T::pieces + h) * 64 + lane] = f[h];
}

// ---- up ---------------------------------------------------------------------------------------------
struct UpArgs {
    const void *h;       // [block of 16 rows][step][piece][lane], scaled
    const void *f;       // count x r x len
    const int32_t *ranks;
    const void *y_in;    // or nullptr
    void *y_out;         // rows x len
    uint32_t pitch_in, pitch_out;
    int len, r, copy;    // copy: rows without adapter are to be written too
    int blocks;          // of columns
};

// A workgroup has 256 bytes of columns and up to `size` rows of one adapter.  It turns the factor's
// columns into operand blocks in LDS once; then each wavefront takes 16 rows at a time: lane l has rows
// 4 (l / 16) + 0 .. 3 and 16 bytes of each, so that 16 lanes make 256 in a row.  (With a row to
// every lane of 16 an access is 64 pieces for the L1, not 16: 128 us for 16384 x 8192 at rank 64.)  HBM
// bounds it: 120 us where it leaves grad its rows, 4.5 TB/s.  bf16: scale h comes in all three of its pieces, so that a
// row's result does not hang on the form that its number of rows takes; rounded to one piece it is 112 us.  The pieces lie
// as the products take them, 1 KB of consecutive memory to a request, where a row to each of 16 lanes took 128 us.  Above rank
// 128 they take 96 registers: one workgroup to a compute unit, 91 us for 4133 rows at rank 256 where two, which spill, take
// 111 (and one piece 54); up to there two, and three are no faster.
constexpr int kUpWaves = 4;
template <typename T, int VEC>
struct UpRows {
    ab_u32x4 y[4];
    __device__ __forceinline__ void load(const UpArgs &a, const int (&t)[4], int j) {
#pragma unroll
        for (int v = 0; v < 4; ++v)
            y[v] = a.y_in ? load16<T, VEC>(row_at<typename T::elem>(a.y_in, t[v], a.pitch_in), j, a.len)
                          : ab_u32x4{0u, 0u, 0u, 0u};
    }
};
template <typename T, int KT, int VEC>
__global__ __launch_bounds__(kUpWaves * 64, KT * T::pieces * sizeof(typename T::Frag) <= 192 ? 2 : 1) void adapter_up_kernel(UpArgs a, Route route, int size) {
    extern __shared__ __attribute__((aligned(16))) char up_lds[];
    typedef typename T::Frag Frag;
    typedef typename T::elem elem;
    Frag *blocks = reinterpret_cast<Frag *>(up_lds);  // [step][tile of columns][lane]
    const uint32_t group = blockIdx.x + blockIdx.y * (uint32_t)kGroupsX;
    const uint32_t block = group % (uint32_t)a.blocks;
    const Tile tile = find_tile<true>(route, size, (int)(group / (uint32_t)a.blocks));  // (beyond the last: none)
    if (tile.adapter < (a.copy ? -1 : 0)) return;
    const int32_t *__restrict__ order = route.order + tile.at;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, row16 = lane & 15, quad = lane >> 4;
    const int j_row = ((int)block * 16 + row16) * T::lane, j = column_base<T>(j_row, a.len);
    const int rank = adapter_rank(tile.adapter, a.ranks, a.r);
    const int steps = (rank + 31) / 32, last = tile.rows - 1;
    constexpr int round = kUpWaves * 16;
    // Two rounds of rows are on their way at any time; the row numbers of a later one go out before an earlier one's rows,
    // and so do the pieces of h of the next round, which take the places of this one's after the products.
    auto index_of = [&](int t0, int (&t)[4]) {
#pragma unroll
        for (int v = 0; v < 4; ++v) t[v] = order[min(t0 + quad * 4 + v, last)];
    };
    UpRows<T, VEC> r0, r1;
    Frag h[KT][T::pieces];
    auto load_h = [&](int t0) {
        const Frag *from = (const Frag *)a.h + (int64_t)(tile.block + min(t0, last) / 16) * (KT * T::pieces * 64) + lane;
#pragma unroll
        for (int s = 0; s < KT; ++s)
#pragma unroll
            for (int k = 0; k < T::pieces; ++k) h[s][k] = from[(s * T::pieces + k) * 64];
    };
    int t0 = wave * 16, i0[4], i1[4], n0[4], n1[4];
    index_of(t0, i0);
    index_of(t0 + round, i1);
    index_of(t0 + 2 * round, n0);
    index_of(t0 + 3 * round, n1);
    r0.load(a, i0, j);
    load_h(t0);
    r1.load(a, i1, j);
    for (int s = wave; s < steps; s += kUpWaves) {
        // (a column from the rank on is the last one again on its way, and zeros in the product)
        const elem *f = (const elem *)a.f + (int64_t)tile.adapter * a.r * a.len;
        ab_u32x4 rows[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            rows[i] = load16<T, VEC ? kAligned : kAnywhere>(f + (int64_t)min(s * 32 + quad * 8 + i, rank - 1) * a.len, j, a.len);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s * 32 + quad * 8 + i >= rank) rows[i] = ab_u32x4{0u, 0u, 0u, 0u};
        Frag turned[T::lane];
        turn(rows, turned);
#pragma unroll
        for (int c = 0; c < T::lane; ++c) blocks[(s * T::lane + c) * 64 + lane] = turned[c];
    }
    __syncthreads();
    auto products = [&](const UpRows<T, VEC> &r, int t0, const int (&t)[4]) {
        f32x4_t acc[T::lane];
#pragma unroll
        for (int c = 0; c < T::lane; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KT; ++s)
            if (s < steps)
#pragma unroll
                for (int c0 = 0; c0 < T::lane; c0 += 4) {
                    Frag f[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) f[c] = blocks[(s * T::lane + c0 + c) * 64 + lane];
#pragma unroll
                    for (int k = 0; k < T::pieces; ++k)
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[c0 + c] = T::mma(h[s][k], f[c], acc[c0 + c]);
                }
        load_h(t0 + round);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const bool valid = t0 + quad * 4 + v <= last;
            elem *out = const_cast<elem *>(row_at<elem>(a.y_out, t[v], a.pitch_out));
            ab_u32x4 w;
            if constexpr (T::lane == 8) {
#pragma unroll
                for (int p = 0; p < 4; ++p)
                    w[p] = pack2(low_bf16(r.y[v][p]) + acc[2 * p][v], high_bf16(r.y[v][p]) + acc[2 * p + 1][v]);
            } else {
#pragma unroll
                for (int p = 0; p < 4; ++p) w[p] = __float_as_uint(__uint_as_float(r.y[v][p]) + acc[p][v]);
            }
            if (valid) store16<T, VEC>(out, w, j, j_row, a.len);
        }
    };
    auto copy = [](int (&to)[4], const int (&from)[4]) {
#pragma unroll
        for (int v = 0; v < 4; ++v) to[v] = from[v];
    };
    for (; t0 <= last; t0 += 2 * round) {
        products(r0, t0, i0);
        copy(i0, n0);
        index_of(t0 + 4 * round, n0);
        r0.load(a, i0, j);
        if (t0 + round > last) break;
        products(r1, t0 + round, i1);
        copy(i1, n1);
        index_of(t0 + 5 * round, n1);
        r1.load(a, i1, j);
    }
}

// ---- few rows -----------------------------------------------------------------------------------------
// Where each row has an adapter of its own there is nothing to share: a workgroup has one row and 512 columns, its
// wavefronts every fourth column of the factor, and h stays in 32 bits.  The shares of h are added by every
// workgroup for itself.  96 rows of 64 adapters beside 28672 columns of ranks 16 and 8: 13 us for 44 MB of factors and 11 of y.
struct RowsArgs {
    const float *splits;  // rows x r, `stride` floats apart
    int64_t stride;
    int n;
    const int32_t *ids, *ranks;
    const float *scale;
    const void *f;        // count x r x len
    const void *y_in;     // or nullptr
    void *y_out;
    float *h_out;         // or nullptr
    uint32_t pitch_in, pitch_out;
    int len, r, count;
};
constexpr int kRowsCols = 512;
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void adapter_rows_kernel(RowsArgs a) {
    typedef typename T::elem elem;
    __shared__ float h[DLCX_MAX_RANK], sums[4][kRowsCols];
    const int t = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x / 64, id = a.ids[t];
    const int adapter = id >= 0 && id < a.count ? id : -1;
    const int rank = adapter_rank(adapter, a.ranks, a.r);
    if ((int)threadIdx.x < a.r) {
        const int c = threadIdx.x;
        float x = 0.f;
        if (c < rank)
            for (int k = 0; k < a.n; k += 8) {
                float part[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) part[u] = a.splits[min(k + u, a.n - 1) * a.stride + (int64_t)t * a.r + c];
#pragma unroll
                for (int u = 0; u < 8; ++u) x += k + u < a.n ? part[u] : 0.f;
            }
        if (a.h_out && blockIdx.x == 0) a.h_out[(int64_t)t * a.r + c] = x;
        h[c] = x * (adapter >= 0 && a.scale ? a.scale[adapter] : 1.f);
    }
    __syncthreads();
    const int j = blockIdx.x * kRowsCols + lane * 8;
    const elem *f = (const elem *)a.f + (int64_t)max(adapter, 0) * a.r * a.len;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const bool whole = j + 8 <= a.len;
#pragma unroll 4
    for (int c = wave; c < rank; c += 4) {
        const typename T::Frag w = whole ? T::template load8<VEC, true>(f + (int64_t)c * a.len, j, a.len)
                                         : T::template load8<false, false>(f + (int64_t)c * a.len, j, a.len);
        const float s = h[c];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += s * T::at(w, i);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave][lane * 8 + i] = acc[i];
    __syncthreads();
    const elem *in = row_at<elem>(a.y_in, t, a.pitch_in);
    elem *out = const_cast<elem *>(row_at<elem>(a.y_out, t, a.pitch_out));
#pragma unroll
    for (int k = threadIdx.x; k < kRowsCols; k += 256) {
        const int col = blockIdx.x * kRowsCols + k;
        if (col >= a.len) break;
        const float y = (sums[0][k] + sums[1][k]) + (sums[2][k] + sums[3][k]);
        out[col] = T::round(y + (a.y_in ? T::value(in[col]) : 0.f));
    }
}

// The same in one launch: every workgroup forms all of h for itself, its wavefronts the columns of h in turn (or,
// where those are fewer, shares of n), before its own kRowCols columns of y.
struct RowArgs {
    const void *x, *q;
    uint32_t pitch;
    int n;
};
constexpr int kRowWaves = 16, kRowParts = 8, kRowCols = kRowWaves / kRowParts * 512;
template <typename T, bool VEC>  // (not VEC and fewer than eight: those that there are)
__device__ __forceinline__ typename T::Frag load_row8(const typename T::elem *row, int at, int len) {
    if (!VEC && len < 8) return T::template load8<false, false>(row, at, len);
    return T::template load8<VEC, true>(row, at, len);
}
template <typename T, bool VEC>
__global__ __launch_bounds__(kRowWaves * 64) void adapter_row_kernel(RowArgs d, RowsArgs a) {
    typedef typename T::elem elem;
    typedef typename T::Frag Frag;
    __shared__ float part[DLCX_MAX_RANK], h[DLCX_MAX_RANK], sums[kRowParts][kRowCols];
    const int t = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x / 64, id = a.ids[t];
    const int adapter = id >= 0 && id < a.count ? id : -1;
    const int rank = adapter_rank(adapter, a.ranks, a.r);
    const elem *q = (const elem *)d.q + (int64_t)max(adapter, 0) * a.r * d.n;
    const elem *p = (const elem *)a.f + (int64_t)max(adapter, 0) * a.r * a.len;
    // what y needs is requested first: it does not depend on h
    const int col = blockIdx.x * kRowCols + (int)threadIdx.x, c0 = wave % kRowParts;
    // eight columns of y a lane; where fewer are left, the last eight, which others have too
    const int j0 = blockIdx.x * kRowCols + wave / kRowParts * 512 + lane * 8, j = min(j0, max(a.len - 8, 0));
    auto load_p = [&](int c) { return load_row8<T, VEC>(p + (int64_t)c * a.len, j, a.len); };
    const float y_in = a.y_in && col < a.len ? T::value(row_at<elem>(a.y_in, t, a.pitch_in)[col]) : 0.f;
    Frag w = rank > c0 ? load_p(c0) : T::zero();

    const elem *x = row_at<elem>(d.x, t, d.pitch);
    const int shares = rank > 0 && rank < kRowWaves ? kRowWaves / rank : 1;
    const int share = (d.n + shares * 512 - 1) / (shares * 512) * 512;
    for (int k = wave; k < rank * shares; k += kRowWaves) {
        const int from = k % shares * share, to = min(from + share, d.n);
        const elem *row = q + (int64_t)(k / shares) * d.n;
        float acc = 0.f;
#pragma unroll 4
        for (int i = from + lane * 8; i < to; i += 512) {
            const int at = VEC ? i : min(i, max(d.n - 8, 0));
            Frag u = load_row8<T, VEC>(row, at, d.n), v = load_row8<T, VEC>(x, at, d.n);
            if (!VEC && at < i) {
                T::drop(u, i - at);
                T::drop(v, i - at);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) acc = fmaf(T::at(u, e), T::at(v, e), acc);
        }
        for (int e = 32; e > 0; e >>= 1) acc += __shfl_xor(acc, e, 64);
        if (lane == 0) part[k] = acc;
    }
    __syncthreads();
    if ((int)threadIdx.x < a.r) {
        const int c = threadIdx.x;
        float sum = 0.f;
        if (c < rank)
            for (int k = 0; k < shares; ++k) sum += part[c * shares + k];
        if (a.h_out && blockIdx.x == 0) a.h_out[(int64_t)t * a.r + c] = sum;
        h[c] = sum * (adapter >= 0 && a.scale ? a.scale[adapter] : 1.f);
    }
    __syncthreads();
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int c = c0; c < rank; c += kRowParts) {
        const Frag next = c + kRowParts < rank ? load_p(c + kRowParts) : T::zero();
        const float s = h[c];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += s * T::at(w, i);
        w = next;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = (VEC ? j0 : j) + i - (int)blockIdx.x * kRowCols;
        if (VEC || at >= 0) sums[c0][at] = acc[i];
    }
    __syncthreads();
    if (col >= a.len) return;
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < kRowParts; ++k) y += sums[k][threadIdx.x];
    const_cast<elem *>(row_at<elem>(a.y_out, t, a.pitch_out))[col] = T::round(y + y_in);
}

// ---- grad -------------------------------------------------------------------------------------------
struct GradProduct {
    const void *u;       // turned operand
    const float *scale;
    const void *z;       // rows x len
    uint32_t pitch;
    float *out;          // count x r x len
    float *slabs;        // slab x r x len
    int len, vec;
};
struct GradArgs {
    GradProduct prod[2];
    const int32_t *ranks;
    int r, steps, blocks0, blocks;  // column blocks of the first product and of both
};

// A wavefront has 256 bytes of columns, CT x 16 columns of the factor and rows of one adapter, 32 at a time, the next
// ones requested before the products of these.  In long tiles the workgroup's wavefronts take rows in
// turn and join their sums in LDS; in tiles of up to kGradShort rows there is little to share (79 rows of 57
// adapters, rank 45, fp32: 82 us that way, 39 this) and each has columns of its own.
// 16384 rows of 8192 + 8192 columns at rank 64: 132 us, 4.1 TB/s.  128 accumulators leave a wavefront registers for
// one set of rows on its way, and requests come back in order: the operands of all but a round's first product are asked
// for behind the rows of the next round and wait for them.
constexpr int kGradWaves = 4;
struct RowIndex {
    int t[8];
    __device__ __forceinline__ void load(const int32_t *__restrict__ order, int t0, int rows) {
        const int quad = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = order[min(t0 + quad * 8 + i, rows - 1)];
    }
};
template <typename T, int VEC>
__device__ __forceinline__ void load_rows(ab_u32x4 (&z)[8], const GradProduct &p, const RowIndex &at, int j) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        z[i] = load16<T, VEC>(row_at<typename T::elem>(p.z, at.t[i], p.pitch), j, p.len);
}
template <typename T, int CT, int VEC, int SPLIT>
__device__ __forceinline__ void adapter_grad_rows(const GradProduct &p, int r, int rank, int steps, const Tile &tile,
                                                  const int32_t *__restrict__ order, int c0, int j0,
                                                  f32x4_t (*sums)[CT * T::lane][64]) {
    typedef typename T::Frag Frag;
    const int lane = threadIdx.x & 63, row16 = lane & 15, quad = lane >> 4;
    const int wave = SPLIT == 1 ? 0 : threadIdx.x / 64;
    f32x4_t acc[CT][T::lane];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int s = 0; s < T::lane; ++s) acc[c][s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int j_row = j0 + T::lane * row16, j = column_base<T>(j_row, p.len);
    const Frag *u = (const Frag *)p.u + ((int64_t)(tile.block / 2) * steps * 2 + c0 / 16) * T::pieces * 64 + lane;
    const int64_t u_block = (int64_t)steps * 2 * T::pieces * 64;
    ab_u32x4 z[8];
    RowIndex at;
    at.load(order, wave * 32, tile.rows);
    load_rows<T, VEC>(z, p, at, j);
    at.load(order, wave * 32 + SPLIT * 32, tile.rows);
    Frag f[2][T::pieces];
    auto load_u = [&](Frag (&to)[T::pieces], int t0, int c) {
#pragma unroll
        for (int h = 0; h < T::pieces; ++h) to[h] = u[(t0 / 32) * u_block + (c * T::pieces + h) * 64];
    };
    const int ct = min(CT, (steps * 32 - c0) / 16);  // columns that there are operands for
    if (wave * 32 < tile.rows) load_u(f[0], wave * 32, 0);
    for (int t0 = wave * 32; t0 < tile.rows; t0 += SPLIT * 32) {
        const int t1 = t0 + SPLIT * 32 < tile.rows ? t0 + SPLIT * 32 : t0;
        if (t0 + 32 > tile.rows)  // zeros in the places of rows beyond the last one, as in u: 0 x Inf would not be 0
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (t0 + quad * 8 + i >= tile.rows) z[i] = ab_u32x4{0u, 0u, 0u, 0u};
        Frag turned[T::lane];
        turn(z, turned);
        load_rows<T, VEC>(z, p, at, j);
        at.load(order, t0 + 2 * SPLIT * 32, tile.rows);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            load_u(f[(c + 1) & 1], c + 1 < CT ? t0 : t1, c + 1 < CT ? min(c + 1, ct - 1) : 0);
            if (c < ct)
#pragma unroll
                for (int h = 0; h < T::pieces; ++h)
#pragma unroll
                    for (int s = 0; s < T::lane; ++s) acc[c][s] = T::mma(f[c & 1][h], turned[s], acc[c][s]);
        }
        if constexpr (CT & 1) {
#pragma unroll
            for (int h = 0; h < T::pieces; ++h) f[0][h] = f[1][h];
        }
    }
#pragma unroll
    for (int half = SPLIT / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int s = 0; s < T::lane; ++s) sums[wave - half][c * T::lane + s][lane] = acc[c][s];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int s = 0; s < T::lane; ++s) acc[c][s] += sums[wave][c * T::lane + s][lane];
        __syncthreads();
    }
    if (wave != 0) return;
    const float scale = p.scale ? p.scale[tile.adapter] : 1.f;
    float *out = tile.slab < 0 ? p.out + (int64_t)tile.adapter * r * p.len : p.slabs + (int64_t)tile.slab * r * p.len;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int col = c0 + c * 16 + quad * 4 + v;
            if (col >= r) continue;
            float *row = out + (int64_t)col * p.len;
#pragma unroll
            for (int s = 0; s < T::lane; s += 4) {
                f32x4_t w = {scale * acc[c][s][v], scale * acc[c][s + 1][v], scale * acc[c][s + 2][v],
                             scale * acc[c][s + 3][v]};
                if (col >= rank) w = f32x4_t{0.f, 0.f, 0.f, 0.f};  // (zeros of u times what is not finite are none)
                if (VEC || j_row + T::lane <= p.len) {
                    if (j_row >= p.len) continue;
                    if constexpr (VEC) *reinterpret_cast<f32x4_t *>(row + j + s) = w;
                    else __builtin_memcpy(row + j + s, &w, sizeof w);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (j + s + i >= j_row && j + s + i < p.len) row[j + s + i] = w[i];
                }
            }
        }
}
// SPLIT wavefronts share the rows of a block of columns, or (1) each has a block of its own.
template <typename T, int CT, int VEC, int SPLIT>
__global__ __launch_bounds__(kGradWaves * 64, 2) void adapter_grad_kernel(GradArgs a, Route route, int size) {
    __shared__ f32x4_t sums[SPLIT == 1 ? 1 : SPLIT / 2][SPLIT == 1 ? 1 : CT * T::lane][64];
    const Tile tile = find_tile<false>(route, size, blockIdx.y);
    if (tile.adapter < 0) return;
    const int32_t *__restrict__ order = route.order + tile.at;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int block = SPLIT == 1 ? (int)blockIdx.x * kGradWaves + wave : (int)blockIdx.x;
    if (block >= a.blocks) return;
    const int second = block >= a.blocks0;
    const GradProduct &p = a.prod[second];
    const int j0 = (block - (second ? a.blocks0 : 0)) * 16 * T::lane, c0 = blockIdx.z * CT * 16;
    adapter_grad_rows<T, CT, VEC, SPLIT>(p, a.r, adapter_rank(tile.adapter, a.ranks, a.r), a.steps, tile, order, c0, j0,
                                         reinterpret_cast<f32x4_t (*)[CT * T::lane][64]>(&sums));
}

// Gradients of adapters with several tiles, as the sum of their slabs in the rows' order, and zeros for
// adapters without rows.
__global__ __launch_bounds__(256) void adapter_sum_kernel(GradArgs a, Route route, int size) {
    int tiles = 0, slab = 0;
    for (int b = threadIdx.x & 63; b <= (int)blockIdx.y; b += 64) {
        const int n = (route.first[b + 1] - route.first[b] + size - 1) / size;
        if (b == (int)blockIdx.y) tiles = n;
        else slab += n > 1 ? n : 0;
    }
    tiles = __builtin_amdgcn_readlane(scan_wave(tiles), 63);
    slab = __builtin_amdgcn_readlane(scan_wave(slab), 63);
    if (tiles == 1) return;
    const GradProduct &p = a.prod[blockIdx.z];
    const int64_t elems = (int64_t)a.r * p.len;
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < elems; e += step) {
        double sum = 0.0;
        for (int k = 0; k < tiles; ++k) sum += p.slabs[(slab + k) * elems + e];
        p.out[blockIdx.y * elems + e] = (float)sum;
    }
}

// ---- launches -----------------------------------------------------------------------------------------
static int launch_route(int64_t rows, const int32_t *ids, const Route &r, hipStream_t st) {
    const size_t lds = (size_t)kRouteWaves * ((r.count + 1) * sizeof(int) + kRouteKept * sizeof(uint16_t));
    static size_t granted = 0;
    int rc = grant_dynamic_lds((const void *)adapter_route_kernel, lds, &granted, "adapter_route lds");
    if (rc != DLCX_OK) return rc;
    Timed timed(KID_ADAPTER_ROUTE, st);
    adapter_route_kernel<<<1, kRouteThreads, lds, st>>>((int)rows, ids, r);
    return check_launch("adapter_route");
}

static inline bool rows_aligned(const void *p, uint32_t pitch) { return aligned16(p) && pitch % 16 == 0; }

// Steps of 32 columns of a factor that the up product is built for.
static int up_steps(int r) { return r <= 32 ? 1 : r <= 64 ? 2 : r <= 128 ? 4 : 8; }
constexpr int kUpRows = 256, kDownRows = 256;  // most rows of a workgroup

static int down_tiles(int r) { return r > 32 ? 4 : r > 16 ? 2 : 1; }
// Shares of a reduction over `len` elements.
template <typename T>
static int down_splits(int64_t len, int r) {
    return (int)ceil_div(len, kDownWaves * 32 * down_steps<T>(down_tiles(r)));
}

template <typename T>
static int access(bool aligned, int64_t rows, int64_t len) {
    if (!aligned) return kAnywhere;
    return rows * len * (int64_t)sizeof(typename T::elem) >= kStreamed ? kStream : kAligned;
}
template <typename T, int CT>
static void down_kernel(const DownArgs &a, int vec, dim3 grid, const Route &v, int size, hipStream_t st) {
    if (vec == kAnywhere) {
        adapter_down_kernel<T, CT, kAnywhere><<<grid, kDownWaves * 64, 0, st>>>(a, v, size);
        return;
    }
    if constexpr (T::lane == 8)  // (fp32 rows: plain)
        if (vec == kStream && grid.y == 1) {
            adapter_down_kernel<T, CT, kStream><<<grid, kDownWaves * 64, 0, st>>>(a, v, size);
            return;
        }
    adapter_down_kernel<T, CT, kAligned><<<grid, kDownWaves * 64, 0, st>>>(a, v, size);
}
template <typename T>
static int launch_down(DownArgs a, int64_t rows, const Route &v, hipStream_t st) {
    const int ct = down_tiles(a.r), splits = down_splits<T>(a.len, a.r);
    const int vec = access<T>(rows_aligned(a.x, a.pitch) && aligned16(a.f) && a.len % 8 == 0, rows, a.len);
    const int64_t cols = ceil_div(a.r, ct * 16);
    // as few rows as two workgroups to a compute unit leave, half a tile more for every adapter
    const int64_t most = ceil_div(512, splits * cols), spare = v.count < most ? v.count / 2 : most / 2;
    int64_t fit = ceil_div(ceil_div(rows, most > spare ? most - spare : 1), 16) * 16;
    const int size = (int)(fit < kDownRows ? fit : kDownRows);
    const int64_t tiles = v.ids ? rows : max_tiles(rows, v.count, size), groups = splits * tiles;
    if (groups > 0x7FFFFFFF) return DLCX_EINVAL;
    a.shares = splits;
    a.tiles = (int)tiles;
    const dim3 grid(groups_x(groups), (unsigned)cols, groups_on(groups));
    Timed timed(KID_ADAPTER_DOWN, st);
    if (ct == 4) down_kernel<T, 4>(a, vec, grid, v, size, st);
    else if (ct == 2) down_kernel<T, 2>(a, vec, grid, v, size, st);
    else down_kernel<T, 1>(a, vec, grid, v, size, st);
    return check_launch("adapter_down");
}

// Few rows in one launch, where forming h in every workgroup costs less than a second launch: Q_a up to 300 KB, read by all
// workgroups together up to 20 MB, and not more of them than the GPU holds at once.  us alone on the GPU and called from
// the host, in two launches -> one: 1 row of 2048 + 2048 columns at rank 8: 6.6, 13 -> 4.6, 10; 128 rows of 64 adapters
// of the same 7.7, 15 -> 5.5, 10; 8192 + 8192 at rank 16, 1 row 7.5, 13 -> 7.5, 9.  Beyond: 16 rows there (33 MB) 8.1, 13
// -> 11.2, 11; rank 64 there (1 MB), 1 row 10.5, 14 -> 20, 20; 512 rows of the first (1024 workgroups) 10.3, 13 -> 15.1, 15.
template <typename T>
static bool one_launch(int64_t rows, int r, int64_t n, int64_t m) {
    const int64_t bytes = r * n * (int64_t)sizeof(typename T::elem), groups = rows * ceil_div(m, kRowCols);
    return bytes <= 300000 && groups <= 512 && groups * bytes <= 20000000;
}

// A row to a workgroup: its time grows with rows x (16 + r) (the matrix instructions take 16 rows at least) and the bytes of a
// row, of which those of an fp32 row count half as much again in the first product and two thirds in the second.  Tiles read
// a factor once for 16 rows or more, but take two launches more, the sorting, and a tile with its columns' blocks for every
// adapter that has rows; which have is known on the device alone, so `count` stands for it, up to 64.  Both sides in us,
// rows / tiles, of one adapter and of 64:
//   8192 x 8192 bf16, forward    rank 1   256 rows 15 / 20, 15 / 33    1024 rows 46 / 28, 47 / 40
//                                rank 16  128 rows 13 / 20, 15 / 34     512 rows 37 / 22, 40 / 40
//                                rank 64   64 rows 17 / 23, 23 / 40     256 rows 50 / 24, 62 / 49
//                     backward   rank 1   128 rows 27 / 28, 31 / 44     256 rows 35 / 31, 38 / 47
//                                rank 64   32 rows 30 / 31, 88 / 93     128 rows 56 / 42, 130 / 134
//   8192 x 8192 fp32, forward    rank 8   128 rows 18 / 23, 20 / 53     512 rows 54 / 32, 55 / 60
//   2048 x 2048 bf16, forward    rank 16  512 rows 14 / 21, 14 / 23    1024 rows 23 / 22, 25 / 25
//   28672 x 8192 bf16, forward   rank 16  128 rows 21 / 22, 28 / 72     512 rows 68 / 34, 78 / 90
// Of 760 calls timed in both forms (64 x 64 to 8192 x 8192, ranks 1 to 64, 16 to 4096 rows, both types) the rule takes the
// slower one by more than an eighth in six.
constexpr int64_t kRowsForward = 250000000, kRowsBackward = 75000000;
template <typename T>
static bool few_rows(int64_t rows, const dlcx_adapter_desc &d, int64_t down, int64_t up, int64_t most) {
    const bool low = T::lane == 8;
    const int64_t one = low ? 2 * (down + up) : 6 * down + 8 * up / 3;
    const int64_t n = rows < 64 ? rows : 64, adapters = d.count < n ? d.count : n;
    return rows <= 4096 &&  // (the launch has them along y)
           rows * (16 + d.r) * (one > 4800 ? one : 4800) <= most + adapters * 188 * up * (low ? 2 : 4);
}

template <typename T>
static bool forward_by_rows(int64_t rows, const dlcx_adapter_desc &d) {
    return one_launch<T>(rows, d.r, d.n, d.m) || few_rows<T>(rows, d, d.n, d.m, kRowsForward);
}
template <typename T>
static bool backward_by_rows(int64_t rows, const dlcx_adapter_desc &d) {
    return few_rows<T>(rows, d, d.m, d.n, kRowsBackward);
}

template <typename T>
static int launch_operands(const OperandArgs &a, int jobs, int64_t rows, const Route &v, hipStream_t st) {
    Timed timed(KID_ADAPTER_OPERAND, st);
    adapter_operand_kernel<T><<<dim3((unsigned)max_tiles(rows, v.count, 32), (unsigned)jobs,
                                              (unsigned)ceil_div(a.steps, 2)), 256, 0, st>>>(a, v);
    return check_launch("adapter_operand");
}

template <typename T, int KT, int VEC>
static int up_kernel(const UpArgs &a, dim3 grid, const Route &v, int size, hipStream_t st) {
    const size_t lds = (size_t)KT * T::lane * 64 * sizeof(typename T::Frag);
    static size_t granted = 0;
    const int rc = grant_dynamic_lds((const void *)adapter_up_kernel<T, KT, VEC>, lds, &granted, "adapter_up lds");
    if (rc != DLCX_OK) return rc;
    Timed timed(KID_ADAPTER_UP, st);
    adapter_up_kernel<T, KT, VEC><<<grid, kUpWaves * 64, lds, st>>>(a, v, size);
    return check_launch("adapter_up");
}
template <typename T, int KT>
static int up_kernel(const UpArgs &a, int vec, dim3 grid, const Route &v, int size, hipStream_t st) {
    return vec == kStream    ? up_kernel<T, KT, kStream>(a, grid, v, size, st)
           : vec == kAligned ? up_kernel<T, KT, kAligned>(a, grid, v, size, st)
                             : up_kernel<T, KT, kAnywhere>(a, grid, v, size, st);
}
template <typename T>
static int launch_up(UpArgs a, int64_t rows, const Route &v, hipStream_t st) {
    const int es = sizeof(typename T::elem);
    const int vec = access<T>(aligned16(a.f) && (int64_t)a.len * es % 16 == 0 && rows_aligned(a.y_out, a.pitch_out) &&
                                  (!a.y_in || rows_aligned(a.y_in, a.pitch_in)),
                              rows, a.len);
    const int64_t cols = ceil_div(a.len, 16 * T::lane);
    int size = kUpRows;
    while (size > 64 && ceil_div(rows, size) * cols < 1024) size /= 2;
    const int64_t groups = cols * max_tiles(rows, v.count, size);
    if (groups > 0x7FFFFFFF) return DLCX_EINVAL;
    a.blocks = (int)cols;
    const dim3 grid(groups_x(groups), groups_on(groups));
    switch (up_steps(a.r)) {
    case 1: return up_kernel<T, 1>(a, vec, grid, v, size, st);
    case 2: return up_kernel<T, 2>(a, vec, grid, v, size, st);
    case 4: return up_kernel<T, 4>(a, vec, grid, v, size, st);
    default: return up_kernel<T, 8>(a, vec, grid, v, size, st);
    }
}

constexpr int kGradGroups = 512;
static int grad_size(int64_t rows, int64_t m, int64_t n, int lane) {
    const int64_t cols = ceil_div(m, 16 * lane) + ceil_div(n, 16 * lane);
    int size = 4096;
    while (size > 64 && ceil_div(rows, size) * cols < kGradGroups) size /= 2;
    return size;
}
constexpr int kGradShort = 128;
template <typename T, int CT>
static void grad_kernel(const GradArgs &a, int vec, dim3 grid, const Route &v, int size, hipStream_t st) {
    if (size <= kGradShort) {  // (rows of kStreamed bytes in tiles as short as these are read plainly)
        grid.x = (grid.x + kGradWaves - 1) / kGradWaves;
        if (vec != kAnywhere)
            adapter_grad_kernel<T, CT, kAligned, 1><<<grid, kGradWaves * 64, 0, st>>>(a, v, size);
        else
            adapter_grad_kernel<T, CT, kAnywhere, 1><<<grid, kGradWaves * 64, 0, st>>>(a, v, size);
    } else if (vec == kStream && grid.z == 1) {
        adapter_grad_kernel<T, CT, kStream, kGradWaves><<<grid, kGradWaves * 64, 0, st>>>(a, v, size);
    } else if (vec != kAnywhere) {
        adapter_grad_kernel<T, CT, kAligned, kGradWaves><<<grid, kGradWaves * 64, 0, st>>>(a, v, size);
    } else {
        adapter_grad_kernel<T, CT, kAnywhere, kGradWaves><<<grid, kGradWaves * 64, 0, st>>>(a, v, size);
    }
}
template <typename T>
static int launch_grad(const GradArgs &a, int64_t rows, int count, int size, const Route &v, hipStream_t st) {
    if (rows > 0) {
        const int ct = a.r > 32 ? 4 : a.r > 16 ? 2 : 1;
        const dim3 grid((unsigned)a.blocks, (unsigned)max_tiles(rows, count, size), (unsigned)ceil_div(a.r, ct * 16));
        Timed timed(KID_ADAPTER_GRAD, st);
        const int64_t longer = a.prod[0].len > a.prod[1].len ? a.prod[0].len : a.prod[1].len;
        const int vec = access<T>(a.prod[0].vec && a.prod[1].vec, rows, longer);
        if (ct == 4) grad_kernel<T, 4>(a, vec, grid, v, size, st);
        else if (ct == 2) grad_kernel<T, 2>(a, vec, grid, v, size, st);
        else grad_kernel<T, 1>(a, vec, grid, v, size, st);
        const int rc = check_launch("adapter_grad");
        if (rc != DLCX_OK) return rc;
    }
    const int64_t most = (int64_t)a.r * (a.prod[0].len > a.prod[1].len ? a.prod[0].len : a.prod[1].len);
    const int64_t gx = ceil_div(most, 1024);
    Timed timed(KID_ADAPTER_SUM, st);
    adapter_sum_kernel<<<dim3((unsigned)(gx < 256 ? gx : 256), (unsigned)count, 2), 256, 0, st>>>(a, v,
                                                                                                      size);
    return check_launch("adapter_sum");
}

// ---- workspace: [own route][shares of h or g][operands][slabs of dP][slabs of dQ] ----------------
// Room for `rows` rows has room for fewer, though their gradients have smaller tiles.  Slabs: at most two for every full tile (of
// adapters with more than one); tiles below the largest size are taken only where twice as large
// ones make less than kGradGroups workgroups, so there are less than 2 kGradGroups / cols of them.
struct AdapterSpace {
    Route route;
    float *split, *slab_p, *slab_q;
    void *up, *turned_h, *turned_g;
};
static size_t adapter_space(const dlcx_adapter_desc *d, int64_t rows, void *base, AdapterSpace *s) {
    AdapterSpace w;
    size_t at = route_view(rows, d->count, (char *)base, &w.route);
    auto take = [&](size_t bytes) {
        char *p = (char *)base + at;
        at += a256x(bytes);
        return (float *)p;
    };
    const bool low = d->dtype == DLCX_BF16;
    const int lane = low ? Bf16::lane : F32::lane;
    const size_t frag = low ? sizeof(Bf16::Frag) * Bf16::pieces : sizeof(F32::Frag) * F32::pieces;
    const int64_t cols = ceil_div(d->m, 16 * lane) + ceil_div(d->n, 16 * lane);
    const size_t row = (size_t)d->r * sizeof(float), steps = (size_t)up_steps(d->r);
    const int64_t longer = d->m > d->n ? d->m : d->n;
    w.split = take(row * (size_t)(rows * (low ? down_splits<Bf16>(longer, d->r) : down_splits<F32>(longer, d->r))));
    const size_t turned = (size_t)max_tiles(rows, d->count, 32) * steps * 2 * 64 * frag;  // (of both forms)
    w.up = take(turned);
    w.turned_h = take(turned);
    w.turned_g = take(turned);
    const int64_t small = 2 * (rows / 64), mid = ceil_div(kGradGroups * 4, cols), large = 2 * (rows / 4096);
    const int64_t slabs = small < mid ? small : mid > large ? mid : large;
    w.slab_p = take(row * (size_t)(slabs * d->m));
    w.slab_q = take(row * (size_t)(slabs * d->n));
    if (s) *s = w;
    return at;
}

// `operands`: the two matrices that the sums over rows need are formed as well (of the first, what down leaves).
template <typename T>
static int down_and_rows(const DownArgs &down, RowsArgs a, int64_t rows, OperandArgs *operands, const AdapterSpace &s,
                         hipStream_t st) {
    DownArgs d = down;
    d.stride = rows * d.r;
    d.out = s.split;
    if (!operands && one_launch<T>(rows, d.r, d.len, a.len)) {
        const RowArgs x = {d.x, d.f, d.pitch, d.len};
        const bool vec = aligned16(d.x) && aligned16(d.f) && aligned16(a.f) && d.pitch % 16 == 0 && d.len % 8 == 0 &&
                         a.len % 8 == 0;
        const dim3 grid((unsigned)ceil_div(a.len, kRowCols), (unsigned)rows);
        Timed timed(KID_ADAPTER_ROWS, st);
        if (vec) adapter_row_kernel<T, true><<<grid, kRowWaves * 64, 0, st>>>(x, a);
        else adapter_row_kernel<T, false><<<grid, kRowWaves * 64, 0, st>>>(x, a);
        return check_launch("adapter_rows");
    }
    const Route by_row = {nullptr, nullptr, a.count, a.ids};
    int rc = launch_down<T>(d, rows, by_row, st);
    if (rc != DLCX_OK) return rc;
    a.splits = s.split;
    a.stride = d.stride;
    a.n = down_splits<T>(d.len, d.r);
    if (operands) {
        OperandJob &g = operands->job[0];
        g.splits = a.splits;
        g.stride = a.stride;
        g.n = a.n;
        rc = launch_operands<T>(*operands, 2, rows, s.route, st);
        if (rc != DLCX_OK) return rc;
    }
    const bool vec = aligned16(a.f) && a.len % 8 == 0;
    const dim3 grid((unsigned)ceil_div(a.len, kRowsCols), (unsigned)rows);
    Timed timed(KID_ADAPTER_ROWS, st);
    if (vec) adapter_rows_kernel<T, true><<<grid, 256, 0, st>>>(a);
    else adapter_rows_kernel<T, false><<<grid, 256, 0, st>>>(a);
    return check_launch("adapter_rows");
}

// h = x F^T, then y_out = y_in + h G: the forward pass, and the first half of the gradient.  `job` says what
// becomes of h; `other` of a second matrix of its form, or nullptr.
template <typename T>
static int down_and_up(const DownArgs &down, OperandJob job, const OperandJob *other, const UpArgs &up, int64_t rows,
                       const AdapterSpace &s, hipStream_t st) {
    DownArgs d = down;
    d.stride = rows * d.r;
    d.out = s.split;
    int rc = launch_down<T>(d, rows, s.route, st);
    if (rc != DLCX_OK) return rc;
    job.splits = s.split;
    job.stride = d.stride;
    job.n = down_splits<T>(d.len, d.r);
    job.up = s.up;
    OperandArgs o = {{job, other ? *other : job}, d.ranks, d.r, up_steps(d.r)};
    rc = launch_operands<T>(o, other ? 2 : 1, rows, s.route, st);
    if (rc != DLCX_OK) return rc;
    UpArgs u = up;
    u.h = s.up;
    u.copy = u.y_in != u.y_out;  // (a row without adapter stays as it is where it is updated in place)
    return launch_up<T>(u, rows, s.route, st);
}

}  // namespace dlcx

using namespace dlcx;

// ---- entry points -------------------------------------------------------------------------------------
extern "C" {

static int check_adapter(const dlcx_adapter_desc *d, int64_t rows) {
    if (!d || rows < 0 || rows > (1 << 24)) return DLCX_EINVAL;
    if (d->m < 1 || d->n < 1 || d->m > (1 << 24) || d->n > (1 << 24)) return DLCX_EINVAL;
    if (d->r < 1 || d->r > DLCX_MAX_RANK || d->count < 1 || d->count > DLCX_MAX_ADAPTERS) return DLCX_EINVAL;
    if (d->dtype != DLCX_F32 && d->dtype != DLCX_BF16) return DLCX_EINVAL;
    return DLCX_OK;
}
constexpr int64_t kMaxStride = 1 << 29;  // elements; 32 bits of bytes
static bool misaligned(const void *p, unsigned to) { return ((uintptr_t)p & (to - 1)) != 0; }

size_t dlcx_adapter_route_bytes(int64_t rows, int32_t count) {
    if (rows < 0 || rows > (1 << 24) || count < 1 || count > DLCX_MAX_ADAPTERS) return 0;
    return route_view(rows, count, nullptr, nullptr);
}

int dlcx_adapter_route(int64_t rows, const int32_t *ids, int32_t count, void *route, void *stream) {
    if (rows < 0 || rows > (1 << 24) || count < 1 || count > DLCX_MAX_ADAPTERS) return DLCX_EINVAL;
    if (!route || misaligned(route, 256) || (rows > 0 && (!ids || misaligned(ids, 4)))) return DLCX_EINVAL;
    Route v;
    route_view(rows, count, (char *)route, &v);
    return launch_route(rows, ids, v, as_stream(stream));
}

size_t dlcx_adapter_workspace_bytes(const dlcx_adapter_desc *desc, int64_t rows) {
    if (check_adapter(desc, rows) != DLCX_OK) return 0;
    return adapter_space(desc, rows, nullptr, nullptr);
}

int dlcx_adapter_forward(const dlcx_adapter_desc *desc, int64_t rows, const void *x, int64_t ldx,
                         const int32_t *ids, const void *q, const void *p, const float *scale,
                         const int32_t *ranks, const void *route, const void *y_in, int64_t ldy_in,
                         void *y_out, int64_t ldy_out, float *h_out, void *workspace, void *stream) {
    int rc = check_adapter(desc, rows);
    if (rc != DLCX_OK) return rc;
    if (rows == 0) return DLCX_OK;
    const unsigned es = desc->dtype == DLCX_BF16 ? 2 : 4;
    if (!x || !ids || !q || !p || !y_out || !h_out || !workspace) return DLCX_EINVAL;
    if (misaligned(x, es) || misaligned(q, es) || misaligned(p, es) || misaligned(y_in, es) || misaligned(y_out, es))
        return DLCX_EINVAL;
    if (misaligned(ids, 4) || misaligned(scale, 4) || misaligned(ranks, 4) || misaligned(h_out, 4)) return DLCX_EINVAL;
    if (misaligned(workspace, 256) || misaligned(route, 256)) return DLCX_EINVAL;
    if (ldx < desc->n || ldy_out < desc->m || (y_in && ldy_in < desc->m)) return DLCX_EINVAL;
    if (ldx > kMaxStride || ldy_out > kMaxStride || (y_in && ldy_in > kMaxStride)) return DLCX_EINVAL;
    if (y_in == y_out && ldy_in != ldy_out) return DLCX_EINVAL;
    hipStream_t st = as_stream(stream);
    auto pitch = [es](int64_t ld) { return (uint32_t)(ld * es); };
    AdapterSpace s;
    adapter_space(desc, rows, workspace, &s);
    const DownArgs down = {x, pitch(ldx), q, ranks, nullptr, 0, (int)desc->n, desc->r, 1, 0};
    if (desc->dtype == DLCX_BF16 ? forward_by_rows<Bf16>(rows, *desc) : forward_by_rows<F32>(rows, *desc)) {
        const RowsArgs a = {nullptr, 0, 0, ids, ranks, scale, p, y_in, y_out, h_out, pitch(ldy_in), pitch(ldy_out),
                            (int)desc->m, desc->r, desc->count};
        return desc->dtype == DLCX_BF16 ? down_and_rows<Bf16>(down, a, rows, nullptr, s, st)
                                        : down_and_rows<F32>(down, a, rows, nullptr, s, st);
    }
    if (route)
        route_view(rows, desc->count, (char *)const_cast<void *>(route), &s.route);
    else if ((rc = launch_route(rows, ids, s.route, st)) != DLCX_OK)
        return rc;
    const OperandJob job = {nullptr, 0, 0, 1, nullptr, scale, h_out, nullptr, nullptr};
    const UpArgs up = {nullptr, p, ranks, y_in, y_out, pitch(ldy_in), pitch(ldy_out), (int)desc->m, desc->r, 0, 1};
    return desc->dtype == DLCX_BF16 ? down_and_up<Bf16>(down, job, nullptr, up, rows, s, st)
                                    : down_and_up<F32>(down, job, nullptr, up, rows, s, st);
}

int dlcx_adapter_backward(const dlcx_adapter_desc *desc, int64_t rows, const void *x, int64_t ldx,
                          const void *dy, int64_t lddy, const int32_t *ids, const void *q,
                          const void *p, const float *scale, const int32_t *ranks, const void *route,
                          const float *h, const void *dx_in, int64_t lddx_in, void *dx_out,
                          int64_t lddx_out, float *dq_out, float *dp_out, void *workspace,
                          void *stream) {
    int rc = check_adapter(desc, rows);
    if (rc != DLCX_OK) return rc;
    const unsigned es = desc->dtype == DLCX_BF16 ? 2 : 4;
    if (!q || !p || !dq_out || !dp_out || !workspace) return DLCX_EINVAL;
    if (rows > 0 && (!x || !dy || !ids || !h || !dx_out)) return DLCX_EINVAL;
    if (misaligned(x, es) || misaligned(dy, es) || misaligned(q, es) || misaligned(p, es) || misaligned(dx_in, es) ||
        misaligned(dx_out, es))
        return DLCX_EINVAL;
    if (misaligned(ids, 4) || misaligned(scale, 4) || misaligned(ranks, 4) || misaligned(h, 4) ||
        misaligned(dq_out, 4) || misaligned(dp_out, 4))
        return DLCX_EINVAL;
    if (misaligned(workspace, 256) || misaligned(route, 256)) return DLCX_EINVAL;
    if (rows > 0 && (ldx < desc->n || lddy < desc->m || lddx_out < desc->n || (dx_in && lddx_in < desc->n)))
        return DLCX_EINVAL;
    if (rows > 0 && (ldx > kMaxStride || lddy > kMaxStride || lddx_out > kMaxStride || (dx_in && lddx_in > kMaxStride)))
        return DLCX_EINVAL;
    if (rows > 0 && dx_in == dx_out && lddx_in != lddx_out) return DLCX_EINVAL;
    hipStream_t st = as_stream(stream);
    auto pitch = [es](int64_t ld) { return (uint32_t)(ld * es); };
    AdapterSpace s;
    adapter_space(desc, rows, workspace, &s);
    if (route)
        route_view(rows, desc->count, (char *)const_cast<void *>(route), &s.route);
    else if ((rc = launch_route(rows, ids, s.route, st)) != DLCX_OK)
        return rc;
    if (rows > 0) {
        const bool low = desc->dtype == DLCX_BF16, few = low ? backward_by_rows<Bf16>(rows, *desc) : backward_by_rows<F32>(rows, *desc);
        const DownArgs down = {dy, pitch(lddy), p, ranks, nullptr, 0, (int)desc->m, desc->r, 1, 0};
        const OperandJob g = {nullptr, 0, 0, few ? 0 : 1, scale, scale, nullptr, nullptr, s.turned_g};
        const OperandJob hj = {h, 0, 1, 0, nullptr, nullptr, nullptr, nullptr, s.turned_h};
        if (few) {
            const RowsArgs a = {nullptr, 0, 0, ids, ranks, scale, q, dx_in, dx_out, nullptr, pitch(lddx_in),
                                pitch(lddx_out), (int)desc->n, desc->r, desc->count};
            OperandArgs o = {{g, hj}, ranks, desc->r, up_steps(desc->r)};
            rc = low ? down_and_rows<Bf16>(down, a, rows, &o, s, st) : down_and_rows<F32>(down, a, rows, &o, s, st);
        } else {
            const UpArgs up = {nullptr, q, ranks, dx_in, dx_out, pitch(lddx_in), pitch(lddx_out), (int)desc->n,
                               desc->r, 0, 1};
            rc = low ? down_and_up<Bf16>(down, g, &hj, up, rows, s, st) : down_and_up<F32>(down, g, &hj, up, rows, s, st);
        }
        if (rc != DLCX_OK) return rc;
    }
    const int lane = desc->dtype == DLCX_BF16 ? Bf16::lane : F32::lane;
    GradArgs a;
    a.prod[0] = {s.turned_h, scale, dy, pitch(lddy), dp_out, s.slab_p, (int)desc->m, 0};
    a.prod[1] = {s.turned_g, nullptr, x, pitch(ldx), dq_out, s.slab_q, (int)desc->n, 0};
    for (GradProduct &g : a.prod)
        g.vec = rows_aligned(g.z, g.pitch) && g.len % lane == 0 && aligned16(g.out);
    a.ranks = ranks;
    a.r = desc->r;
    a.steps = up_steps(desc->r);
    a.blocks0 = (int)ceil_div(desc->m, 16 * lane);
    a.blocks = a.blocks0 + (int)ceil_div(desc->n, 16 * lane);
    const int size = grad_size(rows, desc->m, desc->n, lane);
    return desc->dtype == DLCX_BF16 ? launch_grad<Bf16>(a, rows, desc->count, size, s.route, st)
                                    : launch_grad<F32>(a, rows, desc->count, size, s.route, st);
}

}  // extern "C"
