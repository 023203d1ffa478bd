// Activations kept in 8 bits for the backward pass, and the weight gradient that reads them.
//
// Format.  32 consecutive columns of a row share a power of two 2^s, kept as the byte s + 133, and an element is
// code * 2^s with a signed 8-bit code.  s is the smallest power at which the group's largest magnitude, rounded, is
// at most 127 (so it is 64 at least: an element is off by at most 1/127.5 of half the largest one), and -133 at
// least.  Dividing by a power of two is exact and codes are rounded to nearest even, so the codes are the same in any
// arithmetic; and a code times a power of two from 2^-133 up is a bf16 number: what is read back is not rounded
// again, and enters the bf16 matrix cores as one term.  (Of the largest step, 2^122, the codes from 64 on would be 2^128 and more: they
// stand for the largest finite bf16 number, 63.75 * 2^122, which is within half a step of whatever has the code 64.)  Elements that are not finite do not count for s; their code
// is -128, which nothing else has, and comes back as NaN.
#include <type_traits>

#include "gemm_bf16_tiles.h"
#include "internal.h"
#include "load_rules.h"

namespace mixgcn {
namespace {

constexpr int kGroup = 32;          // columns that share a power of two
constexpr int kStepBias = 133;      // 2^-133 is the smallest bf16

__device__ inline float step_of(uint32_t e) { return ldexpf(1.f, (int)e - kStepBias); }
constexpr float kTopStep = 0x1p122f, kTopCode = 63.75f;  // the largest step, and the largest finite bf16 number in it
__device__ inline float top_code(float code) { return fminf(fmaxf(code, -kTopCode), kTopCode); }

template <bool BF16>
struct Lane {
    static constexpr int VEC = BF16 ? 8 : 4;      // columns of a lane: 16 bytes of features
    static constexpr int LANES = kGroup / VEC;    // lanes of a group
    static constexpr int ITEMS = kBlock / LANES;  // groups that a block works on at a time
    static constexpr int ES = BF16 ? 2 : 4;
    using Codes = typename std::conditional<BF16, uint2, uint32_t>::type;
};

// A block takes rows_per_block rows, and of these a group of columns per `LANES` lanes, four at a time.  Offsets within
// the rows of a block are 32 bits, and where there are several rows these and the pitches have 24, for the multiplications
// that are not done in quarters.
struct Plan {
    int groups;          // per row
    int rows_per_block;
    float per_group;     // 1 / groups, 0 for one row
};

// (item + 1/2) / groups is 1 / (2 groups) from a whole number at least, the product less than 2^-22 of item / groups from
// it: there are less than 2^16 items.
__device__ inline void split_item(const Plan& p, uint32_t item, uint32_t* row, uint32_t* group)
{
    *row = (uint32_t)(((float)item + 0.5f) * p.per_group);
    *group = item - __umul24(*row, (uint32_t)p.groups);
}

// The largest value of the lanes of a group.
template <int LANES>
__device__ inline float group_most(float v)
{
    auto other = [](float x, auto ctrl) {
        const int i = __float_as_int(x);
        return __int_as_float(__builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, 0xF, 0xF, false));
    };
    v = fmaxf(v, other(v, std::integral_constant<int, 0xB1>{}));   // lane ^ 1
    v = fmaxf(v, other(v, std::integral_constant<int, 0x4E>{}));   // lane ^ 2
    if (LANES == 8) v = fmaxf(v, other(v, std::integral_constant<int, 0x141>{}));  // the other four of eight
    return v;
}

// The smallest step that holds the largest magnitude of a group.
__device__ inline int step_for(float top)
{
    int s = (int)(__float_as_uint(top) >> 23) - 127 - 6;
    if (ldexpf(top, -s) >= 127.5f) ++s;
    return s < -kStepBias ? -kStepBias : s;
}

// What bounds it: memory, features in and codes out at 4.3 to 4.7 TB/s (a copy: 5.1): 2^20 x 256 fp32 296 us,
// 2450000 x 100 bf16 183.
template <bool BF16>
__global__ __launch_bounds__(kBlock) void pack_kernel(const void* __restrict__ X, int64_t ldx, int64_t n, int cols,
                                                      int8_t* __restrict__ codes, int64_t ldq,
                                                      uint8_t* __restrict__ steps, int64_t lde, Plan p)
{
    using L = Lane<BF16>;
    constexpr int U = 4;
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
    const int rows = n - row0 < p.rows_per_block ? (int)(n - row0) : p.rows_per_block;
    const uint32_t items = (uint32_t)rows * (uint32_t)p.groups;
    const uint32_t sub = threadIdx.x % L::LANES;
    const char* const xb = (const char*)X + row0 * ldx * L::ES;
    int8_t* const qb = codes + row0 * ldq;
    uint8_t* const eb = steps + row0 * lde;
    const uint32_t xp = (uint32_t)ldx * L::ES, qp = (uint32_t)ldq, ep = (uint32_t)lde;
    const uint32_t padded = (uint32_t)(cols + 15) / 16 * 16;
    for (uint32_t i0 = threadIdx.x / L::LANES; i0 < items; i0 += U * L::ITEMS) {
        uint4 v[U];
        uint32_t row[U], group[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = i0 + u * L::ITEMS;
            split_item(p, i < items ? i : i0, &row[u], &group[u]);
            const uint32_t c = group[u] * kGroup + sub * L::VEC;
            // a lane past the columns reads the row's first ones; its elements are masked below
            v[u] = *reinterpret_cast<const uint4*>(xb + (__umul24(row[u], xp) + (c < (uint32_t)cols ? c : 0u) * L::ES));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t c = group[u] * kGroup + sub * L::VEC;
            float f[L::VEC];
            const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
            for (int e = 0; e < L::VEC; ++e)
                f[e] = BF16 ? ((e & 1) ? high_half(w[e / 2]) : low_half(w[e / 2])) : __uint_as_float(w[e % 4]);
            if (c + L::VEC > (uint32_t)cols)
#pragma unroll
                for (int e = 0; e < L::VEC; ++e)
                    if (c + e >= (uint32_t)cols) f[e] = 0.f;
            float top = 0.f, wild = 0.f;
#pragma unroll
            for (int e = 0; e < L::VEC; ++e) {
                top = fmaxf(top, fabsf(f[e]));
                wild = fmaf(f[e], 0.f, wild);  // NaN after something that is not finite
            }
            uint32_t bad = 0;
            if (__builtin_expect(__any(!(wild == 0.f)), 0)) {
                top = 0.f;
#pragma unroll
                for (int e = 0; e < L::VEC; ++e) {
                    if (fabsf(f[e]) <= 3.402823466e38f) {
                        top = fmaxf(top, fabsf(f[e]));
                    } else {
                        bad |= 1u << e;
                        f[e] = 0.f;
                    }
                }
            }
            const int s = step_for(group_most<L::LANES>(top));
            uint32_t out[L::VEC / 4];
#pragma unroll
            for (int q = 0; q < L::VEC / 4; ++q) {
                uint32_t code[4];
                // the sum is rounded to a whole number, to even in a tie, and has it in its low bits
#pragma unroll
                for (int b = 0; b < 4; ++b) code[b] = __float_as_uint(ldexpf(f[4 * q + b], -s) + 12582912.f);
                out[q] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(code[3], code[2], 0x0c0c0400u),
                                               __builtin_amdgcn_perm(code[1], code[0], 0x0c0c0400u), 0x05040100u);
                if (__builtin_expect(bad != 0, 0))
                    for (int b = 0; b < 4; ++b)
                        if (bad >> (4 * q + b) & 1u) out[q] = (out[q] & ~(255u << (8 * b))) | 128u << (8 * b);
            }
            if (i0 + u * L::ITEMS >= items) continue;
            // the row's padding up to whole 16 bytes becomes zero
            if (c < padded) {
                typename L::Codes o;
                __builtin_memcpy(&o, out, sizeof(o));
                *reinterpret_cast<typename L::Codes*>(qb + (__umul24(row[u], qp) + c)) = o;
            }
            if (sub == 0) eb[__umul24(row[u], ep) + group[u]] = (uint8_t)(s + kStepBias);
        }
    }
}

// What a code stands for.
__device__ inline float value_of(int code, float step)
{
    if (code == -128) return __uint_as_float(0x7FC00000u);
    return (step == kTopStep ? top_code((float)code) : (float)code) * step;
}
// What the codes of N words stand for.  (-128 is the least code, so that the least of them tells whether it is there.)
template <int N>
__device__ inline void values_of(const uint32_t (&w)[N], float step, float (&f)[4 * N])
{
    float least = 0.f;
#pragma unroll
    for (int b = 0; b < 4 * N; ++b) {
        f[b] = (float)(int8_t)(w[b / 4] >> (8 * (b % 4)));
        least = fminf(least, f[b]);
    }
    if (__builtin_expect(step == kTopStep, 0))
#pragma unroll
        for (int b = 0; b < 4 * N; ++b) f[b] = top_code(f[b]);
#pragma unroll
    for (int b = 0; b < 4 * N; ++b) f[b] *= step;
    if (__builtin_expect(least == -128.f, 0))
#pragma unroll
        for (int b = 0; b < 4 * N; ++b) f[b] = value_of((int8_t)(w[b / 4] >> (8 * (b % 4))), step);
}

// Bound by memory, 2^20 x 256 fp32 in 240 us at 5.6 TB/s, 2450000 x 100 bf16 in 152 at 5.2.
template <bool BF16>
__global__ __launch_bounds__(kBlock) void unpack_kernel(const int8_t* __restrict__ codes, int64_t ldq,
                                                        const uint8_t* __restrict__ steps, int64_t lde, int64_t n,
                                                        int cols, void* __restrict__ X, int64_t ldx, Plan p)
{
    using L = Lane<BF16>;
    constexpr int U = 4;
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
    const int rows = n - row0 < p.rows_per_block ? (int)(n - row0) : p.rows_per_block;
    const uint32_t items = (uint32_t)rows * (uint32_t)p.groups;
    const uint32_t sub = threadIdx.x % L::LANES;
    char* const xb = (char*)X + row0 * ldx * L::ES;
    const int8_t* const qb = codes + row0 * ldq;
    const uint8_t* const eb = steps + row0 * lde;
    const uint32_t xp = (uint32_t)ldx * L::ES, qp = (uint32_t)ldq, ep = (uint32_t)lde;
    for (uint32_t i0 = threadIdx.x / L::LANES; i0 < items; i0 += U * L::ITEMS) {
        typename L::Codes v[U];
        uint32_t e[U], row[U], group[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = i0 + u * L::ITEMS;
            split_item(p, i < items ? i : i0, &row[u], &group[u]);
            const uint32_t c = group[u] * kGroup + sub * L::VEC;
            v[u] = *reinterpret_cast<const typename L::Codes*>(qb + (__umul24(row[u], qp) + (c < (uint32_t)cols ? c : 0u)));
            e[u] = eb[__umul24(row[u], ep) + group[u]];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t c = group[u] * kGroup + sub * L::VEC;
            if (i0 + u * L::ITEMS >= items || c >= (uint32_t)cols) continue;
            const float step = step_of(e[u]);
            uint32_t w[L::VEC / 4];
            __builtin_memcpy(w, &v[u], sizeof(w));
            float f[L::VEC];
            values_of(w, step, f);
            // the row's padding up to whole 16 bytes becomes zero (left as it is, 100 bf16 columns took 228 us for 2450000 rows, this
            // way 150: lines with holes are read before they are written)
            if (c + L::VEC > (uint32_t)cols)
#pragma unroll
                for (int b = 0; b < L::VEC; ++b)
                    if (c + b >= (uint32_t)cols) f[b] = 0.f;
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                o[q] = BF16 ? (__float_as_uint(f[(2 * q) % L::VEC]) >> 16) | (__float_as_uint(f[(2 * q + 1) % L::VEC]) & 0xFFFF0000u)
                            : __float_as_uint(f[q]);
            *reinterpret_cast<uint4*>(xb + (__umul24(row[u], xp) + c * L::ES)) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// row_bytes: the largest pitch of the row-wise arrays
Plan plan_rows(int64_t n, int cols, int items, int64_t row_bytes)
{
    Plan p;
    p.groups = (int)ceil_div(cols, kGroup);
    // one group per set of lanes at least, eight rounds of four at most, and between them as many rows as leave
    // 2048 blocks
    int64_t rows = n / 2048;
    const int64_t least = ceil_div(items, p.groups), most = 32 * items / p.groups;
    if (rows > most) rows = most;
    if (rows < least) rows = least;
    if (rows < 1 || row_bytes >= 1 << 24) rows = 1;
    if (rows > (((int64_t)1 << 31) - 1) / row_bytes) rows = (((int64_t)1 << 31) - 1) / row_bytes;
    if (rows < 1) rows = 1;
    p.rows_per_block = (int)rows;
    p.per_group = rows > 1 ? 1.f / (float)p.groups : 0.f;
    return p;
}

int64_t longest_row(int64_t ldx, int es, int64_t ldq, int64_t lde)
{
    int64_t b = ldx * es;
    if (ldq > b) b = ldq;
    return lde > b ? lde : b;
}

// ---- weight gradient ----------------------------------------------------------------------------
// P[slab][KD x MD] = Z8[rows of slab][KD]^T * (G (.) M)[rows][MD].  Z8 is one bf16 term; bf16 gradients are too, and
// fp32 ones the exact sum of three, taken times 2^16 so that the terms of every float are bf16 numbers.
//
// A workgroup has 64 TM x 64 TN cells on 2 x 2 wavefronts and walks its rows 32 at a time.  Global loads run two steps ahead in two
// register sets, LDS is double buffered, one barrier per step: decoding and splitting the next step and the products of
// this one do not wait for each other.  The tiles lie in LDS as in memory, row by row, and the LDS read transposes; of
// a row of 128 or 256 (64) columns the 64-byte block q is at q ^ (row % 4) (row / 2 % 2), so that the four rows that are read
// together come from all banks.
//
// What bounds it: 2^20 x 256 x 256 fp32 with a mask 393 us (464 in the first passes of a load, while the clock is down), 1050 TFLOP/s in its
// three products (a library bf16 product of 8192^3 reaches 1154), matrix cores busy 47 % of the cycles and vector instructions, most
// of them the three terms, 37 %: on one SIMD they take turns.  2450000 x 256 x 256 bf16 410 us, 4.6 TB/s of the 5.1 that a copy
// reaches; 41 and 39 %.
// 4096 x 64 x 32: 8 us, a chain of loads, products and stores of one slab, and 3 us for the slabs' sum.
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

constexpr int BKS = 32;  // rows per step

// halfwords of (row, column) of a tile of WIDTH columns
template <int WIDTH>
__device__ inline int place(int row, int col)
{
    const int block = col / 32 ^ (WIDTH == 64 ? row >> 1 & 1 : row & 3);
    return row * WIDTH + block * 32 + col % 32;
}

// Operand of the 32 columns from col0 on and 16 rows from row0 on.  Lane i of 16 receives element i % 4 of the 8 bytes that
// lanes i / 4, + 4, + 8 and + 12 address: with lane s of the group at row s / 4, columns 4 (s % 4) .. + 3, every lane has
// its own column at four consecutive rows.
template <int WIDTH>
__device__ inline bf16x8 read_transposed(const uint16_t* tile, int col0, int row0, int lane)
{
    const int grp = lane >> 4, gs = lane & 15;
    const uint16_t* const p = tile + place<WIDTH>(row0 + 8 * (grp >> 1) + (gs >> 2), col0 + 16 * (grp & 1) + 4 * (gs & 3));
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)p);
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p + 4 * WIDTH));
    const shortx8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    bf16x8 o;
    __builtin_memcpy(&o, &v, 16);
    return o;
}

__device__ inline uint4 load16(__amdgpu_buffer_rsrc_t rows, uint32_t offset)
{
    const uintx4 v = __builtin_amdgcn_raw_buffer_load_b128(rows, (int)offset, 0, 0);
    return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ inline __amdgpu_buffer_rsrc_t rows_at(const char* first, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(first), 0, bytes, 0x00020000);
}

template <bool BF16, bool MASK, int TM, int TN>
__global__ __launch_bounds__(kBlock, 2) void wgrad_checkpoint_kernel(
    const int8_t* __restrict__ codes, int64_t ldq, const uint8_t* __restrict__ steps, int64_t lde,
    const void* __restrict__ G, int64_t ldg, const uint32_t* __restrict__ mask, int64_t ldm, float* __restrict__ P,
    int KD, int MD, int64_t rows_per_slab, int64_t n_rows, int n_i_tiles, int n_j_tiles)
{
    constexpr int PLANES = BF16 ? 1 : 3, ES = BF16 ? 2 : 4;
    constexpr int WA = 64 * TM, WB = 64 * TN;  // columns of Z8 and of G in a tile
    constexpr int PA = BKS * (WA / 16) / kBlock, PER_ROW_A = WA / 16;  // rows of Z8 per thread and step, threads to a row
    constexpr int PER_ROW = WB / 8;        // threads to a row of G
    constexpr int PB = BKS * PER_ROW / kBlock;  // rows of G per thread and step
    constexpr int APLANE = BKS * WA, BPLANE = BKS * WB;
    __shared__ __attribute__((aligned(16))) uint16_t As[2][APLANE];
    __shared__ __attribute__((aligned(16))) uint16_t Bs[2][PLANES * BPLANE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / 2, wn = wave % 2;
    const int tiles = n_i_tiles * n_j_tiles;
    const unsigned lid = xcd_local_index(blockIdx.x, gridDim.x);
    const int slab = __builtin_amdgcn_readfirstlane((int)(lid / (unsigned)tiles));
    const int t = __builtin_amdgcn_readfirstlane((int)(lid % (unsigned)tiles));
    const int i0 = (t / n_j_tiles) * WA, j0 = (t % n_j_tiles) * WB;
    const int64_t r_begin = slab * rows_per_slab;
    const int64_t r_end = r_begin + rows_per_slab < n_rows ? r_begin + rows_per_slab : n_rows;
    const int n_here = (int)(r_end - r_begin), nk = (n_here + BKS - 1) / BKS;

    floatx16 acc[TM][TN];
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.f;

    // staging: a thread takes 16 codes of PA rows and eight columns of PB rows of G.  Columns past the matrices reach
    // only cells that are not stored: any column of the row will do.
    const int arow = tid / PER_ROW_A, acol = 16 * (tid % PER_ROW_A);
    const int brow = tid / PER_ROW, bcol = 8 * (tid % PER_ROW);
    const int ka = i0 + acol < KD ? i0 + acol : i0, mb = j0 + bcol < MD ? j0 + bcol : j0;
    const int pq = (int)ldq, pe = (int)lde, pg = (int)(ldg * ES), pm = (int)(ldm * 4);  // pitches in bytes
    uint32_t aoff[PA], eoff[PA], boff[PB], moff[PB];
#pragma unroll
    for (int p = 0; p < PA; ++p) {
        aoff[p] = (uint32_t)(arow + p * (BKS / PA)) * (uint32_t)pq + (uint32_t)ka;
        eoff[p] = (uint32_t)(arow + p * (BKS / PA)) * (uint32_t)pe + (uint32_t)(ka / kGroup);
    }
#pragma unroll
    for (int p = 0; p < PB; ++p) {
        boff[p] = (uint32_t)(brow + p * (BKS / PB)) * (uint32_t)pg + (uint32_t)(mb * ES);
        moff[p] = (uint32_t)(brow + p * (BKS / PB)) * (uint32_t)pm + (uint32_t)(mb / 32 * 4);
    }
    const uint32_t second = BF16 ? 0u : (uint32_t)((second_group(mb, MD) - mb) * ES);
    struct Regs {
        uint4 a[PA], b[PB][BF16 ? 1 : 2];
        uint32_t e[PA], m[MASK ? PB : 1];
    };
    // The rows of a step as buffers: rows past the slab's end are read as zeros, and no load is conditional.
    const char* ap = (const char*)codes + r_begin * ldq;
    const char* ep = (const char*)steps + r_begin * lde;
    const char* bp = (const char*)G + r_begin * ldg * ES;
    const char* mp = MASK ? (const char*)mask + r_begin * ldm * 4 : nullptr;
    int left = n_here;  // rows from the load cursor on
    auto load = [&](Regs& g) {
        const int rows = __builtin_amdgcn_readfirstlane(left >= BKS ? BKS : left > 0 ? left : 0);
        const auto ra = rows_at(ap, rows * pq), re = rows_at(ep, rows * pe), rb = rows_at(bp, rows * pg);
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            g.a[p] = load16(ra, aoff[p]);
            g.e[p] = __builtin_amdgcn_raw_buffer_load_b8(re, (int)eoff[p], 0, 0);
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            g.b[p][0] = load16(rb, boff[p]);
            if (!BF16) g.b[p][BF16 ? 0 : 1] = load16(rb, boff[p] + second);
        }
        if (MASK) {
            const auto rm = rows_at(mp, rows * pm);
#pragma unroll
            for (int p = 0; p < PB; ++p) g.m[MASK ? p : 0] = __builtin_amdgcn_raw_buffer_load_b32(rm, (int)moff[p], 0, 0);
            mp += (int64_t)BKS * pm;
        }
        ap += (int64_t)BKS * pq;
        ep += (int64_t)BKS * pe;
        bp += (int64_t)BKS * pg;
        left -= BKS;
    };
    float least = 0.f;  // of the codes that this thread has met
    auto store = [&](const Regs& g, uint16_t* as, uint16_t* bs) {
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const uint32_t w[4] = {g.a[p].x, g.a[p].y, g.a[p].z, g.a[p].w};
            float f[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                f[i] = (float)(int8_t)(w[i / 4] >> (8 * (i % 4)));
                least = fminf(least, f[i]);
            }
            const float unit = step_of(g.e[p]);
            uint32_t d[8];  // pairs of bf16: the upper halves, the lower ones are zero
#pragma unroll
            for (int i = 0; i < 8; ++i)
                d[i] = __builtin_amdgcn_perm(__float_as_uint(f[2 * i + 1] * unit), __float_as_uint(f[2 * i] * unit), 0x07060302u);
            uint16_t* const q = as + place<WA>(arow + p * (BKS / PA), acol);
            lds_store16(q, make_uint4(d[0], d[1], d[2], d[3]));
            lds_store16(q + 8, make_uint4(d[4], d[5], d[6], d[7]));
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const uint32_t m = MASK ? g.m[MASK ? p : 0] >> (mb % 32) : 0u;
            uint16_t* const o = bs + place<WB>(brow + p * (BKS / PB), bcol);
            if (BF16) {
                const uint4 v = g.b[p][0];
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
                if (MASK)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        w[i] &= ((uint32_t)((int32_t)(m << (31 - 2 * i)) >> 31) & 0xFFFFu) |
                                ((uint32_t)((int32_t)(m << (30 - 2 * i)) >> 31) & 0xFFFF0000u);
                lds_store16(o, make_uint4(w[0], w[1], w[2], w[3]));
            } else {
                const uint4 v0 = g.b[p][0], v1 = g.b[p][BF16 ? 0 : 1];
                uint32_t w[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
                if (MASK)
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] &= (uint32_t)((int32_t)(m << (31 - i)) >> 31);
                uint32_t term[3][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = __uint_as_float(w[2 * i]) * kTermScale, y = __uint_as_float(w[2 * i + 1]) * kTermScale;
#pragma unroll
                    for (int s = 0; s < 3; ++s) {
                        term[s][i] = pack_bf16(x, y);
                        x -= low_half(term[s][i]);
                        y -= high_half(term[s][i]);
                    }
                }
#pragma unroll
                for (int s = 0; s < 3; ++s)
                    lds_store16(o + (BF16 ? 0 : s) * BPLANE, make_uint4(term[s][0], term[s][1], term[s][2], term[s][3]));
            }
        }
    };
    auto mma = [&](const uint16_t* as, const uint16_t* bs) {
#pragma unroll
        for (int kc = 0; kc < BKS; kc += 16) {
            bf16x8 a[TM], b[TN][PLANES];
#pragma unroll
            for (int x = 0; x < TM; ++x) a[x] = read_transposed<WA>(as, (wm * TM + x) * 32, kc, lane);
#pragma unroll
            for (int y = 0; y < TN; ++y)
#pragma unroll
                for (int p = 0; p < PLANES; ++p) b[y][p] = read_transposed<WB>(bs + p * BPLANE, (wn * TN + y) * 32, kc, lane);
            // the smaller products first
#pragma unroll
            for (int p = PLANES - 1; p >= 0; --p)
#pragma unroll
                for (int x = 0; x < TM; ++x)
#pragma unroll
                    for (int y = 0; y < TN; ++y)
                        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[x], b[y][p], acc[x][y], 0, 0, 0);
        }
    };
    if (nk > 0) {
        Regs g0, g1;
        load(g0);
        load(g1);
        store(g0, As[0], Bs[0]);
        load(g0);
        __syncthreads();
        for (int i = 0; i + 1 < nk; i += 2) {
            store(g1, As[1], Bs[1]);
            load(g1);
            mma(As[0], Bs[0]);
            __syncthreads();
            store(g0, As[0], Bs[0]);
            load(g0);
            mma(As[1], Bs[1]);
            __syncthreads();
        }
        if (nk & 1) mma(As[0], Bs[0]);
    }
    // Columns of Z8 that have a code -128 are NaN throughout.  It was taken for a number above; which columns they are is
    // looked up only where one was met.
    uint8_t* const not_finite = reinterpret_cast<uint8_t*>(As[0]);
    __syncthreads();
    if (tid < WA) not_finite[tid] = 0;
    __syncthreads();
    // (The row padding may hold one, too: it is looked up in vain, so the looking up reads whole 16 bytes, two rows at a time:
    // 115712 x 72 x 296 bf16 with such padding 54 -> 30 us.)
    if (__builtin_expect(least == -128.f, 0)) {
        uint32_t met[4] = {};
        constexpr int STEP = BKS / PA;
        for (int64_t r = r_begin + arow; r < r_end; r += 2 * STEP) {
            uint4 v[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                v[u] = *reinterpret_cast<const uint4*>(codes + (r + u * STEP < r_end ? r + u * STEP : r) * ldq + ka);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    // the top bit of each byte that is 0x80
                    const uint32_t z = w[q] ^ 0x80808080u;
                    met[q] |= ~(((z & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | z | 0x7F7F7F7Fu);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (met[i / 4] >> (8 * (i % 4) + 7) & 1u) not_finite[acol + i] = 1;
    }
    __syncthreads();

    // D layout: lane l, register v -> row 8 (v / 4) + 4 (l / 32) + v % 4, col l % 32
    const int li = lane & 31, lk = lane >> 5;
    const int iw = wm * TM * 32 + 4 * lk, jw = j0 + wn * TN * 32 + li;
    float* const out = P + ((size_t)slab * KD + i0) * MD;
    const float unscale = BF16 ? 1.f : 1.f / kTermScale;
    float wild = 0.f;  // NaN after a sum that is not finite
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int i = iw + x * 32 + 8 * (v / 4) + (v % 4), j = jw + y * 32;
                if (i0 + i >= KD || j >= MD) continue;
                const float sum = not_finite[i] ? __uint_as_float(0x7FC00000u) : acc[x][y][v] * unscale;
                if (!not_finite[i]) wild = fmaf(sum, 0.f, wild);
                out[(size_t)i * MD + j] = sum;
            }
    bool again = !(wild == 0.f);
    if (BF16 && __builtin_expect(__syncthreads_or(again), 0)) {
        // With one term each they are what fp32 gives, but for codes from 64 on of the largest step, which were taken for infinities.
        bool top = false;
        for (int64_t r = r_begin + tid; r < r_end; r += kBlock)
            for (int q = i0 / kGroup; q * kGroup < KD && q * kGroup < i0 + WA; ++q) top = top || steps[r * lde + q] == 255;
        again = __syncthreads_or(top) && again;
    }
    if (__builtin_expect(again, 0)) {
        // The lane's sums that are not finite again, as chains of fp32 multiply-adds (a term of an infinity is NaN).
        for (int c = 0; c < TM * TN * 16; ++c) {
            const int v = c % 16, i = iw + c / (16 * TN) * 32 + 8 * (v / 4) + (v % 4), j = jw + c / 16 % TN * 32;
            if (i0 + i >= KD || j >= MD || not_finite[i]) continue;
            if (fabsf(out[(size_t)i * MD + j]) <= 3.402823466e38f) continue;
            float sum = 0.f;
            for (int64_t r = r_begin; r < r_end; ++r) {
                const float z = value_of(codes[r * ldq + i0 + i], step_of(steps[r * lde + (i0 + i) / kGroup]));
                const float b = BF16 ? low_half(reinterpret_cast<const uint16_t*>(G)[r * ldg + j]) : reinterpret_cast<const float*>(G)[r * ldg + j];
                const bool on = !MASK || ((mask[r * ldm + j / 32] >> (j % 32)) & 1u);
                sum = fmaf(z, on ? b : 0.f, sum);
            }
            out[(size_t)i * MD + j] = sum;
        }
    }
}

struct Slabs {
    int64_t n, rows;
    int nit, njt, wa, wb;  // tiles and their widths
};
Slabs plan_slabs(int64_t n, int32_t k, int32_t m)
{
    Slabs s;
    // 256 columns of Z8 where they cover no more than tiles of 128 would: what a workgroup does to its part of G, the terms
    // and the mask, is then done for twice the cells
    s.wa = ceil_div(k, 128) % 2 ? 128 : 256;
    s.wb = m > 64 ? 128 : 64;
    s.nit = (int)ceil_div(k, s.wa);
    s.njt = (int)ceil_div(m, s.wb);
    // two workgroups for every compute unit, of 128 rows at least (more of them and the slabs' sums cost more than they
    // gain); four where a slab would have more than 2^14 rows, whose sums are less exact (8500000 x 128 x 128 fp32 1083 us, with two 1073; bf16
    // 618, 562)
    const int64_t tiles = (int64_t)s.nit * s.njt;
    s.n = ceil_div(512, tiles);
    if (ceil_div(n, s.n) > 1 << 14) s.n = ceil_div(1024, tiles);
    if (s.n > ceil_div(n, 128)) s.n = ceil_div(n, 128);
    if (s.n < 1) s.n = 1;
    s.rows = ceil_div(ceil_div(n, s.n), BKS) * BKS;
    if (s.rows < BKS) s.rows = BKS;
    s.n = n > 0 ? ceil_div(n, s.rows) : 1;  // without rows: one slab of zeros
    return s;
}

}  // namespace

int launch_checkpoint_pack(int dtype, const void* X, int64_t ldx, int64_t n, int32_t cols, int8_t* codes, int64_t ldq,
                           uint8_t* steps, int64_t lde, hipStream_t s)
{
    if (n == 0) return MIXGCN_OK;
    const bool bf16 = dtype == MIXGCN_BF16;
    const Plan p = plan_rows(n, cols, bf16 ? Lane<true>::ITEMS : Lane<false>::ITEMS, longest_row(ldx, bf16 ? 2 : 4, ldq, lde));
    const int64_t grid = ceil_div(n, p.rows_per_block);
    if (grid > 0x7FFFFFFF) return fail(MIXGCN_EINVAL, "checkpoint_pack: too many rows");
    if (bf16)
        hipLaunchKernelGGL(pack_kernel<true>, dim3((unsigned)grid), dim3(kBlock), 0, s, X, ldx, n, cols, codes, ldq,
                           steps, lde, p);
    else
        hipLaunchKernelGGL(pack_kernel<false>, dim3((unsigned)grid), dim3(kBlock), 0, s, X, ldx, n, cols, codes, ldq,
                           steps, lde, p);
    MIXGCN_HIP_TRY(hipGetLastError());
    return MIXGCN_OK;
}

int launch_checkpoint_unpack(int dtype, const int8_t* codes, int64_t ldq, const uint8_t* steps, int64_t lde, int64_t n,
                             int32_t cols, void* X, int64_t ldx, hipStream_t s)
{
    if (n == 0) return MIXGCN_OK;
    const bool bf16 = dtype == MIXGCN_BF16;
    const Plan p = plan_rows(n, cols, bf16 ? Lane<true>::ITEMS : Lane<false>::ITEMS, longest_row(ldx, bf16 ? 2 : 4, ldq, lde));
    const int64_t grid = ceil_div(n, p.rows_per_block);
    if (grid > 0x7FFFFFFF) return fail(MIXGCN_EINVAL, "checkpoint_unpack: too many rows");
    if (bf16)
        hipLaunchKernelGGL(unpack_kernel<true>, dim3((unsigned)grid), dim3(kBlock), 0, s, codes, ldq, steps, lde, n,
                           cols, X, ldx, p);
    else
        hipLaunchKernelGGL(unpack_kernel<false>, dim3((unsigned)grid), dim3(kBlock), 0, s, codes, ldq, steps, lde, n,
                           cols, X, ldx, p);
    MIXGCN_HIP_TRY(hipGetLastError());
    return MIXGCN_OK;
}

int64_t checkpoint_wgrad_bytes(int64_t n, int32_t k, int32_t m)
{
    return plan_slabs(n, k, m).n * k * m * (int64_t)sizeof(float);
}

int launch_checkpoint_wgrad(int dtype, const int8_t* codes, int64_t ldq, const uint8_t* steps, int64_t lde,
                            const void* G, int64_t ldg, float* dW, int64_t ldw, int64_t n, int32_t k, int32_t m,
                            const uint32_t* mask, int64_t ldm, float beta, float* P, hipStream_t s)
{
    // the rows of a step are addressed with 31 bits
    const int64_t most = ((int64_t)1 << 31) / BKS;
    if (n > 0 && (ldq >= most || lde >= most || ldg * (dtype == MIXGCN_BF16 ? 2 : 4) >= most || (mask && ldm * 4 >= most)))
        return fail(MIXGCN_EUNSUPPORTED, "checkpoint_wgrad: rows of 2^26 bytes and more");
    const Slabs p = plan_slabs(n, k, m);
    const int64_t grid = p.n * p.nit * p.njt;
    if (grid > 0x7FFFFFFF || p.rows > (1 << 30)) return fail(MIXGCN_EUNSUPPORTED, "checkpoint_wgrad: too many tiles or rows");
#define MIXGCN_WGRAD8_T(BF16, MASK, TM, TN)                                                                               \
    hipLaunchKernelGGL((wgrad_checkpoint_kernel<BF16, MASK, TM, TN>), dim3((unsigned)grid), dim3(kBlock), 0, s, codes, ldq, \
                       steps, lde, G, ldg, mask, ldm, P, k, m, p.rows, n, p.nit, p.njt)
#define MIXGCN_WGRAD8(BF16, MASK)                                         \
    do {                                                                  \
        if (p.wa == 256 && p.wb == 128) MIXGCN_WGRAD8_T(BF16, MASK, 4, 2); \
        else if (p.wa == 256) MIXGCN_WGRAD8_T(BF16, MASK, 4, 1);          \
        else if (p.wb == 128) MIXGCN_WGRAD8_T(BF16, MASK, 2, 2);          \
        else MIXGCN_WGRAD8_T(BF16, MASK, 2, 1);                           \
    } while (0)
    if (dtype == MIXGCN_BF16) {
        if (mask) MIXGCN_WGRAD8(true, true);
        else MIXGCN_WGRAD8(true, false);
    } else {
        if (mask) MIXGCN_WGRAD8(false, true);
        else MIXGCN_WGRAD8(false, false);
    }
#undef MIXGCN_WGRAD8
#undef MIXGCN_WGRAD8_T
    MIXGCN_TRY(launch_wgrad_reduce(P, p.n, (int64_t)k * m, m, dW, ldw, beta, s));
    MIXGCN_HIP_TRY(hipGetLastError());
    return MIXGCN_OK;
}

}  // namespace mixgcn
