// Activations kept in 8 bits for the backward pass, and the weight gradient that reads them.
//
// Format.  32 consecutive columns of a row share a power of two 2^s, kept as the byte s + 133, and an element is
// code * 2^s with a signed 8-bit code.  s is the smallest power at which the group's largest magnitude, rounded, is
// at most 127 (so it is 64 at least: an element is off by at most 1/127.5 of half the largest one), and -133 at
// least.  Dividing by a power of two is exact and codes are rounded to nearest even, so the codes are the same in any
// arithmetic; and a code times a power of two from 2^-133 up is a bf16 number: what is read back is not rounded
// again, and enters the bf16 matrix cores as one term.  Elements that are not finite do not count for s; their code
// is -128, which nothing else has, and comes back as NaN.
#include <type_traits>

#include "gemm_bf16_tiles.h"
#include "internal.h"

namespace mixgcn {
namespace {

constexpr int kGroup = 32;          // columns that share a power of two
constexpr int kStepBias = 133;      // 2^-133 is the smallest bf16

__device__ inline float step_of(uint32_t e) { return ldexpf(1.f, (int)e - kStepBias); }

template <bool BF16>
struct Lane {
    static constexpr int VEC = BF16 ? 8 : 4;      // columns of a lane: 16 bytes of features
    static constexpr int LANES = kGroup / VEC;    // lanes of a group
    static constexpr int ITEMS = kBlock / LANES;  // groups that a block works on at a time
    using Codes = typename std::conditional<BF16, uint2, uint32_t>::type;
};

// A block takes rows_per_block rows, and of these a group of columns per `LANES` lanes, four at a time.
struct Plan {
    int groups;          // per row
    int rows_per_block;
    uint32_t magic;      // item / groups = umulhi(item, magic) where a block has several rows
};

__device__ inline void split_item(const Plan& p, uint32_t item, int* row, int* group)
{
    const uint32_t r = p.groups == 1 ? item : p.rows_per_block > 1 ? __umulhi(item, p.magic) : 0u;
    *row = (int)r;
    *group = (int)(item - r * (uint32_t)p.groups);
}

// What bounds it: memory, features in and codes out.
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
    const int sub = threadIdx.x % L::LANES;
    for (uint32_t i0 = threadIdx.x / L::LANES; i0 < items; i0 += U * L::ITEMS) {
        uint4 v[U];
        int row[U], group[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = i0 + u * L::ITEMS;
            split_item(p, i < items ? i : i0, &row[u], &group[u]);
            const int c = group[u] * kGroup + sub * L::VEC;
            // a lane past the columns reads the row's first ones; its elements are masked below
            const int cc = c < cols ? c : 0;
            const char* const x = (const char*)X + ((row0 + row[u]) * ldx + cc) * (BF16 ? 2 : 4);
            v[u] = *reinterpret_cast<const uint4*>(x);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = group[u] * kGroup + sub * L::VEC;
            float f[L::VEC];
            const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
            for (int e = 0; e < L::VEC; ++e) {
                f[e] = BF16 ? ((e & 1) ? high_half(w[e / 2]) : low_half(w[e / 2])) : __uint_as_float(w[e % 4]);
                if (c + e >= cols) f[e] = 0.f;
            }
            // magnitudes as integers order as the numbers do; those that are not finite do not count
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < L::VEC; ++e) {
                const uint32_t m = __float_as_uint(f[e]) & 0x7FFFFFFFu;
                const uint32_t mm = m < 0x7F800000u ? m : 0u;
                top = mm > top ? mm : top;
            }
#pragma unroll
            for (int o = 1; o < L::LANES; o <<= 1) {
                const uint32_t t = __shfl_xor(top, o, kWave);
                top = t > top ? t : top;
            }
            int s = (int)(top >> 23) - 127 - 6;
            if (ldexpf(__uint_as_float(top), -s) >= 127.5f) ++s;
            if (s < -kStepBias) s = -kStepBias;
            uint32_t out[L::VEC / 4];
#pragma unroll
            for (int q = 0; q < L::VEC / 4; ++q) {
                out[q] = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const float x = f[4 * q + b];
                    const bool finite = (__float_as_uint(x) & 0x7FFFFFFFu) < 0x7F800000u;
                    const int code = finite ? (int)rintf(ldexpf(x, -s)) : -128;
                    out[q] |= ((uint32_t)code & 255u) << (8 * b);
                }
            }
            if (i0 + u * L::ITEMS >= items) continue;
            const int64_t r = row0 + row[u];
            // the row's padding up to whole 16 bytes becomes zero
            if (c < (cols + 15) / 16 * 16) {
                typename L::Codes o;
                __builtin_memcpy(&o, out, sizeof(o));
                *reinterpret_cast<typename L::Codes*>(codes + r * ldq + c) = o;
            }
            if (sub == 0) steps[r * lde + group[u]] = (uint8_t)(s + kStepBias);
        }
    }
}

// What a code stands for.
__device__ inline float value_of(int code, float step) { return code == -128 ? __uint_as_float(0x7FC00000u) : (float)code * step; }

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
    const int sub = threadIdx.x % L::LANES;
    for (uint32_t i0 = threadIdx.x / L::LANES; i0 < items; i0 += U * L::ITEMS) {
        typename L::Codes v[U];
        uint32_t e[U];
        int row[U], group[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = i0 + u * L::ITEMS;
            split_item(p, i < items ? i : i0, &row[u], &group[u]);
            const int c = group[u] * kGroup + sub * L::VEC;
            const int cc = c < cols ? c : 0;
            v[u] = *reinterpret_cast<const typename L::Codes*>(codes + (row0 + row[u]) * ldq + cc);
            e[u] = steps[(row0 + row[u]) * lde + group[u]];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = group[u] * kGroup + sub * L::VEC;
            if (i0 + u * L::ITEMS >= items || c >= cols) continue;
            const float step = step_of(e[u]);
            uint32_t w[L::VEC / 4];
            __builtin_memcpy(w, &v[u], sizeof(w));
            float f[L::VEC];
#pragma unroll
            for (int b = 0; b < L::VEC; ++b) f[b] = value_of((int8_t)(w[b / 4] >> (8 * (b % 4))), step);
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                o[q] = BF16 ? (__float_as_uint(f[(2 * q) % L::VEC]) >> 16) | (__float_as_uint(f[(2 * q + 1) % L::VEC]) & 0xFFFF0000u)
                            : __float_as_uint(f[q]);
            char* const x = (char*)X + ((row0 + row[u]) * ldx + c) * (BF16 ? 2 : 4);
            if (c + L::VEC <= cols) {
                *reinterpret_cast<uint4*>(x) = make_uint4(o[0], o[1], o[2], o[3]);
            } else {
                for (int b = 0; c + b < cols; ++b) {
                    if (BF16) ((uint16_t*)x)[b] = (uint16_t)(__float_as_uint(f[b]) >> 16);
                    else ((float*)x)[b] = f[b];
                }
            }
        }
    }
}

Plan plan_rows(int64_t n, int cols, int items)
{
    Plan p;
    p.groups = (int)ceil_div(cols, kGroup);
    // one group per set of lanes at least, eight rounds of four at most, and between them as many rows as leave
    // 2048 blocks
    int64_t rows = n / 2048;
    const int64_t least = ceil_div(items, p.groups), most = 32 * items / p.groups;
    if (rows > most) rows = most;
    if (rows < least) rows = least;
    p.rows_per_block = (int)rows;
    p.magic = p.groups > 1 ? (uint32_t)(((1ull << 32) + p.groups - 1) / p.groups) : 0u;
    return p;
}

// ---- weight gradient ----------------------------------------------------------------------------
// P[slab][KD x MD] = Z8[rows of slab][KD]^T * (G (.) M)[rows][MD].  Z8 is one bf16 term; bf16 gradients are too, and
// fp32 ones the exact sum of three, taken times 2^16 so that the terms of every float are bf16 numbers.
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

constexpr int BKS = 16;         // rows per step, the reduction depth of an MFMA
constexpr int LDW = 128 + 32;   // halfwords per staged row
constexpr int kTile = BKS * LDW;

// Lane i of 16 receives element i % 4 of the 8 bytes that lanes i / 4, + 4, + 8 and + 12 address: with lane s of the
// group at row s / 4, features 4 (s % 4) .. + 3, every lane has its own feature at four consecutive rows.
__device__ inline bf16x8 read_transposed(const uint16_t* p)
{
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)p);
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p + 4 * LDW));
    const shortx8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    bf16x8 o;
    __builtin_memcpy(&o, &v, 16);
    return o;
}

// four codes as two words of bf16
__device__ inline uint2 decode4(uint32_t w, float step)
{
    uint32_t f[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) f[b] = __float_as_uint(value_of((int8_t)(w >> (8 * b)), step));
    return make_uint2((f[0] >> 16) | (f[1] & 0xFFFF0000u), (f[2] >> 16) | (f[3] & 0xFFFF0000u));
}

template <bool BF16, bool MASK>
__global__ __launch_bounds__(kBlock, 2) void wgrad_checkpoint_kernel(
    const int8_t* __restrict__ codes, int64_t ldq, const uint8_t* __restrict__ steps, int64_t lde,
    const void* __restrict__ G, int64_t ldg, const uint32_t* __restrict__ mask, int64_t ldm, float* __restrict__ P,
    int KD, int MD, int64_t rows_per_slab, int64_t n_rows, int n_i_tiles, int n_j_tiles)
{
    constexpr int PLANES = BF16 ? 1 : 3;
    constexpr int ES = BF16 ? 2 : 4;
    __shared__ __attribute__((aligned(16))) uint16_t As[2][kTile];
    __shared__ __attribute__((aligned(16))) uint16_t Bs[2][PLANES * kTile];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / 2, wn = wave % 2;
    const int tiles = n_i_tiles * n_j_tiles;
    const unsigned lid = xcd_local_index(blockIdx.x, gridDim.x);
    const int64_t slab = lid / (unsigned)tiles;
    const int t = (int)(lid % (unsigned)tiles);
    const int i0 = (t / n_j_tiles) * 128, j0 = (t % n_j_tiles) * 128;
    const int64_t r_begin = slab * rows_per_slab;
    const int64_t r_end = r_begin + rows_per_slab < n_rows ? r_begin + rows_per_slab : n_rows;
    const int nk = r_end > r_begin ? (int)((r_end - r_begin + BKS - 1) / BKS) : 0;

    floatx16 acc[2][2];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.f;

    // staging: a thread takes eight columns of a row, of Z8 and of G.  Columns past the matrices reach only cells that
    // are not stored: any column of the row will do.
    const int row = tid >> 4, col = 8 * (tid & 15);
    const int acol = i0 + col < KD ? i0 + col : i0, bcol = j0 + col < MD ? j0 + col : j0;
    // the last eight codes of a row may lie half past its pitch only where the pitch is not whole: it is
    const int8_t* const a0 = codes + acol;
    const uint8_t* const e0 = steps + acol / kGroup;
    const char* const b0 = (const char*)G + (int64_t)bcol * ES;
    const uint32_t* const m0 = MASK ? mask + bcol / 32 : nullptr;
    struct Regs {
        uint2 a;
        uint4 b[BF16 ? 1 : 2];
        uint32_t e, m;
    } g;
    auto load = [&](int step) {
        const int64_t r = r_begin + (int64_t)step * BKS + row;
        const bool in = r < r_end;
        const int64_t rr = in ? r : r_begin;
        g.a = *reinterpret_cast<const uint2*>(a0 + rr * ldq);
        g.e = e0[rr * lde];
        const uint4* const b = reinterpret_cast<const uint4*>(b0 + rr * ldg * ES);
        g.b[0] = b[0];
        // (fp32: the second four columns exist where the pitch has them)
        if (!BF16) g.b[BF16 ? 0 : 1] = bcol + 4 < ldg ? b[1] : b[0];
        g.m = MASK ? m0[rr * ldm] : 0xFFFFFFFFu;
        if (MASK) g.m >>= bcol % 32;
        if (!in) {
            g.a = make_uint2(0u, 0u);
            g.m = 0u;
        }
    };
    auto store = [&](uint16_t* as, uint16_t* bs) {
        const float step = step_of(g.e);
        const uint2 lo = decode4(g.a.x, step), hi = decode4(g.a.y, step);
        lds_store16(as + row * LDW + col, make_uint4(lo.x, lo.y, hi.x, hi.y));
        uint16_t* const q = bs + row * LDW + col;
        if (BF16) {
            uint32_t w[4] = {g.b[0].x, g.b[0].y, g.b[0].z, g.b[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] &= ((g.m >> (2 * i)) & 1u ? 0xFFFFu : 0u) | ((g.m >> (2 * i)) & 2u ? 0xFFFF0000u : 0u);
            lds_store16(q, make_uint4(w[0], w[1], w[2], w[3]));
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 u = g.b[BF16 ? 0 : h];
                const uint32_t m = g.m >> (4 * h);
                float4 x;
                x.x = m & 1u ? __uint_as_float(u.x) : 0.f;
                x.y = m & 2u ? __uint_as_float(u.y) : 0.f;
                x.z = m & 4u ? __uint_as_float(u.z) : 0.f;
                x.w = m & 8u ? __uint_as_float(u.w) : 0.f;
                split_store<false>(x, x, kTermScale, q + 4 * h, q + kTile + 4 * h, q + 2 * kTile + 4 * h);
            }
        }
    };
    const int grp = lane >> 4, gs = lane & 15;
    const int rpos = (8 * (grp >> 1) + (gs >> 2)) * LDW + 16 * (grp & 1) + 4 * (gs & 3);
    auto mma = [&](const uint16_t* as, const uint16_t* bs) {
        bf16x8 a[2], b[2][PLANES];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            a[x] = read_transposed(as + rpos + (wm * 2 + x) * 32);
#pragma unroll
            for (int p = 0; p < PLANES; ++p) b[x][p] = read_transposed(bs + p * kTile + rpos + (wn * 2 + x) * 32);
        }
#pragma unroll
        for (int p = PLANES - 1; p >= 0; --p)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[x], b[y][p], acc[x][y], 0, 0, 0);
    };
    if (nk > 0) {
        load(0);
        store(As[0], Bs[0]);
        __syncthreads();
        for (int i = 0; i < nk; ++i) {
            if (i + 1 < nk) load(i + 1);
            mma(As[i & 1], Bs[i & 1]);
            if (i + 1 < nk) store(As[(i + 1) & 1], Bs[(i + 1) & 1]);
            __syncthreads();
        }
    }

    // D layout: lane l, register v -> row 8 (v / 4) + 4 (l / 32) + v % 4, col l % 32
    const int li = lane & 31, lk = lane >> 5;
    float* const out = P + (size_t)slab * KD * MD;
    const float unscale = BF16 ? 1.f : 1.f / kTermScale;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int j = j0 + (wn * 2 + y) * 32 + li;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int i = i0 + (wm * 2 + x) * 32 + 8 * (v / 4) + 4 * lk + (v % 4);
                if (i >= KD || j >= MD) continue;
                float sum = acc[x][y][v] * unscale;
                if (!BF16 && __builtin_expect(!(fabsf(sum) <= 3.402823466e38f), 0)) {
                    // Not finite: again as a chain of fp32 multiply-adds (a term of an infinity is NaN).
                    sum = 0.f;
                    for (int64_t r = r_begin; r < r_end; ++r) {
                        const float z = value_of(codes[r * ldq + i], step_of(steps[r * lde + i / kGroup]));
                        const float b = reinterpret_cast<const float*>(G)[r * ldg + j];
                        const bool on = !MASK || ((mask[r * ldm + j / 32] >> (j % 32)) & 1u);
                        sum = fmaf(z, on ? b : 0.f, sum);
                    }
                }
                out[(size_t)i * MD + j] = sum;
            }
        }
}

struct Slabs {
    int64_t n, rows;
    int nit, njt;
};
Slabs plan_slabs(int64_t n, int32_t k, int32_t m)
{
    Slabs s;
    s.nit = (int)ceil_div(k, 128);
    s.njt = (int)ceil_div(m, 128);
    s.n = wgrad_slabs(n, (int64_t)s.nit * s.njt, 1024);
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
    const Plan p = plan_rows(n, cols, bf16 ? Lane<true>::ITEMS : Lane<false>::ITEMS);
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
    const Plan p = plan_rows(n, cols, bf16 ? Lane<true>::ITEMS : Lane<false>::ITEMS);
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
    const Slabs p = plan_slabs(n, k, m);
    const int64_t grid = p.n * p.nit * p.njt;
    if (grid > 0x7FFFFFFF) return fail(MIXGCN_EINVAL, "checkpoint_wgrad: too many tiles");
#define MIXGCN_WGRAD8(BF16, MASK)                                                                                    \
    hipLaunchKernelGGL((wgrad_checkpoint_kernel<BF16, MASK>), dim3((unsigned)grid), dim3(kBlock), 0, s, codes, ldq,  \
                       steps, lde, G, ldg, mask, ldm, P, k, m, p.rows, n, p.nit, p.njt)
    if (dtype == MIXGCN_BF16) {
        if (mask) MIXGCN_WGRAD8(true, true);
        else MIXGCN_WGRAD8(true, false);
    } else {
        if (mask) MIXGCN_WGRAD8(false, true);
        else MIXGCN_WGRAD8(false, false);
    }
#undef MIXGCN_WGRAD8
    MIXGCN_TRY(launch_wgrad_reduce(P, p.n, (int64_t)k * m, m, dW, ldw, beta, s));
    MIXGCN_HIP_TRY(hipGetLastError());
    return MIXGCN_OK;
}

}  // namespace mixgcn
