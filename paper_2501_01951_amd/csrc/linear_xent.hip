// Mean softmax cross-entropy of a linear last layer over many classes, without its logits, with its gradients:
//     S = H W,  lse_r = log sum_c exp S_rc,  loss = 1/N sum_r (lse_r - S_r,y_r),
//     G = (exp(S - lse) - onehot) / N,  dH = G W^T,  dW = H^T G,
// over the N rows that have a label.  The classes are walked in tiles: a first pass keeps the largest logit of a row and
// the sum of exponentials of every 64 classes (a row's are joined afterwards), a second one computes the logits again,
// now with the row's sum known, and hands G on a piece of the classes at a time.
//
// Arithmetic.  The products run on the f16 matrix cores with fp32 sums.  An fp32 number enters as two f16 terms, the
// rounded number and the rounded rest, 22 bits and more together; a bf16 one as one.  Of the products of two terms
// each the one of both rests, below 2^-22, is left out.  f16 has a narrow range, so operands are scaled by powers of
// two, which is exact: feature k by one factor in H and another in W, chosen from the largest magnitudes h_k of its
// column and w_k of its row such that the largest h_k w_k of all features comes to 2^28 at least, 2^14 from either
// side, and a feature whose h_k w_k is smaller by 2^d has both sides smaller by 2^(d / 2), up to a d past which no
// logit shows it.  f16 numbers reach down to 2^-24 and a pair of terms resolves 2^-25: an element keeps its 22 bits
// down to 2^-17 of its column's largest where d is 0, and is off by 2^-39 of it below that.  G (between -1 and 1
// before the division by N) is taken times 2^15.  So a bf16 call has 2 + 2 + 3 + 2 products (logits twice, dH, dW),
// an fp32 one four times 3.  Where products are so large that this is not enough for rows and classes of ordinary
// size beside them, fp32 matrix cores take the operands as they are (kMostExponent).  (dH of bf16 features from one
// term of G and of W each, two products less, was wrong by 2^-11 of its terms: a tenth of the sum where the weights
// of a feature are alike and G W cancels.)
//
// What bounds it: the matrix cores.  16384 x 512 -> 50001 bf16 with both gradients 6.65 ms, 1140 TFLOP/s of these products over
// the whole call (a library f16 product of 8192^3 reaches 1074 here); 4096 x 256 -> 32768 fp32 0.87 ms, 950.  Computing the
// logits again costs 0.19 ms there; writing and reading 4 bytes a logit instead would cost as much.  Calls of few rows and
// few classes are a chain of launches of 3 to 10 us, most of it latency.
#include <type_traits>

#include "gemm_common.h"
#include "internal.h"
#include "load_rules.h"

namespace mixgcn {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx2v __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef unsigned short ushort8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
typedef __attribute__((address_space(3))) uintx4 lds_uintx4;

constexpr int kTile = 128;        // classes and features of a tile
constexpr int kMostTileRows = 256;  // rows of the largest tile
constexpr int kHalfTile = 64;     // classes of a partial sum: what a wavefront holds
constexpr int BK = 32;            // reduction depth of a step
constexpr int kGradShift = 15;
constexpr float kGradScale = 32768.f;  // 2^15
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// What every kernel of a call shares, in the workspace.
struct Meta {
    uint32_t count;  // rows that have a label
    uint32_t wide;   // products on the fp32 matrix cores
    float alpha;     // logit = alpha * sum of the scaled products
};

// Largest exponent of a feature's largest H times its largest W at which the products run on f16 terms.  The terms
// are off by 2^-39 of the largest of a feature, so a logit by 2^(most - 37) per feature, whatever the size of its own
// row: at 16 less than what fp32 sums of rows of ordinary size are off by (at 22, 26, 32 and 38 losses of such rows
// were off by 1e-5, 3e-4, 8e-3 and 0.5).  Past it the planes hold the operands as they are, halves of fp32 numbers,
// and the fp32 matrix cores multiply them: 96 x 256 -> 32000 bf16 153 us instead of 86, 4096 x 256 -> 32768 fp32 2.43
// ms instead of 0.87, 16384 x 512 -> 50001 bf16 27 ms instead of 6.65, at 105 to 125 TFLOP/s.
constexpr int kMostExponent = 16;

// ---- the list of rows with a label --------------------------------------------------------------

__device__ inline bool has_label(int32_t y, int32_t c) { return (uint32_t)y < (uint32_t)c; }

constexpr int kListStep = 4 * kBlock;  // labels that a block looks at at a time, four per thread

__device__ inline uint32_t labelled4(const int32_t* labels, int64_t r, int64_t end, int32_t c)
{
    uint32_t have = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (r + i < end && has_label(labels[r + i], c)) have |= 1u << i;
    return have;
}

// The labels of each block of list_labels.  Clears the maxima of the features.
__global__ __launch_bounds__(kBlock) void count_labels_kernel(const int32_t* __restrict__ labels, int64_t n, int32_t c,
                                                              int per_block, uint32_t* __restrict__ counts,
                                                              uint32_t* __restrict__ top, int n_top)
{
    __shared__ uint32_t part[kBlock / kWave];
    for (int i = blockIdx.x * kBlock + threadIdx.x; i < n_top; i += gridDim.x * kBlock) top[i] = 0u;
    const int64_t r0 = (int64_t)blockIdx.x * per_block, end = r0 + per_block < n ? r0 + per_block : n;
    uint32_t mine = 0;
    for (int64_t r = r0 + 4 * threadIdx.x; r < end; r += kListStep) mine += __popc(labelled4(labels, r, end, c));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, kWave);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    if (threadIdx.x == 0) counts[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

// rows[i]: the i-th row with a label, for block `block` of `blocks`.
__device__ inline void list_labels(int block, int blocks, const int32_t* __restrict__ labels, int64_t n, int32_t c, int per_block,
                                   const uint32_t* __restrict__ counts, uint32_t* __restrict__ rows, Meta* __restrict__ meta)
{
    __shared__ uint64_t lds[4];
    const int tid = threadIdx.x;
    uint64_t before = 0;
    for (int b = tid; b < block; b += kBlock) before += counts[b];
    uint64_t base = 0;
    if (block > 0) block_exclusive_scan_u64(before, &base, lds);
    const int64_t r0 = (int64_t)block * per_block, end = r0 + per_block < n ? r0 + per_block : n;
    for (int64_t s = r0; s < end; s += kListStep) {
        const int64_t r = s + 4 * tid;
        const uint32_t have = labelled4(labels, r, end, c);
        uint64_t total;
        uint64_t at = base + block_exclusive_scan_u64(__popc(have), &total, lds);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (have >> i & 1u) rows[at++] = (uint32_t)(r + i);
        base += total;
    }
    if (block == blocks - 1 && tid == 0) meta->count = (uint32_t)base;
}

// ---- scales -------------------------------------------------------------------------------------

template <bool BF16>
struct Eight {  // eight features of a row of k; the row's pitch holds whole 16 bytes
    static constexpr int V = BF16 ? 1 : 2;
    uint4 v[V];
    __device__ inline void load(const void* p, int64_t row_at, int j, int k)
    {
        if (BF16) {
            v[0] = *reinterpret_cast<const uint4*>((const uint16_t*)p + row_at + j);
        } else {
            v[0] = *reinterpret_cast<const uint4*>((const float*)p + row_at + j);
            v[V - 1] = *reinterpret_cast<const uint4*>((const float*)p + row_at + second_group(j, k));
        }
    }
    __device__ inline float get(int e) const
    {
        const uint4 q = v[BF16 ? 0 : e / 4];
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        if (BF16) return e & 1 ? high_half(w[e / 2]) : low_half(w[e / 2]);
        return __uint_as_float(w[e % 4]);
    }
};
// magnitude as an integer, 0 of what is not finite
__device__ inline uint32_t magnitude(float x)
{
    const uint32_t m = __float_as_uint(x) & 0x7FFFFFFFu;
    return m < 0x7F800000u ? m : 0u;
}
__device__ inline int exponent_of(uint32_t bits)
{
    int e;
    frexpf(__uint_as_float(bits), &e);
    return e - 1;
}

// The exponent of the largest product of a feature's two magnitudes, for a whole block.
__device__ inline int most_exponent(const uint32_t* __restrict__ top, int k, int kp, int* most_of)
{
    int most = -1000;
    for (int i = threadIdx.x; i < k; i += kBlock) {
        const uint32_t h = top[i], w = top[kp + i];
        if (h && w) {
            const int e = exponent_of(h) + exponent_of(w);
            most = e > most ? e : most;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const int t = __shfl_xor(most, o, kWave);
        most = t > most ? t : most;
    }
    if ((threadIdx.x & 63) == 0) most_of[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBlock / kWave; ++w) most = most_of[w] > most ? most_of[w] : most;
    return most == -1000 ? 0 : most;  // 0: all products are zero
}

// The power of two that a feature is taken times on one side: `mine` is its largest magnitude there, `other` the one on
// the other side.  `rest`: this side takes what is left over where their exponents cannot be shared evenly.
// A feature whose products are below 2^-26 in a logit, and below 2^-26 of the largest, is taken for one whose products are as
// large as that: no logit shows it, and either side, which the other one's gradient is made of, stays in the range of f16 however
// small the other one is.  (Left to fall together a side was off by 2^-(39 - d / 2) of its largest, and 0 from d = 84.)
__device__ inline int scale_of(uint32_t mine, uint32_t other, int most, bool rest = false)
{
    if (!mine) return 0;
    const int e = exponent_of(mine);
    if (!other) return 14 - e;
    const int least = -26 - (most > 0 ? most : 0);
    int both = e + exponent_of(other) - most;
    both = both > least ? both : least;
    const int half = both >> 1;
    return 14 + (rest ? both - half : half) - e;
}

constexpr int kTopCols = 4096;  // columns of a row of W per block
constexpr int kTopWidth = 8 * kBlock;  // columns of H that a block takes at a time

// What the roles of the blocks of top_kernel are.
struct TopPlan {
    int list_blocks, list_step;  // the list of the rows with a label
    int w_blocks, w_pieces;      // maxima of the rows of W
    int h_blocks, h_rows;        // maxima of the columns of H, h_rows rows to a block
    int clear_blocks;            // zeros for the rows without a label
    bool alone;                  // every maximum is found by one block, and nothing has cleared them
};

// What a call begins with: the list of the rows with a label; top[k], the largest magnitude of column k of H over these
// rows, and top[kp + k], of row k of W (maxima do not depend on the order of the atomics); zeros for the other rows of
// dH (if it is given) and of the losses of the rows.
// (With the list in a launch of its own before this one 1 x 128 -> 1000 took 23 us instead of 19, 10007 x 256 -> 5003 bf16 86
// instead of 80.)
template <bool BF16>
__global__ __launch_bounds__(kBlock) void top_kernel(const void* __restrict__ H, int64_t ldh,
                                                     const uint32_t* __restrict__ counts, uint32_t* __restrict__ rows,
                                                     Meta* __restrict__ meta, const float* __restrict__ W, int64_t ldw, int k,
                                                     int c, int kp, TopPlan plan, uint32_t* __restrict__ top,
                                                     const int32_t* __restrict__ labels, int64_t n, void* dH,
                                                     int64_t ldd, float* __restrict__ row_loss)
{
    __shared__ uint32_t col_top[kTopWidth];
    const int tid = threadIdx.x;
    int b = blockIdx.x;
    if (b < plan.list_blocks) {
        list_labels(b, plan.list_blocks, labels, n, c, plan.list_step, counts, rows, meta);
        return;
    }
    b -= plan.list_blocks;
    if (b < plan.w_blocks) {
        const int row = b / plan.w_pieces, c0 = b % plan.w_pieces * kTopCols;
        const float* const w = W + (int64_t)row * ldw;
        float4 v[kTopCols / 4 / kBlock];
#pragma unroll
        for (int i = 0; i < kTopCols / 4 / kBlock; ++i) {
            const int j = c0 + 4 * (tid + i * kBlock);
            v[i] = *reinterpret_cast<const float4*>(w + (j < c ? j : c0));
        }
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kTopCols / 4 / kBlock; ++i) {
            const int j = c0 + 4 * (tid + i * kBlock);
            const float f[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t t = j + e < c ? magnitude(f[e]) : 0u;
                m = t > m ? t : m;
            }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint32_t t = __shfl_xor(m, o, kWave);
            m = t > m ? t : m;
        }
        if ((tid & 63) == 0) col_top[tid >> 6] = m;
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int i = 1; i < kBlock / kWave; ++i) m = col_top[i] > m ? col_top[i] : m;
            if (plan.alone) top[kp + row] = m;
            else atomicMax(top + kp + row, m);
        }
    } else if (b < plan.w_blocks + plan.h_blocks) {
        const int64_t i0 = (int64_t)(b - plan.w_blocks) * plan.h_rows;
        const int m_rows = n - i0 < plan.h_rows ? (int)(n - i0) : plan.h_rows;
        for (int j0 = 0; j0 < k; j0 += kTopWidth) {
            const int width = k - j0 < kTopWidth ? k - j0 : kTopWidth;
            const int lanes = (width + 7) / 8, at_once = kBlock / lanes;
            for (int i = tid; i < width; i += kBlock) col_top[i] = 0u;
            __syncthreads();
            const int j = 8 * (tid % lanes);
            uint32_t m[8] = {};
            constexpr int U = 4;
            if (tid < at_once * lanes)
                for (int i = tid / lanes; i < m_rows; i += U * at_once) {
                    bool have[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int iu = i + u * at_once;
                        have[u] = iu < m_rows && has_label(labels[i0 + (iu < m_rows ? iu : i)], c);
                    }
                    Eight<BF16> x[U] = {};
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (have[u]) x[u].load(H, (i0 + i + u * at_once) * ldh, j0 + j, k);
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t t = magnitude(x[u].get(e));
                            m[e] = t > m[e] ? t : m[e];
                        }
                }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (j + e < width && m[e]) atomicMax(&col_top[j + e], m[e]);
            __syncthreads();
            for (int i = tid; i < width; i += kBlock) {
                if (plan.alone) top[j0 + i] = col_top[i];
                else if (col_top[i]) atomicMax(top + j0 + i, col_top[i]);
            }
            __syncthreads();
        }
    } else {
        b -= plan.w_blocks + plan.h_blocks;
        const int cols = dH ? k : 0, per_row = dH ? (k + 7) / 8 : 1, lanes = per_row < kBlock ? per_row : kBlock;
        const int at_once = kBlock / lanes;
        if (tid >= at_once * lanes) return;
        constexpr int U = 4;
        const int64_t step = (int64_t)plan.clear_blocks * at_once;
        for (int64_t r0 = (int64_t)b * at_once + tid / lanes; r0 < n; r0 += U * step) {
            int32_t y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) y[u] = r0 + u * step < n ? labels[r0 + u * step] : 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (has_label(y[u], c)) continue;
                const int64_t r = r0 + u * step;
                if (tid % lanes == 0 && row_loss) row_loss[r] = 0.f;
                for (int j = 8 * (tid % lanes); j < cols; j += 8 * lanes) {
                    const int64_t at = r * ldd + j;
                    if (j + 8 <= cols) {
                        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                        uint4* const o = reinterpret_cast<uint4*>((char*)dH + at * (BF16 ? 2 : 4));
                        o[0] = zero;
                        if (!BF16) o[1] = zero;
                    } else {
                        for (int e = 0; j + e < cols; ++e) {
                            if (BF16) ((uint16_t*)dH)[at + e] = 0;
                            else ((float*)dH)[at + e] = 0.f;
                        }
                    }
                }
            }
        }
    }
}

// ---- operands as f16 terms ----------------------------------------------------------------------

__device__ inline uint32_t pack_f16(float a, float b)
{
    const floatx2v v = {a, b};
    const half2v h = __builtin_convertvector(v, half2v);
    uint32_t u;
    __builtin_memcpy(&u, &h, 4);
    return u;
}
__device__ inline float low_f16(uint32_t u)
{
    half2v h;
    __builtin_memcpy(&h, &u, 4);
    return (float)h[0];
}
__device__ inline float high_f16(uint32_t u)
{
    half2v h;
    __builtin_memcpy(&h, &u, 4);
    return (float)h[1];
}
// a and b less the terms of a pair, as a pair.  minus_one: -1 where the compiler does not see it, for the multiply-adds that
// take and give f16 (of a known -1 it makes a conversion, a subtraction and another conversion).
__device__ inline uint32_t pack_rests(float a, float b, uint32_t terms, float minus_one)
{
    half2v h, r;
    __builtin_memcpy(&h, &terms, 4);
    r[0] = (_Float16)fmaf((float)h[0], minus_one, a);
    r[1] = (_Float16)fmaf((float)h[1], minus_one, b);
    uint32_t u;
    __builtin_memcpy(&u, &r, 4);
    return u;
}
// the rest of x after its first term; none where that is not finite
__device__ inline float rest_of(float x, float t)
{
    const float r = x - t;
    return fabsf(t) <= 65504.f ? r : 0.f;
}

// Eight fp32 numbers as they are: their upper halves to a plane and (bf16 numbers have none) their lower halves to the next.
__device__ inline void put_halves(uint16_t* o, size_t plane, const float (&x)[8], bool both)
{
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t a = __float_as_uint(x[2 * q]), b = __float_as_uint(x[2 * q + 1]);
        hi[q] = a >> 16 | (b & 0xFFFF0000u);
        lo[q] = (a & 0xFFFFu) | b << 16;
    }
    *reinterpret_cast<uint4*>(o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    if (both) *reinterpret_cast<uint4*>(o + plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

// x, and NaN of an infinity: a logit with a term of one is not a number, also where no other term makes it one (left
// an infinity, a logit of -infinity would leave a row's sum of exponentials a number).
__device__ inline float number(float x) { return x + (x - x); }

constexpr int kScaleCols = 2048;  // features whose scales a block keeps in LDS (a multiple of 8)

// The two terms of eight numbers to a plane and the next.
__device__ inline void put_terms(uint16_t* o, size_t plane, const float (&x)[8], bool both)
{
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        hi[q] = pack_f16(x[2 * q], x[2 * q + 1]);
        lo[q] = pack_f16(rest_of(x[2 * q], low_f16(hi[q])), rest_of(x[2 * q + 1], high_f16(hi[q])));
    }
    *reinterpret_cast<uint4*>(o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    if (both) *reinterpret_cast<uint4*>(o + plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

// What the blocks of split_kernel share.  WIDE (the operands as they are) is a function of its own beside the terms: as a branch
// within it made a call of one row 1.3 us longer.
struct Split {
    int k, kp, most;
    const uint32_t* top;
    const int16_t* scale;  // of the first kScaleCols features of the block's operand
};

// A thread takes 32 features of a class.
template <bool WIDE>
__device__ inline void split_weights(const Split& a, int w_blocks, const float* __restrict__ W, int64_t ldw, int c, int cp, int w_rows,
                                     uint16_t* __restrict__ wplanes)
{
    const int64_t items = (int64_t)(a.kp / BK) * cp;
    const size_t plane = (size_t)(a.kp / BK) * w_rows * BK;
    for (int64_t it = (int64_t)blockIdx.x * kBlock + threadIdx.x; it < items; it += (int64_t)w_blocks * kBlock) {
        const int b = (int)(it / cp), j = (int)(it - (int64_t)b * cp);
        uint16_t* const o = wplanes + ((size_t)b * w_rows + j) * BK;
        if (WIDE) {
#pragma unroll 1
            for (int q = 0; q < BK / 8; ++q) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = j < c && b * BK + 8 * q + e < a.k ? number(W[(int64_t)(b * BK + 8 * q + e) * ldw + j]) : 0.f;
                put_halves(o + 8 * q, plane, v, true);
            }
            continue;
        }
        float x[BK];
#pragma unroll
        for (int e = 0; e < BK; ++e) x[e] = j < c && b * BK + e < a.k ? W[(int64_t)(b * BK + e) * ldw + j] : 0.f;
#pragma unroll
        for (int q = 0; q < BK / 8; ++q) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = b * BK + 8 * q + e;
                const int s = i >= a.k ? 0 : b * BK < kScaleCols ? a.scale[i] : scale_of(a.top[a.kp + i], a.top[i], a.most, true);
                v[e] = number(ldexpf(x[8 * q + e], s));
            }
            put_terms(o + 8 * q, plane, v, true);
        }
    }
}

// Four threads take the 32 features of a block in a row.
template <bool BF16, bool WIDE>
__device__ inline void split_rows(const Split& a, int block, int blocks, const void* __restrict__ H, int64_t ldh, const uint32_t* __restrict__ rows,
                                  const int32_t* __restrict__ labels, int live, int h_rows, uint16_t* __restrict__ planes, int32_t* __restrict__ y)
{
    const int end = (live + kMostTileRows - 1) / kMostTileRows * kMostTileRows;
    const size_t plane = (size_t)(a.kp / BK) * h_rows * BK;
    const int64_t items = (int64_t)end * (a.kp / 8), step = (int64_t)blocks * kBlock;
    for (int64_t it = (int64_t)block * kBlock + threadIdx.x; it < items; it += step) {
        const int b = (int)(it / (4 * end)), at = (int)(it - (int64_t)b * (4 * end)), i = at / 4, j = b * BK + at % 4 * 8;
        const bool in = i < live;
        const uint32_t r = in ? rows[i] : 0u;
        if (j == 0) y[i] = in ? labels[r] : -1;
        float x[8] = {};
        if (in && j < a.k) {
            Eight<BF16> v;
            v.load(H, (int64_t)r * ldh, j, a.k);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (j + e < a.k)
                    x[e] = number(ldexpf(v.get(e), WIDE ? 0 : j < kScaleCols ? a.scale[j + e] : scale_of(a.top[j + e], a.top[a.kp + j + e], a.most)));
        }
        uint16_t* const o = planes + ((size_t)b * h_rows + i) * BK + at % 4 * 8;
        if (WIDE) put_halves(o, plane, x, !BF16);
        else put_terms(o, plane, x, !BF16);
    }
}

// planes[t]: the scaled features of the listed rows [first, first + rows of the piece) (or halves of the features themselves),
// zeros past the last one up to a whole tile and past the features.  y[i]: their labels, -1 past the last one.
// Bound by memory: 512 x 50001 weights and 16384 x 512 bf16 features in 70 us (two pieces of rows), 3.4 TB/s;
// 262144 x 128 fp32 50 us, 5.3.
// The first w_blocks blocks: wplanes[t], the two terms of the scaled weights, rows the classes, columns the features,
// zeros past them.
template <bool BF16>
__global__ __launch_bounds__(kBlock, 6) void split_kernel(const void* __restrict__ H, int64_t ldh,
                                                       const uint32_t* __restrict__ rows,
                                                       const int32_t* __restrict__ labels, Meta* __restrict__ meta,
                                                       uint32_t first, int piece_rows, int h_rows, int k, int kp,
                                                       const uint32_t* __restrict__ top, int32_t* __restrict__ shift,
                                                       uint16_t* __restrict__ planes, int32_t* __restrict__ y, int w_blocks,
                                                       const float* __restrict__ W, int64_t ldw, int c, int cp, int w_rows,
                                                       uint16_t* __restrict__ wplanes)
{
    __shared__ int most_of[kBlock / kWave];
    __shared__ int16_t scale_lds[kScaleCols];
    const int most = most_exponent(top, k, kp, most_of);
    const bool wide = most > kMostExponent;
    if (blockIdx.x == 0) {
        // for the kernels that follow
        for (int i = threadIdx.x; i < kp; i += kBlock) {
            shift[i] = wide ? -kGradShift : i < k ? scale_of(top[i], top[kp + i], most) : 0;
            shift[kp + i] = wide ? -kGradShift : i < k ? scale_of(top[kp + i], top[i], most, true) : 0;
        }
        // (not down to zero, which would make NaN of the -infinity past the classes: 2^-100 already leaves all logits at zero)
        if (threadIdx.x == 0) {
            meta->wide = wide;
            meta->alpha = wide ? 1.f : ldexpf(1.f, most < -72 ? -100 : most - 28);
        }
    }
    const bool weights = (int)blockIdx.x < w_blocks;
    const Split a = {k, kp, most, top, scale_lds};
    const uint32_t count = meta->count;
    const int live = first >= count ? 0 : count - first < (uint32_t)piece_rows ? (int)(count - first) : piece_rows;
    if (__builtin_expect(wide, 0)) {
        if (weights) split_weights<true>(a, w_blocks, W, ldw, c, cp, w_rows, wplanes);
        else split_rows<BF16, true>(a, blockIdx.x - w_blocks, gridDim.x - w_blocks, H, ldh, rows + first, labels, live, h_rows, planes, y);
        return;
    }
    for (int i = threadIdx.x; i < k && i < kScaleCols; i += kBlock)
        scale_lds[i] = (int16_t)(weights ? scale_of(top[kp + i], top[i], most, true) : scale_of(top[i], top[kp + i], most));
    __syncthreads();
    if (weights) split_weights<false>(a, w_blocks, W, ldw, c, cp, w_rows, wplanes);
    else split_rows<BF16, false>(a, blockIdx.x - w_blocks, gridDim.x - w_blocks, H, ldh, rows + first, labels, live, h_rows, planes, y);
}

// ---- a tile of a product ------------------------------------------------------------------------
// Operands lie in memory as planes of f16 terms in blocks of 32 columns: column j of row i is at
// [j / 32][i][j % 32], with `rows` rows to a block.  A product takes one with the reduction along its columns (a step of
// 32 is a block, tile rows times 64 contiguous bytes), or, TR, along its rows (a step is 32 rows of each of the tile's
// blocks, 2 KB contiguous); the transposing LDS read turns the latter: lane i of 16 receives element i % 4 of the 8 bytes
// that lanes i / 4, + 4, + 8 and + 12 address.  (With plain rows, of which a step takes 64 bytes each, the second pass over
// the logits of 16384 x 512 -> 50001 bf16 took 1956 us instead of 1676, the product for dH 1923 instead of 1674.)
//
// Sums of A[i][k] B[k][j] over a tile of 64 TM x 64 TN, on 2 x 2 wavefronts of 32 TM x 32 TN.  Steps go straight from
// memory to LDS, 16 bytes per lane and 1 KB per instruction, STAGES - 1 of them ahead; there is one barrier per step,
// before which a wavefront waits for its own part of the step that is due and for what it has read.  LDS holds rows
// without padding, so the 16-byte pieces of a row are put in another order, which each lane fetches from: rows of 64
// bytes have piece p at p ^ (row / 4 % 4), and rows of the free index, in which the transposing read takes 64 bytes of
// four rows at a time, the 64-byte block q at q ^ (row % 4), of rows of two or six blocks at q ^ (row / 2 % 2).  Either way
// the lanes that are served together hit all banks.
struct Operand {
    const uint16_t* p;  // first term of the tile's first element
    int64_t rows;       // rows of a block in memory
    size_t plane;       // halfwords from term to term
};

__device__ inline void clobber() { asm volatile("" ::: "memory"); }
template <int N>
__device__ inline void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    clobber();
}
// 16 bytes per lane from base + offset to LDS at lds + 16 lane (lds in bytes, the same for the wavefront).  The
// compiler does not count this load: wait_and_meet waits for it.  (M0 is no register that the compiler keeps values in,
// and nothing else here uses it.  The instruction after a write of M0 waits one state, one that takes a base from registers
// that a vector instruction may have written waits five.)
__device__ inline void load_to_lds(const uint16_t* base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(lds) : "memory");
}

//
// GRAD: which operand is G (0: neither).  With `wide` the planes of the other ones hold halves of fp32 numbers, G is
// taken from its two terms, without their 2^15, and an f16 instruction over 16 reduction indices is eight fp32 ones
// over two, index i of either half of the wavefront: a lane has the same elements of its operands for either.
template <int TA, int TB, bool TRA, bool TRB, int TM, int TN, int STAGES, int GRAD = 0>
struct Product {
    static constexpr int WA = 64 * TM, WB = 64 * TN;              // extents of the tile
    static constexpr int PA = WA * BK, PB = WB * BK;              // halfwords of a plane
    static constexpr int BUFFER = TA * PA + TB * PB;
    static constexpr int LDS = STAGES * BUFFER;
    static constexpr int IA = PA / 512 / 4, IB = PB / 512 / 4;    // loads of a wavefront per plane
    static constexpr int LOADS = TA * IA + TB * IB;

    // what the 64-byte block of a row of the reduction index is exclusive-ored with
    template <int WIDTH>
    static __device__ inline int turn(int row)
    {
        static_assert(WIDTH == 64 || WIDTH == 128 || WIDTH == 192 || WIDTH == 256, "a multiple of two or of four blocks to a row");
        return WIDTH % 128 ? row >> 1 & 1 : row & 3;
    }
    // where lane `lane` of load `i` of a plane reads, in bytes from the plane's first element of the step
    template <bool TR, int WIDTH>
    static __device__ inline uint32_t source(int64_t rows, int i, int lane)
    {
        if (TR) {
            const int row = (i * 64 + lane) / (WIDTH / 8), slot = (i * 64 + lane) % (WIDTH / 8);
            return (uint32_t)((slot / 4 ^ turn<WIDTH>(row)) * rows * 64) + 64u * (uint32_t)row + 16u * (uint32_t)(slot % 4);
        }
        const int row = i * 16 + lane / 4, slot = lane % 4;
        return 64u * (uint32_t)row + 16u * (uint32_t)(slot ^ ((row >> 2) & 3));
    }
    // halfwords from the plane's start: operand of the 32 free indices from free0 on, 16 reduction indices from kc on
    template <bool TR, int WIDTH>
    static __device__ inline half8 fragment(const uint16_t* t, int free0, int kc, int lane)
    {
        half8 o;
        if (TR) {
            const int grp = lane >> 4, gs = lane & 15, row = kc + 8 * (grp >> 1) + (gs >> 2);
            const uint16_t* const p = t + row * WIDTH + ((free0 / 32 ^ turn<WIDTH>(row)) * 32) + 16 * (grp & 1) + 4 * (gs & 3);
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)p);
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p + 4 * WIDTH));
            const shortx8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            __builtin_memcpy(&o, &v, 16);
        } else {
            const int r = lane & 31;
            o = *reinterpret_cast<const half8*>(t + (free0 + r) * BK + 8 * ((kc / 8 + (lane >> 5)) ^ ((r >> 2) & 3)));
        }
        return o;
    }

    // the numbers that a lane's operand stands for with `wide`
    template <int T, bool G>
    static __device__ inline void widen(const half8 (&f)[T], float (&o)[8])
    {
        ushort8 h[T];
        __builtin_memcpy(h, f, sizeof(h));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (G) o[i] = ((float)f[0][i] + (float)f[T - 1][i]) * (1.f / kGradScale);
            else o[i] = __uint_as_float((uint32_t)h[0][i] << 16 | (T == 2 ? (uint32_t)h[T - 1][i] : 0u));
        }
    }

    // Sums over nk steps into acc (which the caller has cleared or filled).
    static __device__ inline void run(const Operand& a, const Operand& b, int nk, bool wide, uint16_t* lds, floatx16 (&acc)[TM][TN])
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wm = wave / 2, wn = wave % 2;
        const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)lds;
        uint32_t oa[IA], ob[IB];
#pragma unroll
        for (int i = 0; i < IA; ++i) oa[i] = source<TRA, WA>(a.rows, wave * IA + i, lane);
#pragma unroll
        for (int i = 0; i < IB; ++i) ob[i] = source<TRB, WB>(b.rows, wave * IB + i, lane);
        const int64_t sa = TRA ? BK * BK : BK * a.rows, sb = TRB ? BK * BK : BK * b.rows;
        auto load = [&](int step, int buffer) {
            const uint32_t to = lds0 + (uint32_t)buffer * (BUFFER * 2);
#pragma unroll
            for (int t = 0; t < TA; ++t)
#pragma unroll
                for (int i = 0; i < IA; ++i)
                    load_to_lds(a.p + t * a.plane + step * sa, oa[i], to + (uint32_t)(t * PA * 2 + (wave * IA + i) * 1024));
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int i = 0; i < IB; ++i)
                    load_to_lds(b.p + t * b.plane + step * sb, ob[i],
                                to + (uint32_t)((TA * PA + t * PB) * 2 + (wave * IB + i) * 1024));
        };
        auto mma = [&](const uint16_t* buf) {
#pragma unroll
            for (int kc = 0; kc < BK; kc += 16) {
                half8 fa[TA][TM], fb[TB][TN];
#pragma unroll
                for (int t = 0; t < TA; ++t)
#pragma unroll
                    for (int x = 0; x < TM; ++x) fa[t][x] = fragment<TRA, WA>(buf + t * PA, (wm * TM + x) * 32, kc, lane);
#pragma unroll
                for (int t = 0; t < TB; ++t)
#pragma unroll
                    for (int x = 0; x < TN; ++x)
                        fb[t][x] = fragment<TRB, WB>(buf + TA * PA + t * PB, (wn * TN + x) * 32, kc, lane);
                // the smaller products first
#pragma unroll
                for (int q = 1; q >= 0; --q)
#pragma unroll
                    for (int t = 0; t < TA; ++t) {
                        const int u = q - t;
                        if (u < 0 || u >= TB) continue;
#pragma unroll
                        for (int x = 0; x < TM; ++x)
#pragma unroll
                            for (int y = 0; y < TN; ++y)
                                acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[t][x], fb[u][y], acc[x][y], 0, 0, 0);
                    }
            }
        };
        auto mma_wide = [&](const uint16_t* buf) {
#pragma unroll 1
            for (int kc = 0; kc < BK; kc += 16) {
                float fb[TN][8];
#pragma unroll
                for (int y = 0; y < TN; ++y) {
                    half8 f[TB];
#pragma unroll
                    for (int t = 0; t < TB; ++t) f[t] = fragment<TRB, WB>(buf + TA * PA + t * PB, (wn * TN + y) * 32, kc, lane);
                    widen<TB, GRAD == 2>(f, fb[y]);
                }
#pragma unroll
                for (int x = 0; x < TM; ++x) {
                    half8 f[TA];
                    float fa[8];
#pragma unroll
                    for (int t = 0; t < TA; ++t) f[t] = fragment<TRA, WA>(buf + t * PA, (wm * TM + x) * 32, kc, lane);
                    widen<TA, GRAD == 1>(f, fa);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int y = 0; y < TN; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i], fb[y][i], acc[x][y], 0, 0, 0);
                }
            }
        };
        auto walk = [&](auto multiply) {
            clobber();
#pragma unroll
            for (int s = 0; s < STAGES - 1; ++s)
                if (s < nk) load(s, s);
            int cur = 0;  // buffer of the step
            for (int i = 0; i < nk; ++i) {
                // the steps after this one that are on their way may stay so, where all of them are
                if (i + STAGES - 2 < nk) wait_and_meet<(STAGES - 2) * LOADS>();
                else wait_and_meet<0>();
                const int free = cur == 0 ? STAGES - 1 : cur - 1;
                if (i + STAGES - 1 < nk) load(i + STAGES - 1, free);
                multiply(lds + cur * BUFFER);
                cur = cur + 1 == STAGES ? 0 : cur + 1;
            }
        };
        if (__builtin_expect(wide, 0)) walk(mma_wide);
        else walk(mma);
    }
};

template <int TM, int TN>
__device__ inline void clear(floatx16 (&acc)[TM][TN])
{
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.f;
}
// row of a 32 x 32 tile that register v of a lane holds (its column is lane % 32)
__device__ inline int tile_row(int v, int lane) { return 8 * (v / 4) + 4 * (lane >> 5) + (v % 4); }

// rows of the piece that starts at `first`
__device__ inline int rows_here(const Meta* meta, uint32_t first, int piece_rows)
{
    const uint32_t count = meta->count;
    return first >= count ? 0 : count - first < (uint32_t)piece_rows ? (int)(count - first) : piece_rows;
}

// ---- logits -------------------------------------------------------------------------------------
// Tiles of logits come transposed, classes x rows, so that a lane holds classes of one row: sums over the classes stay
// in the lane, but for one exchange of its halves.  A sum of products times a2 = alpha log2(e) is a logit in units of log 2.
// Exponentials are of the difference from the largest sum, which is exact where it is small: the largest term of a row is
// 1, no loss is below zero, and one next to it is off by the rounding of 1 + what is beside it.  (Products with a2 before the
// difference round by 2^-24 of the logit, and a loss next to zero was off by that, to either side.)
//
// A workgroup takes 128 classes (a wavefront 64) and 64 TN rows; few rows, for which there are few workgroups, have more steps on
// their way.  Tiles are walked in groups of 8 tiles of classes: their
// weights stay in the L2 of an XCD while the rows pass by.
template <int TH, int TN>
struct Logits {
    static constexpr int STAGES = TN > 1 ? 2 : TH == 1 ? 4 : 3;
    using P = Product<2, TH, false, false, 2, TN, STAGES>;
    static constexpr int ROWS = 64 * TN, GROUP = 8;  // (4, 8, 16: 4096 x 256 -> 32768 fp32 879 873 885 us, 16384 x 512 -> 50001 bf16 within 0.4 %)
    int c0, r0;  // first class and row of the tile

    // false: no such tile.  The tiles of the rows there are, not of the grid, are dealt to the XCDs.
    __device__ inline bool find(int live, int class_tiles)
    {
        const unsigned row_tiles = (unsigned)(live + ROWS - 1) / ROWS, tiles = row_tiles * (unsigned)class_tiles;
        if (blockIdx.x >= tiles) return false;
        const unsigned lid = xcd_local_index(blockIdx.x, tiles);
        const unsigned group = lid / (GROUP * row_tiles), at = lid - group * (GROUP * row_tiles);
        const unsigned width = (unsigned)class_tiles - group * GROUP < GROUP ? (unsigned)class_tiles - group * GROUP : GROUP;
        r0 = __builtin_amdgcn_readfirstlane((int)(at / width) * ROWS);
        c0 = __builtin_amdgcn_readfirstlane((int)(group * GROUP + at % width) * kTile);
        return true;
    }
};

// 16384 x 512 -> 50001 bf16 1.26 ms, 1330 TFLOP/s: matrix cores busy 67 % of the cycles, at 1.7 GHz (the clock falls
// under this load). No bank conflicts, 11 % of the reads miss the L2s.  4096 x 256 -> 32768 fp32 190 us, 1090.
// sums[piece of 64 classes][row] = { largest sum of products, sum of 2^(a2 (each less the largest)) }; at_label[row]:
// that of the row's label.
template <int TH, int TN>
__global__ __launch_bounds__(kBlock, 2) void logit_sums_kernel(const uint16_t* __restrict__ Wp, int kp, int w_rows, int c, int nk,
                                                               const uint16_t* __restrict__ Hp, int h_rows, const int32_t* __restrict__ y,
                                                               const Meta* __restrict__ meta, uint32_t first, int piece_rows,
                                                               int class_tiles, float2* __restrict__ sums,
                                                               float* __restrict__ at_label)
{
    using L = Logits<TH, TN>;
    __shared__ __attribute__((aligned(1024))) uint16_t lds[L::P::LDS];
    L tile;
    if (!tile.find(rows_here(meta, first, piece_rows), class_tiles)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
    floatx16 acc[2][TN];
    clear(acc);
    L::P::run({Wp + (size_t)tile.c0 * BK, w_rows, (size_t)kp * w_rows}, {Hp + (size_t)tile.r0 * BK, h_rows, (size_t)kp * h_rows}, nk,
              meta->wide, lds, acc);
    const float a2 = meta->alpha * kLog2e;
    const int cw = tile.c0 + wm * 64;
    if (cw + kHalfTile > c)  // the last classes
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (cw + x * 32 + tile_row(v, lane) >= c)
#pragma unroll
                    for (int yy = 0; yy < TN; ++yy) acc[x][yy][v] = -INFINITY;
#pragma unroll
    for (int yy = 0; yy < TN; ++yy) {
        const int row = tile.r0 + (wn * TN + yy) * 32 + (lane & 31);
        float most = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v) most = fmaxf(most, acc[x][yy][v]);
        most = fmaxf(most, __shfl_xor(most, 32, kWave));
        const float base = most == -INFINITY ? 0.f : most;
        float sum = 0.f;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v) sum += __builtin_amdgcn_exp2f((acc[x][yy][v] - base) * a2);
        sum += __shfl_xor(sum, 32, kWave);
        if (lane < 32) sums[(size_t)(cw / kHalfTile) * piece_rows + row] = make_float2(most, sum);
        const int at = y[row] - cw;
        if (__any(at >= 0 && at < kHalfTile)) {
            float mine = 0.f;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (at == x * 32 + tile_row(v, lane)) mine = acc[x][yy][v];
            if (at >= 0 && at < kHalfTile && ((at >> 2) & 1) == (lane >> 5)) at_label[row] = mine;
        }
    }
}

// A row's largest sum of products and what its exponentials are taken times for G, from the sums of its pieces; the loss of the row.
// A block takes ROWS rows, kBlock / ROWS lanes walk the pieces of each; losses[block]: the sum of its rows' losses.
template <int ROWS>
__global__ __launch_bounds__(kBlock) void join_sums_kernel(const float2* __restrict__ sums, int pieces,
                                                           const float* __restrict__ at_label,
                                                           const Meta* __restrict__ meta, uint32_t first, int piece_rows,
                                                           const uint32_t* __restrict__ rows, float2* __restrict__ norm,
                                                           double* __restrict__ losses, float* __restrict__ row_loss)
{
    constexpr int LANES = kBlock / ROWS;
    __shared__ float tops[LANES][ROWS + 1], parts[LANES][ROWS + 1];
    const int live = rows_here(meta, first, piece_rows);
    const int j = threadIdx.x % ROWS, q = threadIdx.x / ROWS;
    const int row = blockIdx.x * ROWS + j;
    if ((int)blockIdx.x * ROWS >= live) return;
    const int rr = row < live ? row : live - 1;
    const float a2 = meta->alpha * kLog2e;
    float top = -INFINITY, sum = 0.f;
    bool bad = false;
    for (int p0 = q; p0 < pieces; p0 += 4 * LANES) {
        float2 s[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int p = p0 + u * LANES;
            s[u] = sums[(size_t)(p < pieces ? p : p0) * piece_rows + rr];
            if (p >= pieces) s[u] = make_float2(-INFINITY, 0.f);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            bad = bad || !(s[u].y == s[u].y);
            if (s[u].x > top) {
                sum = sum * __builtin_amdgcn_exp2f((top - s[u].x) * a2) + s[u].y;
                top = s[u].x;
            } else if (s[u].x > -INFINITY) {
                sum += s[u].y * __builtin_amdgcn_exp2f((s[u].x - top) * a2);
            }
        }
    }
    tops[q][j] = top;
    parts[q][j] = bad ? __uint_as_float(0x7FC00000u) : sum;
    __syncthreads();
    float l = 0.f;
    if (q == 0 && row < live) {
        float m = -INFINITY;
        for (int i = 0; i < LANES; ++i) m = fmaxf(m, tops[i][j]);
        float s = 0.f;
        // (what is not a number stays one: the lanes before it and after it add to it)
        for (int i = 0; i < LANES; ++i)
            s += parts[i][j] * (tops[i][j] > -INFINITY ? __builtin_amdgcn_exp2f((tops[i][j] - m) * a2) : 0.f);
        if (!(m > -INFINITY)) s = __uint_as_float(0x7FC00000u);
        norm[row] = make_float2(m, kGradScale / s);
        l = ((m - at_label[row]) * a2 + log2f(s)) * kLn2;
        if (row_loss) row_loss[rows[first + row]] = l;
    }
    __syncthreads();
    if (q == 0) parts[0][j] = l;
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (int i = 0; i < ROWS; ++i) sum += (double)parts[0][i];
        losses[first / ROWS + blockIdx.x] = sum;
    }
}

// Mean of the losses, from the sums of `per` rows each, in a fixed order; 0 without rows.
__device__ inline void mean_loss(const double* __restrict__ losses, int per, uint32_t count, double* __restrict__ loss)
{
    __shared__ double sh[kBlock / kWave];
    const int64_t parts = ((int64_t)count + per - 1) / per;
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < parts; i += 8 * kBlock) {
        double v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = i + u * kBlock < parts ? losses[i + u * kBlock] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u) s += v[u];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) *loss = count ? ((sh[0] + sh[1]) + (sh[2] + sh[3])) / (double)count : 0.0;
}

__global__ __launch_bounds__(kBlock) void mean_loss_kernel(const double* __restrict__ losses, int per,
                                                           const Meta* __restrict__ meta, double* __restrict__ loss)
{
    mean_loss(losses, per, meta->count, loss);
}

// ---- gradient with respect to the logits --------------------------------------------------------

// The two terms of a 32 x 32 tile of G, from registers as the matrix instruction leaves them to its place in either plane.  tmp:
// 4 KB that only this wavefront uses.
__device__ inline void store_grad(const float (&g)[16], float minus_one, int lane, uint16_t* tmp, uint16_t* o, size_t plane)
{
    // groups of 8 classes, of which this lane has the four at 4 (lane / 32)
    uint32_t hi[8], lo[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        hi[p] = pack_f16(g[2 * p], g[2 * p + 1]);
        lo[p] = pack_rests(g[2 * p], g[2 * p + 1], hi[p], minus_one);
    }
    // The halves of the wavefront exchange, so that each has eight classes of a row, and the 32 rows of 64 bytes go
    // through LDS into the order they have in memory (piece p of row r at p ^ (r / 4 % 4)): a store is then 1 KB in a
    // row (72640 x 32 -> 8123 fp32 1518 -> 1479 us).
    auto put = [&](uint16_t* to, uint16_t* t, const uint32_t (&w)[8]) {
#pragma unroll
        for (int q = 0; q < 8; q += 4) {
            const auto s0 = __builtin_amdgcn_permlane32_swap(w[q], w[q + 2], false, false);
            const auto s1 = __builtin_amdgcn_permlane32_swap(w[q + 1], w[q + 3], false, false);
            const uintx4 v = {s0[0], s1[0], s0[1], s1[1]};
            const int r = lane & 31, p = q / 2 + (lane >> 5);
            *(lds_uintx4*)(t + r * BK + 8 * (p ^ (r >> 2 & 3))) = v;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 16 * i + lane / 4, p = lane % 4;
            const uintx4 v = *(lds_uintx4*)(t + r * BK + 8 * (p ^ (r >> 2 & 3)));
            *reinterpret_cast<uint4*>(to + i * 512) = make_uint4(v.x, v.y, v.z, v.w);
        }
    };
    put(o, tmp, hi);
    put(o + plane, tmp + 1024, lo);
}

// The two passes over 16384 x 512 -> 50001 bf16 take 1.26 and 1.69 ms: beside its products (41 % of the cycles) this one takes
// exponentials, terms and their way through LDS, 13 vector instructions to a logit, and writes 2 TB/s; 15 % of its LDS cycles are
// bank conflicts.
// planes[t], rows the listed ones and columns the classes from col0 on: 2^15 (softmax - onehot), zeros past the rows up to
// a whole tile and past the classes up to whole blocks of 32; what blocks past these hold reaches no result.
template <int TH, int TN>
__global__ __launch_bounds__(kBlock, 2) void logit_grad_kernel(const uint16_t* __restrict__ Wp, int kp, int w_rows, int c, int nk,
                                                               const uint16_t* __restrict__ Hp, int h_rows, const int32_t* __restrict__ y,
                                                               const float2* __restrict__ norm,
                                                               const Meta* __restrict__ meta, uint32_t first, int piece_rows,
                                                               int col0, int g_rows, int class_tiles,
                                                               uint16_t* __restrict__ planes)
{
    using L = Logits<TH, TN>;
    __shared__ __attribute__((aligned(1024))) uint16_t lds[L::P::LDS];
    const int live = rows_here(meta, first, piece_rows);
    L tile;
    if (!tile.find(live, class_tiles)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
    floatx16 acc[2][TN];
    clear(acc);
    L::P::run({Wp + (size_t)(col0 + tile.c0) * BK, w_rows, (size_t)kp * w_rows},
              {Hp + (size_t)tile.r0 * BK, h_rows, (size_t)kp * h_rows}, nk, meta->wide, lds, acc);
    const float a2 = meta->alpha * kLog2e;
    const int cw = col0 + tile.c0 + wm * 64;
    const bool edge = cw + kHalfTile > c;
    float minus_one = -1.f;
    asm("" : "+v"(minus_one));
    uint16_t* const mine = lds + wave * 4096;  // 8 KB that only this wavefront uses
    __syncthreads();
    const size_t plane = (size_t)class_tiles * kTile * g_rows;
#pragma unroll
    for (int yy = 0; yy < TN; ++yy) {
        const int row = tile.r0 + (wn * TN + yy) * 32 + (lane & 31);
        // rows past the last one have no features and so no logits: times zero they have no gradient
        const float2 nm = row < live ? norm[row] : make_float2(0.f, 0.f);
        const int at = y[row] - cw;
        const bool mark = __any(at >= 0 && at < kHalfTile);
        uint16_t* const out = planes + ((size_t)((tile.c0 + wm * 64) / BK) * g_rows + tile.r0 + (wn * TN + yy) * 32) * BK + 8 * lane;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (cw + x * 32 >= c) continue;
            float g[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) g[v] = __builtin_amdgcn_exp2f((acc[x][yy][v] - nm.x) * a2);
#pragma unroll
            for (int v = 0; v < 16; ++v) g[v] *= nm.y;
            if (mark || edge)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int i = x * 32 + tile_row(v, lane);
                    if (at == i) g[v] -= kGradScale;
                    if (cw + i >= c) g[v] = 0.f;
                }
            store_grad(g, minus_one, lane, mine + 2 * x * 1024, out + (size_t)x * g_rows * BK, plane);
        }
    }
}

// Few classes, all in one tile: a workgroup has its rows' logits at once, and their losses and G come from one pass over them.
// (262144 x 128 -> 172 fp32 506 -> 400 us, 2000 x 100 -> 220 bf16 54 -> 38.)  losses: a
// sum per 64 rows.  planes may be null.
template <int TH, int TM, int TN>
__global__ __launch_bounds__(kBlock, 2) void logit_rows_kernel(const uint16_t* __restrict__ Wp, int kp, int w_rows, int c, int nk,
                                                               const uint16_t* __restrict__ Hp, int h_rows, const int32_t* __restrict__ y,
                                                               const Meta* __restrict__ meta, uint32_t first, int piece_rows,
                                                               const uint32_t* __restrict__ rows, double* __restrict__ losses,
                                                               float* __restrict__ row_loss, int g_rows, int cols, uint16_t* __restrict__ planes)
{
    constexpr int STEP = 64 * BK * (2 * TM + TH * TN), MOST = 40960 / STEP;  // halfwords
    using P = Product<2, TH, false, false, TM, TN, MOST < 4 ? MOST : 4>;
    constexpr int ROWS = 64 * TN;
    __shared__ __attribute__((aligned(1024))) uint16_t lds[P::LDS];
    static_assert(P::LDS >= 4 * 2048 + 2 * 5 * ROWS, "LDS of the end");
    const int live = rows_here(meta, first, piece_rows), r0 = blockIdx.x * ROWS;
    if (r0 >= live) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
    floatx16 acc[TM][TN];
    clear(acc);
    P::run({Wp, w_rows, (size_t)kp * w_rows}, {Hp + (size_t)r0 * BK, h_rows, (size_t)kp * h_rows}, nk, meta->wide, lds, acc);
    const float a2 = meta->alpha * kLog2e;
    uint16_t* const mine = lds + wave * 2048;
    float(*const tops)[ROWS] = reinterpret_cast<float(*)[ROWS]>(lds + 4 * 2048);  // of the two halves of the classes
    float(*const sums)[ROWS] = tops + 2;
    float* const at_label = sums[2];
    __syncthreads();
    const int cw = wm * TM * 32;
#pragma unroll
    for (int x = 0; x < TM; ++x)
        if (cw + (x + 1) * 32 > c)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (cw + x * 32 + tile_row(v, lane) >= c)
#pragma unroll
                    for (int yy = 0; yy < TN; ++yy) acc[x][yy][v] = -INFINITY;
#pragma unroll
    for (int yy = 0; yy < TN; ++yy) {
        const int row = (wn * TN + yy) * 32 + (lane & 31), at = y[r0 + row] - cw;
        float most = -INFINITY, label = 0.f;
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                most = fmaxf(most, acc[x][yy][v]);
                if (at == x * 32 + tile_row(v, lane)) label = acc[x][yy][v];
            }
        most = fmaxf(most, __shfl_xor(most, 32, kWave));
        if (lane < 32) tops[wm][row] = most;
        if (at >= 0 && at < TM * 32 && (at >> 2 & 1) == lane >> 5) at_label[row] = label;
    }
    __syncthreads();
#pragma unroll
    for (int yy = 0; yy < TN; ++yy) {
        const int row = (wn * TN + yy) * 32 + (lane & 31);
        const float most = fmaxf(tops[0][row], tops[1][row]), base = most == -INFINITY ? 0.f : most;
        float sum = 0.f;
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                acc[x][yy][v] = __builtin_amdgcn_exp2f((acc[x][yy][v] - base) * a2);
                sum += acc[x][yy][v];
            }
        sum += __shfl_xor(sum, 32, kWave);
        if (most == -INFINITY) sum = __uint_as_float(0x7FC00000u);
        if (lane < 32) sums[wm][row] = sum;
    }
    __syncthreads();
    if (planes) {
        float minus_one = -1.f;
        asm("" : "+v"(minus_one));
        const size_t plane = (size_t)cols * g_rows;
#pragma unroll
        for (int yy = 0; yy < TN; ++yy) {
            const int row = (wn * TN + yy) * 32 + (lane & 31), at = y[r0 + row] - cw;
            // rows past the last one have no gradient
            const float unit = r0 + row < live ? kGradScale / (sums[0][row] + sums[1][row]) : 0.f;
            uint16_t* const out = planes + ((size_t)(wm * TM) * g_rows + r0 + (wn * TN + yy) * 32) * BK + 8 * lane;
#pragma unroll
            for (int x = 0; x < TM; ++x) {
                if (cw + x * 32 >= c) continue;
                float g[16];
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    g[v] = acc[x][yy][v] * unit;
                    if (at == x * 32 + tile_row(v, lane)) g[v] -= kGradScale;
                }
                if (cw + (x + 1) * 32 > c)  // where the row is not a number
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (cw + x * 32 + tile_row(v, lane) >= c) g[v] = 0.f;
                store_grad(g, minus_one, lane, mine, out + (size_t)x * g_rows * BK, plane);
            }
        }
    }
    if (threadIdx.x < ROWS) {
        const int row = threadIdx.x, r = r0 + row;
        double l = 0.0;
        if (r < live) {
            const float f = ((fmaxf(tops[0][row], tops[1][row]) - at_label[row]) * a2 + log2f(sums[0][row] + sums[1][row])) * kLn2;
            if (row_loss) row_loss[rows[first + r]] = f;
            l = (double)f;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, kWave);
        if (lane == 0 && r < live) losses[first / 64 + blockIdx.x * TN + wave] = l;
    }
}

// ---- dH and dW ----------------------------------------------------------------------------------
// Of a block of G (the listed rows from `first` on, the classes from col0 on):
//   dh[slab][row][kp] (+)= G[row][classes of the slab] W'^T,     dw[slab][kp][piece_cols] = H'^T[rows of the slab] G.
// One launch has the workgroups of both, row_blocks of dH first, so that the products of one fill the end of the other.
// 16384 x 512 -> 50001 bf16, 14 blocks of 8192 classes and rows: 3.41 ms, 1230 TFLOP/s, matrix cores busy 61 % of the
// cycles; 4096 x 256 -> 32768 fp32 373 us, 1100.  262144 x 128 -> 172 fp32: 172 us, 3.9 TB/s of G, features and dH.

// The classes of a block of G are dealt to slabs for dH, so that every compute unit has a workgroup; how many are
// needed depends on the rows with a label that there are (12839 x 352 -> 29071 bf16, a twentieth labelled, 681 -> 318
// us while dH was one product).  There is room for the sums of `planned` slabs of all rows; 0: the product writes dH
// itself, in one.
struct RowSlabs {
    int tiles;         // of features
    int tile_rows;
    int cols;          // classes of a whole block of G
    int planned, piece_rows;

    __host__ __device__ int row_tiles(int live) const { return (live + tile_rows - 1) / tile_rows; }
    __host__ __device__ int slab_cols(int live) const
    {
        const int rt = row_tiles(live) > 0 ? row_tiles(live) : 1, col_tiles = cols / kTile;
        const int room = planned * piece_rows / (rt * tile_rows);  // (planned * piece_rows < 2^20)
        int n = 256 / (tiles * rt);
        n = n < room ? n : room;
        n = n < col_tiles ? n : col_tiles;
        n = n > 1 ? n : 1;
        return (col_tiles + n - 1) / n * kTile;
    }
    __host__ __device__ int slabs(int live) const { return (cols + slab_cols(live) - 1) / slab_cols(live); }
    __host__ __device__ int64_t slab_rows(int live) const { return (int64_t)row_tiles(live) * tile_rows; }
};

struct Gradients {
    const uint16_t *g, *hp, *wp;
    int kp, h_rows, w_rows, g_rows;
    const Meta* meta;
    uint32_t first;
    int piece_rows, piece_cols, col0;
    int row_blocks;
    RowSlabs row_slabs;
    bool add;
    float* dh;
    int w_slabs, class_tiles;                  // dW: its rows are dealt to slabs
    float* dw;
    // where that is one slab and one block of rows, dW itself takes the sums, and dH where it is one slab and one block of classes
    float* dW;
    int64_t ldg;
    int k, c;
    const int32_t* shift;
    void* dH;
    int64_t ldd;
    const uint32_t* rows;
};

constexpr int kGradRows = 128;  // rows of a tile of dH

// Tiles of 128 rows x 64 TN features, of `BF16` or fp32 features.
template <bool BF16, int TN>
struct GradRows {
    static constexpr int TM = kGradRows / 64, ROWS = kGradRows;
    using P = Product<2, 2, false, true, TM, TN, 2, 1>;

    // Rows of dH from the wavefront's sums, of features f0 on and listed rows r0 on.
    static __device__ inline void write(const Gradients& a, int r0, int live, int f0, int lane, const floatx16 (&acc)[TM][TN])
    {
        const float inv = 1.f / (float)a.meta->count;
        const int f = f0 + (lane & 31);
        int e[TN];
#pragma unroll
        for (int y = 0; y < TN; ++y) e[y] = -kGradShift - a.shift[a.kp + f + y * 32];
#pragma unroll
        for (int x = 0; x < TM; ++x) {
            if (r0 + x * 32 >= live) continue;
            uint32_t row[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int r = r0 + x * 32 + tile_row(v, lane);
                row[v] = a.rows[a.first + (r < live ? r : live - 1)];
            }
#pragma unroll
            for (int y = 0; y < TN; ++y)
#pragma unroll
                for (int v = 0; v < 16; v += 2) {
                    const float g0 = ldexpf(acc[x][y][v] * inv, e[y]), g1 = ldexpf(acc[x][y][v + 1] * inv, e[y]);
                    const int r = r0 + x * 32 + tile_row(v, lane), col = f + y * 32;
                    if (BF16) {
                        // neighboring lanes exchange, so that each has two features of one of the rows
                        const bool odd = lane & 1;
                        const int send = __float_as_int(odd ? g0 : g1);
                        const float got = __int_as_float(__builtin_amdgcn_update_dpp(send, send, 0xB1, 0xF, 0xF, false));
                        const uint32_t w = odd ? pack_bf16(got, g1) : pack_bf16(g0, got);
                        const int c0 = col & ~1;
                        if (r + (odd ? 1 : 0) >= live) continue;
                        uint16_t* const o = (uint16_t*)a.dH + (int64_t)(odd ? row[v + 1] : row[v]) * a.ldd + c0;
                        if (c0 + 1 < a.k) *reinterpret_cast<uint32_t*>(o) = w;
                        else if (c0 < a.k) *o = (uint16_t)w;
                    } else if (col < a.k) {
                        float* const o = (float*)a.dH + col;
                        if (r < live) o[(int64_t)row[v] * a.ldd] = g0;
                        if (r + 1 < live) o[(int64_t)row[v + 1] * a.ldd] = g1;
                    }
                }
        }
    }

    static __device__ inline void run(const Gradients& a, uint16_t* lds)
    {
        const int k_tiles = a.kp / P::WB, live = rows_here(a.meta, a.first, a.piece_rows);
        const unsigned row_tiles = (unsigned)(live + ROWS - 1) / ROWS;
        const int slab_cols = a.row_slabs.slab_cols(live), slabs = a.row_slabs.slabs(live);
        const unsigned tiles = row_tiles * (unsigned)(k_tiles * slabs);
        if (blockIdx.x >= tiles) return;
        const unsigned lid = xcd_local_index(blockIdx.x, tiles);
        const int kt = __builtin_amdgcn_readfirstlane((int)(lid % k_tiles));
        const int slab = __builtin_amdgcn_readfirstlane((int)(lid / k_tiles % slabs));
        const int r0 = __builtin_amdgcn_readfirstlane((int)(lid / (k_tiles * slabs)) * ROWS);
        const int s0 = slab * slab_cols;
        const int cols = a.c - a.col0 < a.piece_cols ? (a.c - a.col0 + BK - 1) / BK * BK : a.piece_cols;
        const int s1 = s0 + slab_cols < cols ? s0 + slab_cols : cols;
        if (a.add && s1 <= s0) return;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
        floatx16 acc[TM][TN];
        clear(acc);
        P::run({a.g + ((size_t)(s0 / BK) * a.g_rows + r0) * BK, a.g_rows, (size_t)a.piece_cols * a.g_rows},
               {a.wp + ((size_t)(kt * P::WB / BK) * a.w_rows + a.col0 + s0) * BK, a.w_rows, (size_t)a.kp * a.w_rows},
               s1 > s0 ? (s1 - s0) / BK : 0, a.meta->wide, lds, acc);
        if (a.dH) {
            write(a, r0 + wm * TM * 32, live, kt * P::WB + wn * TN * 32, lane, acc);
            return;
        }
        float* const out =
            a.dh + ((size_t)slab * a.row_slabs.slab_rows(live) + r0 + wm * TM * 32) * a.kp + kt * P::WB + wn * TN * 32 + (lane & 31);
#pragma unroll
        for (int x = 0; x < TM; ++x) {
            if (r0 + (wm * TM + x) * 32 >= live) continue;
            if (a.add) {
                // all loads of a row of tiles before its first store (left to follow each other they cost 56 us a piece)
                float had[TN][16];
#pragma unroll
                for (int y = 0; y < TN; ++y)
#pragma unroll
                    for (int v = 0; v < 16; ++v) had[y][v] = out[(size_t)(x * 32 + tile_row(v, lane)) * a.kp + y * 32];
#pragma unroll
                for (int y = 0; y < TN; ++y)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[x][y][v] += had[y][v];
            }
#pragma unroll
            for (int y = 0; y < TN; ++y)
#pragma unroll
                for (int v = 0; v < 16; ++v) out[(size_t)(x * 32 + tile_row(v, lane)) * a.kp + y * 32] = acc[x][y][v];
        }
    }
};

// Tiles of 64 TM features x 64 TN classes.
template <int T, int TM, int TN>
struct GradWeights {
    using P = Product<T, 2, true, true, TM, TN, 2, 2>;

    static __device__ inline void run(const Gradients& a, uint16_t* lds)
    {
        const int k_tiles = a.kp / P::WA, class_tiles = a.class_tiles;
        const unsigned lid = xcd_local_index(blockIdx.x - a.row_blocks, gridDim.x - a.row_blocks);
        const int kt = __builtin_amdgcn_readfirstlane((int)(lid % k_tiles));
        const int ct = __builtin_amdgcn_readfirstlane((int)(lid / k_tiles % class_tiles));
        const int slab = __builtin_amdgcn_readfirstlane((int)(lid / (k_tiles * class_tiles)));
        const int live = rows_here(a.meta, a.first, a.piece_rows);
        const int per = ((live + a.w_slabs - 1) / a.w_slabs + BK - 1) / BK * BK;
        const int r0 = slab * per, r1 = r0 + per < live ? r0 + per : live;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
        floatx16 acc[TM][TN];
        clear(acc);
        P::run({a.hp + ((size_t)(kt * P::WA / BK) * a.h_rows + r0) * BK, a.h_rows, (size_t)a.kp * a.h_rows},
               {a.g + ((size_t)(ct * P::WB / BK) * a.g_rows + r0) * BK, a.g_rows, (size_t)a.piece_cols * a.g_rows},
               r1 > r0 ? (r1 - r0 + BK - 1) / BK : 0, a.meta->wide, lds, acc);
        if (a.dW) {
            const float inv = a.meta->count ? 1.f / (float)a.meta->count : 0.f;
            const int f0 = kt * P::WA + wm * TM * 32, col = a.col0 + ct * P::WB + wn * TN * 32 + (lane & 31);
#pragma unroll
            for (int x = 0; x < TM; ++x)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int f = f0 + x * 32 + tile_row(v, lane);
                    if (f >= a.k) continue;
                    const int e = -kGradShift - a.shift[f];
#pragma unroll
                    for (int y = 0; y < TN; ++y)
                        if (col + y * 32 < a.c) a.dW[(int64_t)f * a.ldg + col + y * 32] = ldexpf(acc[x][y][v] * inv, e);
                }
            return;
        }
        float* const out = a.dw + ((size_t)slab * a.kp + kt * P::WA + wm * TM * 32) * a.piece_cols + ct * P::WB + wn * TN * 32 + (lane & 31);
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
            for (int y = 0; y < TN; ++y)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    out[(size_t)(x * 32 + tile_row(v, lane)) * a.piece_cols + y * 32] = acc[x][y][v];
    }
};

template <int T, int TN, int TM, int CN>
__global__ __launch_bounds__(kBlock, 2) void gradients_kernel(Gradients a)
{
    using R = GradRows<T == 1, TN>;
    using W = GradWeights<T, TM, CN>;
    __shared__ __attribute__((aligned(1024))) uint16_t lds[R::P::LDS > W::P::LDS ? R::P::LDS : W::P::LDS];
    if ((int)blockIdx.x < a.row_blocks) R::run(a, lds);
    else W::run(a, lds);
}

// The sum of four neighboring cells over the slabs, for SL lanes that share the cells: lane 0 of them has it.
template <int SL>
__device__ inline float4 sum_slabs(const float* p, size_t slab, int slabs, bool in, float4 (*lds)[kBlock / SL])
{
    const int item = threadIdx.x % (kBlock / SL), l = threadIdx.x / (kBlock / SL);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int b = l; in && b < slabs; b += 4 * SL) {
        float4 t[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            t[u] = b + u * SL < slabs ? *reinterpret_cast<const float4*>(p + (b + u * SL) * slab) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            s.x += t[u].x;
            s.y += t[u].y;
            s.z += t[u].z;
            s.w += t[u].w;
        }
    }
    if (SL == 1) return s;
    lds[l][item] = s;
    __syncthreads();
    if (l == 0)
#pragma unroll
        for (int i = 1; i < SL; ++i) {
            const float4 t = lds[i][item];
            s.x += t.x;
            s.y += t.y;
            s.z += t.z;
            s.w += t.w;
        }
    return s;
}

// What ends a block of G: dH of the listed rows from the slabs' sums (row_blocks blocks), dW[k][classes of the piece] (+)= the slabs'
// sums (w_blocks), and the mean of the losses (one more, where loss is given).
struct Finish {
    const float* dh;
    int row_blocks, piece_rows;
    RowSlabs row_slabs;
    const uint32_t* rows;
    void* dH;
    int64_t ldd;
    const float* dw;
    int w_blocks, w_slabs, piece_cols, cols;
    bool add;
    float* dW;
    int64_t ldg;
    int k, kp;
    const int32_t* shift;
    const Meta* meta;
    uint32_t first;
    const double* losses;
    int loss_rows;
    double* loss;
};

template <bool BF16, int SL>
__device__ inline void finish_rows(const Finish& a)
{
    __shared__ float4 lds[SL][kBlock / SL];
    const int live = rows_here(a.meta, a.first, a.piece_rows);
    const int per_row = (a.k + 3) / 4;
    const float inv = 1.f / (float)a.meta->count;
    const int slabs = a.row_slabs.slabs(live);
    const size_t slab = (size_t)a.row_slabs.slab_rows(live) * a.kp;
    for (int64_t it0 = (int64_t)blockIdx.x * (kBlock / SL); it0 < (int64_t)live * per_row; it0 += (int64_t)a.row_blocks * (kBlock / SL)) {
        const int64_t it = it0 + threadIdx.x % (kBlock / SL);
        const bool in = it < (int64_t)live * per_row;
        const int i = in ? (int)(it / per_row) : 0, j = in ? (int)(it - (int64_t)i * per_row) * 4 : 0;
        const float4 s = sum_slabs<SL>(a.dh + (size_t)i * a.kp + j, slab, slabs, in, lds);
        if (SL > 1) __syncthreads();  // before the next ones are written
        if (!in || threadIdx.x >= kBlock / SL) continue;
        const float v[4] = {s.x, s.y, s.z, s.w};
        float o[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) o[b] = ldexpf(v[b] * inv, -kGradShift - a.shift[a.kp + j + b]);
        const int64_t at = (int64_t)a.rows[a.first + i] * a.ldd + j;
        if (BF16) {
            const uint32_t w[2] = {pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
            if (j + 4 <= a.k) *reinterpret_cast<uint2*>((uint16_t*)a.dH + at) = make_uint2(w[0], w[1]);
            else
                for (int b = 0; j + b < a.k; ++b) ((uint16_t*)a.dH)[at + b] = (uint16_t)(w[b / 2] >> (16 * (b % 2)));
        } else {
            if (j + 4 <= a.k) *reinterpret_cast<float4*>((float*)a.dH + at) = make_float4(o[0], o[1], o[2], o[3]);
            else
                for (int b = 0; j + b < a.k; ++b) ((float*)a.dH)[at + b] = o[b];
        }
    }
}

template <int SL>
__device__ inline void finish_weights(const Finish& a)
{
    __shared__ float4 lds[SL][kBlock / SL];
    const uint32_t count = a.meta->count;
    if (a.add && a.first >= count) return;
    const int per_row = (a.cols + 3) / 4;
    const int64_t it = (int64_t)(blockIdx.x - a.row_blocks) * (kBlock / SL) + threadIdx.x % (kBlock / SL);
    const bool in = it < (int64_t)a.k * per_row;
    const int i = in ? (int)(it / per_row) : 0, j = in ? (int)(it - (int64_t)i * per_row) * 4 : 0;
    const float4 s = sum_slabs<SL>(a.dw + (size_t)i * a.piece_cols + j, (size_t)a.kp * a.piece_cols, a.w_slabs, in, lds);
    if (!in || threadIdx.x >= kBlock / SL) return;
    const float inv = count ? 1.f / (float)count : 0.f;
    const float v[4] = {s.x, s.y, s.z, s.w};
    float* const o = a.dW + (int64_t)i * a.ldg + j;
    const int e = -kGradShift - a.shift[i];
    if (j + 4 <= a.cols) {
        float4 g = make_float4(ldexpf(v[0] * inv, e), ldexpf(v[1] * inv, e), ldexpf(v[2] * inv, e), ldexpf(v[3] * inv, e));
        if (a.add) {
            const float4 d = *reinterpret_cast<const float4*>(o);
            g = make_float4(d.x + g.x, d.y + g.y, d.z + g.z, d.w + g.w);
        }
        *reinterpret_cast<float4*>(o) = g;
    } else {
        for (int b = 0; j + b < a.cols; ++b) {
            const float g = ldexpf(v[b] * inv, e);
            o[b] = a.add ? o[b] + g : g;
        }
    }
}

// WL: lanes that share a cell of dW, 16 where there are many slabs (as for dH)
template <bool BF16, int WL>
__global__ __launch_bounds__(kBlock) void finish_kernel(Finish a)
{
    if ((int)blockIdx.x < a.row_blocks) {
        if (a.row_slabs.slabs(rows_here(a.meta, a.first, a.piece_rows)) > 4) finish_rows<BF16, 16>(a);
        else finish_rows<BF16, 1>(a);
    } else if ((int)blockIdx.x < a.row_blocks + a.w_blocks) finish_weights<WL>(a);
    else mean_loss(a.losses, a.loss_rows, a.meta->count, a.loss);
}

// ---- plan ---------------------------------------------------------------------------------------

struct Layout {
    int kp, cp, terms;              // padded widths; terms of a feature
    int h_rows, w_rows, g_rows;     // rows of a block of 32 columns of the features, the weights and G
    int piece_rows, piece_cols;     // a block of G
    int row_pieces, col_pieces;
    RowSlabs row_slabs;             // dH: classes of a piece dealt to slabs
    int w_slabs;                    // dW: rows of a piece dealt to slabs
    bool rows_direct, w_direct;     // the product writes dH, dW itself
    int r_width, w_width, c_width;  // features of a tile of dH, of dW, classes of the latter
    bool one_tile;                  // all classes are in one tile of logits
    int loss_rows;                  // rows of a partial sum of the losses
    int list_step, list_blocks;
    size_t meta, counts, rows, top, shift, hp, wp, y, sums, at_label, norm, losses, g, dh, dw, bytes;
};

int64_t up(int64_t x, int64_t to) { return ceil_div(x, to) * to; }
int64_t between(int64_t lo, int64_t x, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

Layout plan(int dtype, int64_t n, int32_t k, int32_t c, bool gradients)
{
    Layout l;
    l.terms = dtype == MIXGCN_BF16 ? 1 : 2;
    // tiles of 64 features where they are a quarter less than tiles of 128 (k up to 64, 129 to 192)
    l.kp = (int)(4 * up(k, 64) <= 3 * up(k, 128) ? up(k, 64) : up(k, 128));
    l.cp = (int)up(c, kTile);
    // G, four bytes a logit, is handed on in blocks of at most 2^26 logits, of 8192 classes and as many rows (us of
    // 16384 x 512 -> 50001 bf16 and 72640 x 32 -> 8123 fp32, 2^24, 2^25, 2^26, 2^27: 8090 7080 6780 7400, 2270 1790
    // 1610 1740; of 30000 x 200 -> 20000 bf16 with 4096 rows of 16384 classes 3490, 8192 of 8192 3150).  Where twice
    // the rows are all of them they are one block (in two blocks 16384 x 256 -> 50001 fp32 5440 -> 5550 us, 9000 x 64
    // -> 60000 bf16 1510 -> 1670; 100000 x 64 -> 1000 fp32 would gain, 444 -> 394); of many features, whose sums of
    // dH each block of classes reads and writes, where 5/4 of them are (in two blocks 16384 x 512 -> 50001 bf16 7350
    // -> 6920, 12000 x 384 -> 20001 fp32 2670 -> 2580, but 9000 x 512 -> 20001 bf16 1690 -> 1770).
    const int64_t most = (int64_t)1 << 26, all_rows = up(n > 0 ? n : 1, kMostTileRows);
    int64_t cols = between(kTile, l.cp, 8192);
    // (2^18 rows at most, and 2^32 cells of dH: a launch has less than 2^32 threads)
    const int64_t most_rows = between(kMostTileRows, ((int64_t)1 << 32) / l.kp / kMostTileRows * kMostTileRows, (int64_t)1 << 18);
    int64_t rows = between(kMostTileRows, most / cols / kMostTileRows * kMostTileRows, most_rows);
    l.one_tile = l.cp <= 2 * kTile;
    if (all_rows <= (l.kp <= 256 ? 2 * rows : rows + rows / 4) && !l.one_tile) rows = all_rows;
    if (all_rows < rows) rows = all_rows;
    cols = between(kTile, most / rows / kTile * kTile, l.cp);
    l.piece_rows = (int)rows;
    l.piece_cols = (int)cols;
    // (two more: blocks a power of two apart would begin in the same channel of the L2)
    l.h_rows = l.g_rows = (int)rows + 2;
    l.w_rows = l.cp + 2;
    l.row_pieces = (int)ceil_div(all_rows, rows);
    l.col_pieces = (int)ceil_div(l.cp, cols);
    l.r_width = l.kp % 128 ? 64 : 128;
    // dW: up to 192 classes in one tile (262144 x 128 -> 172 fp32 398 -> 379 us, -> 47 bf16 198 -> 177)
    l.c_width = l.one_tile && c <= 192 ? (int)up(c, 64) : kTile;
    // tiles of 256 features where the rows make slabs long (2000 x 256 -> 5000 bf16 with them 128 us, without 115; 30000 x 256 -> 2000
    // 385, 392)
    l.w_width = l.kp % 128 ? 64 : l.terms == 1 && l.kp % 256 == 0 && n > 2048 && l.c_width <= kTile ? 256 : 128;
    // a workgroup of either gradient for every compute unit
    const int64_t col_tiles = cols / kTile, row_tiles = ceil_div(rows, kGradRows);
    const int64_t s = between(1, 256 / (l.kp / l.r_width * row_tiles), col_tiles);
    const int planned = (int)ceil_div(col_tiles, ceil_div(col_tiles, s));
    l.w_slabs = (int)between(1, 256 / (l.kp / l.w_width * (l.one_tile ? ceil_div(c, l.c_width) : col_tiles)), rows / kTile);
    l.rows_direct = planned == 1 && l.col_pieces == 1;
    l.row_slabs = {l.kp / l.r_width, kGradRows, (int)cols, l.rows_direct ? 0 : planned, (int)rows};
    l.w_direct = l.w_slabs == 1 && l.row_pieces == 1;
    l.loss_rows = l.one_tile ? 64 : rows <= 4096 ? 4 : 16;
    // (few rows: more lanes to each.  us with 4 and 16 rows to a block: 100 x 64 -> 60000 fp32 41 46, 96 x 256 ->
    // 32000 bf16 with gradients 86 88, 1000 x 64 -> 5000 27 26, 4096 x 64 -> 5000 40 34; 6000 x 64 -> 5000 47 42,
    // 10007 x 256 -> 5003 bf16 81 76)
    l.list_step = (int)between(kListStep, up(ceil_div(n, 2048), kListStep), (int64_t)1 << 30);
    l.list_blocks = (int)(n > 0 ? ceil_div(n, l.list_step) : 1);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    l.meta = take(sizeof(Meta));
    l.counts = take((size_t)l.list_blocks * 4);
    l.rows = take((size_t)n * 4);
    l.top = take((size_t)l.kp * 8);
    l.shift = take((size_t)l.kp * 8);
    l.hp = take((size_t)l.terms * l.h_rows * l.kp * 2);
    l.wp = take((size_t)2 * l.kp * l.w_rows * 2);
    l.y = take((size_t)rows * 4);
    l.sums = take(l.one_tile ? 0 : (size_t)(l.cp / kHalfTile) * rows * 8);
    l.at_label = take(l.one_tile ? 0 : (size_t)rows * 4);
    l.norm = take(l.one_tile ? 0 : (size_t)rows * 8);
    l.losses = take((size_t)(ceil_div(n, l.loss_rows) + 1) * 8);
    l.g = l.dh = l.dw = 0;
    if (gradients) {
        l.g = take((size_t)2 * l.g_rows * cols * 2);
        l.dh = take(l.rows_direct ? 0 : (size_t)planned * rows * l.kp * 4);
        l.dw = take(l.w_direct ? 0 : (size_t)l.w_slabs * l.kp * cols * 4);
    }
    l.bytes = at;
    return l;
}

unsigned grid_for(int64_t items) { return (unsigned)between(1, ceil_div(items, kBlock), 8192); }

}  // namespace

int64_t linear_xent_bytes(int dtype, int64_t n, int32_t k, int32_t c, bool gradients)
{
    return (int64_t)plan(dtype, n, k, c, gradients).bytes;
}

int launch_linear_xent(int dtype, const void* H, int64_t ldh, const float* W, int64_t ldw, const int32_t* labels, int64_t n,
                       int32_t k, int32_t c, double* loss, float* row_loss, void* dH, int64_t ldd, float* dW, int64_t ldg,
                       void* workspace, hipStream_t s)
{
    const bool bf16 = dtype == MIXGCN_BF16, grads = dH || dW;
    const Layout l = plan(dtype, n, k, c, grads);
    char* const ws = (char*)workspace;
    Meta* const meta = (Meta*)(ws + l.meta);
    uint32_t* const counts = (uint32_t*)(ws + l.counts);
    uint32_t* const rows = (uint32_t*)(ws + l.rows);
    uint32_t* const top = (uint32_t*)(ws + l.top);
    int32_t* const shift = (int32_t*)(ws + l.shift);
    uint16_t* const hp = (uint16_t*)(ws + l.hp);
    uint16_t* const wp = (uint16_t*)(ws + l.wp);
    int32_t* const y = (int32_t*)(ws + l.y);
    float2* const sums = (float2*)(ws + l.sums);
    float* const at_label = (float*)(ws + l.at_label);
    float2* const norm = (float2*)(ws + l.norm);
    double* const losses = (double*)(ws + l.losses);
    uint16_t* const g = (uint16_t*)(ws + l.g);
    float* const dhp = (float*)(ws + l.dh);
    float* const dwp = (float*)(ws + l.dw);
#define MIXGCN_RUN(KERNEL, GRID, ...) hipLaunchKernelGGL((KERNEL), dim3((unsigned)(GRID)), dim3(kBlock), 0, s, __VA_ARGS__)
#define MIXGCN_RUN_T(KERNEL, GRID, ...)                         \
    do {                                                        \
        if (bf16) MIXGCN_RUN(KERNEL<true>, GRID, __VA_ARGS__);  \
        else MIXGCN_RUN(KERNEL<false>, GRID, __VA_ARGS__);      \
    } while (0)
#define MIXGCN_RUN_T2(KERNEL, W, GRID, ...)                         \
    do {                                                            \
        if (bf16) MIXGCN_RUN((KERNEL<true, W>), GRID, __VA_ARGS__); \
        else MIXGCN_RUN((KERNEL<false, W>), GRID, __VA_ARGS__);     \
    } while (0)
    TopPlan tp;
    tp.list_blocks = l.list_blocks;
    tp.list_step = l.list_step;
    tp.w_pieces = (int)ceil_div(c, kTopCols);
    tp.w_blocks = tp.w_pieces * k;
    // (the blocks' atomics meet in a few lines: 262144 x 128 -> 172 fp32, a tenth labelled, over one input again and
    // again, 97 us with 1024 blocks, 94 with 512, 101 with 256; with 1024, 2048 or 4096 blocks to clear 105, 104,
    // 104)
    tp.h_rows = (int)between(64, ceil_div(n, 512), (int64_t)1 << 30);
    tp.h_blocks = (int)between(1, ceil_div(n, tp.h_rows), 512);
    tp.clear_blocks = row_loss || dH ? (int)between(0, ceil_div(n * (dH ? (k + 7) / 8 : 1), 4 * kBlock), 2048) : 0;
    tp.alone = tp.list_blocks == 1 && tp.w_pieces == 1 && tp.h_blocks == 1;
    if (!tp.alone) MIXGCN_RUN(count_labels_kernel, l.list_blocks, labels, n, c, l.list_step, counts, top, 2 * l.kp);
    MIXGCN_RUN_T(top_kernel, tp.list_blocks + tp.w_blocks + tp.h_blocks + tp.clear_blocks, H, ldh, counts, rows, meta, W, ldw, k, c,
                 l.kp, tp, top, labels, n, dH, ldd, row_loss);
    const int nk = (int)ceil_div(k, BK), class_tiles = l.cp / kTile, pr = l.piece_rows;
    const int pieces = l.cp / kHalfTile;
    // rows of a tile of logits: as many as the registers hold for bf16 features, whose one plane is read from LDS for two planes
    // of weights; 64, with more steps on their way, where they do not fill one or that leaves 128 tiles or less for the compute units
    // (373 x 512 -> 381 bf16 78 -> 57 us, 300 x 100 -> 5000 fp32 54 -> 51; up to 256 tiles 10007 x 256 -> 600 bf16 95 either way)
    const int logit_rows = n <= 128 || (int64_t)class_tiles * ceil_div(n, bf16 ? 256 : 128) <= 128 ? 64 : bf16 ? 256 : 128;
#define MIXGCN_LOGITS(KERNEL, CLASS_TILES, ...)                                                         \
    do {                                                                                                \
        const int64_t grid = (int64_t)(CLASS_TILES) * (pr / logit_rows);                                \
        if (bf16 && logit_rows == 64) MIXGCN_RUN((KERNEL<1, 1>), grid, __VA_ARGS__);                    \
        else if (bf16) MIXGCN_RUN((KERNEL<1, 4>), grid, __VA_ARGS__);                                   \
        else if (logit_rows == 64) MIXGCN_RUN((KERNEL<2, 1>), grid, __VA_ARGS__);                       \
        else MIXGCN_RUN((KERNEL<2, 2>), grid, __VA_ARGS__);                                             \
    } while (0)
    for (int rp = 0; rp < l.row_pieces; ++rp) {
        const uint32_t first = (uint32_t)rp * (uint32_t)pr;
        const int w_blocks = rp == 0 ? (int)grid_for((int64_t)l.kp / BK * l.cp) : 0;
        MIXGCN_RUN_T(split_kernel, w_blocks + grid_for((int64_t)pr * l.kp / 8), H, ldh, rows, labels, meta, first, pr, l.h_rows, k,
                     l.kp, top, shift, hp, y, w_blocks, W, ldw, c, l.cp, l.w_rows, wp);
        if (l.one_tile) {
            // rows of a tile: what two workgroups of a compute unit have registers and LDS for
#define MIXGCN_ROWS(TH, TM, TN)                                                                                                          \
    MIXGCN_RUN((logit_rows_kernel<TH, TM, TN>), pr / (64 * TN), wp, l.kp, l.w_rows, c, nk, hp, l.h_rows, y, meta, first, pr, rows, losses, \
               row_loss, l.g_rows, l.cp, grads ? g : nullptr)
            // rows of a tile likewise (40000 x 100 -> 47 bf16 with 128 tiles 65 us, with 256 62)
            const int tm = (int)ceil_div(c, 64);
            const bool few = ceil_div(n, tm == 1 || (tm == 2 && bf16) ? 256 : 128) <= 256;
            switch (tm) {
            case 1:
                if (bf16 && few) MIXGCN_ROWS(1, 1, 1);
                else if (bf16) MIXGCN_ROWS(1, 1, 4);
                else if (few) MIXGCN_ROWS(2, 1, 1);
                else MIXGCN_ROWS(2, 1, 4);
                break;
            case 2:
                if (bf16 && few) MIXGCN_ROWS(1, 2, 1);
                else if (bf16) MIXGCN_ROWS(1, 2, 4);
                else if (few) MIXGCN_ROWS(2, 2, 1);
                else MIXGCN_ROWS(2, 2, 2);
                break;
            case 3:
                if (bf16 && few) MIXGCN_ROWS(1, 3, 1);
                else if (bf16) MIXGCN_ROWS(1, 3, 2);
                else if (few) MIXGCN_ROWS(2, 3, 1);
                else MIXGCN_ROWS(2, 3, 2);
                break;
            default:
                if (bf16 && few) MIXGCN_ROWS(1, 4, 1);
                else if (bf16) MIXGCN_ROWS(1, 4, 2);
                else MIXGCN_ROWS(2, 4, 1);
            }
#undef MIXGCN_ROWS
        } else {
            MIXGCN_LOGITS(logit_sums_kernel, class_tiles, wp, l.kp, l.w_rows, c, nk, hp, l.h_rows, y, meta, first, pr, class_tiles, sums,
                          at_label);
            if (l.loss_rows == 4)
                MIXGCN_RUN(join_sums_kernel<4>, pr / 4, sums, pieces, at_label, meta, first, pr, rows, norm, losses, row_loss);
            else
                MIXGCN_RUN(join_sums_kernel<16>, pr / 16, sums, pieces, at_label, meta, first, pr, rows, norm, losses, row_loss);
        }
        for (int q = 0; grads && q < l.col_pieces; ++q) {
            const int col0 = q * l.piece_cols;
            const int pc = l.cp - col0 < l.piece_cols ? l.cp - col0 : l.piece_cols, ct = pc / kTile;
            if (!l.one_tile)
                MIXGCN_LOGITS(logit_grad_kernel, ct, wp, l.kp, l.w_rows, c, nk, hp, l.h_rows, y, norm, meta, first, pr, col0, l.g_rows, ct, g);
            Gradients ga = {g, hp, wp, l.kp, l.h_rows, l.w_rows, l.g_rows, meta, first, pr, pc, col0, 0, l.row_slabs,
                            q > 0, dhp, l.w_slabs, (int)(l.one_tile ? ceil_div(c, l.c_width) : ct), dwp, nullptr, ldg, k, c, shift, nullptr, ldd, rows};
            if (l.w_direct) ga.dW = dW;
            if (l.rows_direct) ga.dH = dH;
            // (256 at least: fewer rows with a label have more slabs)
            if (dH) ga.row_blocks = (int)between(256, (int64_t)l.row_slabs.tiles * l.row_slabs.slabs(pr) * l.row_slabs.row_tiles(pr), 0x7FFFFFFF);
            const int64_t grid = ga.row_blocks + (dW ? (int64_t)(l.kp / l.w_width) * ga.class_tiles * l.w_slabs : 0);
#define MIXGCN_GRADIENTS(T, TN, TM)                                             \
    do {                                                                        \
        if (l.c_width == 64) MIXGCN_RUN((gradients_kernel<T, TN, TM, 1>), grid, ga);       \
        else if (l.c_width == 128) MIXGCN_RUN((gradients_kernel<T, TN, TM, 2>), grid, ga); \
        else MIXGCN_RUN((gradients_kernel<T, TN, TM == 4 ? 2 : TM, 3>), grid, ga); \
    } while (0)
            if (bf16 && l.w_width == 256) MIXGCN_GRADIENTS(1, 2, 4);
            else if (bf16 && l.w_width == 128) MIXGCN_GRADIENTS(1, 2, 2);
            else if (bf16) MIXGCN_GRADIENTS(1, 1, 1);
            else if (l.w_width == 128) MIXGCN_GRADIENTS(2, 2, 2);
            else MIXGCN_GRADIENTS(2, 1, 1);
#undef MIXGCN_GRADIENTS

            const bool last = q == l.col_pieces - 1, mean = loss && last && rp == l.row_pieces - 1;
            Finish fa = {dhp, 0, pr, l.row_slabs, rows, dH, ldd, dwp, 0, l.w_slabs, pc, c - col0 < pc ? c - col0 : pc, rp > 0, dW ? dW + col0 : nullptr, ldg,
                         k, l.kp, shift, meta, first, losses, l.loss_rows, loss};
            const bool w16 = l.w_slabs > 4;
            if (dH && last && !l.rows_direct) {
                const int64_t cells = (int64_t)pr * ceil_div(k, 4);
                fa.row_blocks = (int)between(between(1, ceil_div(cells, kBlock / 16), 2048), ceil_div(cells, kBlock), 0x7FFFFFFF);
            }
            if (dW && !l.w_direct) fa.w_blocks = (int)ceil_div((int64_t)k * ceil_div(fa.cols, 4), w16 ? kBlock / 16 : kBlock);
            const int64_t blocks = (int64_t)fa.row_blocks + fa.w_blocks + (mean ? 1 : 0);
            if (blocks > 0) {
                if (w16) MIXGCN_RUN_T2(finish_kernel, 16, blocks, fa);
                else MIXGCN_RUN_T2(finish_kernel, 1, blocks, fa);
            }
        }
    }
    if (loss && !grads) MIXGCN_RUN(mean_loss_kernel, 1, losses, l.loss_rows, meta, loss);
#undef MIXGCN_LOGITS
#undef MIXGCN_RUN_T2
#undef MIXGCN_RUN_T
#undef MIXGCN_RUN
    MIXGCN_HIP_TRY(hipGetLastError());
    return MIXGCN_OK;
}

}  // namespace mixgcn
