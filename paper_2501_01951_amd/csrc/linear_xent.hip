// Mean softmax cross-entropy of a linear last layer over many classes, without its logits, with its gradients:
//     S = H W,  lse_r = log sum_c exp S_rc,  loss = 1/N sum_r (lse_r - S_r,y_r),
//     G = (exp(S - lse) - onehot) / N,  dH = G W^T,  dW = H^T G,
// over the N rows that have a label.  The classes are walked in tiles: a first pass keeps the largest logit of a row and
// the sum of exponentials of every 64 classes (a row's are joined afterwards), a second one computes the logits again,
// now with the row's sum known, and hands G on a piece of the classes at a time.
//
// Arithmetic.  The products run on the f16 matrix cores with fp32 sums.  An fp32 number enters as two f16 terms, the
// rounded number and the rounded rest, 22 bits and more together; a bf16 one as one.  Of the products of two terms each
// the one of both rests, below 2^-22, is left out.  f16 has a narrow range, so operands are scaled by powers of two,
// which is exact: feature k by one factor in H and another in W, chosen from the largest magnitudes h_k of its column
// and w_k of its row such that the largest h_k w_k of all features comes to 2^28 at least, 2^14 from either side, and a
// feature whose h_k w_k is smaller by 2^d has both sides smaller by 2^(d / 2).  f16 numbers reach down to 2^-24 and a
// pair of terms resolves 2^-25: an element keeps its 22 bits down to 2^-17 of its column's largest where d is 0, and is off by
// 2^-39 of it below that.  G (between -1 and 1 before the division by N) is taken times 2^15.
#include <type_traits>

#include "gemm_common.h"
#include "internal.h"

namespace mixgcn {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx2v __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
typedef __attribute__((address_space(3))) uintx4 lds_uintx4;

constexpr int kTile = 128;        // rows, classes and features of a tile
constexpr int kHalfTile = 64;     // classes of a partial sum: what a wavefront holds
constexpr int BK = 32;            // reduction depth of a step
constexpr int kListRows = 4096;   // labels of a block of the list kernels
constexpr float kGradScale = 32768.f;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// What every kernel of a call shares, in the workspace.
struct Meta {
    uint32_t count;  // rows that have a label
    float alpha;     // logit = alpha * sum of the scaled products
};

// ---- the list of rows with a label --------------------------------------------------------------

__device__ inline bool has_label(int32_t y, int32_t c) { return (uint32_t)y < (uint32_t)c; }

__global__ __launch_bounds__(kBlock) void count_labels_kernel(const int32_t* __restrict__ labels, int64_t n, int32_t c,
                                                              uint32_t* __restrict__ counts)
{
    __shared__ uint32_t part[kBlock / kWave];
    const int64_t r0 = (int64_t)blockIdx.x * kListRows;
    uint32_t mine = 0;
    for (int i = threadIdx.x; i < kListRows; i += kBlock)
        if (r0 + i < n && has_label(labels[r0 + i], c)) ++mine;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, kWave);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    if (threadIdx.x == 0) counts[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

// rows[i]: the i-th row with a label.  Clears the maxima of the features, too.
__global__ __launch_bounds__(kBlock) void list_labels_kernel(const int32_t* __restrict__ labels, int64_t n, int32_t c,
                                                             const uint32_t* __restrict__ counts, uint32_t* __restrict__ rows,
                                                             Meta* __restrict__ meta, uint32_t* __restrict__ top, int n_top)
{
    __shared__ uint64_t lds[4];
    const int tid = threadIdx.x;
    uint64_t before = 0;
    for (unsigned b = tid; b < blockIdx.x; b += kBlock) before += counts[b];
    uint64_t base;
    block_exclusive_scan_u64(before, &base, lds);
    constexpr int PER = kListRows / kBlock;
    const int64_t r0 = (int64_t)blockIdx.x * kListRows + tid * PER;
    uint32_t have = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (r0 + i < n && has_label(labels[r0 + i], c)) have |= 1u << i;
    uint64_t total;
    uint64_t at = base + block_exclusive_scan_u64(__popc(have), &total, lds);
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (have >> i & 1u) rows[at++] = (uint32_t)(r0 + i);
    if (blockIdx.x == gridDim.x - 1 && tid == 0) meta->count = (uint32_t)(base + total);
    if (blockIdx.x == 0)
        for (int i = tid; i < n_top; i += kBlock) top[i] = 0u;
}

// ---- scales -------------------------------------------------------------------------------------

template <bool BF16>
__device__ inline float feature(const void* p, int64_t i)
{
    return BF16 ? __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16) : ((const float*)p)[i];
}
// magnitude as an integer, 0 of what is not finite
__device__ inline uint32_t magnitude(float x)
{
    const uint32_t m = __float_as_uint(x) & 0x7FFFFFFFu;
    return m < 0x7F800000u ? m : 0u;
}

constexpr int kMaxCols = 4096;    // columns of a row of W per block

// top[k]: largest magnitude of column k of H over the rows with a label; top[kp + k]: of row k of W.  (Maxima do not
// depend on the order of the atomics.)
template <bool BF16>
__global__ __launch_bounds__(kBlock) void top_kernel(const void* __restrict__ H, int64_t ldh,
                                                     const uint32_t* __restrict__ rows, const Meta* __restrict__ meta,
                                                     const float* __restrict__ W, int64_t ldw, int k, int c, int kp,
                                                     int w_blocks, int w_pieces, int h_rows, uint32_t* __restrict__ top)
{
    if ((int)blockIdx.x < w_blocks) {
        const int row = blockIdx.x / w_pieces, c0 = (int)(blockIdx.x % w_pieces) * kMaxCols;
        const int c1 = c - c0 < kMaxCols ? c : c0 + kMaxCols;
        uint32_t m = 0;
        for (int j = c0 + threadIdx.x; j < c1; j += kBlock) {
            const uint32_t t = magnitude(W[(int64_t)row * ldw + j]);
            m = t > m ? t : m;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint32_t t = __shfl_xor(m, o, kWave);
            m = t > m ? t : m;
        }
        if ((threadIdx.x & 63) == 0) atomicMax(top + kp + row, m);
        return;
    }
    const uint32_t count = meta->count;
    const uint32_t i0 = (blockIdx.x - w_blocks) * (uint32_t)h_rows;
    if (i0 >= count) return;
    const int m_rows = count - i0 < (uint32_t)h_rows ? (int)(count - i0) : h_rows;
    for (int j = threadIdx.x; j < k; j += kBlock) {
        uint32_t m = 0;
        for (int i = 0; i < m_rows; ++i) {
            const uint32_t t = magnitude(feature<BF16>(H, (int64_t)rows[i0 + i] * ldh + j));
            m = t > m ? t : m;
        }
        atomicMax(top + j, m);
    }
}

__device__ inline int exponent_of(uint32_t bits)
{
    int e;
    frexpf(__uint_as_float(bits), &e);
    return e - 1;
}

// shift[k], shift[kp + k]: powers of two that feature k is taken times in H and in W.
__global__ __launch_bounds__(kBlock) void scale_kernel(const uint32_t* __restrict__ top, int k, int kp,
                                                       int32_t* __restrict__ shift, Meta* __restrict__ meta)
{
    __shared__ int most_of[kBlock / kWave];
    int most = -1000;
    for (int i = threadIdx.x; i < k; i += kBlock)
        if (top[i] && top[kp + i]) {
            const int e = exponent_of(top[i]) + exponent_of(top[kp + i]);
            most = e > most ? e : most;
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
    if (most == -1000) most = 28;      // all products are zero
    if (most > 155) most = 155;        // larger logits are not finite: alpha is
    for (int i = threadIdx.x; i < kp; i += kBlock) {
        int sh = 0, sw = 0;
        const bool h = i < k && top[i], w = i < k && top[kp + i];
        if (h && w) {
            const int eh = exponent_of(top[i]), ew = exponent_of(top[kp + i]);
            const int both = eh + ew - most, half = both >> 1;
            sh = 14 + half - eh;
            sw = 14 + (both - half) - ew;
        } else if (h) {
            sh = 14 - exponent_of(top[i]);
        } else if (w) {
            sw = 14 - exponent_of(top[kp + i]);
        }
        shift[i] = sh;
        shift[kp + i] = sw;
    }
    if (threadIdx.x == 0) meta->alpha = ldexpf(1.f, most - 28);
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
// the rest of x after its first term; none where that is not finite
__device__ inline float rest_of(float x, float t)
{
    const float r = x - t;
    return fabsf(t) <= 65504.f ? r : 0.f;
}

// planes[t][i][kp]: the scaled features of the listed rows [first, first + rows of the piece), zeros past the last one
// up to a whole tile and past the features.  y[i]: their labels, -1 past the last one.
template <bool BF16>
__global__ __launch_bounds__(kBlock) void split_rows_kernel(const void* __restrict__ H, int64_t ldh,
                                                            const uint32_t* __restrict__ rows,
                                                            const int32_t* __restrict__ labels,
                                                            const Meta* __restrict__ meta, uint32_t first, int piece_rows,
                                                            int k, int kp, const int32_t* __restrict__ shift,
                                                            uint16_t* __restrict__ planes, int32_t* __restrict__ y)
{
    const uint32_t count = meta->count;
    if (first >= count) return;
    const int live = count - first < (uint32_t)piece_rows ? (int)(count - first) : piece_rows;
    const int end = (live + kTile - 1) / kTile * kTile;
    const int per_row = kp / 8;
    const int64_t items = (int64_t)end * per_row;
    const size_t plane = (size_t)piece_rows * kp;
    for (int64_t it = (int64_t)blockIdx.x * kBlock + threadIdx.x; it < items; it += (int64_t)gridDim.x * kBlock) {
        const int i = (int)(it / per_row), j = (int)(it % per_row) * 8;
        const bool in = i < live;
        const uint32_t r = in ? rows[first + i] : 0u;
        if (j == 0) y[i] = in ? labels[r] : -1;
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float x[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int col = j + 2 * q + b;
                x[b] = in && col < k ? ldexpf(feature<BF16>(H, (int64_t)r * ldh + col), shift[col]) : 0.f;
            }
            hi[q] = pack_f16(x[0], x[1]);
            lo[q] = pack_f16(rest_of(x[0], low_f16(hi[q])), rest_of(x[1], high_f16(hi[q])));
        }
        uint16_t* const o = planes + (size_t)i * kp + j;
        *reinterpret_cast<uint4*>(o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        if (!BF16) *reinterpret_cast<uint4*>(o + plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}

// planes[t][k][cp]: the two terms of the scaled weights, zeros past them.
__global__ __launch_bounds__(kBlock) void split_weights_kernel(const float* __restrict__ W, int64_t ldw, int k, int c,
                                                               int kp, int cp, const int32_t* __restrict__ shift,
                                                               uint16_t* __restrict__ planes)
{
    const int per_row = cp / 8;
    const int64_t items = (int64_t)kp * per_row;
    const size_t plane = (size_t)kp * cp;
    for (int64_t it = (int64_t)blockIdx.x * kBlock + threadIdx.x; it < items; it += (int64_t)gridDim.x * kBlock) {
        const int i = (int)(it / per_row), j = (int)(it % per_row) * 8;
        const int s = shift[kp + i];
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float x[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int col = j + 2 * q + b;
                x[b] = i < k && col < c ? ldexpf(W[(int64_t)i * ldw + col], s) : 0.f;
            }
            hi[q] = pack_f16(x[0], x[1]);
            lo[q] = pack_f16(rest_of(x[0], low_f16(hi[q])), rest_of(x[1], high_f16(hi[q])));
        }
        uint16_t* const o = planes + (size_t)i * cp + j;
        *reinterpret_cast<uint4*>(o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(o + plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}

// ---- a tile of a product ------------------------------------------------------------------------
// 128 x 128 sums of A[i][k] B[k][j] on four wavefronts of 64 x 64, the operands as planes of f16 terms in memory that
// holds whole tiles.  An operand lies either with the reduction index contiguous (rows of its free index) or, TR, with
// the free index contiguous (rows of the reduction index); the transposing LDS read turns the latter: lane i of 16
// receives element i % 4 of the 8 bytes that lanes i / 4, + 4, + 8 and + 12 address.
struct Operand {
    const uint16_t* p;  // first term of the tile's first element
    int64_t ld;         // halfwords from row to row
    size_t plane;       // halfwords from term to term
};

template <int TA, int TB, bool TRA, bool TRB>
struct Product {
    static constexpr int PITCH_N = BK + 8;      // 80 bytes: 16 rows of 16 bytes hit all banks
    static constexpr int PITCH_T = kTile + 32;  // 320 bytes: four rows of 64 bytes, too
    static constexpr int PLANE = kTile * PITCH_N;
    static_assert(PLANE == BK * PITCH_T, "both layouts take the same room");
    static constexpr int BUFFER = (TA + TB) * PLANE;   // halfwords
    static constexpr int LDS = 2 * BUFFER;

    template <bool TR>
    static __device__ inline int64_t source(int64_t ld, int piece)
    {
        return TR ? (int64_t)(piece / 16) * ld + 8 * (piece % 16) : (int64_t)(piece / 4) * ld + 8 * (piece % 4);
    }
    template <bool TR>
    static __device__ inline int place(int piece)
    {
        return TR ? (piece / 16) * PITCH_T + 8 * (piece % 16) : (piece / 4) * PITCH_N + 8 * (piece % 4);
    }
    template <bool TR>
    static __device__ inline half8 fragment(const uint16_t* t, int free0, int kc, int lane)
    {
        half8 o;
        if (TR) {
            const int grp = lane >> 4, gs = lane & 15;
            const uint16_t* const p = t + (kc + 8 * (grp >> 1) + (gs >> 2)) * PITCH_T + free0 + 16 * (grp & 1) + 4 * (gs & 3);
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)p);
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p + 4 * PITCH_T));
            const shortx8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            __builtin_memcpy(&o, &v, 16);
        } else {
            o = *reinterpret_cast<const half8*>(t + (free0 + (lane & 31)) * PITCH_N + kc + 8 * (lane >> 5));
        }
        return o;
    }

    // Sums over nk steps into acc (which the caller has cleared or filled); ends with a barrier, after which the LDS
    // is the caller's.
    static __device__ inline void run(const Operand& a, const Operand& b, int nk, uint16_t* lds, floatx16 (&acc)[2][2])
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int wm = wave / 2, wn = wave % 2;
        uint4 ra[TA][2], rb[TB][2];
        int64_t oa[2], ob[2];
        int pa[2], pb[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            oa[h] = source<TRA>(a.ld, tid + h * kBlock);
            ob[h] = source<TRB>(b.ld, tid + h * kBlock);
            pa[h] = place<TRA>(tid + h * kBlock);
            pb[h] = place<TRB>(tid + h * kBlock);
        }
        auto load = [&](int step) {
            const int64_t sa = (int64_t)step * (TRA ? BK * a.ld : BK), sb = (int64_t)step * (TRB ? BK * b.ld : BK);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int t = 0; t < TA; ++t) ra[t][h] = *reinterpret_cast<const uint4*>(a.p + t * a.plane + sa + oa[h]);
#pragma unroll
                for (int t = 0; t < TB; ++t) rb[t][h] = *reinterpret_cast<const uint4*>(b.p + t * b.plane + sb + ob[h]);
            }
        };
        auto put = [](uint16_t* p, const uint4& v) {
            const uintx4 q = {v.x, v.y, v.z, v.w};
            *(lds_uintx4*)p = q;
        };
        auto store = [&](uint16_t* buf) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int t = 0; t < TA; ++t) put(buf + t * PLANE + pa[h], ra[t][h]);
#pragma unroll
                for (int t = 0; t < TB; ++t) put(buf + (TA + t) * PLANE + pb[h], rb[t][h]);
            }
        };
        auto mma = [&](const uint16_t* buf) {
#pragma unroll
            for (int kc = 0; kc < BK; kc += 16) {
                half8 fa[TA][2], fb[TB][2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
#pragma unroll
                    for (int t = 0; t < TA; ++t) fa[t][x] = fragment<TRA>(buf + t * PLANE, wm * 64 + x * 32, kc, lane);
#pragma unroll
                    for (int t = 0; t < TB; ++t)
                        fb[t][x] = fragment<TRB>(buf + (TA + t) * PLANE, wn * 64 + x * 32, kc, lane);
                }
                // the smaller products first
#pragma unroll
                for (int q = TA + TB - 2; q >= 0; --q)
#pragma unroll
                    for (int t = 0; t < TA; ++t) {
                        const int u = q - t;
                        if (u < 0 || u >= TB || t + u > 1) continue;
#pragma unroll
                        for (int x = 0; x < 2; ++x)
#pragma unroll
                            for (int y = 0; y < 2; ++y)
                                acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[t][x], fb[u][y], acc[x][y], 0, 0, 0);
                    }
            }
        };
        if (nk > 0) {
            load(0);
            store(lds);
            __syncthreads();
            for (int i = 0; i < nk; ++i) {
                if (i + 1 < nk) load(i + 1);
                mma(lds + (i & 1) * BUFFER);
                if (i + 1 < nk) store(lds + ((i + 1) & 1) * BUFFER);
                __syncthreads();
            }
        }
    }
};

__device__ inline void clear(floatx16 (&acc)[2][2])
{
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
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
// in the lane, but for one exchange of its halves.  In units of log 2: t = logit * log2(e).

// sums[piece of 64 classes][row] = { largest t, sum of 2^(t - largest) }; at_label[row] = t of the row's label.
template <int TH>
__global__ __launch_bounds__(kBlock, 2) void logit_sums_kernel(const uint16_t* __restrict__ Wp, int kp, int cp, int c, int nk,
                                                               const uint16_t* __restrict__ Hp, const int32_t* __restrict__ y,
                                                               const Meta* __restrict__ meta, uint32_t first, int piece_rows,
                                                               int class_tiles, float2* __restrict__ sums,
                                                               float* __restrict__ at_label)
{
    using P = Product<2, TH, true, false>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS];
    const unsigned lid = xcd_local_index(blockIdx.x, gridDim.x);
    const int c0 = (int)(lid % class_tiles) * kTile, r0 = (int)(lid / class_tiles) * kTile;
    if (r0 >= rows_here(meta, first, piece_rows)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
    floatx16 acc[2][2];
    clear(acc);
    P::run({Wp + c0, cp, (size_t)kp * cp}, {Hp + (size_t)r0 * kp, kp, (size_t)piece_rows * kp}, nk, lds, acc);
    const float a2 = meta->alpha * kLog2e;
    const int cw = c0 + wm * 64;
#pragma unroll
    for (int yy = 0; yy < 2; ++yy) {
        const int row = r0 + wn * 64 + yy * 32 + (lane & 31);
        float t[2][16];
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                t[x][v] = cw + x * 32 + tile_row(v, lane) < c ? acc[x][yy][v] * a2 : -INFINITY;
                top = fmaxf(top, t[x][v]);
            }
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v) sum += __builtin_amdgcn_exp2f(t[x][v] - base);
        sum += __shfl_xor(sum, 32, kWave);
        if (lane < 32) sums[(size_t)(cw / kHalfTile) * piece_rows + row] = make_float2(top, sum);
        const int at = y[row] - cw;
        if (__any(at >= 0 && at < kHalfTile)) {
            float mine = 0.f;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (at == x * 32 + tile_row(v, lane)) mine = t[x][v];
            if (at >= 0 && at < kHalfTile && ((at >> 2) & 1) == (lane >> 5)) at_label[row] = mine;
        }
    }
}

// A row's largest t and what its exponentials are taken times for G, from the sums of its pieces; the loss of the row.
__global__ __launch_bounds__(kBlock) void join_sums_kernel(const float2* __restrict__ sums, int pieces,
                                                           const float* __restrict__ at_label,
                                                           const Meta* __restrict__ meta, uint32_t first, int piece_rows,
                                                           const uint32_t* __restrict__ rows, float2* __restrict__ norm,
                                                           float* __restrict__ losses, float* __restrict__ row_loss)
{
    // 16 rows per block, 16 lanes walk the pieces of each
    __shared__ float tops[16][17], parts[16][17];
    const int live = rows_here(meta, first, piece_rows);
    const int j = threadIdx.x % 16, q = threadIdx.x / 16;
    const int row = blockIdx.x * 16 + j;
    if ((int)blockIdx.x * 16 >= live) return;
    const int rr = row < live ? row : live - 1;
    float top = -INFINITY, sum = 0.f;
    bool bad = false;
    for (int p = q; p < pieces; p += 16) {
        const float2 s = sums[(size_t)p * piece_rows + rr];
        bad = bad || !(s.y == s.y);
        if (s.x > top) {
            sum = sum * __builtin_amdgcn_exp2f(top - s.x) + s.y;
            top = s.x;
        } else if (s.x > -INFINITY) {
            sum += s.y * __builtin_amdgcn_exp2f(s.x - top);
        }
    }
    tops[q][j] = top;
    parts[q][j] = bad ? __uint_as_float(0x7FC00000u) : sum;
    __syncthreads();
    if (q == 0 && row < live) {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fmaxf(m, tops[i][j]);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += parts[i][j] * (tops[i][j] > -INFINITY ? __builtin_amdgcn_exp2f(tops[i][j] - m) : 0.f);
        // what is not a number stays one
        if (!(m > -INFINITY)) s = __uint_as_float(0x7FC00000u);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (!(parts[i][j] == parts[i][j])) s = parts[i][j];
        norm[row] = make_float2(m, kGradScale / s);
        const float l = ((m - at_label[row]) + log2f(s)) * kLn2;
        losses[first + row] = l;
        if (row_loss) row_loss[rows[first + row]] = l;
    }
}

// Mean of the losses in a fixed order; 0 without rows.
__global__ __launch_bounds__(1024) void mean_loss_kernel(const float* __restrict__ losses, const Meta* __restrict__ meta,
                                                         double* __restrict__ loss)
{
    __shared__ double sh[1024];
    const uint32_t count = meta->count;
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < count; i += 1024) s += (double)losses[i];
    sh[threadIdx.x] = s;
    __syncthreads();
    for (int o = 512; o > 0; o >>= 1) {
        if ((int)threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) *loss = count ? sh[0] / (double)count : 0.0;
}

// ---- gradient with respect to the logits --------------------------------------------------------
// planes[t][row][piece_cols]: 2^15 (softmax - onehot) of the classes [col0, col0 + piece_cols), zeros past the classes
// and past the rows up to a whole tile.
template <int TH>
__global__ __launch_bounds__(kBlock, 2) void logit_grad_kernel(const uint16_t* __restrict__ Wp, int kp, int cp, int c, int nk,
                                                               const uint16_t* __restrict__ Hp, const int32_t* __restrict__ y,
                                                               const float2* __restrict__ norm,
                                                               const Meta* __restrict__ meta, uint32_t first, int piece_rows,
                                                               int col0, int piece_cols, int class_tiles,
                                                               uint16_t* __restrict__ planes)
{
    using P = Product<2, TH, true, false>;
    constexpr int PITCH = kTile + 8;  // 272 bytes
    constexpr int NEED = kTile * PITCH > P::LDS ? kTile * PITCH : P::LDS;
    __shared__ __attribute__((aligned(16))) uint16_t lds[NEED];
    const unsigned lid = xcd_local_index(blockIdx.x, gridDim.x);
    const int ct = (int)(lid % class_tiles) * kTile, r0 = (int)(lid / class_tiles) * kTile;
    const int live = rows_here(meta, first, piece_rows);
    if (r0 >= live) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / 2, wn = wave % 2;
    floatx16 acc[2][2];
    clear(acc);
    P::run({Wp + col0 + ct, cp, (size_t)kp * cp}, {Hp + (size_t)r0 * kp, kp, (size_t)piece_rows * kp}, nk, lds, acc);
    const float a2 = meta->alpha * kLog2e;
    const int cw = col0 + ct + wm * 64;
    uint2 lo[2][2][4];
#pragma unroll
    for (int yy = 0; yy < 2; ++yy) {
        const int rt = wn * 64 + yy * 32 + (lane & 31), row = r0 + rt;
        const bool in = row < live;
        const float2 nm = in ? norm[row] : make_float2(0.f, 0.f);
        const int at = in ? y[row] - cw : -1;
        const bool mark = __any(at >= 0 && at < kHalfTile);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float g[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int i = x * 32 + tile_row(4 * q + b, lane);
                    g[b] = __builtin_amdgcn_exp2f(fmaf(acc[x][yy][4 * q + b], a2, -nm.x)) * nm.y;
                    if (mark && at == i) g[b] -= kGradScale;
                    if (!in || cw + i >= c) g[b] = 0.f;
                }
                const uint2 hi = make_uint2(pack_f16(g[0], g[1]), pack_f16(g[2], g[3]));
                lo[x][yy][q] = make_uint2(pack_f16(g[0] - low_f16(hi.x), g[1] - high_f16(hi.x)),
                                          pack_f16(g[2] - low_f16(hi.y), g[3] - high_f16(hi.y)));
                *reinterpret_cast<uint2*>(lds + rt * PITCH + wm * 64 + x * 32 + 8 * q + 4 * (lane >> 5)) = hi;
            }
    }
    auto flush = [&](uint16_t* out) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kTile * kTile / 8 / kBlock; ++i) {
            const int p = tid + i * kBlock, r = p / 16, q = p % 16;
            *reinterpret_cast<uint4*>(out + (size_t)(r0 + r) * piece_cols + ct + 8 * q) =
                *reinterpret_cast<const uint4*>(lds + r * PITCH + 8 * q);
        }
        __syncthreads();
    };
    flush(planes);
#pragma unroll
    for (int yy = 0; yy < 2; ++yy)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<uint2*>(lds + (wn * 64 + yy * 32 + (lane & 31)) * PITCH + wm * 64 + x * 32 + 8 * q +
                                          4 * (lane >> 5)) = lo[x][yy][q];
    flush(planes + (size_t)piece_rows * piece_cols);
}

// ---- dH -----------------------------------------------------------------------------------------
// part[slab][row][kp] (+)= G[row][classes of the slab] W'^T
template <int T>
__global__ __launch_bounds__(kBlock, 2) void grad_rows_kernel(const uint16_t* __restrict__ Gp, int piece_cols, int piece_rows,
                                                              const uint16_t* __restrict__ Wp, int kp, int cp, int col0,
                                                              const Meta* __restrict__ meta, uint32_t first, int slab_cols,
                                                              int k_tiles, int slabs, bool add, float* __restrict__ part)
{
    using P = Product<T, T, false, false>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS];
    const unsigned lid = xcd_local_index(blockIdx.x, gridDim.x);
    const int kt = (int)(lid % k_tiles), slab = (int)(lid / k_tiles) % slabs, r0 = (int)(lid / (k_tiles * slabs)) * kTile;
    if (r0 >= rows_here(meta, first, piece_rows)) return;
    const int s0 = slab * slab_cols;
    const int s1 = s0 + slab_cols < piece_cols ? s0 + slab_cols : piece_cols;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
    float* const out = part + ((size_t)slab * piece_rows + r0 + wm * 64) * kp + kt * kTile + wn * 64 + (lane & 31);
    floatx16 acc[2][2];
    clear(acc);
    P::run({Gp + (size_t)r0 * piece_cols + s0, piece_cols, (size_t)piece_rows * piece_cols},
           {Wp + (size_t)kt * kTile * cp + col0 + s0, cp, (size_t)kp * cp}, s1 > s0 ? (s1 - s0) / BK : 0, lds, acc);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                float* const o = out + (size_t)(x * 32 + tile_row(v, lane)) * kp + y * 32;
                *o = add ? *o + acc[x][y][v] : acc[x][y][v];
            }
}

// dH of the listed rows from the slabs' sums.
template <bool BF16>
__global__ __launch_bounds__(kBlock) void finish_rows_kernel(const float* __restrict__ part, int slabs, int piece_rows, int k,
                                                             int kp, const int32_t* __restrict__ shift,
                                                             const Meta* __restrict__ meta, uint32_t first,
                                                             const uint32_t* __restrict__ rows, void* __restrict__ dH,
                                                             int64_t ldd)
{
    const int live = rows_here(meta, first, piece_rows);
    const float inv = 1.f / (float)meta->count;
    const int per_row = (k + 3) / 4;
    const int64_t items = (int64_t)live * per_row;
    const size_t slab = (size_t)piece_rows * kp;
    for (int64_t it = (int64_t)blockIdx.x * kBlock + threadIdx.x; it < items; it += (int64_t)gridDim.x * kBlock) {
        const int i = (int)(it / per_row), j = (int)(it % per_row) * 4;
        const float* const p = part + (size_t)i * kp + j;
        float4 s = *reinterpret_cast<const float4*>(p);
        for (int b = 1; b < slabs; ++b) {
            const float4 t = *reinterpret_cast<const float4*>(p + b * slab);
            s.x += t.x;
            s.y += t.y;
            s.z += t.z;
            s.w += t.w;
        }
        const float v[4] = {s.x, s.y, s.z, s.w};
        float o[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) o[b] = ldexpf(v[b] * inv, -15 - shift[kp + j + b]);
        const int64_t at = (int64_t)rows[first + i] * ldd + j;
        if (BF16) {
            const uint32_t w[2] = {pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
            if (j + 4 <= k) *reinterpret_cast<uint2*>((uint16_t*)dH + at) = make_uint2(w[0], w[1]);
            else
                for (int b = 0; j + b < k; ++b) ((uint16_t*)dH)[at + b] = (uint16_t)(w[b / 2] >> (16 * (b % 2)));
        } else {
            if (j + 4 <= k) *reinterpret_cast<float4*>((float*)dH + at) = make_float4(o[0], o[1], o[2], o[3]);
            else
                for (int b = 0; j + b < k; ++b) ((float*)dH)[at + b] = o[b];
        }
    }
}

// Zeros for the rows without a label: of dH (cols > 0) and of the losses of the rows.
template <bool BF16>
__global__ __launch_bounds__(kBlock) void clear_rows_kernel(const int32_t* __restrict__ labels, int64_t n, int32_t c,
                                                            void* __restrict__ dH, int64_t ldd, int k,
                                                            float* __restrict__ row_loss)
{
    const int per_row = (k + 3) / 4 + (k == 0);
    const int64_t items = n * per_row;
    for (int64_t it = (int64_t)blockIdx.x * kBlock + threadIdx.x; it < items; it += (int64_t)gridDim.x * kBlock) {
        const int64_t r = it / per_row;
        const int j = (int)(it - r * per_row) * 4;
        if (has_label(labels[r], c)) continue;
        if (j == 0 && row_loss) row_loss[r] = 0.f;
        const int64_t at = r * ldd + j;
        if (j + 4 <= k) {
            if (BF16) *reinterpret_cast<uint2*>((uint16_t*)dH + at) = make_uint2(0u, 0u);
            else *reinterpret_cast<float4*>((float*)dH + at) = make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
            for (int b = 0; j + b < k; ++b) {
                if (BF16) ((uint16_t*)dH)[at + b] = 0;
                else ((float*)dH)[at + b] = 0.f;
            }
        }
    }
}

// ---- dW -----------------------------------------------------------------------------------------
// part[slab][kp][piece_cols] = H'^T[rows of the slab] G
template <int TH>
__global__ __launch_bounds__(kBlock, 2) void grad_weights_kernel(const uint16_t* __restrict__ Hp, int kp,
                                                                 const uint16_t* __restrict__ Gp, int piece_cols,
                                                                 int piece_rows, const Meta* __restrict__ meta, uint32_t first,
                                                                 int class_tiles, int k_tiles, int slabs,
                                                                 float* __restrict__ part)
{
    using P = Product<TH, 2, true, true>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[P::LDS];
    const unsigned lid = xcd_local_index(blockIdx.x, gridDim.x);
    const int kt = (int)(lid % k_tiles), ct = (int)(lid / k_tiles) % class_tiles, slab = (int)(lid / (k_tiles * class_tiles));
    const int live = rows_here(meta, first, piece_rows);
    const int per = ((live + slabs - 1) / slabs + BK - 1) / BK * BK;
    const int r0 = slab * per, r1 = r0 + per < live ? r0 + per : live;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
    floatx16 acc[2][2];
    clear(acc);
    P::run({Hp + (size_t)r0 * kp + kt * kTile, kp, (size_t)piece_rows * kp},
           {Gp + (size_t)r0 * piece_cols + ct * kTile, piece_cols, (size_t)piece_rows * piece_cols},
           r1 > r0 ? (r1 - r0 + BK - 1) / BK : 0, lds, acc);
    float* const out = part + ((size_t)slab * kp + kt * kTile + wm * 64) * piece_cols + ct * kTile + wn * 64 + (lane & 31);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                out[(size_t)(x * 32 + tile_row(v, lane)) * piece_cols + y * 32] = acc[x][y][v];
}

// dW[k][classes of the piece] (+)= the slabs' sums, unscaled.
__global__ __launch_bounds__(kBlock) void finish_weights_kernel(const float* __restrict__ part, int slabs, int k, int kp,
                                                                int piece_cols, int cols, const int32_t* __restrict__ shift,
                                                                const Meta* __restrict__ meta, uint32_t first, bool add,
                                                                float* __restrict__ dW, int64_t ldw)
{
    const uint32_t count = meta->count;
    if (add && first >= count) return;
    const float inv = count ? 1.f / (float)count : 0.f;
    const int per_row = (cols + 3) / 4;
    const int64_t items = (int64_t)k * per_row;
    const size_t slab = (size_t)kp * piece_cols;
    for (int64_t it = (int64_t)blockIdx.x * kBlock + threadIdx.x; it < items; it += (int64_t)gridDim.x * kBlock) {
        const int i = (int)(it / per_row), j = (int)(it % per_row) * 4;
        const float* const p = part + (size_t)i * piece_cols + j;
        float4 s = *reinterpret_cast<const float4*>(p);
        for (int b = 1; b < slabs; ++b) {
            const float4 t = *reinterpret_cast<const float4*>(p + b * slab);
            s.x += t.x;
            s.y += t.y;
            s.z += t.z;
            s.w += t.w;
        }
        const float v[4] = {s.x, s.y, s.z, s.w};
        float* const o = dW + (int64_t)i * ldw + j;
        const int e = -15 - shift[i];
        for (int b = 0; b < 4 && j + b < cols; ++b) {
            const float g = ldexpf(v[b] * inv, e);
            o[b] = add ? o[b] + g : g;
        }
    }
}

// ---- plan ---------------------------------------------------------------------------------------

struct Layout {
    int kp, cp, terms;              // padded widths; terms of a feature
    int piece_rows, piece_cols;     // a block of G
    int row_pieces, col_pieces;
    int row_slabs, row_slab_cols;   // dH: classes of a piece dealt to slabs
    int w_slabs;                    // dW: rows of a piece dealt to slabs
    int64_t list_blocks;
    size_t meta, counts, rows, top, shift, hp, wp, y, sums, at_label, norm, losses, g, dh, dw, bytes;
};

int up(int64_t x, int to) { return (int)(ceil_div(x, to) * to); }

Layout plan(int dtype, int64_t n, int32_t k, int32_t c, bool gradients)
{
    Layout l;
    l.terms = dtype == MIXGCN_BF16 ? 1 : 2;
    l.kp = up(k, kTile);
    l.cp = up(c, kTile);
    // G of a block of rows and classes takes at most 128 MB, which the last-level cache holds
    const int64_t most = ((int64_t)128 << 20) / 4;
    const int64_t all_rows = n > 0 ? up(n < (1 << 30) ? n : (1 << 30), kTile) : kTile;
    int64_t rows = most / l.cp / kTile * kTile;
    if (rows < 16384) rows = 16384;
    if (rows > all_rows) rows = all_rows;
    if (rows > 131072) rows = 131072;
    l.piece_rows = (int)rows;
    int64_t cols = most / rows / kTile * kTile;
    if (cols > l.cp) cols = l.cp;
    l.piece_cols = (int)cols;
    l.row_pieces = (int)ceil_div(all_rows, rows);
    l.col_pieces = (int)ceil_div(l.cp, cols);
    const int64_t k_tiles = l.kp / kTile, row_tiles = rows / kTile, col_tiles = cols / kTile;
    // enough workgroups for every compute unit
    int64_t s = 512 / (k_tiles * row_tiles);
    if (s > col_tiles) s = col_tiles;
    if (s < 1) s = 1;
    l.row_slab_cols = (int)(ceil_div(col_tiles, s) * kTile);
    l.row_slabs = (int)ceil_div(cols, l.row_slab_cols);
    s = 512 / (k_tiles * col_tiles);
    if (s > row_tiles) s = row_tiles;
    if (s < 1) s = 1;
    l.w_slabs = (int)s;
    l.list_blocks = ceil_div(n, kListRows);
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
    l.hp = take((size_t)l.terms * rows * l.kp * 2);
    l.wp = take((size_t)2 * l.kp * l.cp * 2);
    l.y = take((size_t)rows * 4);
    l.sums = take((size_t)(l.cp / kHalfTile) * rows * 8);
    l.at_label = take((size_t)rows * 4);
    l.norm = take((size_t)rows * 8);
    l.losses = take((size_t)n * 4);
    l.g = l.dh = l.dw = 0;
    if (gradients) {
        l.g = take((size_t)2 * rows * cols * 2);
        l.dh = take((size_t)l.row_slabs * rows * l.kp * 4);
        l.dw = take((size_t)l.w_slabs * l.kp * cols * 4);
    }
    l.bytes = at;
    return l;
}

unsigned grid_for(int64_t items)
{
    const int64_t g = ceil_div(items, kBlock);
    return (unsigned)(g < 1 ? 1 : g > 8192 ? 8192 : g);
}

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
    float* const losses = (float*)(ws + l.losses);
    uint16_t* const g = (uint16_t*)(ws + l.g);
    float* const dhp = (float*)(ws + l.dh);
    float* const dwp = (float*)(ws + l.dw);
#define MIXGCN_RUN(KERNEL, GRID, ...) hipLaunchKernelGGL(KERNEL, dim3((unsigned)(GRID)), dim3(kBlock), 0, s, __VA_ARGS__)
#define MIXGCN_RUN_T(KERNEL, YES, NO, GRID, ...)              \
    do {                                                      \
        if (bf16) MIXGCN_RUN(KERNEL<YES>, GRID, __VA_ARGS__); \
        else MIXGCN_RUN(KERNEL<NO>, GRID, __VA_ARGS__);       \
    } while (0)
    const unsigned list_grid = (unsigned)(l.list_blocks > 0 ? l.list_blocks : 1);
    if (list_grid > 1) MIXGCN_RUN(count_labels_kernel, list_grid, labels, n, c, counts);
    MIXGCN_RUN(list_labels_kernel, list_grid, labels, n, c, counts, rows, meta, top, 2 * l.kp);
    const int w_pieces = (int)ceil_div(c, kMaxCols), w_blocks = w_pieces * k;
    const int h_rows = n > 65536 ? (int)ceil_div(n, 1024) : 64;
    MIXGCN_RUN_T(top_kernel, true, false, w_blocks + ceil_div(n, h_rows), H, ldh, rows, meta, W, ldw, k, c, l.kp, w_blocks,
                 w_pieces, h_rows, top);
    MIXGCN_RUN(scale_kernel, 1, top, k, l.kp, shift, meta);
    MIXGCN_RUN(split_weights_kernel, grid_for((int64_t)l.kp * l.cp / 8), W, ldw, k, c, l.kp, l.cp, shift, wp);
    if (row_loss || dH) MIXGCN_RUN_T(clear_rows_kernel, true, false, grid_for(n * (dH ? (k + 3) / 4 : 1)), labels, n, c, dH, ldd,
                                     dH ? k : 0, row_loss);
    const int nk = (int)ceil_div(k, BK), k_tiles = l.kp / kTile, class_tiles = l.cp / kTile, row_tiles = l.piece_rows / kTile;
    for (int rp = 0; rp < l.row_pieces; ++rp) {
        const uint32_t first = (uint32_t)rp * (uint32_t)l.piece_rows;
        const int pr = l.piece_rows;
        MIXGCN_RUN_T(split_rows_kernel, true, false, grid_for((int64_t)pr * l.kp / 8), H, ldh, rows, labels, meta, first, pr, k,
                     l.kp, shift, hp, y);
        MIXGCN_RUN_T(logit_sums_kernel, 1, 2, (int64_t)class_tiles * row_tiles, wp, l.kp, l.cp, c, nk, hp, y, meta, first, pr,
                     class_tiles, sums, at_label);
        MIXGCN_RUN(join_sums_kernel, ceil_div(pr, 16), sums, l.cp / kHalfTile, at_label, meta, first, pr, rows, norm, losses,
                   row_loss);
        for (int q = 0; grads && q < l.col_pieces; ++q) {
            const int col0 = q * l.piece_cols;
            const int pc = l.cp - col0 < l.piece_cols ? l.cp - col0 : l.piece_cols, ct = pc / kTile;
            const int cols = c - col0 < pc ? c - col0 : pc;
            MIXGCN_RUN_T(logit_grad_kernel, 1, 2, (int64_t)ct * row_tiles, wp, l.kp, l.cp, c, nk, hp, y, norm, meta, first, pr, col0,
                         pc, ct, g);
            if (dH)
                MIXGCN_RUN_T(grad_rows_kernel, 1, 2, (int64_t)k_tiles * l.row_slabs * row_tiles, g, pc, pr, wp, l.kp, l.cp, col0,
                             meta, first, l.row_slab_cols, k_tiles, l.row_slabs, q > 0, dhp);
            if (dW) {
                MIXGCN_RUN_T(grad_weights_kernel, 1, 2, (int64_t)k_tiles * ct * l.w_slabs, hp, l.kp, g, pc, pr, meta, first, ct,
                             k_tiles, l.w_slabs, dwp);
                MIXGCN_RUN(finish_weights_kernel, grid_for((int64_t)k * ceil_div(cols, 4)), dwp, l.w_slabs, k, l.kp, pc, cols,
                           shift, meta, first, rp > 0, dW + col0, ldg);
            }
        }
        if (dH)
            MIXGCN_RUN_T(finish_rows_kernel, true, false, grid_for((int64_t)pr * ceil_div(k, 4)), dhp, l.row_slabs, pr, k, l.kp,
                         shift, meta, first, rows, dH, ldd);
    }
    if (loss) hipLaunchKernelGGL(mean_loss_kernel, dim3(1), dim3(1024), 0, s, losses, meta, loss);
#undef MIXGCN_RUN_T
#undef MIXGCN_RUN
    MIXGCN_HIP_TRY(hipGetLastError());
    return MIXGCN_OK;
}

}  // namespace mixgcn
