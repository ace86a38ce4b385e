// Orthogonalised updates: a matrix with its singular values brought near 1 by Newton-Schulz products, and the training step
// made of it (momentum, weight decay).
//
// With X the matrix, or its transpose where that has fewer rows: m x n, m <= n, X <- X / (|X|_F + eps), and for every step
//     A = X X^T,   B = b A + c A^2,   X <- a X + B X.
// A step maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors as they are.
//
// All three products are rows times rows (A_ij = x_i . x_j; A is symmetric, so A^2 is rows times rows, too; for B X there is X^T
// beside X), so one kernel does them: fp16 operands of 64 values of k a tile in LDS, fp32 sums on the matrix cores.  Of the symmetric
// ones the tiles on and below the diagonal are computed and stored twice.
//
// Precision.  The polynomial multiplies what a rounding adds to a small singular value by up to a^steps (485 for five of the usual steps), so
// roundings of X to 11 bits alone leave 1e-2 in the result of a gradient whose singular values are spread over two decades, to 8 bits
// (bf16) 8e-2.  Two things take that away at no cost in products: the linear term a X is carried in 22 bits (two
// fp16 numbers, x = high + low), and the diagonals of A and B, which hold most of their size, stay in fp32 outside of the products
// (A = D + F:  A^2 = F^2 + D F + F D + D^2,  B X = E X + H X).  That leaves (HB_TENSOR_BF16) 6e-4 to 9e-4 of the result's norm where
// singular values are spread over two decades, and more the more of them are near 0: all but one at 1e-4 of the largest 4e-4 (520 x 513), 2.4e-3 (134 x 176), of small
// matrices beside a larger one 7e-3 (64 x 512) to 5e-2 (2 x 2).  A result in bf16 is rounded (2^-8 at most, 1.7e-3 of its norm) besides; fp32 weights are not.
// HB_TENSOR_F32 takes the products of high and low parts, too (three products of the four; low times low is 2^-22): the errors are those of fp32 products, about 1e-6,
// and 4e-5 to 1e-4 with all but one singular value at 1e-4 of the largest, as plain fp32 has there.
// Operands are scaled by powers of two so that neither what they hold nor its low part leaves fp16's range: X by 2^12 (entries are at most the largest
// singular value s, 1.2 for the usual steps, and around (m n)^-1/2 at the start), A by 2^8 and B by 2^10 (entries beside the diagonal are at most half
// the range of s^2, and of b s^2 + c s^4): s up to 16 and b s^2 + c s^4 up to 64 have room.
// X is padded with zeros to whole k-tiles, which the steps keep zero, and the workspace has whole tiles: no kernel between the first and the last has a bounds
// check.  What a tile makes of the rows behind the last k-tile is not defined, but stays in such rows: no k gets that far.
#include "gemm_device.h"
#include "operators.h"
#include <math.h>

namespace hb {
namespace {

typedef _Float16 half_t;
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) const void *gptr_t;
typedef __attribute__((address_space(3))) void *lptr_t;

constexpr float SX = 4096.f, SA = 256.f, SB = 1024.f;
constexpr int BK = 64, ROW_BYTES = 2 * BK;  // a row of an operand tile: one cache line
constexpr int SUM_NT = 256, SUM_BLOCKS = 1024, SUM_MIN = 4096;
constexpr int PREP = 64;  // tiles of the kernel that lays X out

// a matrix as the caller has it
struct Matrix {
    int rows, cols;
    bool flip;                // X is its transpose
    // every row begins at a boundary of four elements (of a result in two bytes eight), so that these can be moved at once
    bool whole_g : 1, whole_m : 1, whole_out : 1;
    // ... of four elements, the first row does: what counts where rows follow one another without gaps
    bool begins_g : 1, begins_m : 1, begins_out : 1;
    float scale;              // lr times the matrix's factor
    const void *g;
    void *out;                // the result, or the weights
    float *mom;
    long long ldg, ldo, ldm;
};
// and what is the same for all of them
struct How {
    int g_tensor, out_tensor;  // TENSOR_* of G and of the result
    bool muon, nesterov;
    float momentum, eps, decay;  // decay: lr weight_decay
};
// what the kernels of the products read of it besides, in the workspace
struct Mat : Matrix {
    int m, n, mp, np;         // rows and columns of X in whole k-tiles (zeros behind the last), and pitches: whole tiles
    int sums, sum0;           // blocks of the sum of squares, and the first
    int prep0, sym0, all0;    // first block of the others: X's layout, tiles on and below the diagonal of m x m, tiles of m x n
    size_t x[2], xt[2], f, h; // byte offsets from the workspace: X and X^T (two of each, in turn), A and B; low parts follow
    size_t d, e;              // diagonals of A and B
};
struct List : How {
    int count, planes;
    int syms, splits;          // tiles of the symmetric products, and parts of k in GRAM_PART
    size_t part;               // byte offset of its sums
    Mat mat[ORTHO_GROUP];
};

static_assert(sizeof(List) < 4000, "arguments of a launch");

typedef __bf16 v4b __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

// elements at .. at + 3 of a row of which `left` are there (0 for the others); whole: the four lie at a boundary of their size
__device__ __forceinline__ v4f load_four(const void *p, long long at, int tensor, int left, bool whole)
{
    v4f x = {0.f, 0.f, 0.f, 0.f};
    if (tensor == TENSOR_BF16) {
        const __bf16 *q = static_cast<const __bf16 *>(p) + at;
        if (whole && left >= 4) {
            const v4b u = *reinterpret_cast<const v4b *>(q);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (float)u[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) x[e] = (float)q[e];
        }
    } else {
        const float *q = static_cast<const float *>(p) + at;
        if (whole && left >= 4) {
            x = *reinterpret_cast<const v4f *>(q);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) x[e] = q[e];
        }
    }
    return x;
}

__device__ __forceinline__ void store_four(float *q, const v4f &x, int left, bool whole)
{
    if (whole && left >= 4) {
        *reinterpret_cast<v4f *>(q) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) q[e] = x[e];
    }
}

// the matrix of a block, from the first blocks of each
template <typename F>
__device__ __forceinline__ int find(const List &l, int block, F first)
{
    int k = 0;
    while (k + 1 < l.count && block >= first(l.mat[k + 1])) ++k;
    return k;
}

// what is orthogonalised: G, or with momentum m' = mu m + g (the new one): g + mu m' or m'
__device__ __forceinline__ float updated(const How &l, float g, float m_new)
{
    if (!l.muon) return g;
    return l.nesterov ? __builtin_fmaf(l.momentum, m_new, g) : m_new;
}

// ---------------------------------------------------------------- the norm
// Sums of squares in 64 bits (neither 1e30 nor 1e-30 leaves their range), a fixed part of the rows a block; the momentum on the way.
// A power of two of lanes has a row, four elements each at a time, and loads four times before it waits; a matrix without gaps is one long row.
// The first block puts the list where the other kernels read it: it is longer than what a launch should carry.
// Bound by memory: 45 M elements with momenta (451 MB) in 91 us, 5.0 TB/s; 4096 x 4096 bf16 15 us.
template <int NT>
__device__ __forceinline__ double sum_of_block(const How &l, const Matrix &a, int block, int blocks, double *red)
{
    const bool gaps = a.ldg != a.cols || (l.muon && a.ldm != a.cols);
    const int rows = gaps ? a.rows : 1, cols = gaps ? a.cols : a.rows * a.cols;
    const bool whole_g = gaps ? a.whole_g : a.begins_g, whole_m = gaps ? a.whole_m : a.begins_m;
    int lanes = NT;
    while (lanes > 1 && 2 * lanes >= cols) lanes >>= 1;
    const int per_block = NT / lanes, step = 4 * lanes;
    // one long row goes to all blocks in turn, else rows do
    const int stride = rows == 1 ? blocks * step : step, c0 = 4 * ((int)threadIdx.x % lanes) + (rows == 1 ? block * step : 0);
    const int r0 = rows == 1 ? (int)threadIdx.x / lanes : block * per_block + (int)threadIdx.x / lanes;
    double s = 0.0;
    for (int r = r0; r < rows; r += blocks * per_block) {
        const long long g = (long long)r * a.ldg, m = (long long)r * a.ldm;
        for (long long c = c0; c < cols; c += 4LL * stride) {
            v4f x[4], y[4];
            int left[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const long long at = c + (long long)u * stride;
                left[u] = at < cols ? (int)min(4LL, cols - at) : 0;
                x[u] = load_four(a.g, g + at, l.g_tensor, left[u], whole_g);
                if (l.muon) y[u] = load_four(a.mom, m + at, TENSOR_F32, left[u], whole_m);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (l.muon) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[u][e] = __builtin_fmaf(l.momentum, y[u][e], x[u][e]);
                        x[u][e] = updated(l, x[u][e], y[u][e]);
                    }
                    store_four(a.mom + m + c + (long long)u * stride, y[u], left[u], whole_m);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) s += (double)x[u][e] * (double)x[u][e];
            }
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    s = red[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) s += red[i];
    return s;
}

__global__ __launch_bounds__(SUM_NT) void sum_kernel(List l, List *to, double *partial)
{
    if (blockIdx.x == 0) {
        const unsigned *from = reinterpret_cast<const unsigned *>(&l);
        for (unsigned i = threadIdx.x; i < sizeof(List) / 4; i += SUM_NT) reinterpret_cast<unsigned *>(to)[i] = from[i];
    }
    __shared__ double red[SUM_NT / 64];
    const Mat &a = l.mat[find(l, blockIdx.x, [](const Mat &x) { return x.sum0; })];
    const double s = sum_of_block<SUM_NT>(l, a, blockIdx.x - a.sum0, a.sums, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ void split(float x, half_t &hi, half_t &lo)
{
    hi = (half_t)x;
    lo = (half_t)(x - (float)hi);
}

// ---------------------------------------------------------------- X, X^T from G
// Bound by memory: a 64 x 64 tile is read once and leaves in both layouts (4096 x 4096 bf16, 134 MB: 26.6 us, 5.0 TB/s).
__global__ __launch_bounds__(256) void prep_kernel(const List *lp, unsigned char *ws, const double *partial)
{
    const List &l = *lp;
    const int k = find(l, blockIdx.x, [](const Mat &a) { return a.prep0; });
    const Mat &a = l.mat[k];
    __shared__ double red[4];
    __shared__ float tile[PREP][PREP + 1];
    const int tid = threadIdx.x;
    double s = 0.0;
    for (int i = tid; i < a.sums; i += 256) s += partial[a.sum0 + i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((tid & 63) == 0) red[tid >> 6] = s;
    __syncthreads();
    const double inv = (double)SX / (sqrt((red[0] + red[1]) + (red[2] + red[3])) + (double)l.eps);
    // tile of X: rows i0 .., columns j0 ..; of G the same or exchanged
    const int per_row = a.n / PREP, t = blockIdx.x - a.prep0;
    const int i0 = (t / per_row) * PREP, j0 = (t % per_row) * PREP;
    const int r0 = a.flip ? j0 : i0, c0 = a.flip ? i0 : j0;
    v4f x[PREP / 16], y[PREP / 16];
    const int c = 4 * (tid & 15), there = a.cols - (c0 + c);
#pragma unroll
    for (int i = 0; i < PREP / 16; ++i) {
        const int r = 16 * i + (tid >> 4), left = r0 + r < a.rows ? there : 0;
        x[i] = load_four(a.g, (long long)(r0 + r) * a.ldg + c0 + c, l.g_tensor, left, a.whole_g);
        if (l.muon) y[i] = load_four(a.mom, (long long)(r0 + r) * a.ldm + c0 + c, TENSOR_F32, left, a.whole_m);
    }
#pragma unroll
    for (int i = 0; i < PREP / 16; ++i) {
        const int r = 16 * i + (tid >> 4), left = r0 + r < a.rows ? there : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = l.muon ? updated(l, x[i][e], y[i][e]) : x[i][e];
            const float v = e < left ? (float)((double)u * inv) : 0.f;  // (inv may be inf)
            if (a.flip) tile[c + e][r] = v;
            else tile[r][c + e] = v;
        }
    }
    __syncthreads();
    half_t *const X = reinterpret_cast<half_t *>(ws + a.x[0]), *const XT = reinterpret_cast<half_t *>(ws + a.xt[0]);
    const size_t low = (size_t)a.mp * a.np;
    for (int q = tid; q < PREP * PREP / 8; q += 256) {  // 8 values of a row of X, and of a row of X^T
        const int r = q >> 3, c = (q & 7) * 8;
        v8h hi, lo, thi, tlo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            half_t p, w;
            split(tile[r][c + e], p, w);
            hi[e] = p;
            lo[e] = w;
            split(tile[c + e][r], p, w);
            thi[e] = p;
            tlo[e] = w;
        }
        const size_t at = (size_t)(i0 + r) * a.np + j0 + c, tat = (size_t)(j0 + r) * a.mp + i0 + c;
        *reinterpret_cast<v8h *>(X + at) = hi;
        if (l.planes == 2) *reinterpret_cast<v8h *>(X + low + at) = lo;
        *reinterpret_cast<v8h *>(XT + tat) = thi;
        *reinterpret_cast<v8h *>(XT + low + tat) = tlo;
    }
}

// ---------------------------------------------------------------- products
// GRAM_PART, GRAM_JOIN: the first product of few rows and many columns in two launches: sums over parts of k, and what is made of them
enum { GRAM = 0, SQUARE = 1, NEXT = 2, LAST = 3, GRAM_PART = 4, GRAM_JOIN = 5 };

// slot of 16-byte chunk c of tile row R: c ^ swz(R), so that the sixteen rows of a fragment read lie on different banks
__device__ __forceinline__ int swz(int R) { return (R >> 1) & 7; }

template <int N>
__device__ __forceinline__ void wait_loads_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// T x T tile of rows times rows, WM x WN wavefronts, S stages of both operands in LDS.  Two planes of an operand are in a stage together, so that each is
// loaded once for the three products (instead of one segment of k behind the other: 983 x 512 fp32 18.0 -> 13.7, 11.9 -> 9.6, 11.4 -> 8.9 us for the
// three products of a step, 1024 x 1024 30 -> 18); with one plane, 64 x 64 tiles have two k-tiles in a stage.  KG = 2, where there is no more
// than a workgroup a compute unit: twice the wavefronts, each half with one of two k-tiles or k-steps of a stage, and four stages.
// Bound by the loads into LDS where tiles are small (1000 x 4096: 1024 tiles of 64, the 8.2 GFLOP of a X + B X in 21.6 us, 380 TFLOP/s), by the
// matrix cores and the units that have no tile where they are large.
template <int T, int WM, int WN, int S, int PL, int KG>
struct Product {
    static constexpr int NW = WM * WN * KG, NT = 64 * NW;
    static constexpr int RM = T / WM, RN = T / WN, MB = RM / 16, NB = RN / 16;
    static constexpr int LOADS = T * 8 / NT;  // 16-byte loads a lane and operand tile
    static constexpr int KT = T == 64 && PL == 1 ? 2 : 1, SUB = PL * KT;  // k-tiles in a stage
    static constexpr int OPERAND = T * ROW_BYTES, STAGE = 2 * SUB * OPERAND;
    static constexpr int HM = RM < 64 ? RM : 64, AHEAD = 2, REGION = RN * (HM + 4) * 4;  // of the results: rows at a time, loads before one is used
    static constexpr size_t LDS = (size_t)(S * STAGE > WM * WN * REGION ? S * STAGE : WM * WN * REGION);
    v4f acc[MB][NB];

    // the sums as they lie in the first WM x WN wavefronts, and from several such parts in their order
    __device__ __forceinline__ void keep(v4f *to, int tid) const
    {
        if (tid >= 64 * WM * WN) return;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) to[(i * NB + j) * (64 * WM * WN) + tid] = acc[i][j];
    }
    __device__ __forceinline__ void join(const v4f *from, size_t step, int parts, int tid)
    {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = from[(i * NB + j) * (64 * WM * WN) + tid];
#pragma unroll 4
        for (int s = 1; s < parts; ++s)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] += from[s * step + (i * NB + j) * (64 * WM * WN) + tid];
    }

    // P, Q: first rows of the tile, of `pitch` bytes; nk k-tiles; low_p, low_q: bytes to the low parts
    __device__ __forceinline__ void run(unsigned char *lds, const unsigned char *P, const unsigned char *Q, unsigned pitch, int nk, size_t low_p,
                                        size_t low_q, int tid)
    {
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wm = wave % WM, wn = wave / WM % WN, group = wave / (WM * WN);
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
        unsigned off[LOADS];
#pragma unroll
        for (int v = 0; v < LOADS; ++v) {
            const int R = (wave + NW * v) * 8 + (lane >> 3);
            off[v] = (unsigned)R * pitch + (((lane & 7) ^ swz(R)) << 4);
        }
        const int steps = (nk + KT - 1) / KT;
        auto issue = [&](int t, int stage) {
            const size_t k = (size_t)t * (KT * ROW_BYTES);
            unsigned char *to = lds + stage * STAGE;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                if (kt == 1 && 2 * t + 1 >= nk) continue;  // (an odd number of k-tiles)
#pragma unroll
                for (int pl = 0; pl < PL; ++pl)
#pragma unroll
                    for (int v = 0; v < LOADS; ++v) {
                        unsigned char *const to_v = to + 2 * (kt * PL + pl) * OPERAND + (wave + NW * v) * 1024;
                        __builtin_amdgcn_global_load_lds((gptr_t)(P + (pl ? low_p : 0) + k + kt * ROW_BYTES + off[v]), (lptr_t)to_v, 16, 0, 0);
                        __builtin_amdgcn_global_load_lds((gptr_t)(Q + (pl ? low_q : 0) + k + kt * ROW_BYTES + off[v]), (lptr_t)(to_v + OPERAND), 16, 0, 0);
                    }
            }
        };
        const int full = nk / KT;  // (the last step may have fewer loads)
#pragma unroll
        for (int t = 0; t < S - 1; ++t)
            if (t < steps) issue(t, t);
        const int c16 = lane & 15, g4 = lane >> 4;
        const int p_off = (wm * RM + c16) * ROW_BYTES + ((g4 ^ swz(c16)) << 4);
        const int q_off = OPERAND + (wn * RN + c16) * ROW_BYTES + ((g4 ^ swz(c16)) << 4);
        int stage = 0;
        for (int t = 0; t < steps; ++t) {
            // tile t has landed, and everybody is done with tile t - 1
            if (S > 2 && t + S - 2 < full) wait_loads_and_meet<2 * SUB * LOADS *(S - 2)>();
            else wait_loads_and_meet<0>();
            if (t + S - 1 < steps) issue(t + S - 1, stage == 0 ? S - 1 : stage - 1);
            const unsigned char *at = lds + stage * STAGE;
#pragma unroll
            for (int ks = 0; ks < 2 * KT / KG; ++ks) {
                const int kk = KG == 1 || KT == 2 ? ks & 1 : group, kt = KT == 1 ? 0 : KG == 2 ? group : ks / 2;
                if (KT == 2 && (KG == 2 || ks == 2) && kt == 1 && 2 * t + 1 >= nk) break;
                v8h fp[PL][MB], fq[PL][NB];
#pragma unroll
                for (int pl = 0; pl < PL; ++pl) {
                    const unsigned char *from = at + 2 * (kt * PL + pl) * OPERAND;
#pragma unroll
                    for (int i = 0; i < MB; ++i) fp[pl][i] = *reinterpret_cast<const v8h *>(from + (p_off ^ (kk << 6)) + i * 16 * ROW_BYTES);
#pragma unroll
                    for (int j = 0; j < NB; ++j) fq[pl][j] = *reinterpret_cast<const v8h *>(from + (q_off ^ (kk << 6)) + j * 16 * ROW_BYTES);
                }
#pragma unroll
                for (int s = 0; s < 2 * PL - 1; ++s)  // high x high, high x low, low x high
#pragma unroll
                    for (int i = 0; i < MB; ++i)
#pragma unroll
                        for (int j = 0; j < NB; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[s == 2 ? PL - 1 : 0][i], fq[s == 1 ? PL - 1 : 0][j], acc[i][j], 0, 0, 0);
            }
            stage = stage == S - 1 ? 0 : stage + 1;
        }
        if (KG == 1) return;
        // the second group's sums to the first
        v4f *const sums = reinterpret_cast<v4f *>(lds) + (wave % (WM * WN)) * (MB * NB * 64) + lane;
        __syncthreads();
        if (group == 1) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j2 = 0; j2 < NB; ++j2) sums[(i * NB + j2) * 64] = acc[i][j2];
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j2 = 0; j2 < NB; ++j2) acc[i][j2] += sums[(i * NB + j2) * 64];
        }
    }
};

// 256 x 256 tiles of eight wavefronts, as 2 x 4, of 128 x 64 each: two stages of the left operand and three of the right one (all 160 KB of LDS).
// The sixteen products of a group (half of the rows at one k-step of 32) are issued with the requests of the next group's fragments and two
// loads from memory between them, so that neither the LDS nor the address unit gets them all at once; loads have two groups or more to land.
template <int PL>
struct Product<256, 2, 4, 2, PL, 1> {
    static constexpr int T = 256, WM = 2, NW = 8, NT = 512, RM = 128, RN = 64, MB = 8, NB = 4;
    static constexpr int OPERAND = T * ROW_BYTES, Q_BASE = 2 * OPERAND;
    static constexpr int HM = 64, AHEAD = 4, REGION = RN * (HM + 4) * 4;
    static constexpr size_t LDS = 5 * (size_t)OPERAND;
    static_assert(NW * REGION <= (int)LDS, "LDS");
    v4f acc[MB][NB];

    __device__ __forceinline__ void run(unsigned char *lds, const unsigned char *P, const unsigned char *Q, unsigned pitch, int nk, size_t low_p,
                                        size_t low_q, int tid)
    {
        constexpr int segs = 2 * PL - 1;  // high x high, high x low, low x high: one behind the other
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wm = wave % WM, wn = wave / WM;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
        unsigned off[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int R = (wave + NW * v) * 8 + (lane >> 3);
            off[v] = (unsigned)R * pitch + (((lane & 7) ^ swz(R)) << 4);
        }
        const int total = nk * segs;
        auto issue_p = [&](int t, int stage, int v) {
            const int seg = t >= 2 * nk ? 2 : t >= nk ? 1 : 0;
            const unsigned char *p = P + (seg == 2 ? low_p : 0) + (size_t)(t - seg * nk) * ROW_BYTES;
            __builtin_amdgcn_global_load_lds((gptr_t)(p + off[v]), (lptr_t)(lds + stage * OPERAND + (wave + NW * v) * 1024), 16, 0, 0);
        };
        auto issue_q = [&](int t, int stage, int v) {
            const int seg = t >= 2 * nk ? 2 : t >= nk ? 1 : 0;
            const unsigned char *q = Q + (seg == 1 ? low_q : 0) + (size_t)(t - seg * nk) * ROW_BYTES;
            __builtin_amdgcn_global_load_lds((gptr_t)(q + off[v]), (lptr_t)(lds + Q_BASE + stage * OPERAND + (wave + NW * v) * 1024), 16, 0, 0);
        };
        const int c16 = lane & 15, g4 = lane >> 4;
        const int p_off = (wm * RM + c16) * ROW_BYTES + ((g4 ^ swz(c16)) << 4);
        const int q_off = Q_BASE + (wn * RN + c16) * ROW_BYTES + ((g4 ^ swz(c16)) << 4);
        v8h fp[2][4], fq[2][4];  // half of the rows, all columns at one k-step
        auto read = [&](int off_, int q, int kk) { return *reinterpret_cast<const v8h *>(lds + ((off_ ^ (kk << 6)) + q * 16 * ROW_BYTES)); };
        auto group = [&](auto half_c, int bs, bool rd, int sp, int sq, int kk, bool ld, bool is_p, int t, int stage, int first) {
            constexpr int half = decltype(half_c)::value;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    acc[4 * half + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[half][i], fq[bs][j], acc[4 * half + i][j], 0, 0, 0);
                    const int b = 4 * i + j;
                    __builtin_amdgcn_sched_barrier(0);
                    if (rd) {
                        if (b < 4) fp[half ^ 1][b] = read(p_off + sp * OPERAND, b + (half ? 0 : 4), kk);
                        else if (half && b < 8) fq[bs ^ 1][b - 4] = read(q_off + sq * OPERAND, b - 4, kk);
                    }
                    if (ld && (b == (half ? 10 : 5) || b == (half ? 14 : 10))) {
                        const int v = first + (b == (half ? 14 : 10) ? 1 : 0);
                        if (is_p) issue_p(t, stage, v);
                        else issue_q(t, stage, v);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
        };
        constexpr IntC<0> LO = {};
        constexpr IntC<1> HI = {};
#pragma unroll
        for (int v = 0; v < 4; ++v) issue_p(0, 0, v);
#pragma unroll
        for (int v = 0; v < 4; ++v) issue_q(0, 0, v);
        if (total > 1) {
#pragma unroll
            for (int v = 0; v < 4; ++v) issue_q(1, 1, v);
            issue_p(1, 1, 0);
            issue_p(1, 1, 1);
            wait_loads_and_meet<6>();  // tile 0 has landed
        } else {
            wait_loads_and_meet<0>();
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) fp[0][q] = read(p_off, q, 0);
#pragma unroll
        for (int q = 0; q < 4; ++q) fq[0][q] = read(q_off, q, 0);
        int q_cur = 0, q_nxt = 1, q_ld = 2;  // stages of the right operand of tiles t, t + 1, t + 2
        for (int t = 0; t < total; ++t) {
            const int cur = t & 1;
            const bool next = t + 1 < total, next2 = t + 2 < total;
            // (the fragments of a group were requested during the one before; the compiler cannot tell across the branches)
            __builtin_amdgcn_s_waitcnt(0xc07f);
            group(LO, 0, true, cur, q_cur, 0, next, true, t + 1, cur ^ 1, 2);  // + second half of the left tile t + 1
            __builtin_amdgcn_s_waitcnt(0xc07f);
            group(HI, 0, true, cur, q_cur, 1, next2, false, t + 2, q_ld, 0);   // + the right tile t + 2, whose stage held t - 1
            __builtin_amdgcn_s_waitcnt(0xc07f);
            group(LO, 1, true, cur, q_cur, 1, next2, false, t + 2, q_ld, 2);
            // tile t + 1 has landed (the right tile t + 2 may be on its way), and nobody reads tile t any more
            if (next2) wait_loads_and_meet<4>();
            else wait_loads_and_meet<0>();
            __builtin_amdgcn_s_waitcnt(0xc07f);
            group(HI, 1, next, cur ^ 1, q_nxt, 0, next2, true, t + 2, cur, 0);  // + first half of the left tile t + 2
            const int u = q_cur;
            q_cur = q_nxt;
            q_nxt = q_ld;
            q_ld = u;
        }
    }
};

// row of tile t of the tiles on and below the diagonal, in row order
__device__ __forceinline__ int triangle_row(int t)
{
    int r = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((r + 1) * (r + 2) / 2 <= t) ++r;
    while (r * (r + 1) / 2 > t) --r;
    return r;
}

// eight values of a row: high parts, and low ones `low` elements further on
struct Eight {
    float v[8];
    __device__ __forceinline__ void load(const half_t *p, size_t low, bool two)
    {
        const v8h hi = *reinterpret_cast<const v8h *>(p);
        v8h lo = {};
        if (two) lo = *reinterpret_cast<const v8h *>(p + low);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)hi[e] + (float)lo[e];
    }
    __device__ __forceinline__ void store(half_t *p, size_t low, bool two) const
    {
        v8h hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            half_t u, w;
            split(v[e], u, w);
            hi[e] = u;
            lo[e] = w;
        }
        *reinterpret_cast<v8h *>(p) = hi;
        if (two) *reinterpret_cast<v8h *>(p + low) = lo;
    }
};

// Eight neighbours in a row of the result, of which `left` are there
__device__ __forceinline__ void put_result(const How &l, const Matrix &a, int r, int c, const float *v)
{
    if (r >= a.rows || c >= a.cols) return;
    const int left = a.cols - c;
    const long long at = (long long)r * a.ldo + c;
    if (l.out_tensor == TENSOR_BF16) {
        __bf16 *const q = static_cast<__bf16 *>(a.out) + at;
        if (a.whole_out && left >= 8) {
            v8b u;
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = (__bf16)(v[e] * (1.f / SX));
            *reinterpret_cast<v8b *>(q) = u;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) q[e] = (__bf16)(v[e] * (1.f / SX));
        }
        return;
    }
    float *const q = static_cast<float *>(a.out) + at;
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
        v4f x;
        if (l.muon) x = load_four(q, h, TENSOR_F32, left - h, a.whole_out);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float o = v[h + e] * (1.f / SX);
            x[e] = l.muon ? __builtin_fmaf(-a.scale, o, __builtin_fmaf(-l.decay, x[e], x[e])) : o;
        }
        store_four(q + h, x, left - h, a.whole_out);
    }
}

template <int T, int WM, int WN, int S, int PL, int KG, int WHAT>
__global__ __launch_bounds__(64 * WM *WN *KG) void product_kernel(const List *lp, unsigned char *ws, int from, float ca, float cb, float cc)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    typedef Product<T, WM, WN, S, PL, KG> P;
    const List &l = *lp;
    constexpr int KIND = WHAT == GRAM_PART || WHAT == GRAM_JOIN ? (int)GRAM : WHAT;
    constexpr bool SYM = KIND == GRAM || KIND == SQUARE;
    const int slice = WHAT == GRAM_PART ? (int)blockIdx.x / l.syms : 0, block = (int)blockIdx.x - slice * l.syms;
    const int k = find(l, block, [](const Mat &a) { return SYM ? a.sym0 : a.all0; });
    const Mat &a = l.mat[k];
    const int t = block - (SYM ? a.sym0 : a.all0);
    int ti, tj;
    if (SYM) {
        ti = triangle_row(t);
        tj = t - ti * (ti + 1) / 2;
    } else {
        const int per_row = (a.n + T - 1) / T;
        ti = t / per_row;
        tj = t - ti * per_row;
    }
    const int i0 = ti * T, j0 = tj * T;
    const size_t xlow = (size_t)a.mp * a.np, alow = (size_t)a.mp * a.mp;
    const int tid = threadIdx.x;
    P p;
    if constexpr (WHAT == GRAM_JOIN) {
        p.join(reinterpret_cast<const v4f *>(ws + l.part) + (size_t)block * (T * T / 4), (size_t)l.syms * (T * T / 4), l.splits, tid);
    } else {
        const unsigned char *x = ws + (KIND == GRAM ? a.x[from] : KIND == SQUARE ? a.f : a.h);
        const unsigned char *y = KIND == GRAM || KIND == SQUARE ? x : ws + a.xt[from];
        const unsigned pitch = 2u * (unsigned)(KIND == GRAM ? a.np : a.mp);
        int nk = (KIND == GRAM ? a.n : a.m) / BK;
        if (WHAT == GRAM_PART) {
            const int chunk = (nk + l.splits - 1) / l.splits, k0 = min(slice * chunk, nk);
            nk = min(chunk, nk - k0);
            x += (size_t)k0 * ROW_BYTES;
            y += (size_t)k0 * ROW_BYTES;
        }
        p.run(lds, x + (size_t)i0 * pitch, y + (size_t)j0 * pitch, pitch, nk, 2 * (KIND == GRAM ? xlow : alow), 2 * (SYM ? (KIND == GRAM ? xlow : alow) : xlow), tid);
    }
    if constexpr (WHAT == GRAM_PART) {
        p.keep(reinterpret_cast<v4f *>(ws + l.part) + (size_t)blockIdx.x * (T * T / 4), tid);
        return;
    }
    // The results leave through LDS, HM rows of the wavefront's block at a time: lane 16 g + c of a 16 x 16 block has column c, rows 4 g .. 4 g + 3, in LDS
    // they lie a column after the other.  From there lanes take eight rows of a column each (whole lines of the transposed
    // layouts, which the terms to be added are read from, too), and eight columns of a row.  Loops that are not unrolled throughout: code that every
    // workgroup runs once comes from memory, a line after the other (unrolled for all blocks it took 40 to 80 us of a launch).
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int bi0 = i0 + (wave % WM) * P::RM, bj0 = j0 + (wave / WM) * P::RN;  // of this wavefront
    float *const D = reinterpret_cast<float *>(ws + a.d), *const E = reinterpret_cast<float *>(ws + a.e);
    half_t *const F = reinterpret_cast<half_t *>(ws + a.f), *const H = reinterpret_cast<half_t *>(ws + a.h);
    half_t *const xt = reinterpret_cast<half_t *>(ws + a.xt[from]);
    half_t *const new_xt = reinterpret_cast<half_t *>(ws + a.xt[from ^ 1]), *const new_x = reinterpret_cast<half_t *>(ws + a.x[from ^ 1]);
    constexpr int HM = P::HM, PITCH = HM + 4, PER = HM / 8, ITEMS = P::RN * PER / 64;
    constexpr bool two = PL == 2;
    const bool rows_too = SYM ? ti != tj : KIND == NEXT || !a.flip;
    __syncthreads();  // nobody reads the operands any more: their place is for the results
    if (KG == 2 && wave >= WM * WN) return;  // (no wavefront waits for another from here on)
    float *const mine = reinterpret_cast<float *>(lds + wave * P::REGION);
#pragma unroll
    for (int half = 0; half < P::RM / HM; ++half) {
#pragma unroll
        for (int bj = 0; bj < P::NB; ++bj)
#pragma unroll
            for (int bi = 0; bi < HM / 16; ++bi)
                *reinterpret_cast<v4f *>(mine + (16 * bj + (lane & 15)) * PITCH + 16 * bi + 4 * (lane >> 4)) = p.acc[half * (HM / 16) + bi][bj];
        const int ih = bi0 + half * HM;
#pragma unroll 1
        for (int it0 = 0; it0 < ITEMS; it0 += P::AHEAD) {
            Eight x[P::AHEAD];
            if (KIND != GRAM) {
#pragma unroll
                for (int u = 0; u < P::AHEAD; ++u) {
                    const int item = (it0 + u) * 64 + lane, j = bj0 + item / PER, i = ih + 8 * (item % PER);
                    if (KIND == SQUARE) x[u].load(F + (size_t)j * a.mp + i, alow, two);
                    else x[u].load(xt + (size_t)j * a.mp + i, xlow, true);
                }
            }
#pragma unroll
            for (int u = 0; u < P::AHEAD; ++u) {
                const int item = (it0 + u) * 64 + lane, jl = item / PER, il = 8 * (item % PER), j = bj0 + jl, i = ih + il;
                float *const at = mine + jl * PITCH + il;
                Eight v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v.v[e] = at[e];
                const v4f *const di = reinterpret_cast<const v4f *>((KIND == SQUARE ? D : E) + i);
                if (KIND == GRAM) {
                    if (ti == tj && i <= j && j < i + 8) D[j] = at[j - i] * (1.f / (SX * SX));
#pragma unroll
                    for (int e = 0; e < 8; ++e) v.v[e] *= SA / (SX * SX);
                } else if (KIND == SQUARE) {
                    const float dj = D[j];
                    if (ti == tj && i <= j && j < i + 8) E[j] = __builtin_fmaf(cc, __builtin_fmaf(dj, dj, at[j - i] * (1.f / (SA * SA))), cb * dj);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float sq = v.v[e] * (1.f / (SA * SA)), f = x[u].v[e] * (1.f / SA);
                        v.v[e] = SB * __builtin_fmaf(cc, __builtin_fmaf(di[e / 4][e % 4] + dj, f, sq), cb * f);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v.v[e] = __builtin_fmaf(ca + di[e / 4][e % 4], x[u].v[e], v.v[e] * (1.f / SB));
                }
                if (SYM && ti == tj) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v.v[e] = i + e == j ? 0.f : v.v[e];
                }
                if (SYM) v.store((KIND == GRAM ? F : H) + (size_t)j * a.mp + i, alow, two);
                else if (KIND == NEXT) v.store(new_xt + (size_t)j * a.mp + i, xlow, true);
                else if (a.flip) put_result(l, a, j, i, v.v);
                if (rows_too) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) at[e] = v.v[e];
                }
            }
        }
        if (rows_too) {
#pragma unroll 1
            for (int it = 0; it < ITEMS; ++it) {
                const int item = it * 64 + lane, il = item / (P::RN / 8), jl = 8 * (item % (P::RN / 8)), i = ih + il, j = bj0 + jl;
                Eight v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v.v[e] = mine[(jl + e) * PITCH + il];
                if (SYM) v.store((KIND == GRAM ? F : H) + (size_t)i * a.mp + j, alow, two);
                else if (KIND == NEXT) v.store(new_x + (size_t)i * a.np + j, xlow, two);
                else put_result(l, a, i, j, v.v);
            }
        }
    }
}

// ---------------------------------------------------------------- small matrices
// X of up to 128 rows: a workgroup has a block of its columns (all of them where they are few: then one launch does everything), and
// several steps need X once.  With A = X X^T and P_k = a + b A_k + c A_k^2,
//     X_k+1 = P_k X_k,   A_k+1 = P_k A_k P_k,   X_k+l = Q X_k,   Q = P_k+l-1 ... P_k
// so a run of steps is products of m x m matrices, which commute and are symmetric.  A value of A near 0 keeps an absolute error while A_k+1 gives it the factor
// p(0)^2, so the error of a long run is as of a square root of the precision: runs end where the product of the largest factors
// passes 12 (HB_TENSOR_F32: two of the usual steps), or 500 (HB_TENSOR_BF16: five; 2e-5 to 1e-4 of the result's norm where singular values are spread over two decades, 6e-4 to
// 1.6e-3 at worst, where they are 3e-3 of the largest); of HB_TENSOR_F32 with up to 16 rows every step is a run,
// since roundings do not average out over few of them (2 x 5 6.0e-6 in runs of two, 0.9e-6; 16 x 8192 takes 67 us for 53).
// Everything but diagonals is held in 22 bits.  A wavefront has a strip of 16 columns of the m x m matrices in its registers.  A result of the matrix core holds four
// rows of a column a lane, so two blocks of a strip are its operand of 32 values of k (in an order of their own, the same for both operands); rows go through LDS.
// What bounds it is latency: 512 x 54 fp32 takes 58 us in one workgroup, of which reading and writing 220 KB are 17, the products with X 18, the m x m ones 16.
constexpr int SMALL_NT = 512, SMALL_WAVES = 8;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

struct SmallStep {
    float a, b, c;
    float sa, sp, sq;  // powers of two: scales of A before the step, of its P, and of Q after it
    int end;           // of a run
};
struct SmallMat : Matrix {
    int m, n;
    int blocks, block0;  // of columns, and the first workgroup
    int sums, sum0;      // as in Mat
    size_t x;            // byte offset in the workspace: X^T, between launches
    size_t part[2];      // sums of X X^T over each block's columns, in turn
};
struct SmallArgs : How {
    int count;
    int steps;
    SmallStep step[ORTHO_STEPS];
    SmallMat mat[ORTHO_GROUP];
};
static_assert(sizeof(SmallArgs) < 4000, "arguments of a launch");

// MP: rows of X, padded; NB: columns of a block
template <int MP, int NB>
struct Small {
    static constexpr int S = MP / 16, PARTS = SMALL_WAVES / S, KS = (MP + 31) / 32;  // strips; parts that share a strip's sums; k-steps of m
    static constexpr int CHUNKS = MP / 8;
    static constexpr int PLANE = NB * MP * 2, FILE = S * KS * 2 * 1024, RED = (PARTS - 1) * MP * MP * 4;
    static constexpr int X = 0, SHARED = 2 * PLANE;  // X^T, high and low; then rows of the m x m matrices, or sums to be added up
    static constexpr int DIAG = FILE > RED ? FILE : RED;  // behind the rows: their matrix's diagonal
    static constexpr size_t LDS = 2 * (size_t)PLANE + DIAG + 4 * MP;

    // byte of element (column j, row i) in a plane of X^T: the 16-byte pieces of a row are exchanged so that 16 rows lie on different banks, and so do the four
    // rows of 32 bytes of a transposing read
    static __device__ __forceinline__ int turn(int j)
    {
        if (MP == 128) return ((j & 7) << 1) | ((j >> 3) & 1);
        if (MP == 64) return (j & 6) | ((j >> 3) & 1);
        if (MP == 32) return (j >> 2) & 3;
        return (j >> 3) & 1;
    }
    static __device__ __forceinline__ int at(int j, int i) { return j * (2 * MP) + (((i >> 3) ^ turn(j)) << 4) + 2 * (i & 7); }

    struct Strip {
        v4f v[S];  // rows 16 i + 4 g + e of column 16 strip + c
    };
    struct Frag {
        v8h hi[KS], lo[KS];
    };

    static __device__ __forceinline__ void frag_of(const Strip &m, float scale, Frag &f)
    {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                half_t hi = 0, lo = 0;
                if (2 * ks + e / 4 < S) split(m.v[2 * ks + e / 4 < S ? 2 * ks + e / 4 : 0][e % 4] * scale, hi, lo);
                f.hi[ks][e] = hi;
                f.lo[ks][e] = lo;
            }
    }
    // The strip's part of the rows, for everybody, in the order in which the lanes ask for it.  (The matrices are symmetric but for roundings: columns in place of
    // rows would save the exchange, but what is not symmetric grows from step to step then, 8e-4 of the result after five.)
    // The diagonal goes beside them in 32 bits: it is as large as all the rest of a row, and its rounding to 22 bits would be the same for every
    // column of a product (1 x 6 2.3e-6 then).
    static __device__ __forceinline__ void put_rows(unsigned char *file, const Strip &m, float scale, int strip, int lane)
    {
        const int g4 = lane >> 4, c16 = lane & 15, ks = strip >> 1;
        float d = 0.f;
        unsigned char *const to = file + ks * 2048 + (16 * (c16 >> 2) + 4 * g4) * 16 + (4 * (strip & 1) + (c16 & 3)) * 2;
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool on = i == strip && 4 * g4 + e == c16;
                d = on ? m.v[i][e] : d;
                half_t hi, lo;
                split(on ? 0.f : m.v[i][e] * scale, hi, lo);
                *reinterpret_cast<half_t *>(to + i * KS * 2048 + 16 * e) = hi;
                *reinterpret_cast<half_t *>(to + i * KS * 2048 + 16 * e + 1024) = lo;
            }
        if (g4 == c16 >> 2) *reinterpret_cast<float *>(file + DIAG + 4 * (16 * strip + c16)) = d;
        if (S == 1) {  // there is no second block of 16 values of k
            *reinterpret_cast<v4h *>(file + 16 * lane + 8) = v4h{0, 0, 0, 0};
            *reinterpret_cast<v4h *>(file + 1024 + 16 * lane + 8) = v4h{0, 0, 0, 0};
        }
    }
    // scale (rows in LDS times columns) + d_scale (diagonal times the same columns in 32 bits, of(block, row))
    template <typename Of>
    static __device__ __forceinline__ void times(const unsigned char *file, const Frag &f, float scale, float d_scale, Of of, Strip &out, int lane)
    {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const v8h hi = *reinterpret_cast<const v8h *>(file + ((i * KS + ks) * 2) * 1024 + 16 * lane);
                const v8h lo = *reinterpret_cast<const v8h *>(file + ((i * KS + ks) * 2 + 1) * 1024 + 16 * lane);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, f.hi[ks], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, f.lo[ks], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, f.hi[ks], acc, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                out.v[i][e] = __builtin_fmaf(d_scale * *reinterpret_cast<const float *>(file + DIAG + 4 * (16 * i + 4 * (lane >> 4) + e)), of(i, e), acc[e] * scale);
            if (S == 8) __builtin_amdgcn_sched_barrier(0);  // (requests for all rows at once leave no registers)
        }
    }

    // A matrix as the caller has it, lanes along its rows: f(first row, column, step to the next row, rows) for ROWS_AT_ONCE rows at a time
    static constexpr int ROWS_AT_ONCE = 8;
    template <typename F>
    static __device__ __forceinline__ void rows_of(const SmallMat &a, int j0, int columns, F f)
    {
        const int rows = a.flip ? min(columns, a.rows - j0) : a.rows, cols = a.flip ? a.cols : min(columns, a.cols - j0);
        int shift = 9;  // of the lanes of a row
        while (shift > 0 && (1 << (shift - 1)) >= cols) --shift;
        const int step = SMALL_NT >> shift;
#pragma unroll 1
        for (int c = threadIdx.x & ((1 << shift) - 1); c < cols; c += 1 << shift)
#pragma unroll 1
            for (int r = threadIdx.x >> shift; r < rows; r += ROWS_AT_ONCE * step) f(r, c, step, rows);
    }
    // Rows without gaps between them, four elements at a time from a 16-byte boundary (8 for two bytes): f(first element, how many) for all of a thread's
    static constexpr int FLAT = NB * MP / (4 * SMALL_NT);
    static __device__ __forceinline__ int elements(const SmallMat &a, int j0, int columns) { return a.flip ? min(columns, a.rows - j0) * a.cols : a.rows * a.cols; }
    static __device__ __forceinline__ bool flat(const SmallMat &a, long long ld, bool begins)
    {
        return ld == a.cols && begins && (a.flip || a.blocks == 1);  // (a block is then a run of rows that begins at a multiple of NB of them)
    }
    // the places in LDS of elements first .. first + 3
    struct Places {
        int r, c, cols;
        bool flip;
        __device__ __forceinline__ Places(const SmallMat &a, int first) : cols(a.cols), flip(a.flip)
        {
            r = (int)(((float)first + 0.5f) * __builtin_amdgcn_rcpf((float)cols));  // first < 2^16: off by less than 1 / (2 cols)
            c = first - r * cols;
        }
        __device__ __forceinline__ int next()
        {
            const int p = flip ? at(r, c) : at(c, r);
            if (++c == cols) {
                c = 0;
                ++r;
            }
            return p;
        }
    };
    static __device__ __forceinline__ void keep(unsigned char *lds, int p, float x)
    {
        *reinterpret_cast<unsigned short *>(lds + p) = (unsigned short)(__float_as_uint(x) >> 16);
        *reinterpret_cast<unsigned short *>(lds + PLANE + p) = (unsigned short)__float_as_uint(x);
    }
    static __device__ __forceinline__ float kept(const unsigned char *lds, int p)
    {
        return __uint_as_float((unsigned)*reinterpret_cast<const unsigned short *>(lds + p) << 16 | *reinterpret_cast<const unsigned short *>(lds + PLANE + p));
    }
    // Columns j0 .. of X as they are, a float in the two halves of an element's places in LDS, and this thread's part of the sum of their squares.
    // with_momentum: M gets its new value on the way (else it has it)
    static __device__ __forceinline__ double load_g(unsigned char *lds, const How &l, const SmallMat &a, int j0, int columns, bool with_momentum)
    {
        double sum = 0.0;
        const bool bf16 = l.g_tensor == TENSOR_BF16;
        const long long first_g = a.flip ? j0 * a.ldg : j0, first_m = a.flip ? j0 * a.ldm : j0;
        if (flat(a, a.ldg, a.begins_g) && (!l.muon || flat(a, a.ldm, a.begins_m))) {
            const int n = elements(a, j0, columns);
            v4f x[FLAT];
#pragma unroll
            for (int u = 0; u < FLAT; ++u) {  // all of them are asked for before one is waited for
                const int q = 4 * (threadIdx.x + u * SMALL_NT);
                if (4 * u * SMALL_NT < n) x[u] = load_four(a.g, first_g + q, l.g_tensor, n - q, true);
            }
#pragma unroll
            for (int u = 0; u < FLAT; ++u) {
                const int q = 4 * (threadIdx.x + u * SMALL_NT);
                if (4 * u * SMALL_NT >= n) continue;
                if (l.muon) {
                    v4f y = load_four(a.mom, first_m + q, TENSOR_F32, n - q, true);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (with_momentum) y[e] = __builtin_fmaf(l.momentum, y[e], x[u][e]);
                        x[u][e] = updated(l, x[u][e], y[e]);
                    }
                    if (with_momentum) store_four(a.mom + first_m + q, y, n - q, true);
                }
                Places at_x(a, q);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sum += (double)x[u][e] * (double)x[u][e];
                    const int p = at_x.next();
                    if (q + e < n) keep(lds, p, x[u][e]);
                }
            }
            return sum;
        }
        rows_of(a, j0, columns, [&](int r, int c, int step, int rows) {
            constexpr int U = ROWS_AT_ONCE;
            float x[U], y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long q = first_g + min(r + u * step, rows - 1) * a.ldg + c;
                x[u] = bf16 ? (float)static_cast<const __bf16 *>(a.g)[q] : static_cast<const float *>(a.g)[q];
            }
            if (l.muon) {
#pragma unroll
                for (int u = 0; u < U; ++u) y[u] = a.mom[first_m + min(r + u * step, rows - 1) * a.ldm + c];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + u * step >= rows) continue;
                if (l.muon) {
                    if (with_momentum) {
                        y[u] = __builtin_fmaf(l.momentum, y[u], x[u]);
                        a.mom[first_m + (r + u * step) * a.ldm + c] = y[u];
                    }
                    x[u] = updated(l, x[u], y[u]);
                }
                sum += (double)x[u] * (double)x[u];
                keep(lds, a.flip ? at(r + u * step, c) : at(c, r + u * step), x[u]);
            }
        });
        return sum;
    }
    // ... and as X, with zeros behind its rows and columns
    static __device__ __forceinline__ void scale_g(unsigned char *lds, const SmallMat &a, int j0, int columns, double inv)
    {
        const int n = (a.flip ? a.rows : a.cols) - j0, m = a.flip ? a.cols : a.rows;
#pragma unroll 1
        for (int item = threadIdx.x; item < columns * CHUNKS; item += SMALL_NT) {
            const int j = item / CHUNKS, i = 8 * (item % CHUNKS), p = at(j, i);
            const v8s up = *reinterpret_cast<const v8s *>(lds + p), down = *reinterpret_cast<const v8s *>(lds + PLANE + p);
            v8h hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __uint_as_float((unsigned)(unsigned short)up[e] << 16 | (unsigned short)down[e]);
                half_t u, w;
                split(j < n && i + e < m ? (float)((double)x * inv) : 0.f, u, w);  // (inv may be inf)
                hi[e] = u;
                lo[e] = w;
            }
            *reinterpret_cast<v8h *>(lds + p) = hi;
            *reinterpret_cast<v8h *>(lds + PLANE + p) = lo;
        }
    }

    // X X^T over the block's columns, a strip each; of several wavefronts with one strip the first has it
    static __device__ __forceinline__ void gram(unsigned char *lds, int columns, Strip &m, int strip, int part, int lane)
    {
#pragma unroll
        for (int i = 0; i < S; ++i) m.v[i] = v4f{0.f, 0.f, 0.f, 0.f};
        const int g4 = lane >> 4, row = (lane & 15) >> 2, col = 4 * (lane & 3);
        for (int k = 32 * part; k < columns; k += 32 * PARTS) {
            // the transposing read: lane 4 r + q of sixteen gives the place of columns 4 q .. of row r, and gets column lane of rows 0 .. 3
            auto read = [&](int plane, int s) {
                v8h f;
                v4s u[2];
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    u[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) v4s *)(lds + plane * PLANE + at(k + 8 * g4 + 4 * t + row, 16 * s + col)));
                __builtin_memcpy(&f, u, sizeof(f));
                return f;
            };
            const v8h hi = read(0, strip), lo = read(1, strip);
#pragma unroll
            for (int i = 0; i < S; ++i) {
                const v8h ph = read(0, i), pl = read(1, i);
                m.v[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, hi, m.v[i], 0, 0, 0);
                m.v[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, lo, m.v[i], 0, 0, 0);
                m.v[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl, hi, m.v[i], 0, 0, 0);
                if (S == 8) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    static __device__ __forceinline__ void add_parts(unsigned char *shared, Strip &m, int strip, int part, int lane)
    {
        if (PARTS == 1) return;
        v4f *const red = reinterpret_cast<v4f *>(shared);
        if (part > 0) {
#pragma unroll
            for (int i = 0; i < S; ++i) red[(((part - 1) * S + strip) * S + i) * 64 + lane] = m.v[i];
        }
        __syncthreads();
        if (part == 0) {
#pragma unroll 1
            for (int q = 0; q < PARTS - 1; ++q)
#pragma unroll
                for (int i = 0; i < S; ++i) m.v[i] += red[((q * S + strip) * S + i) * 64 + lane];
        }
        __syncthreads();
    }

    // A run of steps from step k: A (in `m` of the first wavefronts) to the rows of Q in LDS; returns the step behind it
    static __device__ __forceinline__ int run(const SmallStep *steps, unsigned char *file, Strip &m, int k, int strip, int part, int lane)
    {
        Strip q, p;
        Frag f;
        const bool mine = part == 0;
        auto of = [](const Strip &x) { return [&x](int i, int e) { return x.v[i][e]; }; };
        for (;; ++k) {
            const SmallStep s = steps[k];
            const bool first = k == 0 || steps[k - 1].end != 0, end = __builtin_amdgcn_readfirstlane(s.end) != 0;
            if (mine) {
                put_rows(file, m, s.sa, strip, lane);
                frag_of(m, s.sa, f);
            }
            __syncthreads();
            if (mine) {
                times(file, f, s.c / (s.sa * s.sa), s.c, of(m), p, lane);
#pragma unroll
                for (int i = 0; i < S; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p.v[i][e] = __builtin_fmaf(s.b, m.v[i][e], p.v[i][e]);
                        if (i == strip && 4 * (lane >> 4) + e == (lane & 15)) p.v[i][e] += s.a;
                    }
            }
            __syncthreads();
            if (mine) put_rows(file, p, s.sp, strip, lane);
            __syncthreads();
            if (mine) {
                if (first) {
                    q = p;
                } else {
                    const float before = steps[k - 1].sq;
                    frag_of(q, before, f);
                    times(file, f, 1.f / (s.sp * before), 1.f, of(q), q, lane);
                }
                if (!end) {
                    const float next = steps[k + 1].sa;
                    frag_of(m, s.sa, f);
                    times(file, f, 1.f / (s.sp * s.sa), 1.f, of(m), p, lane);  // P A
                    frag_of(p, next, f);
                    times(file, f, 1.f / (s.sp * next), 1.f, of(p), m, lane);
                }
            }
            __syncthreads();
            if (end) {
                if (mine) put_rows(file, q, s.sq, strip, lane);
                __syncthreads();
                return k + 1;
            }
        }
    }

    // Q X for the block's columns, in its place
    static __device__ __forceinline__ void apply(unsigned char *lds, int columns, float inv_sq, bool last, int wave, int lane)
    {
        const unsigned char *const file = lds + SHARED;
        const int g4 = lane >> 4, c16 = lane & 15;
#pragma unroll 1
        for (int jb = 16 * wave; jb < columns; jb += 16 * SMALL_WAVES) {
            const int j = jb + c16;
            Frag f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v4h hi = {0, 0, 0, 0}, lo = {0, 0, 0, 0};
                    if (2 * ks + h < S) {
                        hi = *reinterpret_cast<const v4h *>(lds + at(j, 32 * ks + 16 * h + 4 * g4));
                        lo = *reinterpret_cast<const v4h *>(lds + PLANE + at(j, 32 * ks + 16 * h + 4 * g4));
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        f.hi[ks][4 * h + e] = hi[e];
                        f.lo[ks][4 * h + e] = lo[e];
                    }
                }
            Strip x;
            times(file, f, inv_sq, 1.f, [&f](int i, int e) { return (float)f.hi[i / 2][4 * (i % 2) + e] + (float)f.lo[i / 2][4 * (i % 2) + e]; }, x, lane);
#pragma unroll
            for (int i = 0; i < S; ++i) {
                v4s hi, lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (last) {  // the two halves of a float
                        const unsigned bits = __float_as_uint(x.v[i][e] * (1.f / SX));
                        hi[e] = (short)(bits >> 16);
                        lo[e] = (short)(bits & 0xffffu);
                    } else {
                        half_t u, w;
                        split(x.v[i][e], u, w);
                        hi[e] = __builtin_bit_cast(short, u);
                        lo[e] = __builtin_bit_cast(short, w);
                    }
                }
                *reinterpret_cast<v4s *>(lds + at(j, 16 * i + 4 * g4)) = hi;
                *reinterpret_cast<v4s *>(lds + PLANE + at(j, 16 * i + 4 * g4)) = lo;
            }
        }
    }

    // the result from there
    static __device__ __forceinline__ void put_out(const unsigned char *lds, const How &l, const SmallMat &a, int j0, int columns)
    {
        const long long first = a.flip ? j0 * a.ldo : j0;
        const bool bf16 = l.out_tensor == TENSOR_BF16;
        if (flat(a, a.ldo, a.begins_out)) {
            const int n = elements(a, j0, columns);
            v4f w[FLAT];
            if (l.muon) {
#pragma unroll
                for (int u = 0; u < FLAT; ++u) {
                    const int q = 4 * (threadIdx.x + u * SMALL_NT);
                    if (4 * u * SMALL_NT < n) w[u] = load_four(a.out, first + q, TENSOR_F32, n - q, true);
                }
            }
#pragma unroll
            for (int u = 0; u < FLAT; ++u) {
                const int q = 4 * (threadIdx.x + u * SMALL_NT);
                if (q >= n) continue;
                Places at_x(a, q);
                v4f o;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = at_x.next();
                    o[e] = q + e < n ? kept(lds, p) : 0.f;
                    if (l.muon) o[e] = __builtin_fmaf(-a.scale, o[e], __builtin_fmaf(-l.decay, w[u][e], w[u][e]));
                }
                if (bf16) {
                    __bf16 *const to = static_cast<__bf16 *>(a.out) + first + q;
                    if (q + 4 <= n) {
                        v4b b;
#pragma unroll
                        for (int e = 0; e < 4; ++e) b[e] = (__bf16)o[e];
                        *reinterpret_cast<v4b *>(to) = b;
                    } else {
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            if (q + e < n) to[e] = (__bf16)o[e];
                    }
                } else {
                    store_four(static_cast<float *>(a.out) + first + q, o, n - q, true);
                }
            }
            return;
        }
        rows_of(a, j0, columns, [&](int r, int c, int step, int rows) {
            constexpr int U = ROWS_AT_ONCE;
            float w[U];
            if (l.muon) {
#pragma unroll
                for (int u = 0; u < U; ++u) w[u] = static_cast<const float *>(a.out)[first + min(r + u * step, rows - 1) * a.ldo + c];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + u * step >= rows) continue;
                const float o = kept(lds, a.flip ? at(r + u * step, c) : at(c, r + u * step));
                const long long q = first + (r + u * step) * a.ldo + c;
                if (bf16) static_cast<__bf16 *>(a.out)[q] = (__bf16)o;
                else static_cast<float *>(a.out)[q] = l.muon ? __builtin_fmaf(-a.scale, o, __builtin_fmaf(-l.decay, w[u], w[u])) : o;
            }
        });
    }
};

__device__ __forceinline__ double factor_of(double sum, float eps) { return (double)SX / (sqrt(sum) + (double)eps); }

template <typename F>
__device__ __forceinline__ int find_small(const SmallArgs &l, int block, F first)
{
    int k = 0;
    while (k + 1 < l.count && block >= first(l.mat[k + 1])) ++k;
    return k;
}

// The arguments of a launch are in the host's memory, and every line of them that is read is a trip there of more than a microsecond: what is needed of them comes
// at once, in front of everything else, and is not read again where it is used
template <typename T>
__device__ __forceinline__ void here(T &x)
{
    asm volatile("" : "+s"(x));
}
__device__ __forceinline__ void args_here(How &l, SmallMat &a)
{
    int flip = a.flip, muon = l.muon, nesterov = l.nesterov;
    here(flip);
    here(muon);
    here(nesterov);
    here(a.rows);
    here(a.cols);
    here(a.scale);
    here(a.g);
    here(a.out);
    here(a.mom);
    here(a.ldg);
    here(a.ldo);
    here(a.ldm);
    here(a.n);
    here(l.g_tensor);
    here(l.out_tensor);
    here(l.momentum);
    here(l.eps);
    here(l.decay);
    a.flip = flip != 0;
    l.muon = muon != 0;
    l.nesterov = nesterov != 0;
}
__device__ __forceinline__ void copy_steps(const SmallArgs &l, SmallStep *steps)
{
    const unsigned *const from = reinterpret_cast<const unsigned *>(l.step);
    for (unsigned i = threadIdx.x; i < sizeof(l.step) / 4; i += SMALL_NT) reinterpret_cast<unsigned *>(steps)[i] = from[i];
}

// over a workgroup, in a fixed order
__device__ __forceinline__ double sum_of_all(double s, double *red, int lane, int wave)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    s = red[0];
#pragma unroll
    for (int i = 1; i < SMALL_WAVES; ++i) s += red[i];
    __syncthreads();
    return s;
}

// A matrix a workgroup, everything in one launch
template <int MP, int NB>
__global__ __launch_bounds__(SMALL_NT) void small_kernel(SmallArgs l)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    __shared__ SmallStep steps[ORTHO_STEPS];
    __shared__ double red[SMALL_WAVES];
    typedef Small<MP, NB> M;
    copy_steps(l, steps);
    SmallMat a = l.mat[blockIdx.x];
    How how = l;
    int count = l.steps;
    args_here(how, a);
    here(count);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), strip = wave % M::S, part = wave / M::S;
    const int columns = (a.n + 31) / 32 * 32;
    const double sum = sum_of_all(M::load_g(lds, how, a, 0, columns, true), red, lane, wave);
    M::scale_g(lds, a, 0, columns, factor_of(sum, how.eps));
    __syncthreads();
    typename M::Strip m;
#pragma unroll 1
    for (int k = 0; k < count;) {
        M::gram(lds, columns, m, strip, part, lane);
        M::add_parts(lds + M::SHARED, m, strip, part, lane);
#pragma unroll
        for (int i = 0; i < M::S; ++i) m.v[i] *= 1.f / (SX * SX);
        k = M::run(steps, lds + M::SHARED, m, k, strip, part, lane);
        M::apply(lds, columns, 1.f / steps[k - 1].sq, k == count, wave, lane);
        __syncthreads();
    }
    M::put_out(lds, how, a, 0, columns);
}

// The sums of a matrix's blocks, added up in their order where the first one's lie, four of them a lane
template <int MP>
__global__ __launch_bounds__(MP < 32 ? 64 : 128) void small_join_kernel(SmallArgs l, unsigned char *ws, int turn)
{
    constexpr int N = MP * MP / 4, NT = MP < 32 ? 64 : 128;
    const int k = blockIdx.x / (N / NT), e = (blockIdx.x - k * (N / NT)) * NT + threadIdx.x, blocks = l.mat[k].blocks;
    v4f *const sums = reinterpret_cast<v4f *>(ws + l.mat[k].part[turn]);
    v4f m = sums[e];
#pragma unroll 8
    for (int b = 1; b < blocks; ++b) m += sums[b * N + e];
    sums[e] = m;
}

__global__ __launch_bounds__(SUM_NT) void small_sum_kernel(SmallArgs l, double *partial)
{
    __shared__ double red[SUM_NT / 64];
    const SmallMat &a = l.mat[find_small(l, blockIdx.x, [](const SmallMat &x) { return x.sum0; })];
    const double s = sum_of_block<SUM_NT>(l, a, blockIdx.x - a.sum0, a.sums, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// A workgroup a block of columns.  from = -1: X from G and the sums of its products; else the run of steps from `from` on (every workgroup makes its Q itself:
// one more launch would take longer), X times Q, and for another run the sums of its products.  turn: which of the sums are read
template <int MP, int NB>
__global__ __launch_bounds__(SMALL_NT) void small_part_kernel(SmallArgs l, unsigned char *ws, const double *partial, int from, int turn, int joined)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    __shared__ SmallStep steps[ORTHO_STEPS];
    __shared__ double red[SMALL_WAVES];
    typedef Small<MP, NB> M;
    const SmallMat &a = l.mat[find_small(l, blockIdx.x, [](const SmallMat &x) { return x.block0; })];
    copy_steps(l, steps);
    const int block = blockIdx.x - a.block0, j0 = block * NB, columns = (min(a.n - j0, NB) + 31) / 32 * 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), strip = wave % M::S, part = wave / M::S;
    __syncthreads();
    half_t *const kept = reinterpret_cast<half_t *>(ws + a.x) + (size_t)block * NB * MP * 2;  // the planes as they are in LDS
    if (from <= 0) {
        M::load_g(lds, l, a, j0, columns, false);
        double s = 0.0;
        for (int i = threadIdx.x; i < a.sums; i += SMALL_NT) s += partial[a.sum0 + i];
        s = sum_of_all(s, red, lane, wave);
        M::scale_g(lds, a, j0, columns, factor_of(s, l.eps));
    } else {
        const int n = columns * (2 * MP) / 16;
        for (int plane = 0; plane < 2; ++plane)
            for (int i = threadIdx.x; i < n; i += SMALL_NT)
                reinterpret_cast<v8h *>(lds + plane * M::PLANE)[i] = reinterpret_cast<const v8h *>(kept + plane * NB * MP)[i];
    }
    typename M::Strip m;
    int k = from;
    if (from >= 0) {
#pragma unroll
        for (int i = 0; i < M::S; ++i) m.v[i] = v4f{0.f, 0.f, 0.f, 0.f};
        const v4f *const sums = reinterpret_cast<const v4f *>(ws + a.part[turn]);
#pragma unroll 2
        for (int b = part; b < (joined ? 1 : a.blocks); b += M::PARTS)
#pragma unroll
            for (int i = 0; i < M::S; ++i) m.v[i] += sums[((b * M::S + strip) * M::S + i) * 64 + lane];
        M::add_parts(lds + M::SHARED, m, strip, part, lane);
#pragma unroll
        for (int i = 0; i < M::S; ++i) m.v[i] *= 1.f / (SX * SX);
        k = M::run(steps, lds + M::SHARED, m, from, strip, part, lane);
        M::apply(lds, columns, 1.f / steps[k - 1].sq, k == l.steps, wave, lane);
        if (k == l.steps) {
            __syncthreads();
            M::put_out(lds, l, a, j0, columns);
            return;
        }
    } else {
        k = 0;
    }
    __syncthreads();
    if (from >= 0) {
        const int n = columns * (2 * MP) / 16;
        for (int plane = 0; plane < 2; ++plane)
            for (int i = threadIdx.x; i < n; i += SMALL_NT)
                reinterpret_cast<v8h *>(kept + plane * NB * MP)[i] = reinterpret_cast<const v8h *>(lds + plane * M::PLANE)[i];
    }
    M::gram(lds, columns, m, strip, part, lane);
    M::add_parts(lds + M::SHARED, m, strip, part, lane);
    if (part == 0) {
        v4f *const sums = reinterpret_cast<v4f *>(ws + a.part[from < 0 ? turn : turn ^ 1]);
#pragma unroll
        for (int i = 0; i < M::S; ++i) sums[((block * M::S + strip) * M::S + i) * 64 + lane] = m.v[i];
    }
}

// ---------------------------------------------------------------- launches
// the passes of a call, for who asks for their times: norms and layouts (small matrices: everything), products
enum { PASS_NORM = 0, PASS_PRODUCT = 1 };

template <typename K, typename... Args>
hipError_t go(K kernel, int blocks, int threads, size_t lds, hipStream_t stream, const LaunchEvents &ev, Args... args)
{
    if (ev.start != nullptr)
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3((unsigned)threads), (unsigned)lds, stream, ev.start, ev.stop, 0, args...);
    else
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3((unsigned)threads), lds, stream, args...);
    return hipGetLastError();
}

long long round_to(long long v, int t) { return (v + t - 1) / t * t; }
size_t aligned(size_t v) { return (v + 255) / 256 * 256; }

struct Tiles {
    int sym, all;  // of the symmetric products, and of those with as many columns as X
    int most() const { return sym > all ? sym : all; }
};

// Time of a product of `tiles` tiles of T x T over the longest k, in us, from what the kernels take for a k-tile of 64 (all planes of it) where a compute unit has a
// workgroup, and where it has two (T = 64: one plane 0.25 and 0.40, two 0.55 and 0.80 us; 128: 0.68, 1.20; 1.70; 256: 1.40; 4.20), and for first loads and
// results: 4, 8, 18.
double product_time(int T, int planes, double tiles, double k_tiles)
{
    const double one = planes == 1 ? (T == 64 ? 0.25 : T == 128 ? 0.68 : 1.40) : T == 64 ? 0.55 : T == 128 ? 1.70 : 4.20;
    const double two = planes == 1 ? (T == 64 ? 0.40 : T == 128 ? 1.20 : 1.40) : T == 64 ? 0.80 : one;
    const double at_once = T == 256 || (T == 128 && planes == 2) ? 256 : 512, rounds = floor(tiles / at_once), rest = tiles - rounds * at_once;
    return k_tiles * (rounds * two + (rest == 0.0 ? 0.0 : rest <= 256 ? one : two)) + (T == 64 ? 4.0 : T == 128 ? 8.0 : 18.0);
}

// Large tiles read less for a product, small ones are more of them.  (4096 x 4096 bf16: sym 64 158, 128 120, 256 120 us, all 249, 165, 147;
// 1000 x 4096: sym 19, 48, 105, all 22.6, 22.4, 43.)
Tiles tiles_for(const OrthoShape *s, int n, int planes)
{
    Tiles best = {64, 64};
    double sym_time = 0.0, all_time = 0.0;
    for (int T : {64, 128, 256}) {
        double sym = 0.0, all = 0.0, m_most = 0.0, n_most = 0.0;
        for (int k = 0; k < n; ++k) {
            const double mt = (double)((s[k].m() + T - 1) / T), nt = (double)((s[k].n() + T - 1) / T);
            sym += mt * (mt + 1) / 2;
            all += mt * nt;
            m_most = fmax(m_most, s[k].m());
            n_most = fmax(n_most, s[k].n());
        }
        const double km = ceil(m_most / BK), kn = ceil(n_most / BK);
        const double ts = product_time(T, planes, sym, kn) + product_time(T, planes, sym, km), ta = product_time(T, planes, all, km);
        if (T == 64 || ts < sym_time) {
            sym_time = ts;
            best.sym = T;
        }
        if (T == 64 || ta < all_time) {
            all_time = ta;
            best.all = T;
        }
    }
    return best;
}

struct Layout {
    size_t partial, end;
    int sums, preps, syms, alls, splits;
    Tiles tiles;
};

Layout lay_out(List &l, const OrthoShape *s, int n, int planes)
{
    l.count = n;
    l.planes = planes;
    const Tiles tiles = tiles_for(s, n, planes);
    Layout y = {};
    y.tiles = tiles;
    size_t at = aligned(sizeof(List));
    y.partial = at;
    at += aligned(sizeof(double) * SUM_BLOCKS * (size_t)n);
    for (int k = 0; k < n; ++k) {
        Mat &a = l.mat[k];
        a.rows = s[k].rows;
        a.cols = s[k].cols;
        a.m = (int)round_to(s[k].m(), BK);
        a.n = (int)round_to(s[k].n(), BK);
        a.mp = (int)round_to(a.m, tiles.most());
        a.np = (int)round_to(a.n, tiles.all);
        const size_t x = 2 * (size_t)a.mp * a.np, sq = 2 * (size_t)a.mp * a.mp;
        for (int i = 0; i < 2; ++i) {
            a.x[i] = at;
            at += planes * x;
            a.xt[i] = at;
            at += 2 * x;
        }
        a.f = at;
        at += planes * sq;
        a.h = at;
        at += planes * sq;
        a.d = at;
        at += sizeof(float) * (size_t)a.mp;
        a.e = at;
        at = aligned(at + sizeof(float) * (size_t)a.mp);
        const long long total = (long long)a.rows * a.cols;
        a.sums = (int)(total >= (long long)SUM_MIN * SUM_BLOCKS ? SUM_BLOCKS : (total + SUM_MIN - 1) / SUM_MIN);
        a.sum0 = y.sums;
        a.prep0 = y.preps;
        a.sym0 = y.syms;
        a.all0 = y.alls;
        const int mt = (a.m + tiles.sym - 1) / tiles.sym;
        y.sums += a.sums;
        y.preps += (a.m / PREP) * (a.n / PREP);
        y.syms += mt * (mt + 1) / 2;
        y.alls += ((a.m + tiles.all - 1) / tiles.all) * ((a.n + tiles.all - 1) / tiles.all);
    }
    // Few tiles over a long k leave most compute units without one: parts of at least 8 k-tiles, where that takes away more than the second launch takes
    // (5 us; 140 x 8192 fp32 358 us without it, 149 with; 300 x 8192 392, 202)
    l.syms = y.syms;
    l.splits = 1;
    l.part = at;
    if (tiles.sym == 64 && y.syms > 0) {
        int nk = 0;
        for (int k = 0; k < n; ++k) nk = l.mat[k].n / BK > nk ? l.mat[k].n / BK : nk;
        const int most = 256 / y.syms < nk / 8 ? 256 / y.syms : nk / 8;
        if (most > 1 && nk * (planes == 1 ? 0.25 : 0.55) * (1.0 - 1.0 / most) > 6.0) {
            l.splits = most;
            at = aligned(at + (size_t)most * y.syms * (64 * 64 * 4));
        }
    }
    y.splits = l.splits;
    y.end = at;
    return y;
}

void describe(How &l, const OrthoSteps &how)
{
    l.g_tensor = how.g_tensor;
    l.out_tensor = how.muon ? (int)TENSOR_F32 : how.out_tensor;
    l.muon = how.muon;
    l.nesterov = how.nesterov;
    l.momentum = how.momentum;
    l.eps = how.eps;
    l.decay = how.lr * how.weight_decay;
}

void describe(Matrix &a, const OrthoMatrix &o, const OrthoShape &s, const OrthoSteps &how)
{
    const size_t size = how.g_tensor == TENSOR_BF16 ? 2 : 4;
    a.rows = s.rows;
    a.cols = s.cols;
    a.flip = s.rows > s.cols;
    a.g = o.g;
    a.ldg = o.ldg;
    a.out = o.out;
    a.ldo = o.ldo;
    a.mom = o.momentum;
    a.ldm = o.ldm;
    a.scale = how.lr * o.scale;
    auto begins = [](const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; };
    const bool two = how.out_tensor == TENSOR_BF16 && !how.muon;
    a.begins_g = begins(o.g, 4 * size);
    a.begins_m = begins(o.momentum, 16);
    a.begins_out = begins(o.out, two ? 8 : 16);
    a.whole_g = a.begins_g && (o.ldg % 4 == 0 || a.rows == 1);
    a.whole_m = a.begins_m && (o.ldm % 4 == 0 || a.rows == 1);
    a.whole_out = begins(o.out, 16) && (o.ldo % (two ? 8 : 4) == 0 || a.rows == 1);
}

template <int T, int PL>
struct Form;
template <int PL>
struct Form<64, PL> {
    static constexpr int WM = 2, WN = 2;
};
template <int PL>
struct Form<128, PL> {
    static constexpr int WM = 2, WN = 2;
};
template <int PL>
struct Form<256, PL> {
    static constexpr int WM = 2, WN = 4;
};

template <int T, int PL, int KIND, int KG = 1>
hipError_t product(int blocks, const List *dl, unsigned char *ws, int from, const float *c, hipStream_t stream, const LaunchEvents &ev)
{
    if constexpr (T == 64 && KG == 1 && KIND != GRAM_JOIN)
        if (blocks <= 256) return product<T, PL, KIND, 2>(blocks, dl, ws, from, c, stream, ev);
    typedef Form<T, PL> F;
    constexpr int S = KG == 2 ? 4 : 2;
    typedef Product<T, F::WM, F::WN, S, PL, KG> P;
    const auto kernel = product_kernel<T, F::WM, F::WN, S, PL, KG, KIND>;
    static LdsGrant grant;
    const hipError_t e = grant_lds(grant, P::LDS, kernel);
    if (e != hipSuccess) return e;
    return go(kernel, blocks, P::NT, P::LDS, stream, ev, dl, ws, from, c[0], c[1], c[2]);
}

template <int KIND>
hipError_t product(int tile, int planes, int blocks, const List *dl, unsigned char *ws, int from, const float *c, hipStream_t stream,
                   const PassEvents &passes)
{
    const LaunchEvents ev = passes(PASS_PRODUCT, 0.0);
    if (planes == 2) {
        if (tile == 256) return product<256, 2, KIND>(blocks, dl, ws, from, c, stream, ev);
        if (tile == 128) return product<128, 2, KIND>(blocks, dl, ws, from, c, stream, ev);
        return product<64, 2, KIND>(blocks, dl, ws, from, c, stream, ev);
    }
    if (tile == 256) return product<256, 1, KIND>(blocks, dl, ws, from, c, stream, ev);
    if (tile == 128) return product<128, 1, KIND>(blocks, dl, ws, from, c, stream, ev);
    return product<64, 1, KIND>(blocks, dl, ws, from, c, stream, ev);
}

template <int KIND>
hipError_t product64(int planes, int blocks, const List *dl, unsigned char *ws, int from, const float *c, hipStream_t stream, const PassEvents &passes)
{
    const LaunchEvents ev = passes(PASS_PRODUCT, 0.0);
    return planes == 2 ? product<64, 2, KIND>(blocks, dl, ws, from, c, stream, ev) : product<64, 1, KIND>(blocks, dl, ws, from, c, stream, ev);
}

hipError_t products(const List *dl, unsigned char *ws, const Layout &y, const OrthoSteps &how, hipStream_t stream, const PassEvents &ev)
{
    hipError_t e = hipSuccess;
    for (int i = 0; i < how.steps && e == hipSuccess; ++i) {
        const float *c = how.coef + 3 * (how.n_coef == 1 ? 0 : i);
        const int from = i & 1, planes = how.products == TENSOR_F32 ? 2 : 1;
        if (y.splits == 1) {
            e = product<GRAM>(y.tiles.sym, planes, y.syms, dl, ws, from, c, stream, ev);
        } else {
            e = product64<GRAM_PART>(planes, y.syms * y.splits, dl, ws, from, c, stream, ev);
            if (e == hipSuccess) e = product64<GRAM_JOIN>(planes, y.syms, dl, ws, from, c, stream, ev);
        }
        if (e == hipSuccess) e = product<SQUARE>(y.tiles.sym, planes, y.syms, dl, ws, from, c, stream, ev);
        if (e != hipSuccess) return e;
        e = i + 1 < how.steps ? product<NEXT>(y.tiles.all, planes, y.alls, dl, ws, from, c, stream, ev)
                              : product<LAST>(y.tiles.all, planes, y.alls, dl, ws, from, c, stream, ev);
    }
    return e;
}

// Runs of steps, and the scales: singular values of X are at most 1 at the start; the largest factor and value of a step are looked for
bool plan_steps(SmallArgs &l, const OrthoSteps &how, int rows)
{
    const double limit = how.products != TENSOR_F32 ? 500.0 : rows > 16 ? 12.0 : 1.0;
    auto scale = [](double most, double cap) {  // a power of two that leaves room to 2^14
        double s = cap;
        while (s > 1.0 && most * s > 16384.0) s *= 0.5;
        return (float)s;
    };
    double top = 1.002, last = top, product = 1.0;  // of the singular values, and before the step; of the factors in a run
    l.steps = how.steps;
    for (int k = 0; k < how.steps; ++k) {
        const float *c = how.coef + 3 * (how.n_coef == 1 ? 0 : k);
        SmallStep &s = l.step[k];
        s.a = c[0];
        s.b = c[1];
        s.c = c[2];
        double most = 0.0, next = 0.0;
        for (int i = 0; i <= 256; ++i) {
            const double x = top * i / 256, p = fabs(c[0] + x * x * (c[1] + x * x * c[2]));
            most = p > most ? p : most;
            next = p * x > next ? p * x : next;
        }
        if (k > 0) {
            l.step[k - 1].end = product * most > limit;
            if (l.step[k - 1].end) product = 1.0;
        }
        product *= most > 1.0 ? most : 1.0;
        s.sa = scale(top * (top > last ? top : last), 4096.0);  // (P A of the step before, too)
        s.sp = scale(most, 4096.0);
        s.sq = scale(product, 4096.0);
        s.end = k + 1 == how.steps;
        last = top;
        top = 1.002 * next;  // (between the places that are looked at)
        if (!(top < 16.0) || most > 8192.0) return false;  // (or X leaves fp16 anyway)
    }
    return true;
}

struct SmallForm {
    int rows, columns;
};
SmallForm small_form(int m)
{
    if (m <= 16) return {16, 1024};
    if (m <= 32) return {32, 1024};
    if (m <= 64) return {64, 512};
    return {128, 128};
}

// The rows of the largest matrix of a call decide; 0: not for it
int small_rows(const OrthoShape *s, int n)
{
    int m = 0;
    for (int k = 0; k < n; ++k) m = s[k].m() > m ? s[k].m() : m;
    return m <= 128 ? small_form(m).rows : 0;
}

struct SmallLayout {
    size_t partial, end;
    int sums, blocks;
    bool one;  // every matrix is one block
};
SmallLayout lay_out_small(SmallArgs &l, const OrthoShape *s, int n, int rows)
{
    const int nb = small_form(rows).columns;
    SmallLayout y = {};
    l.count = n;
    size_t at = 0;
    y.partial = at;
    at += aligned(sizeof(double) * SUM_BLOCKS * (size_t)n);
    y.one = true;
    for (int k = 0; k < n; ++k) {
        SmallMat &a = l.mat[k];
        a.m = s[k].m();
        a.n = s[k].n();
        a.blocks = (int)((a.n + nb - 1) / nb);
        a.block0 = y.blocks;
        y.blocks += a.blocks;
        y.one = y.one && a.blocks == 1;
        const long long total = (long long)s[k].rows * s[k].cols;
        a.sums = (int)(total >= (long long)SUM_MIN * SUM_BLOCKS ? SUM_BLOCKS : (total + SUM_MIN - 1) / SUM_MIN);
        a.sum0 = y.sums;
        y.sums += a.sums;
        a.x = at;
        at = aligned(at + (size_t)a.blocks * nb * rows * 4);
        for (int i = 0; i < 2; ++i) {
            a.part[i] = at;
            at = aligned(at + (size_t)a.blocks * rows * rows * 4);
        }
    }
    y.end = y.one ? 16 : at;
    return y;
}

template <int MP, int NB>
hipError_t small_launches(const SmallArgs &l, const SmallLayout &y, unsigned char *ws, hipStream_t stream, const PassEvents &ev)
{
    typedef Small<MP, NB> M;
    static LdsGrant grant;
    hipError_t e = grant_lds(grant, M::LDS, small_kernel<MP, NB>, small_part_kernel<MP, NB>);
    if (e != hipSuccess) return e;
    if (y.one) return go(small_kernel<MP, NB>, l.count, SMALL_NT, M::LDS, stream, ev(PASS_NORM, 0.0), l);
    double *const partial = reinterpret_cast<double *>(ws + y.partial);
    e = go(small_sum_kernel, y.sums, SUM_NT, 0, stream, ev(PASS_NORM, 0.0), l, partial);
    // every workgroup adds up the blocks' sums itself (64 KB in about 1 us), but for many, which a launch joins (6 us; 100 x 8192 fp32 227 us without it,
    // 138 with; 128 x 4096 172, 131)
    int joined = 0;
    for (int k = 0; k < l.count; ++k) joined = joined || (long long)l.mat[k].blocks * MP * MP * 4 > (512 << 10);
    auto sums_are_there = [&](int turn) {
        constexpr int THREADS = MP < 32 ? 64 : 128;
        return joined ? go(small_join_kernel<MP>, l.count * (MP * MP / 4 / THREADS), THREADS, 0, stream, ev(PASS_PRODUCT, 0.0), l, ws, turn) : hipSuccess;
    };
    if (e == hipSuccess)
        e = go(small_part_kernel<MP, NB>, y.blocks, SMALL_NT, M::LDS, stream, ev(PASS_PRODUCT, 0.0), l, ws, (const double *)partial, -1, 0, joined);
    if (e == hipSuccess) e = sums_are_there(0);
    int turn = 0;
    for (int k = 0; k < l.steps && e == hipSuccess;) {
        e = go(small_part_kernel<MP, NB>, y.blocks, SMALL_NT, M::LDS, stream, ev(PASS_PRODUCT, 0.0), l, ws, (const double *)partial, k, turn, joined);
        while (!l.step[k].end) ++k;
        ++k;
        turn ^= 1;
        if (k < l.steps && e == hipSuccess) e = sums_are_there(turn);
    }
    return e;
}

}  // namespace

size_t ortho_workspace(const OrthoShape *shapes, int n, int products)
{
    size_t most = 0;
    List l;
    const int rows = small_rows(shapes, n);
    for (int k = 0; rows && k < n; k += ORTHO_GROUP) {
        SmallArgs a;
        const size_t b = lay_out_small(a, shapes + k, n - k < ORTHO_GROUP ? n - k : ORTHO_GROUP, rows).end;
        most = b > most ? b : most;
    }
    // (also of small ones: the steps decide, too)
    for (int k = 0; k < n; k += ORTHO_GROUP) {
        const size_t b = lay_out(l, shapes + k, n - k < ORTHO_GROUP ? n - k : ORTHO_GROUP, products == TENSOR_F32 ? 2 : 1).end;
        most = b > most ? b : most;
    }
    return most;
}

// Groups of at most ORTHO_GROUP matrices, one after the other in the same workspace
hipError_t launch_ortho(const OrthoMatrix *list, const OrthoShape *shapes, int n, const OrthoSteps &how, void *ws, hipStream_t stream,
                        const PassEvents &ev)
{
    const int rows = small_rows(shapes, n);
    SmallArgs small = {};
    if (rows && plan_steps(small, how, rows)) {
        describe(small, how);
        for (int k0 = 0; k0 < n; k0 += ORTHO_GROUP) {
            const int count = n - k0 < ORTHO_GROUP ? n - k0 : ORTHO_GROUP;
            const SmallLayout y = lay_out_small(small, shapes + k0, count, rows);
            for (int k = 0; k < count; ++k) describe(small.mat[k], list[k0 + k], shapes[k0 + k], how);
            unsigned char *const w = static_cast<unsigned char *>(ws);
            const hipError_t e = rows == 16   ? small_launches<16, 1024>(small, y, w, stream, ev)
                                 : rows == 32 ? small_launches<32, 1024>(small, y, w, stream, ev)
                                 : rows == 64 ? small_launches<64, 512>(small, y, w, stream, ev)
                                              : small_launches<128, 128>(small, y, w, stream, ev);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    for (int k0 = 0; k0 < n; k0 += ORTHO_GROUP) {
        const int count = n - k0 < ORTHO_GROUP ? n - k0 : ORTHO_GROUP;
        List l = {};
        const Layout y = lay_out(l, shapes + k0, count, how.products == TENSOR_F32 ? 2 : 1);
        describe(l, how);
        for (int k = 0; k < count; ++k) {
            Mat &a = l.mat[k];
            const OrthoMatrix &o = list[k0 + k];
            describe(a, o, shapes[k0 + k], how);
        }
        unsigned char *const w = static_cast<unsigned char *>(ws);
        List *const dl = reinterpret_cast<List *>(w);
        double *const partial = reinterpret_cast<double *>(w + y.partial);
        hipError_t e = go(sum_kernel, y.sums, SUM_NT, 0, stream, ev(PASS_NORM, 0.0), l, dl, partial);
        if (e == hipSuccess) e = go(prep_kernel, y.preps, 256, 0, stream, ev(PASS_NORM, 0.0), (const List *)dl, w, (const double *)partial);
        if (e == hipSuccess) e = products(dl, w, y, how, stream, ev);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace hb
