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
// (A = D + F:  A^2 = F^2 + D F + F D + D^2,  B X = E X + H X).  That leaves 1e-3 (HB_TENSOR_BF16, whose results are rounded to 2^-8 anyway).
// HB_TENSOR_F32 takes the products of high and low parts, too (three products of the four; low times low is 2^-22): the errors are
// those of fp32 products.
// Operands are scaled by powers of two so that neither what they hold nor its low part leaves fp16's range: X by 2^12 (entries are at most the largest
// singular value, 1.2, and around (m n)^-1/2 at the start), A by 2^12, B by 2^10 (entries up to the range of b s^2 + c s^4).
// Everything in the workspace is padded with zeros to whole tiles, which the steps keep zero: no kernel between the first and the last
// has a bounds check.
#include "operators.h"

namespace hb {
namespace {

typedef _Float16 half_t;
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) const void *gptr_t;
typedef __attribute__((address_space(3))) void *lptr_t;

constexpr float SX = 4096.f, SA = 4096.f, SB = 1024.f;
constexpr int BK = 64, ROW_BYTES = 2 * BK;  // a row of an operand tile: one cache line
constexpr int SUM_NT = 256, SUM_BLOCKS = 256, SUM_MIN = 8192;
constexpr int PREP = 64;  // tiles of the kernel that lays X out

// one matrix: what the kernels read of it, in the workspace
struct Mat {
    int m, n, mp, np;         // rows and columns of X, and padded to whole tiles
    int rows, cols, flip;     // of G; X is its transpose
    int sums, sum0;           // blocks of the sum of squares, and the first
    int prep0, sym0, all0;    // first block of the others: X's layout, tiles on and below the diagonal of m x m, tiles of m x n
    size_t x[2], xt[2], f, h; // byte offsets from the workspace: X and X^T (two of each, in turn), A and B; low parts follow
    size_t d, e;              // diagonals of A and B
    const void *g;
    long long ldg;
    void *out;                // the result, or the weights
    long long ldo;
    float *mom;
    long long ldm;
    float scale;              // lr times the matrix's factor
};
struct List {
    int count, tile, planes;
    int g_tensor, out_tensor, step_kind;  // HB_TENSOR_* of G and of the result
    int nesterov;
    float momentum, eps, decay;           // lr weight_decay
    Mat mat[ORTHO_GROUP];
};
enum { PLAIN = 0, MUON = 1 };  // step_kind

__device__ __forceinline__ float load_one(const void *p, long long at, int tensor)
{
    return tensor == TENSOR_BF16 ? (float)static_cast<const __bf16 *>(p)[at] : static_cast<const float *>(p)[at];
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
__device__ __forceinline__ float updated(const List &l, float g, float m_new)
{
    if (l.step_kind == PLAIN) return g;
    return l.nesterov ? __builtin_fmaf(l.momentum, m_new, g) : m_new;
}

// ---------------------------------------------------------------- the norm
// Sums of squares in 64 bits (neither 1e30 nor 1e-30 leaves their range), a fixed part of the rows a block; the momentum on the way.
// The first block puts the list where the other kernels read it: it is longer than what a launch should carry.
__global__ __launch_bounds__(SUM_NT) void sum_kernel(List l, List *to, double *partial)
{
    if (blockIdx.x == 0) {
        const unsigned *from = reinterpret_cast<const unsigned *>(&l);
        for (unsigned i = threadIdx.x; i < sizeof(List) / 4; i += SUM_NT) reinterpret_cast<unsigned *>(to)[i] = from[i];
    }
    const int k = find(l, blockIdx.x, [](const Mat &a) { return a.sum0; });
    const Mat &a = l.mat[k];
    const int b = blockIdx.x - a.sum0;
    const long long total = (long long)a.rows * a.cols;
    double s = 0.0;
    for (long long i = (long long)b * SUM_NT + threadIdx.x; i < total; i += (long long)a.sums * SUM_NT) {
        const long long r = i / a.cols, c = i - r * a.cols;
        float v = load_one(a.g, r * a.ldg + c, l.g_tensor);
        if (l.step_kind == MUON) {
            const float m_new = __builtin_fmaf(l.momentum, a.mom[r * a.ldm + c], v);
            a.mom[r * a.ldm + c] = m_new;
            v = updated(l, v, m_new);
        }
        s += (double)v * (double)v;
    }
    __shared__ double red[SUM_NT / 64];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ void split(float x, half_t &hi, half_t &lo)
{
    hi = (half_t)x;
    lo = (half_t)(x - (float)hi);
}

// ---------------------------------------------------------------- X, X^T from G
__global__ __launch_bounds__(256) void prep_kernel(const List *lp, unsigned char *ws, const double *partial)
{
    const List &l = *lp;
    const int k = find(l, blockIdx.x, [](const Mat &a) { return a.prep0; });
    const Mat &a = l.mat[k];
    __shared__ double red[4];
    __shared__ float tile[PREP][PREP + 1];
    const int tid = threadIdx.x;
    double s = tid < a.sums ? partial[a.sum0 + tid] : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((tid & 63) == 0) red[tid >> 6] = s;
    __syncthreads();
    const double inv = (double)SX / (sqrt((red[0] + red[1]) + (red[2] + red[3])) + (double)l.eps);
    // tile of X: rows i0 .., columns j0 ..; of G the same or exchanged
    const int per_row = a.np / PREP, t = blockIdx.x - a.prep0;
    const int i0 = (t / per_row) * PREP, j0 = (t % per_row) * PREP;
    const int r0 = a.flip ? j0 : i0, c0 = a.flip ? i0 : j0;
    for (int q = tid; q < PREP * PREP; q += 256) {
        const int r = q / PREP, c = q % PREP;
        float v = 0.f;
        if (r0 + r < a.rows && c0 + c < a.cols) {
            v = load_one(a.g, (long long)(r0 + r) * a.ldg + c0 + c, l.g_tensor);
            if (l.step_kind == MUON) v = updated(l, v, a.mom[(long long)(r0 + r) * a.ldm + c0 + c]);
            v = (float)((double)v * inv);
        }
        if (a.flip) tile[c][r] = v;
        else tile[r][c] = v;
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
enum { GRAM = 0, SQUARE = 1, NEXT = 2, LAST = 3 };

// slot of 16-byte chunk c of tile row R: c ^ swz(R), so that the sixteen rows of a fragment read lie on different banks
__device__ __forceinline__ int swz(int R) { return (R >> 1) & 7; }

template <int N>
__device__ __forceinline__ void wait_loads_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// T x T tile of rows times rows, WM x WN wavefronts, S stages of both operands in LDS.
template <int T, int WM, int WN, int S>
struct Product {
    static constexpr int NW = WM * WN, NT = 64 * NW;
    static constexpr int RM = T / WM, RN = T / WN, MB = RM / 16, NB = RN / 16;
    static constexpr int LOADS = T * 8 / NT;  // 16-byte loads a lane and operand tile
    static constexpr int OPERAND = T * ROW_BYTES, STAGE = 2 * OPERAND;
    static constexpr size_t LDS = (size_t)S * STAGE;
    v4f acc[MB][NB];

    // P, Q: first rows of the tile, of `pitch` bytes; segments of nk k-tiles with the offsets (bytes) of their operands
    __device__ __forceinline__ void run(unsigned char *lds, const unsigned char *P, const unsigned char *Q, unsigned pitch, int nk, int segs,
                                        size_t low_p, size_t low_q, int tid)
    {
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wm = wave % WM, wn = wave / WM;
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
        const int total = nk * segs;
        // segment 0: high x high, 1: high x low, 2: low x high
        auto issue = [&](int t, int stage) {
            const int seg = t >= 2 * nk ? 2 : t >= nk ? 1 : 0;
            const size_t k = (size_t)(t - seg * nk) * ROW_BYTES;
            const unsigned char *p = P + (seg == 2 ? low_p : 0) + k, *q = Q + (seg == 1 ? low_q : 0) + k;
            unsigned char *to = lds + stage * STAGE;
#pragma unroll
            for (int v = 0; v < LOADS; ++v) {
                __builtin_amdgcn_global_load_lds((gptr_t)(p + off[v]), (lptr_t)(to + (wave + NW * v) * 1024), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((gptr_t)(q + off[v]), (lptr_t)(to + OPERAND + (wave + NW * v) * 1024), 16, 0, 0);
            }
        };
#pragma unroll
        for (int t = 0; t < S - 1; ++t)
            if (t < total) issue(t, t);
        const int c16 = lane & 15, g4 = lane >> 4;
        const int p_off = (wm * RM + c16) * ROW_BYTES + ((g4 ^ swz(c16)) << 4);
        const int q_off = OPERAND + (wn * RN + c16) * ROW_BYTES + ((g4 ^ swz(c16)) << 4);
        int stage = 0;
        for (int t = 0; t < total; ++t) {
            // tile t has landed, and everybody is done with tile t - 1
            if (t + S - 2 < total) wait_loads_and_meet<2 * LOADS *(S - 2)>();
            else wait_loads_and_meet<0>();
            if (t + S - 1 < total) issue(t + S - 1, stage == 0 ? S - 1 : stage - 1);
            const unsigned char *at = lds + stage * STAGE;
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                v8h fp[MB], fq[NB];
#pragma unroll
                for (int i = 0; i < MB; ++i) fp[i] = *reinterpret_cast<const v8h *>(at + (p_off ^ (kk << 6)) + i * 16 * ROW_BYTES);
#pragma unroll
                for (int j = 0; j < NB; ++j) fq[j] = *reinterpret_cast<const v8h *>(at + (q_off ^ (kk << 6)) + j * 16 * ROW_BYTES);
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[i], fq[j], acc[i][j], 0, 0, 0);
            }
            stage = stage == S - 1 ? 0 : stage + 1;
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

// 4 values of a row: high parts, and low ones `low` elements further on
__device__ __forceinline__ v4f load4(const half_t *p, size_t low, bool two)
{
    const v4h hi = *reinterpret_cast<const v4h *>(p);
    v4f x = {(float)hi[0], (float)hi[1], (float)hi[2], (float)hi[3]};
    if (two) {
        const v4h lo = *reinterpret_cast<const v4h *>(p + low);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += (float)lo[e];
    }
    return x;
}

template <int T, int WM, int WN, int S, int KIND>
__global__ __launch_bounds__(64 * WM *WN) void product_kernel(const List *lp, unsigned char *ws, int from, float ca, float cb, float cc)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    typedef Product<T, WM, WN, S> P;
    const List &l = *lp;
    constexpr bool SYM = KIND == GRAM || KIND == SQUARE;
    const int k = find(l, blockIdx.x, [](const Mat &a) { return SYM ? a.sym0 : a.all0; });
    const Mat &a = l.mat[k];
    const int t = blockIdx.x - (SYM ? a.sym0 : a.all0);
    int ti, tj;
    if (SYM) {
        ti = triangle_row(t);
        tj = t - ti * (ti + 1) / 2;
    } else {
        const int per_row = a.np / T;
        ti = t / per_row;
        tj = t - ti * per_row;
    }
    const int i0 = ti * T, j0 = tj * T, planes = l.planes;
    const size_t xlow = (size_t)a.mp * a.np, alow = (size_t)a.mp * a.mp;
    const int tid = threadIdx.x;
    P p;
    {
        const unsigned char *x = ws + (KIND == GRAM ? a.x[from] : KIND == SQUARE ? a.f : a.h);
        const unsigned char *y = KIND == GRAM || KIND == SQUARE ? x : ws + a.xt[from];
        const unsigned pitch = 2u * (unsigned)(KIND == GRAM ? a.np : a.mp);
        const int nk = ((KIND == GRAM ? a.n : a.m) + BK - 1) / BK;
        p.run(lds, x + (size_t)i0 * pitch, y + (size_t)j0 * pitch, pitch, nk, planes == 2 ? 3 : 1, 2 * (KIND == GRAM ? xlow : alow),
              2 * (SYM ? (KIND == GRAM ? xlow : alow) : xlow), tid);
    }
    // lane 16 g + c of a 16 x 16 block: column c, rows 4 g .. 4 g + 3
    const int lane = tid & 63, wave = tid >> 6;
    const int wi = i0 + (wave % WM) * P::RM + 4 * (lane >> 4), wj = j0 + (wave / WM) * P::RN + (lane & 15);
    float *const D = reinterpret_cast<float *>(ws + a.d), *const E = reinterpret_cast<float *>(ws + a.e);
    const half_t *const F = reinterpret_cast<const half_t *>(ws + a.f);
#pragma unroll
    for (int bj = 0; bj < P::NB; ++bj) {
        const int j = wj + 16 * bj;
        const float dj = KIND == SQUARE ? D[j] : 0.f;
#pragma unroll
        for (int bi = 0; bi < P::MB; ++bi) {
            const int i = wi + 16 * bi;
            v4f v = p.acc[bi][bj];
            if (KIND == GRAM) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (i + e == j) {
                        D[j] = v[e] * (1.f / (SX * SX));
                        v[e] = 0.f;
                    } else {
                        v[e] *= SA / (SX * SX);
                    }
                }
            } else if (KIND == SQUARE) {
                const v4f f = load4(F + (size_t)j * a.mp + i, alow, planes == 2);
                const v4f di = *reinterpret_cast<const v4f *>(D + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float sq = v[e] * (1.f / (SA * SA)), fe = f[e] * (1.f / SA);
                    if (i + e == j) {
                        E[j] = __builtin_fmaf(cc, __builtin_fmaf(dj, dj, sq), cb * dj);
                        v[e] = 0.f;
                    } else {
                        v[e] = SB * __builtin_fmaf(cc, __builtin_fmaf(di[e] + dj, fe, sq), cb * fe);
                    }
                }
            } else {
                const v4f x = load4(reinterpret_cast<const half_t *>(ws + a.xt[from]) + (size_t)j * a.mp + i, xlow, true);
                const v4f ei = *reinterpret_cast<const v4f *>(E + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(ca + ei[e], x[e], v[e] * (1.f / SB));
            }
            if (KIND == LAST) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = a.flip ? j : i + e, c = a.flip ? i + e : j;
                    if (r < a.rows && c < a.cols) {
                        const long long at = (long long)r * a.ldo + c;
                        const float o = v[e] * (1.f / SX);
                        if (l.step_kind == MUON) {
                            float *const w = static_cast<float *>(a.out) + at;
                            *w = __builtin_fmaf(-a.scale, o, __builtin_fmaf(-l.decay, *w, *w));
                        } else if (l.out_tensor == TENSOR_BF16) {
                            static_cast<__bf16 *>(a.out)[at] = (__bf16)o;
                        } else {
                            static_cast<float *>(a.out)[at] = o;
                        }
                    }
                }
                continue;
            }
            v4h hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                half_t u, w;
                split(v[e], u, w);
                hi[e] = u;
                lo[e] = w;
            }
            if (SYM) {
                half_t *const to = reinterpret_cast<half_t *>(ws + (KIND == GRAM ? a.f : a.h));
                *reinterpret_cast<v4h *>(to + (size_t)j * a.mp + i) = hi;
                if (planes == 2) *reinterpret_cast<v4h *>(to + alow + (size_t)j * a.mp + i) = lo;
                if (ti != tj) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        to[(size_t)(i + e) * a.mp + j] = hi[e];
                        if (planes == 2) to[alow + (size_t)(i + e) * a.mp + j] = lo[e];
                    }
                }
            } else {
                half_t *const xt = reinterpret_cast<half_t *>(ws + a.xt[from ^ 1]), *const x = reinterpret_cast<half_t *>(ws + a.x[from ^ 1]);
                *reinterpret_cast<v4h *>(xt + (size_t)j * a.mp + i) = hi;
                *reinterpret_cast<v4h *>(xt + xlow + (size_t)j * a.mp + i) = lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[(size_t)(i + e) * a.np + j] = hi[e];
                    if (planes == 2) x[xlow + (size_t)(i + e) * a.np + j] = lo[e];
                }
            }
        }
    }
}

// ---------------------------------------------------------------- launches
long long round_to(long long v, int t) { return (v + t - 1) / t * t; }
size_t aligned(size_t v) { return (v + 255) / 256 * 256; }

// Tile size of a call
int tile_of(const OrthoShape *s, int n)
{
    double best = 0.0;
    int tile = 64;
    for (int t : {64, 128, 256}) {
        double cost = 0.0, sym = 0.0, all = 0.0, depth = 0.0;
        for (int k = 0; k < n; ++k) {
            const double mt = (double)round_to(s[k].m(), t) / t, nt = (double)round_to(s[k].n(), t) / t;
            sym += mt * (mt + 1) / 2;
            all += mt * nt;
            depth = depth > (double)s[k].n() ? depth : (double)s[k].n();
        }
        cost = (2 * ceil(sym / 256) + ceil(all / 256)) * t * t;
        if (t == 64 || cost < best) {
            best = cost;
            tile = t;
        }
    }
    return tile;
}

struct Layout {
    size_t partial, end;
    int sums, preps, syms, alls;
};

Layout lay_out(List &l, const OrthoShape *s, int n, int planes)
{
    l.count = n;
    l.planes = planes;
    l.tile = tile_of(s, n);
    Layout y = {};
    size_t at = aligned(sizeof(List));
    y.partial = at;
    at += aligned(sizeof(double) * SUM_BLOCKS * (size_t)n);
    for (int k = 0; k < n; ++k) {
        Mat &a = l.mat[k];
        a.rows = s[k].rows;
        a.cols = s[k].cols;
        a.flip = s[k].rows > s[k].cols;
        a.m = s[k].m();
        a.n = s[k].n();
        a.mp = (int)round_to(a.m, l.tile);
        a.np = (int)round_to(a.n, l.tile);
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
        const int mt = a.mp / l.tile, nt = a.np / l.tile;
        y.sums += a.sums;
        y.preps += (a.mp / PREP) * (a.np / PREP);
        y.syms += mt * (mt + 1) / 2;
        y.alls += mt * nt;
    }
    y.end = at;
    return y;
}

template <int T, int WM, int WN, int S>
hipError_t products(const List *dl, unsigned char *ws, const Layout &y, const OrthoSteps &how, hipStream_t stream)
{
    typedef Product<T, WM, WN, S> P;
    static LdsGrant grant;
    hipError_t e = grant_lds(grant, P::LDS, product_kernel<T, WM, WN, S, GRAM>, product_kernel<T, WM, WN, S, SQUARE>,
                             product_kernel<T, WM, WN, S, NEXT>, product_kernel<T, WM, WN, S, LAST>);
    for (int i = 0; i < how.steps && e == hipSuccess; ++i) {
        const float *c = how.coef + 3 * (how.n_coef == 1 ? 0 : i);
        const int from = i & 1;
        hipLaunchKernelGGL((product_kernel<T, WM, WN, S, GRAM>), dim3(y.syms), dim3(P::NT), P::LDS, stream, dl, ws, from, c[0], c[1], c[2]);
        hipLaunchKernelGGL((product_kernel<T, WM, WN, S, SQUARE>), dim3(y.syms), dim3(P::NT), P::LDS, stream, dl, ws, from, c[0], c[1], c[2]);
        if (i + 1 < how.steps)
            hipLaunchKernelGGL((product_kernel<T, WM, WN, S, NEXT>), dim3(y.alls), dim3(P::NT), P::LDS, stream, dl, ws, from, c[0], c[1], c[2]);
        else
            hipLaunchKernelGGL((product_kernel<T, WM, WN, S, LAST>), dim3(y.alls), dim3(P::NT), P::LDS, stream, dl, ws, from, c[0], c[1], c[2]);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

size_t ortho_workspace(const OrthoShape *shapes, int n, int products)
{
    size_t most = 0;
    List l;
    for (int k = 0; k < n; k += ORTHO_GROUP) {
        const size_t b = lay_out(l, shapes + k, n - k < ORTHO_GROUP ? n - k : ORTHO_GROUP, products == TENSOR_F32 ? 2 : 1).end;
        most = b > most ? b : most;
    }
    return most;
}

// Groups of at most ORTHO_GROUP matrices, one after the other in the same workspace
hipError_t launch_ortho(const OrthoMatrix *list, const OrthoShape *shapes, int n, const OrthoSteps &how, void *ws, hipStream_t stream)
{
    for (int k0 = 0; k0 < n; k0 += ORTHO_GROUP) {
        const int count = n - k0 < ORTHO_GROUP ? n - k0 : ORTHO_GROUP;
        List l = {};
        const Layout y = lay_out(l, shapes + k0, count, how.products == TENSOR_F32 ? 2 : 1);
        l.g_tensor = how.g_tensor;
        l.out_tensor = how.out_tensor;
        l.step_kind = how.muon ? MUON : PLAIN;
        l.nesterov = how.nesterov;
        l.momentum = how.momentum;
        l.eps = how.eps;
        l.decay = how.lr * how.weight_decay;
        for (int k = 0; k < count; ++k) {
            Mat &a = l.mat[k];
            const OrthoMatrix &o = list[k0 + k];
            a.g = o.g;
            a.ldg = o.ldg;
            a.out = o.out;
            a.ldo = o.ldo;
            a.mom = o.momentum;
            a.ldm = o.ldm;
            a.scale = how.lr * o.scale;
        }
        unsigned char *const w = static_cast<unsigned char *>(ws);
        List *const dl = reinterpret_cast<List *>(w);
        double *const partial = reinterpret_cast<double *>(w + y.partial);
        hipLaunchKernelGGL(sum_kernel, dim3(y.sums), dim3(SUM_NT), 0, stream, l, dl, partial);
        hipLaunchKernelGGL(prep_kernel, dim3(y.preps), dim3(256), 0, stream, dl, w, partial);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (l.tile == 256) e = products<256, 2, 4, 2>(dl, w, y, how, stream);
        else if (l.tile == 128) e = products<128, 2, 2, 2>(dl, w, y, how, stream);
        else e = products<64, 2, 2, 4>(dl, w, y, how, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace hb
