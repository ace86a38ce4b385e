// Log-probabilities of chosen classes, and the losses that start from them: the clipped policy loss with a KL term and the
// preference loss over paired log ratios, with their gradients in the logits.
//
// Row z of K logits, chosen class y.  With m = max z, o = sum over k != y of exp(z_k - m), e = exp(z_y - m), s = o + e:
//     lp = log softmax(z)_y = -log(1 + o / e),   p_k = exp(z_k - m) / s,   1 - p_y = o / s,
//     d lp / d z_k = [k = y] - p_k.
// The chosen class is kept out of the sum o, so that lp and 1 - p_y of a choice that is all but certain keep their digits
// (s - e would cancel).  Exponentials and their sums are fp32, what is computed once per row is in 64 bits.
#include "operators.h"

namespace hb {
namespace {

constexpr int NT = 256;
constexpr int MAX_SUM_BLOCKS = 1024;  // blocks that leave partial sums of a loss, at most
constexpr int MAX_CHUNKED = 2048;     // (row, chunk) pairs of the calls that split their rows, at most

// ---------------------------------------------------------------- rows in memory
// A 16-byte piece of a row, as it is stored: four values, or eight of two bytes.
template <typename T>
struct Piece {
    static constexpr int V = 16 / sizeof(T);
    unsigned w[4];
    __device__ __forceinline__ float get(int e) const
    {
        if (sizeof(T) == 4) return __uint_as_float(w[e]);
        return __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
    __device__ __forceinline__ void set(int e, T v)
    {
        if constexpr (sizeof(T) == 4) {
            w[e] = __float_as_uint(v);
        } else {
            const unsigned h = __builtin_bit_cast(unsigned short, v);
            w[e >> 1] = (e & 1) ? (w[e >> 1] & 0xffffu) | h << 16 : (w[e >> 1] & 0xffff0000u) | h;
        }
    }
    __device__ __forceinline__ void set_none()
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    }
    // Between two passes over pieces in registers: what the first has made of them (eight floats of four words) is made
    // again in the second, not kept.
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(w[i]));
    }
    // without element y of the row, where the piece begins with element j0
    __device__ __forceinline__ void drop(int j0, int y)
    {
        if ((unsigned)(y - j0) < (unsigned)V) {
            const int at = y - j0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (sizeof(T) == 4) {
                    w[i] = i == at ? 0xff800000u : w[i];
                } else {
                    const unsigned low = (w[i] & 0xffff0000u) | 0xff80u, high = (w[i] & 0xffffu) | 0xff800000u;
                    w[i] = 2 * i == at ? low : 2 * i + 1 == at ? high : w[i];
                }
            }
        }
    }
};

// The pieces of a row begin at 16-byte boundaries in memory: piece p has the elements p * V - lead .. + V, the first and
// the last may be cut by the row's ends.
template <typename T>
struct Row {
    static constexpr int V = Piece<T>::V;
    const T *z;
    int K, lead, pieces;
    __device__ __forceinline__ Row(const void *Z, long long ld, long long row, int K_)
        : z(static_cast<const T *>(Z) + row * ld), K(K_)
    {
        lead = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
        pieces = (K + lead + V - 1) / V;
    }
    __device__ __forceinline__ int first(int piece) const { return piece * V - lead; }
    // what is outside of the row reads as -inf
    __device__ __forceinline__ Piece<T> load(int j0) const
    {
        Piece<T> t;
        if (j0 >= 0 && j0 + V <= K) {
            const uint4 u = *reinterpret_cast<const uint4 *>(z + j0);
            t.w[0] = u.x, t.w[1] = u.y, t.w[2] = u.z, t.w[3] = u.w;
        } else {
            t.set_none();
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (j0 + e >= 0 && j0 + e < K) t.set(e, z[j0 + e]);
        }
        return t;
    }
};

// V elements of a row of dZ from j0 on, those in [0, K)
template <typename T, int V>
__device__ __forceinline__ void store(T *dz, int j0, int K, const float *x)
{
    if (j0 >= 0 && j0 + V <= K) {
        T t[V];
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = T(x[e]);
        __builtin_memcpy(dz + j0, t, sizeof(t));
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (j0 + e >= 0 && j0 + e < K) dz[j0 + e] = T(x[e]);
    }
}

__device__ __forceinline__ float logit(const ChoiceRows &r, long long row, int k)
{
    const long long i = row * r.ldz + k;
    return r.tensor == TENSOR_BF16 ? (float)static_cast<const __bf16 *>(r.Z)[i] : static_cast<const float *>(r.Z)[i];
}

__device__ __forceinline__ bool has_choice(const ChoiceRows &r, long long row)
{
    const int y = r.y[row];
    return y >= 0 && y < r.K && (r.weight == nullptr || r.weight[row] != 0.f);
}

// exp(t).  Of log2 e = 1.4426950 + 1.9e-8 the second part matters in sums: without it every term is too small by 1.3e-8 |t|
// relative, all in one direction, which the log-probabilities of a sequence add up.
__device__ __forceinline__ float exp_for_sum(float t)
{
    return __builtin_amdgcn_exp2f(__builtin_fmaf(t, 0x1.715476p+0f, t * 0x1.4ae0cp-26f));
}

// log(s) for a positive s, in two parts whose sum is off by less than 2^-23: of s = 2^k f, f in [1/2, 1), the first is k times the
// leading bits of log 2 (exact), the second, at most 1, the rest.
struct TwoLog {
    float hi, lo;
};
__device__ __forceinline__ TwoLog two_log(float s)
{
    const int k = __builtin_amdgcn_frexp_expf(s);
    const float f = __builtin_amdgcn_frexp_mantf(s);
    return {(float)k * 0.693359375f, __builtin_fmaf((float)k, -2.12194440e-4f, __logf(f))};
}

// exp(d) - 1 - d, to a few roundings where d is small, too: d^2 times a series
__device__ __forceinline__ float kl_of(float d, float em /* exp(d) - 1 */)
{
    if (fabsf(d) < 0.5f) {
        float c = 1.f / 40320.f;
        c = __builtin_fmaf(c, d, 1.f / 5040.f);
        c = __builtin_fmaf(c, d, 1.f / 720.f);
        c = __builtin_fmaf(c, d, 1.f / 120.f);
        c = __builtin_fmaf(c, d, 1.f / 24.f);
        c = __builtin_fmaf(c, d, 1.f / 6.f);
        c = __builtin_fmaf(c, d, 0.5f);
        return d * d * c;
    }
    return em == INFINITY ? INFINITY : em - d;
}

// ---------------------------------------------------------------- what a row comes down to
// part: the row takes part.  One without a choice has lp = lse = 0, one whose logits are all -inf has -inf.
struct RowTerms {
    bool part;
    float top;               // the maximum, 0 where that is -inf
    float inv_sum, others;   // 1 / s, 1 - p_y
    double lp, lse;          // log-probability, log of the sum of exponentials: off by 1e-7 beside what s is
};

// zy: the chosen logit; top: the maximum; o: the sum over the others of exp(z - top) (z itself where top = -inf).
// 64-bit additions, but no function of 64 bits: those would take more registers than the rows do.
__device__ __forceinline__ RowTerms finish_row(float zy, float top, float o)
{
    RowTerms t = {false, 0.f, 0.f, 0.f, 0.0, 0.0};
    if (top == -INFINITY && o == 0.f && zy == zy) {  // NaN in o or zy: no maximum either, but a row that takes part
        t.lp = t.lse = -INFINITY;
        return t;
    }
    t.part = true;
    t.top = top == -INFINITY ? 0.f : top;
    const float e = exp_for_sum(zy - t.top), s = o + e;
    const TwoLog l = two_log(s);
    t.inv_sum = 1.f / s;
    t.others = o * t.inv_sum;
    t.lse = (double)t.top + (double)l.hi + (double)l.lo;
    t.lp = o < e ? -(double)log1pf(o / e) : (double)zy - t.lse;
    return t;
}

// The gradient of a row: dz_k = scale * exp(z_k - base) for k != y and `chosen` for k = y; all zero where both are
struct RowCoef {
    float base, scale, chosen, pad;
};

struct Four {
    double v[4];
};
__device__ __forceinline__ Four add_four(const Four &a, const Four &b)
{
    Four s;
#pragma unroll
    for (int i = 0; i < 4; ++i) s.v[i] = a.v[i] + b.v[i];
    return s;
}
// stats = sum of n partial sums in a fixed order
struct SumFour {
    const Four *partial;
    int n;  // 0: nothing to do
    float *stats;
};

// What is done with a row's terms
enum { HEAD_LOGPROB, HEAD_TERMS, HEAD_POLICY };
struct RowHead {
    int kind;
    float *logp, *lse;  // LOGPROB: results (lse may be null).  POLICY: in p
    double *row_lp;     // TERMS: 0 where a row takes no part
    RowCoef *coef;      // TERMS: {top, 1 / s, 1 - p_y}.  POLICY: null, or the gradient's coefficients
    PolicyTerms p;
};

__device__ __forceinline__ RowCoef head_row(const RowHead &h, const ChoiceRows &r, long long row, const RowTerms &t, bool write,
                                            Four &sums)
{
    RowCoef c = {0.f, 0.f, 0.f, 0.f};
    if (h.kind == HEAD_LOGPROB) {
        if (write) {
            h.logp[row] = (float)t.lp;
            if (h.lse) h.lse[row] = (float)t.lse;
        }
        return c;
    }
    if (h.kind == HEAD_TERMS) {
        if (write) {
            h.row_lp[row] = t.part ? t.lp : 0.0;
            if (h.coef) h.coef[row] = RowCoef{t.top, t.inv_sum, t.others, 0.f};
        }
        return c;
    }
    const PolicyTerms &p = h.p;
    if (t.part) {
        const float A = p.adv[row];
        float pg = 0.f, g = 0.f, kl = 0.f;
        bool cut = false;
        if (A != 0.f) {  // (NaN too); without an advantage the ratio does not matter, however large
            const float ratio = expf((float)(t.lp - (double)p.old_logp[row]));
            const float lo = 1.f - p.clip_low, hi = 1.f + p.clip_high;
            cut = (A > 0.f && ratio > hi) || (A < 0.f && ratio < lo);
            pg = cut ? -(A > 0.f ? hi : lo) * A : -ratio * A;
            g = cut ? 0.f : pg;
        }
        if (p.ref_logp) {
            const float d = (float)((double)p.ref_logp[row] - t.lp), em = expm1f(d);
            kl = kl_of(d, em);
            if (p.kl_coef != 0.f) g -= p.kl_coef * em;
        }
        const float w = r.weight ? r.weight[row] : p.uniform;
        if (write) {
            const double pgw = (double)w * pg, klw = (double)w * kl;
            sums = add_four(sums, Four{{p.kl_coef != 0.f ? pgw + (double)p.kl_coef * klw : pgw, pgw, klw, cut ? (double)w : 0.0}});
        }
        g *= w;
        c.base = t.top;
        c.scale = -g * t.inv_sum;
        c.chosen = g * t.others;
    }
    if (write) {
        if (p.logp) p.logp[row] = (float)t.lp;
        if (h.coef) h.coef[row] = c;
    }
    return c;
}

__device__ __forceinline__ Four sum_block(Four s, Four *red /* a wavefront each */)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s.v[i] += __shfl_xor(s.v[i], o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    s = red[0];
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) s = add_four(s, red[w]);
    return s;
}

__device__ __forceinline__ void store_stats(float *stats, const Four &s)
{
    if (threadIdx.x == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) stats[i] = (float)s.v[i];
}

__device__ __forceinline__ void sum_four(const SumFour &f, Four *red)
{
    Four s = {};
    for (int i = threadIdx.x; i < f.n; i += blockDim.x) s = add_four(s, f.partial[i]);
    store_stats(f.stats, sum_block(s, red));
}

__global__ __launch_bounds__(NT) void sum_four_kernel(SumFour f)
{
    __shared__ Four red[NT / 64];
    sum_four(f, red);
}

// ---------------------------------------------------------------- whole rows in registers
struct RowsArgs {
    ChoiceRows r;
    RowHead h;
    ChoiceGrad d;   // POLICY
    Four *sums;     // POLICY: one a block, or with one block ...
    float *stats;   // ... the statistics themselves
};

// G lanes have a row between them, N pieces each: it is read once, whole, for the maximum, the sum and the gradient.
template <typename T, typename TO, int G, int N>
__global__ __launch_bounds__(G > NT ? G : NT) void rows_kernel(RowsArgs a)
{
    constexpr int V = Piece<T>::V, THREADS = G > NT ? G : NT, WAVES = THREADS / 64, ROWS = THREADS / G;
    __shared__ float red_top[WAVES], red_sum[WAVES];
    __shared__ RowCoef red_coef;
    __shared__ Four red_four[WAVES];
    const int g = threadIdx.x % G;
    Four sums = {};
    for (long long row = (long long)blockIdx.x * ROWS + threadIdx.x / G; row < a.r.B; row += (long long)gridDim.x * ROWS) {
        const Row<T> z(a.r.Z, a.r.ldz, row, a.r.K);
        const int y = a.r.y[row];
        const bool choice = has_choice(a.r, row);
        Piece<T> x[N];
        RowCoef c = {0.f, 0.f, 0.f, 0.f};
        RowTerms t = {false, 0.f, 0.f, 0.f, 0.0, 0.0};
        if (choice) {
            const float zy = logit(a.r, row, y);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = z.load(z.first(i * G + g));
            float top = zy;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i].drop(z.first(i * G + g), y);
#pragma unroll
                for (int e = 0; e < V; ++e) top = fmaxf(top, x[i].get(e));
            }
#pragma unroll
            for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
            if (G > 64) {
                if ((threadIdx.x & 63) == 0) red_top[threadIdx.x >> 6] = top;
                __syncthreads();
                top = red_top[0];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) top = fmaxf(top, red_top[w]);
            }
            const float ref = top == -INFINITY ? 0.f : top;
            float o4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i].forget();
#pragma unroll
                for (int e = 0; e < V; ++e) o4[e & 3] += exp_for_sum(x[i].get(e) - ref);
            }
            float others = (o4[0] + o4[1]) + (o4[2] + o4[3]);
#pragma unroll
            for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1) others += __shfl_xor(others, o, 64);
            if (G <= 64) {
                t = finish_row(zy, top, others);
                c = head_row(a.h, a.r, row, t, g == 0, sums);
            } else {
                if ((threadIdx.x & 63) == 0) red_sum[threadIdx.x >> 6] = others;
                __syncthreads();
                if (threadIdx.x < 64) {
                    others = red_sum[0];
#pragma unroll
                    for (int w = 1; w < WAVES; ++w) others += red_sum[w];
                    t = finish_row(zy, top, others);
                    c = head_row(a.h, a.r, row, t, g == 0, sums);
                    if (threadIdx.x == 0) red_coef = c;
                }
                __syncthreads();
                c = red_coef;
            }
        } else if (g == 0) {
            head_row(a.h, a.r, row, t, true, sums);
        }
        if (a.d.dZ) {
            TO *dz = static_cast<TO *>(a.d.dZ) + row * a.d.ld;
            const bool none = c.scale == 0.f && c.chosen == 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int j0 = z.first(i * G + g);
                if (j0 >= a.r.K) break;
                float out[V];
                if (none) {
#pragma unroll
                    for (int e = 0; e < V; ++e) out[e] = 0.f;
                } else {
                    x[i].forget();
#pragma unroll
                    for (int e = 0; e < V; ++e) out[e] = c.scale * __expf(x[i].get(e) - c.base);
                    if ((unsigned)(y - j0) < (unsigned)V)
#pragma unroll
                        for (int e = 0; e < V; ++e) out[e] = e == y - j0 ? c.chosen : out[e];
                }
                store<TO, V>(dz, j0, a.r.K, out);
            }
            for (int j = a.r.K + g; j < a.d.pad; j += G) dz[j] = TO(0.f);
        }
    }
    if (a.h.kind == HEAD_POLICY) {
        sums = sum_block(sums, red_four);
        if (a.stats) store_stats(a.stats, sums);
        else if (threadIdx.x == 0) a.sums[blockIdx.x] = sums;
    }
}

// ---------------------------------------------------------------- rows in chunks
// A running maximum and the sum of exponentials under it.  top = -inf: nothing but -inf so far (sum 0), or NaN (sum NaN)
struct TopSum {
    float top, sum;
};

__device__ __forceinline__ float under(float x, float top) { return exp_for_sum(x - (top == -INFINITY ? 0.f : top)); }

__device__ __forceinline__ TopSum join(TopSum a, TopSum b)
{
    const float top = fmaxf(a.top, b.top);
    return {top, a.sum * under(a.top, top) + b.sum * under(b.top, top)};
}

// Without the chosen class.
template <typename T>
__global__ __launch_bounds__(NT) void row_sums_kernel(ChoiceRows r, int chunks, int pieces_per_chunk, TopSum *partial)
{
    constexpr int V = Piece<T>::V, U = 4;
    __shared__ TopSum red[NT / 64];
    const long long row = blockIdx.x / chunks;
    const int c = blockIdx.x % chunks;
    if (!has_choice(r, row)) return;
    const Row<T> z(r.Z, r.ldz, row, r.K);
    const int y = r.y[row], end = min(z.pieces, (c + 1) * pieces_per_chunk);
    TopSum t = {-INFINITY, 0.f};
    for (int p = c * pieces_per_chunk + (int)threadIdx.x; p < end; p += U * NT) {
        Piece<T> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * NT < end) x[u] = z.load(z.first(p + u * NT));
            else x[u].set_none();
        }
        float top = t.top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u].drop(z.first(p + u * NT), y);
#pragma unroll
            for (int e = 0; e < V; ++e) top = fmaxf(top, x[u].get(e));
        }
        const float ref = top == -INFINITY ? 0.f : top;
        float o = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) o += exp_for_sum(x[u].get(e) - ref);
        t.sum = t.sum * under(t.top, top) + o;
        t.top = top;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t = join(t, TopSum{__shfl_xor(t.top, o, 64), __shfl_xor(t.sum, o, 64)});
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < NT / 64; ++w) t = join(t, red[w]);
        partial[blockIdx.x] = t;
    }
}

// The rows' terms from their chunks, a thread a row.
__global__ __launch_bounds__(NT) void merge_kernel(RowsArgs a, int chunks, const TopSum *partial)
{
    __shared__ Four red[NT / 64];
    Four sums = {};
    for (long long row = (long long)blockIdx.x * NT + threadIdx.x; row < a.r.B; row += (long long)gridDim.x * NT) {
        RowTerms t = {false, 0.f, 0.f, 0.f, 0.0, 0.0};
        if (has_choice(a.r, row)) {
            const TopSum *part = partial + row * chunks;
            const float zy = logit(a.r, row, a.r.y[row]);
            float top = zy;
            for (int c = 0; c < chunks; ++c) top = fmaxf(top, part[c].top);
            float o = 0.f;
            for (int c = 0; c < chunks; ++c) o += part[c].sum * under(part[c].top, top);
            t = finish_row(zy, top, o);
        }
        head_row(a.h, a.r, row, t, true, sums);
    }
    if (a.h.kind == HEAD_POLICY) {
        sums = sum_block(sums, red);
        if (a.stats) store_stats(a.stats, sums);
        else if (threadIdx.x == 0) a.sums[blockIdx.x] = sums;
    }
}

// ---------------------------------------------------------------- the gradient in the logits, from the rows' coefficients
// Rows [*first_row, *end_row) only where there are bounds; the first block adds the sums up where there are any.
struct GradArgs {
    ChoiceRows r;
    ChoiceGrad d;
    const RowCoef *coef;              // or
    const float *logp, *lse, *g;      // ... of hb_logprob_grad
    const int32_t *first_row, *end_row;
    int chunks, pieces_per_chunk;     // G = NT
    SumFour fin;
};

__device__ __forceinline__ RowCoef coef_of(const GradArgs &a, long long row)
{
    if (a.coef) return a.coef[row];
    RowCoef c = {0.f, 0.f, 0.f, 0.f};
    const float lse = a.lse[row], g = a.g[row];
    if (!has_choice(a.r, row) || lse == -INFINITY || g == 0.f) return c;
    c.base = lse;
    c.scale = -g;
    c.chosen = -g * expm1f(a.logp[row]);
    return c;
}

// G lanes have a row, or a chunk of one, between them.  The last rows come first: they are what the pass over the logits
// before this one has left in the caches.
template <typename T, typename TO, int G>
__global__ __launch_bounds__(NT) void logit_grad_kernel(GradArgs a)
{
    constexpr int V = Piece<T>::V, U = 4;
    __shared__ Four red[NT / 64];
    const int first = a.fin.n > 0;
    if ((int)blockIdx.x < first) {
        sum_four(a.fin, red);
        return;
    }
    const int g = threadIdx.x % G;
    long long row = blockIdx.x - first;
    int c = 0;
    if (G == NT) {
        c = (int)(row % a.chunks);
        row /= a.chunks;
    } else {
        row = row * (NT / G) + threadIdx.x / G;
        if (row >= a.r.B) return;
    }
    row = a.r.B - 1 - row;
    if (a.first_row && (row < *a.first_row || row >= *a.end_row)) return;
    const Row<T> z(a.r.Z, a.r.ldz, row, a.r.K);
    TO *dz = static_cast<TO *>(a.d.dZ) + row * a.d.ld;
    const RowCoef k = coef_of(a, row);
    const int y = a.r.y[row], end = G == NT ? min(z.pieces, (c + 1) * a.pieces_per_chunk) : z.pieces;
    const bool none = k.scale == 0.f && k.chosen == 0.f;
    for (int p = c * a.pieces_per_chunk + g; p < end; p += U * G) {
        Piece<T> x[U];
        if (!none)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * G < end) x[u] = z.load(z.first(p + u * G));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * G >= end) break;
            const int j0 = z.first(p + u * G);
            float out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = none ? 0.f : k.scale * __expf(x[u].get(e) - k.base);
            if ((unsigned)(y - j0) < (unsigned)V)
#pragma unroll
                for (int e = 0; e < V; ++e) out[e] = e == y - j0 ? k.chosen : out[e];
            store<TO, V>(dz, j0, a.r.K, out);
        }
    }
    if (c == a.chunks - 1)
        for (int j = a.r.K + g; j < a.d.pad; j += G) dz[j] = TO(0.f);
}

// ---------------------------------------------------------------- pairs of sequences
__device__ __forceinline__ double softplus(double v) { return fmax(v, 0.0) + log1p(exp(-fabs(v))); }
__device__ __forceinline__ double sigma(double v) { return v >= 0.0 ? 1.0 / (1.0 + exp(-v)) : exp(v) / (1.0 + exp(v)); }

// One block per pair.
__global__ __launch_bounds__(NT) void preference_kernel(PreferenceTerms p, long long B, const double *row_lp, RowCoef *coef,
                                                        Four *sums)
{
    __shared__ Four red[NT / 64];
    const int n = blockIdx.x;
    long long at[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) at[i] = min(max((long long)p.seq[2 * n + i], i ? at[i - 1] : 0ll), B);
    Four s = {};
#pragma unroll
    for (int q = 0; q < 2; ++q)
        for (long long row = at[q] + threadIdx.x; row < at[q + 1]; row += NT) s.v[q] += row_lp[row];
    s = sum_block(s, red);
    const double up = s.v[0] - (p.ref ? (double)p.ref[2 * n] : 0.0), down = s.v[1] - (p.ref ? (double)p.ref[2 * n + 1] : 0.0);
    const double h = up - down, b = p.beta, eps = p.smoothing;
    const double mean = 1.0 / (double)p.pairs;
    if (threadIdx.x == 0) {
        double loss = (1.0 - eps) * softplus(-b * h);
        if (eps != 0.0) loss += eps * softplus(b * h);
        sums[n] = Four{{mean * loss, h > 0.0 ? mean : 0.0, mean * b * up, mean * b * down}};
        if (p.seq_logp) {
            p.seq_logp[2 * n] = (float)s.v[0];
            p.seq_logp[2 * n + 1] = (float)s.v[1];
        }
    }
    if (!coef) return;
    const double slope = b * mean * (eps * sigma(b * h) - (1.0 - eps) * sigma(-b * h));
#pragma unroll
    for (int q = 0; q < 2; ++q)
        for (long long row = at[q] + threadIdx.x; row < at[q + 1]; row += NT) {
            const float g = (float)(q ? -slope : slope);
            RowCoef c = coef[row];
            c.scale *= -g;
            c.chosen *= g;
            coef[row] = c;
        }
}

// ---------------------------------------------------------------- launches
struct Workspace {
    Four *sums;
    RowCoef *coef;
    double *row_lp;
    TopSum *partial;
    Workspace(void *ws, long long B, int pairs)
    {
        char *p = static_cast<char *>(ws);
        sums = reinterpret_cast<Four *>(p);
        p += sizeof(Four) * (size_t)(pairs > MAX_SUM_BLOCKS ? pairs : MAX_SUM_BLOCKS);
        coef = reinterpret_cast<RowCoef *>(p);
        p += sizeof(RowCoef) * (size_t)B;
        row_lp = reinterpret_cast<double *>(p);
        p += sizeof(double) * (size_t)B;
        partial = reinterpret_cast<TopSum *>(p);
    }
};

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
int most_pieces(const ChoiceRows &r)  // of a row at any alignment
{
    const int V = r.tensor == TENSOR_BF16 ? 8 : 4;
    return (r.K + V - 1 + V - 1) / V;
}

struct Split {
    int chunks, pieces_per_chunk;
};

constexpr int ROW_PIECES = 20 * 1024;  // the longest row that rows_kernel has a form for

// Rows go through registers unless they are too long for a workgroup, or too few to fill the device.
bool rows_in_registers(const ChoiceRows &r) { return most_pieces(r) <= ROW_PIECES; }

Split split_for(const ChoiceRows &r)
{
    const int pieces = most_pieces(r);
    int chunks = ceil_div(pieces, 4 * NT);
    const long long room = r.B < MAX_CHUNKED ? MAX_CHUNKED / (r.B > 0 ? r.B : 1) : 1;
    if (chunks > room) chunks = (int)room;
    return {chunks, ceil_div(pieces, chunks)};
}

template <typename T, typename TO, int G, int N>
hipError_t rows_form(RowsArgs a, int *blocks_out, hipStream_t stream, const LaunchEvents &ev)
{
    constexpr int ROWS = G > NT ? 1 : NT / G;
    int blocks = ceil_div(a.r.B, ROWS);
    if (a.h.kind == HEAD_POLICY && blocks > MAX_SUM_BLOCKS) blocks = MAX_SUM_BLOCKS;
    if (blocks > 1) a.stats = nullptr;
    *blocks_out = blocks;
    return launch_kernel(rows_kernel<T, TO, G, N>, dim3((unsigned)blocks), dim3(G > NT ? G : NT), stream, ev, a);
}

template <typename T, typename TO>
hipError_t rows_of_type(const RowsArgs &a, int *blocks, hipStream_t s, const LaunchEvents &ev)
{
    const int n = most_pieces(a.r);
    if (n <= 8) return rows_form<T, TO, 8, 1>(a, blocks, s, ev);
    if (n <= 32) return rows_form<T, TO, 16, 2>(a, blocks, s, ev);
    if (n <= 128) return rows_form<T, TO, 64, 2>(a, blocks, s, ev);
    if (n <= 256) return rows_form<T, TO, 64, 4>(a, blocks, s, ev);
    if (n <= 512) return rows_form<T, TO, 64, 8>(a, blocks, s, ev);
    if (n <= 1024) return rows_form<T, TO, 256, 4>(a, blocks, s, ev);
    if (n <= 2048) return rows_form<T, TO, 256, 8>(a, blocks, s, ev);
    if (n <= 4096) return rows_form<T, TO, 512, 8>(a, blocks, s, ev);
    if (n <= 8192) return rows_form<T, TO, 1024, 8>(a, blocks, s, ev);
    if (n <= 12288) return rows_form<T, TO, 1024, 12>(a, blocks, s, ev);
    if (n <= 16384) return rows_form<T, TO, 1024, 16>(a, blocks, s, ev);
    return rows_form<T, TO, 1024, 20>(a, blocks, s, ev);
}

hipError_t rows(const RowsArgs &a, int *blocks, hipStream_t stream, const LaunchEvents &ev)
{
    if (a.r.tensor == TENSOR_BF16) return rows_of_type<__bf16, __bf16>(a, blocks, stream, ev);
    return a.d.dZ && a.d.tensor == TENSOR_BF16 ? rows_of_type<float, __bf16>(a, blocks, stream, ev)
                                               : rows_of_type<float, float>(a, blocks, stream, ev);
}

// The heads of rows in chunks.  blocks: those that leave sums
hipError_t chunked_rows(RowsArgs a, const Split &s, TopSum *partial, int *blocks, hipStream_t stream, const LaunchEvents &ev)
{
    const dim3 grid((unsigned)(a.r.B * s.chunks)), block(NT);
    const hipError_t e = a.r.tensor == TENSOR_BF16
                             ? launch_kernel(row_sums_kernel<__bf16>, grid, block, stream, ev, a.r, s.chunks, s.pieces_per_chunk, partial)
                             : launch_kernel(row_sums_kernel<float>, grid, block, stream, ev, a.r, s.chunks, s.pieces_per_chunk, partial);
    if (e != hipSuccess) return e;
    *blocks = ceil_div(a.r.B, NT);
    if (*blocks > MAX_SUM_BLOCKS) *blocks = MAX_SUM_BLOCKS;
    if (*blocks > 1) a.stats = nullptr;
    return launch_kernel(merge_kernel, dim3((unsigned)*blocks), block, stream, LaunchEvents(), a, s.chunks, (const TopSum *)partial);
}

template <typename T, typename TO>
hipError_t grad_of_type(GradArgs a, hipStream_t stream, const LaunchEvents &ev)
{
    const int n = most_pieces(a.r), fin = a.fin.n > 0 ? 1 : 0;
    a.chunks = 1;
    a.pieces_per_chunk = 0;
    if (n <= 16) return launch_kernel(logit_grad_kernel<T, TO, 8>, dim3((unsigned)(ceil_div(a.r.B, NT / 8) + fin)), dim3(NT), stream, ev, a);
    if (n <= 512)
        return launch_kernel(logit_grad_kernel<T, TO, 64>, dim3((unsigned)(ceil_div(a.r.B, NT / 64) + fin)), dim3(NT), stream, ev, a);
    const Split s = split_for(a.r);
    a.chunks = s.chunks;
    a.pieces_per_chunk = s.pieces_per_chunk;
    return launch_kernel(logit_grad_kernel<T, TO, NT>, dim3((unsigned)(a.r.B * s.chunks + fin)), dim3(NT), stream, ev, a);
}

hipError_t logit_grad(const GradArgs &a, hipStream_t stream, const LaunchEvents &ev)
{
    if (a.r.tensor == TENSOR_BF16) return grad_of_type<__bf16, __bf16>(a, stream, ev);
    return a.d.tensor == TENSOR_BF16 ? grad_of_type<float, __bf16>(a, stream, ev) : grad_of_type<float, float>(a, stream, ev);
}

hipError_t add_sums(const SumFour &f, hipStream_t stream)
{
    return launch_kernel(sum_four_kernel, dim3(1), dim3(NT), stream, LaunchEvents(), f);
}

}  // namespace

size_t choice_workspace(long long B, int pairs)
{
    return sizeof(Four) * (size_t)(pairs > MAX_SUM_BLOCKS ? pairs : MAX_SUM_BLOCKS) + (sizeof(RowCoef) + sizeof(double)) * (size_t)B +
           sizeof(TopSum) * (size_t)(B > MAX_CHUNKED ? B : MAX_CHUNKED);
}

hipError_t launch_logprob(const ChoiceRows &r, float *logp, float *lse, void *ws, hipStream_t stream, const LaunchEvents &ev)
{
    if (r.B == 0) return hipSuccess;
    RowsArgs a = {};
    a.r = r;
    a.h.kind = HEAD_LOGPROB;
    a.h.logp = logp;
    a.h.lse = lse;
    int blocks = 0;
    if (rows_in_registers(r)) return rows(a, &blocks, stream, ev);
    return chunked_rows(a, split_for(r), Workspace(ws, r.B, 0).partial, &blocks, stream, ev);
}

hipError_t launch_logprob_grad(const ChoiceRows &r, const float *logp, const float *lse, const float *g, const ChoiceGrad &d,
                               hipStream_t stream, const LaunchEvents &ev)
{
    if (r.B == 0) return hipSuccess;
    GradArgs a = {};
    a.r = r;
    a.d = d;
    a.logp = logp;
    a.lse = lse;
    a.g = g;
    return logit_grad(a, stream, ev);
}

hipError_t launch_policy(const ChoiceRows &r, const PolicyTerms &t, const ChoiceGrad &d, void *ws, hipStream_t stream,
                         const LaunchEvents &ev)
{
    const Workspace w(ws, r.B, 0);
    SumFour fin = {w.sums, 0, t.stats};
    if (r.B == 0) return add_sums(fin, stream);
    RowsArgs a = {};
    a.r = r;
    a.h.kind = HEAD_POLICY;
    a.h.p = t;
    a.sums = w.sums;
    a.stats = t.stats;
    if (rows_in_registers(r)) {
        a.d = d;
        const hipError_t e = rows(a, &fin.n, stream, ev);
        return e != hipSuccess || fin.n == 1 ? e : add_sums(fin, stream);
    }
    a.h.coef = d.dZ ? w.coef : nullptr;
    const hipError_t e = chunked_rows(a, split_for(r), w.partial, &fin.n, stream, ev);
    if (e != hipSuccess) return e;
    if (fin.n == 1) fin.n = 0;
    if (!d.dZ) return fin.n ? add_sums(fin, stream) : hipSuccess;
    GradArgs g = {};
    g.r = r;
    g.d = d;
    g.coef = w.coef;
    g.fin = fin;
    return logit_grad(g, stream, LaunchEvents());
}

hipError_t launch_preference(const ChoiceRows &r, const PreferenceTerms &t, const ChoiceGrad &d, void *ws, hipStream_t stream,
                             const LaunchEvents &ev)
{
    const Workspace w(ws, r.B, t.pairs);
    RowsArgs a = {};
    a.r = r;
    a.h.kind = HEAD_TERMS;
    a.h.row_lp = w.row_lp;
    a.h.coef = d.dZ ? w.coef : nullptr;
    int blocks = 0;
    hipError_t e = hipSuccess;
    if (r.B > 0) e = rows_in_registers(r) ? rows(a, &blocks, stream, ev) : chunked_rows(a, split_for(r), w.partial, &blocks, stream, ev);
    if (e == hipSuccess)
        e = launch_kernel(preference_kernel, dim3((unsigned)t.pairs), dim3(NT), stream, LaunchEvents(), t, r.B,
                          (const double *)w.row_lp, d.dZ ? w.coef : nullptr, w.sums);
    const SumFour fin = {w.sums, t.pairs, t.stats};
    if (e != hipSuccess || !d.dZ || r.B == 0) return e != hipSuccess ? e : add_sums(fin, stream);
    GradArgs g = {};
    g.r = r;
    g.d = d;
    g.coef = w.coef;
    g.first_row = t.seq;
    g.end_row = t.seq + 2 * t.pairs;
    g.fin = fin;
    return logit_grad(g, stream, LaunchEvents());
}

}  // namespace hb
