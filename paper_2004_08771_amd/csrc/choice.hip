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
constexpr int MAX_CHUNKED = 4096;   // (row, chunk) pairs of the calls that split their rows, at most
constexpr int MAX_SUM_BLOCKS = 512;

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__bf16 v) { return (float)v; }

// A row in 16-byte pieces that are aligned in memory: piece v has the elements v * V - lead .. + V.  The first and the
// last may be cut by the row's ends.
template <typename T>
struct Row {
    static constexpr int V = 16 / sizeof(T);
    const T *z;
    int K, lead, pieces;
    __device__ __forceinline__ Row(const void *Z, long long ld, long long row, int K_)
        : z(static_cast<const T *>(Z) + row * ld), K(K_)
    {
        lead = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
        pieces = (K + lead + V - 1) / V;
    }
    __device__ __forceinline__ int first(int piece) const { return piece * V - lead; }
    __device__ __forceinline__ bool whole(int j0) const { return j0 >= 0 && j0 + V <= K; }
    // what is outside of the row reads as -inf
    __device__ __forceinline__ void load(int j0, float *x) const
    {
        if (whole(j0)) {
            T t[V];
            __builtin_memcpy(t, __builtin_assume_aligned(z + j0, 16), 16);
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = widen(t[e]);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = (j0 + e >= 0 && j0 + e < K) ? widen(z[j0 + e]) : -INFINITY;
        }
    }
};

// n elements of a row of dZ from j0 on, those in [0, K)
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

// A running maximum and the sum of exponentials under it.  top = -inf: nothing but -inf so far (sum 0), or NaN (sum NaN)
struct TopSum {
    float top, sum;
};

__device__ __forceinline__ float under(float x, float top) { return __expf(x - (top == -INFINITY ? 0.f : top)); }

__device__ __forceinline__ TopSum join(TopSum a, TopSum b)
{
    const float top = fmaxf(a.top, b.top);
    return {top, a.sum * under(a.top, top) + b.sum * under(b.top, top)};
}

template <int V>
__device__ __forceinline__ void add(TopSum &t, const float *x)
{
    float top = t.top;
#pragma unroll
    for (int e = 0; e < V; ++e) top = fmaxf(top, x[e]);
    t.sum *= under(t.top, top);
#pragma unroll
    for (int e = 0; e < V; ++e) t.sum += under(x[e], top);
    t.top = top;
}

__device__ __forceinline__ TopSum join_block(TopSum t, TopSum *red)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t = join(t, TopSum{__shfl_xor(t.top, o, 64), __shfl_xor(t.sum, o, 64)});
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = t;
    __syncthreads();
    t = red[0];
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) t = join(t, red[w]);
    return t;
}

__device__ __forceinline__ bool has_choice(const ChoiceRows &r, long long row)
{
    const int y = r.y[row];
    return y >= 0 && y < r.K && (r.weight == nullptr || r.weight[row] != 0.f);
}

__device__ __forceinline__ float logit(const ChoiceRows &r, long long row, int k)
{
    const long long i = row * r.ldz + k;
    return r.tensor == TENSOR_BF16 ? (float)static_cast<const __bf16 *>(r.Z)[i] : static_cast<const float *>(r.Z)[i];
}

// What a row comes down to, in 64 bits.  part: it takes part.  One without a choice has lp = lse = 0, one whose logits
// are all -inf has -inf.
struct RowTerms {
    bool part;
    float top;
    double inv_sum, others, lp, lse;  // 1 / s, 1 - p_y, log-probability, log of the sum of exponentials
};

__device__ __forceinline__ RowTerms finish_row(const ChoiceRows &r, long long row, const TopSum *partial, int chunks)
{
    RowTerms t = {false, 0.f, 0.0, 0.0, 0.0, 0.0};
    if (!has_choice(r, row)) return t;
    const float zy = logit(r, row, r.y[row]);
    float top = zy;
    for (int c = 0; c < chunks; ++c) top = fmaxf(top, partial[c].top);
    const float ref = top == -INFINITY ? 0.f : top;
    double o = 0.0;
    for (int c = 0; c < chunks; ++c) o += (double)partial[c].sum * exp((double)partial[c].top - (double)ref);
    const double d = (double)zy - (double)ref, e = exp(d), s = o + e;
    if (top == -INFINITY && o == 0.0 && zy == zy) {
        t.lp = t.lse = -INFINITY;
        return t;
    }
    t.part = true;
    t.top = ref;
    t.inv_sum = 1.0 / s;
    t.others = o / s;
    t.lp = o < e ? -log1p(o / e) : d - log(s);
    t.lse = (double)ref + log(s);
    return t;
}

// ---------------------------------------------------------------- sums over the rows
template <typename T>
__global__ __launch_bounds__(NT) void row_sums_kernel(ChoiceRows r, int chunks, int pieces_per_chunk, TopSum *partial)
{
    __shared__ TopSum red[NT / 64];
    const long long row = blockIdx.x / chunks;
    const int c = blockIdx.x % chunks;
    if (!has_choice(r, row)) return;
    const Row<T> z(r.Z, r.ldz, row, r.K);
    const int y = r.y[row], end = min(z.pieces, (c + 1) * pieces_per_chunk);
    TopSum t = {-INFINITY, 0.f};
    for (int p = c * pieces_per_chunk + (int)threadIdx.x; p < end; p += NT) {
        float x[Row<T>::V];
        const int j0 = z.first(p);
        z.load(j0, x);
        if (y >= j0 && y < j0 + Row<T>::V) {
#pragma unroll
            for (int e = 0; e < Row<T>::V; ++e)
                if (j0 + e == y) x[e] = -INFINITY;
        }
        add<Row<T>::V>(t, x);
    }
    t = join_block(t, red);
    if (threadIdx.x == 0) partial[(long long)blockIdx.x] = t;
}

__global__ __launch_bounds__(NT) void logprob_kernel(ChoiceRows r, int chunks, const TopSum *partial, float *logp, float *lse)
{
    const long long row = (long long)blockIdx.x * NT + threadIdx.x;
    if (row >= r.B) return;
    const RowTerms t = finish_row(r, row, partial + row * chunks, chunks);
    if (logp) logp[row] = (float)t.lp;
    if (lse) lse[row] = (float)t.lse;
}

// ---------------------------------------------------------------- the gradient in the logits
// dz_k = scale * exp(z_k - base) for k != y and `chosen` for k = y; all zero where both are
struct RowCoef {
    float base, scale, chosen, pad;
};

struct Four {
    double v[4];
};
// stats = sum of n partial sums in a fixed order
struct SumFour {
    const Four *partial;
    int n;  // 0: nothing to do
    float *stats;
};

__device__ __forceinline__ Four add_four(const Four &a, const Four &b)
{
    Four s;
#pragma unroll
    for (int i = 0; i < 4; ++i) s.v[i] = a.v[i] + b.v[i];
    return s;
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

__device__ __forceinline__ void sum_four(const SumFour &f, Four *red)
{
    Four s = {};
    for (int i = threadIdx.x; i < f.n; i += blockDim.x) s = add_four(s, f.partial[i]);
    s = sum_block(s, red);
    if (threadIdx.x == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) f.stats[i] = (float)s.v[i];
}

__global__ __launch_bounds__(NT) void sum_four_kernel(SumFour f)
{
    __shared__ Four red[NT / 64];
    sum_four(f, red);
}

// Rows [bounds[0], bounds[1]) only where there are bounds; the first block adds the sums up where there are any.
struct GradArgs {
    ChoiceRows r;
    ChoiceGrad d;
    const RowCoef *coef;              // or
    const float *logp, *lse, *g;      // ... of hb_logprob_grad
    const int32_t *first_row, *end_row;
    int chunks, pieces_per_chunk;
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

template <typename T, typename TO>
__global__ __launch_bounds__(NT) void logit_grad_kernel(GradArgs a)
{
    __shared__ Four red[NT / 64];
    const int first = a.fin.n > 0;
    if ((int)blockIdx.x < first) {
        sum_four(a.fin, red);
        return;
    }
    const long long row = (blockIdx.x - first) / a.chunks;
    const int c = (blockIdx.x - first) % a.chunks;
    if (a.first_row && (row < *a.first_row || row >= *a.end_row)) return;
    constexpr int V = Row<T>::V;
    const Row<T> z(a.r.Z, a.r.ldz, row, a.r.K);
    TO *dz = static_cast<TO *>(a.d.dZ) + row * a.d.ld;
    const RowCoef k = coef_of(a, row);
    const int y = a.r.y[row], end = min(z.pieces, (c + 1) * a.pieces_per_chunk);
    const bool none = k.scale == 0.f && k.chosen == 0.f;
    for (int p = c * a.pieces_per_chunk + (int)threadIdx.x; p < end; p += NT) {
        float x[V];
        const int j0 = z.first(p);
        if (none) {
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = 0.f;
        } else {
            z.load(j0, x);
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = j0 + e == y ? k.chosen : k.scale * __expf(x[e] - k.base);
        }
        store<TO, V>(dz, j0, a.r.K, x);
    }
    if (c == a.chunks - 1)
        for (int j = a.r.K + (int)threadIdx.x; j < a.d.pad; j += NT) dz[j] = TO(0.f);
}

// ---------------------------------------------------------------- the losses, from the rows' sums
__global__ __launch_bounds__(NT) void policy_kernel(ChoiceRows r, PolicyTerms p, int chunks, const TopSum *partial,
                                                    RowCoef *coef, Four *sums)
{
    __shared__ Four red[NT / 64];
    Four s = {};
    for (long long row = (long long)blockIdx.x * NT + threadIdx.x; row < r.B; row += (long long)gridDim.x * NT) {
        const RowTerms t = finish_row(r, row, partial + row * chunks, chunks);
        RowCoef c = {0.f, 0.f, 0.f, 0.f};
        if (t.part) {
            const double w = r.weight ? r.weight[row] : p.uniform, A = p.adv[row];
            double pg = 0.0, g = 0.0, kl = 0.0, cut = 0.0;
            if (A != 0.0) {  // (NaN too); without an advantage the ratio does not matter, however large
                const double ratio = exp(t.lp - (double)p.old_logp[row]);
                const double lo = 1.0 - (double)p.clip_low, hi = 1.0 + (double)p.clip_high;
                const double held = ratio < lo ? lo : ratio > hi ? hi : ratio;
                cut = (A > 0.0 && ratio > hi) || (A < 0.0 && ratio < lo) ? 1.0 : 0.0;
                pg = cut != 0.0 ? -held * A : -ratio * A;
                g = cut != 0.0 ? 0.0 : -ratio * A;
            }
            if (p.ref_logp) {
                const double d = (double)p.ref_logp[row] - t.lp, em = expm1(d);
                kl = em == INFINITY ? INFINITY : em - d;
                if (p.kl_coef != 0.f) g -= (double)p.kl_coef * em;
            }
            const double penalty = p.kl_coef != 0.f ? (double)p.kl_coef * kl : 0.0;
            s = add_four(s, Four{{w * (pg + penalty), w * pg, w * kl, w * cut}});
            g *= w;
            c.base = t.top;
            c.scale = (float)(-g * t.inv_sum);
            c.chosen = (float)(g * t.others);
        }
        if (p.logp) p.logp[row] = (float)t.lp;
        if (coef) coef[row] = c;
    }
    s = sum_block(s, red);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__device__ __forceinline__ double softplus(double v) { return fmax(v, 0.0) + log1p(exp(-fabs(v))); }
__device__ __forceinline__ double sigma(double v) { return v >= 0.0 ? 1.0 / (1.0 + exp(-v)) : exp(v) / (1.0 + exp(v)); }

// One block per pair of sequences.
__global__ __launch_bounds__(NT) void preference_kernel(ChoiceRows r, PreferenceTerms p, int chunks, const TopSum *partial,
                                                        RowCoef *coef, Four *sums)
{
    __shared__ Four red[NT / 64];
    const int n = blockIdx.x;
    long long at[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) at[i] = min(max((long long)p.seq[2 * n + i], i ? at[i - 1] : 0ll), r.B);
    Four s = {};
#pragma unroll
    for (int q = 0; q < 2; ++q)
        for (long long row = at[q] + threadIdx.x; row < at[q + 1]; row += NT) {
            const RowTerms t = finish_row(r, row, partial + row * chunks, chunks);
            if (t.part) s.v[q] += t.lp;
            if (coef) coef[row] = RowCoef{t.top, (float)t.inv_sum, (float)t.others, 0.f};
        }
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
        for (long long row = at[q] + threadIdx.x; row < at[q + 1]; row += NT) {  // each thread its own of above
            const float g = (float)(q ? -slope : slope);
            RowCoef c = coef[row];
            c.scale *= -g;
            c.chosen *= g;
            coef[row] = c;
        }
}

// Chunks that a call of B rows splits each of them into.
struct Split {
    int chunks, pieces_per_chunk;
};

template <typename T>
Split split_rows(long long B, int K)
{
    const int pieces = K / Row<T>::V + 2;  // at any alignment
    (void)B;
    return {1, pieces};
}

struct Workspace {
    RowCoef *coef;
    TopSum *partial;
    Four *sums;
    Workspace(void *ws, long long B, int pairs)
    {
        char *p = static_cast<char *>(ws);
        sums = reinterpret_cast<Four *>(p);
        p += sizeof(Four) * (size_t)(pairs > MAX_SUM_BLOCKS ? pairs : MAX_SUM_BLOCKS);
        coef = reinterpret_cast<RowCoef *>(p);
        p += sizeof(RowCoef) * (size_t)B;
        partial = reinterpret_cast<TopSum *>(p);
    }
};

template <typename T>
hipError_t row_sums(const ChoiceRows &r, const Split &s, TopSum *partial, hipStream_t stream, const LaunchEvents &ev)
{
    return launch_kernel(row_sums_kernel<T>, dim3((unsigned)(r.B * s.chunks)), dim3(NT), stream, ev, r, s.chunks,
                         s.pieces_per_chunk, partial);
}

hipError_t logit_grad(const GradArgs &a, hipStream_t stream, const LaunchEvents &ev)
{
    const dim3 grid((unsigned)(a.r.B * a.chunks + (a.fin.n > 0 ? 1 : 0))), block(NT);
    if (a.r.tensor == TENSOR_BF16) return launch_kernel(logit_grad_kernel<__bf16, __bf16>, grid, block, stream, ev, a);
    return a.d.tensor == TENSOR_BF16 ? launch_kernel(logit_grad_kernel<float, __bf16>, grid, block, stream, ev, a)
                                     : launch_kernel(logit_grad_kernel<float, float>, grid, block, stream, ev, a);
}

Split split_for(const ChoiceRows &r)
{
    return r.tensor == TENSOR_BF16 ? split_rows<__bf16>(r.B, r.K) : split_rows<float>(r.B, r.K);
}

hipError_t sums_for(const ChoiceRows &r, const Split &s, TopSum *partial, hipStream_t stream, const LaunchEvents &ev)
{
    return r.tensor == TENSOR_BF16 ? row_sums<__bf16>(r, s, partial, stream, ev) : row_sums<float>(r, s, partial, stream, ev);
}

// What is left when the rows' coefficients and the partial sums are there: the gradient, and the sums
hipError_t finish_loss(const ChoiceRows &r, const ChoiceGrad &d, const Split &s, const RowCoef *coef, const int32_t *first_row,
                       const int32_t *end_row, const SumFour &fin, hipStream_t stream, const LaunchEvents &ev)
{
    if (d.dZ == nullptr || r.B == 0) return launch_kernel(sum_four_kernel, dim3(1), dim3(NT), stream, ev, fin);
    GradArgs a = {};
    a.r = r;
    a.d = d;
    a.coef = coef;
    a.first_row = first_row;
    a.end_row = end_row;
    a.chunks = s.chunks;
    a.pieces_per_chunk = s.pieces_per_chunk;
    a.fin = fin;
    return logit_grad(a, stream, ev);
}

}  // namespace

size_t choice_workspace(long long B, int pairs)
{
    return sizeof(Four) * (size_t)(pairs > MAX_SUM_BLOCKS ? pairs : MAX_SUM_BLOCKS) + sizeof(RowCoef) * (size_t)B +
           sizeof(TopSum) * (size_t)(B > MAX_CHUNKED ? B : MAX_CHUNKED);
}

hipError_t launch_logprob(const ChoiceRows &r, float *logp, float *lse, void *ws, hipStream_t stream, const LaunchEvents &ev)
{
    if (r.B == 0) return hipSuccess;
    const Workspace w(ws, r.B, 0);
    const Split s = split_for(r);
    const hipError_t e = sums_for(r, s, w.partial, stream, ev);
    if (e != hipSuccess) return e;
    return launch_kernel(logprob_kernel, dim3((unsigned)((r.B + NT - 1) / NT)), dim3(NT), stream, LaunchEvents(), r, s.chunks,
                         (const TopSum *)w.partial, logp, lse);
}

hipError_t launch_logprob_grad(const ChoiceRows &r, const float *logp, const float *lse, const float *g, const ChoiceGrad &d,
                               hipStream_t stream, const LaunchEvents &ev)
{
    if (r.B == 0) return hipSuccess;
    const Split s = split_for(r);
    GradArgs a = {};
    a.r = r;
    a.d = d;
    a.logp = logp;
    a.lse = lse;
    a.g = g;
    a.chunks = s.chunks;
    a.pieces_per_chunk = s.pieces_per_chunk;
    return logit_grad(a, stream, ev);
}

hipError_t launch_policy(const ChoiceRows &r, const PolicyTerms &t, const ChoiceGrad &d, void *ws, hipStream_t stream,
                         const LaunchEvents &ev)
{
    const Workspace w(ws, r.B, 0);
    const Split s = split_for(r);
    int blocks = (int)((r.B + NT - 1) / NT < MAX_SUM_BLOCKS ? (r.B + NT - 1) / NT : MAX_SUM_BLOCKS);
    if (r.B > 0) {
        hipError_t e = sums_for(r, s, w.partial, stream, ev);
        if (e == hipSuccess)
            e = launch_kernel(policy_kernel, dim3((unsigned)blocks), dim3(NT), stream, LaunchEvents(), r, t, s.chunks,
                              (const TopSum *)w.partial, d.dZ ? w.coef : nullptr, w.sums);
        if (e != hipSuccess) return e;
    }
    return finish_loss(r, d, s, w.coef, nullptr, nullptr, SumFour{w.sums, blocks, t.stats}, stream, LaunchEvents());
}

hipError_t launch_preference(const ChoiceRows &r, const PreferenceTerms &t, const ChoiceGrad &d, void *ws, hipStream_t stream,
                             const LaunchEvents &ev)
{
    const Workspace w(ws, r.B, t.pairs);
    const Split s = split_for(r);
    hipError_t e = r.B > 0 ? sums_for(r, s, w.partial, stream, ev) : hipSuccess;
    if (e == hipSuccess)
        e = launch_kernel(preference_kernel, dim3((unsigned)t.pairs), dim3(NT), stream, LaunchEvents(), r, t, s.chunks,
                          (const TopSum *)w.partial, d.dZ ? w.coef : nullptr, w.sums);
    if (e != hipSuccess) return e;
    return finish_loss(r, d, s, w.coef, t.seq, t.seq + 2 * t.pairs, SumFour{w.sums, t.pairs, t.stats}, stream, LaunchEvents());
}

}  // namespace hb
