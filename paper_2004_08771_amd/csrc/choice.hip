// Log-probabilities of chosen classes, and the losses that start from them: the clipped policy loss with a KL term and the
// preference loss over paired log ratios, with their gradients in the logits.
//
// Row z of K logits, chosen class y.  With m = max z, o = sum over k != y of exp(z_k - m), e = exp(z_y - m), s = o + e:
//     lp = log softmax(z)_y = -log(1 + o / e),   p_k = exp(z_k - m) / s,   1 - p_y = o / s,
//     d lp / d z_k = [k = y] - p_k.
// The chosen class is kept out of the sum o, so that lp and 1 - p_y of a choice that is all but certain keep their digits
// (s - e would cancel).  Exponentials, their sums and what follows from them are fp32; a log-probability is put together in 64
// bits from parts that are each fp32, and sums over rows are in 64 bits.
//
// All of it is bound by memory (but for short rows, whose once-a-row part counts, and small calls, which are launches).  Measured on
// one MI355X, a large copy there 5.2 TB/s: policy loss 8192 x 50257 bf16 288 us (10 % of the rows padding; 1.56 GB, 5.4 TB/s),
// 100000 x 2000 bf16 120 us (800 MB, partly from the last cache); log-probabilities 8192 x 32000 bf16 80 us (5.9 TB/s); of
// 4096 x 32000 bf16 38 us, and their gradient 75 us; preference loss of 16 pairs x 32000 bf16, 8111 rows, 246 us: the logits come
// twice, because a token's gradient takes the whole pair (1.43 GB, 5.8 TB/s; splitting the call by pairs, so that the second pass
// finds the logits in the last cache, costs more in launches than it saves: 286 -> 311 us in two parts, 347 us in four).
#include "operators.h"

namespace hb {
namespace {

constexpr int NT = 256;
constexpr int MAX_SUM_BLOCKS = 1024;  // blocks of merge_kernel, at most
constexpr int SUM_THREADS = 1024;
constexpr int SUM_SLICES = 256;       // more than 16 partial sums for each of SUM_THREADS are added up in two steps
constexpr int MAX_CHUNKED = 2048;     // (row, chunk) pairs of the calls that split their rows, at most

// ---------------------------------------------------------------- rows in memory
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

// 16 bytes of a row, as they are stored: four values, or eight of two bytes.
template <typename T>
struct Piece {
    static constexpr int V = 16 / sizeof(T);
    unsigned w[4];
    __device__ __forceinline__ float get(int e) const
    {
        if (sizeof(T) == 4) return __uint_as_float(w[e]);
        return __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
    __device__ __forceinline__ void set_none()  // -inf
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    }
    // without element `at` of it, where `own`
    __device__ __forceinline__ void drop(int at, bool own)
    {
        const unsigned half = sizeof(T) == 4 ? 0xffffffffu : (at & 1) ? 0xffff0000u : 0xffffu;
        const int word = sizeof(T) == 4 ? at : at >> 1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned m = own && i == word ? half : 0u;
            w[i] = (m & (sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u)) | (~m & w[i]);
        }
    }
    // Between two passes over pieces in registers: what the first has made of them (eight floats of four words) is made
    // again in the second, not kept.
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(w[i]));
    }
};

// A row is whole pieces that begin at 16-byte boundaries in memory, and an edge of fewer than V single elements at either
// end.  Piece p has the elements first(p) .. + V.
template <typename T>
struct Row {
    static constexpr int V = Piece<T>::V;
    static constexpr int EDGE = 2 * V;  // places: V for either end
    const T *z;
    int K, head, pieces;
    __device__ __forceinline__ Row(const void *Z, long long ld, long long row, int K_)
        : z(static_cast<const T *>(Z) + row * ld), K(K_)
    {
        const int past = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
        head = past ? min(V - past, K) : 0;
        pieces = (K - head) / V;
    }
    __device__ __forceinline__ int first(int piece) const { return head + piece * V; }
    __device__ __forceinline__ Piece<T> load(int piece) const
    {
        Piece<T> t;
        const v4u *from = reinterpret_cast<const v4u *>(z + first(piece));
        const v4u u = *from;
#pragma unroll
        for (int i = 0; i < 4; ++i) t.w[i] = u[i];
        return t;
    }
    // The pieces as a buffer, for wavefronts that have one row (z the same in all lanes): what is behind the last reads as 0
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const
    {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(z + head), (short)0, pieces * 16, 0x00027000);
    }
    template <int POLICY>
    __device__ __forceinline__ static Piece<T> load(__amdgpu_buffer_rsrc_t rs, int lane_piece, int first_piece)
    {
        const v4u u = __builtin_amdgcn_raw_buffer_load_b128(rs, 16 * lane_piece, 16 * first_piece, POLICY);
        Piece<T> t;
#pragma unroll
        for (int i = 0; i < 4; ++i) t.w[i] = u[i];
        return t;
    }
    // the element in place i of the edges, -1 if there is none
    __device__ __forceinline__ int edge(int i) const
    {
        const int tail = first(pieces);
        const int j = i < V ? i : tail + i - V;
        return i < V ? (j < head ? j : -1) : (j < K && i < EDGE ? j : -1);
    }
    __device__ __forceinline__ float at(int j) const { return j >= 0 ? (float)z[j] : -INFINITY; }
};

template <int B>
struct Bytes {
    typedef v2u type;
};
template <>
struct Bytes<16> {
    typedef v4u type;
};

// V elements of a row of dZ, as they are stored
template <typename T, int V>
__device__ __forceinline__ typename Bytes<V * sizeof(T)>::type narrow(const float *x)
{
    T t[V];
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = T(x[e]);
    typename Bytes<V * sizeof(T)>::type u;
    __builtin_memcpy(&u, t, sizeof(u));
    return u;
}

// ... at any address.  past: past the caches, if it is aligned to its size
template <typename T, int V>
__device__ __forceinline__ void store(T *dz, const float *x, bool past)
{
    typedef typename Bytes<V * sizeof(T)>::type B;
    const B u = narrow<T, V>(x);
    if (past) __builtin_nontemporal_store(u, reinterpret_cast<B *>(dz));
    else __builtin_memcpy(dz, &u, sizeof(u));
}

// ... through a buffer
constexpr int PAST = 2;  // cache policy of a buffer access: non-temporal
template <typename T, int V, int POLICY>
__device__ __forceinline__ void store_buffer(__amdgpu_buffer_rsrc_t rs, int lane_piece, int first_piece, const float *x)
{
    constexpr int B = V * sizeof(T);
    const auto u = narrow<T, V>(x);
    if constexpr (B == 16) __builtin_amdgcn_raw_buffer_store_b128(u, rs, B * lane_piece, B * first_piece, POLICY);
    else __builtin_amdgcn_raw_buffer_store_b64(u, rs, B * lane_piece, B * first_piece, POLICY);
}

// Exponentials are powers of two of (z - top) * LOG2E: the difference first, since it is exact near the maximum and 0 there whatever the
// logits' size, where z * LOG2E - top * LOG2E would leave the rounding error of a product (+-64 at 1e9, past fp32's range from
// 1e10 on).  LOG2E is log2 e to 24 bits, so what is added up is the softmax of logits that are 1.3e-8 smaller; log-probabilities
// are made of (z_y - top) * LOG2E and that sum in the same way, which leaves an error of 1.3e-8 (E z - z_y) in them, of both signs
// (with the exact factor outside it would be 1.3e-8 times the entropy, always of one sign, which the tokens of a sequence add up).
constexpr float LOG2E = 0x1.715476p+0f;
constexpr double LN2 = 0.693147180559945309;
__device__ __forceinline__ float exp2_of(float u) { return __builtin_amdgcn_exp2f(u); }

// Exponentials under a maximum (under 0 where that is -inf)
struct Under {
    float ref;
    __device__ __forceinline__ explicit Under(float top) : ref(top == -INFINITY ? 0.f : top) {}
    __device__ __forceinline__ float exp(float z) const { return exp2_of((z - ref) * LOG2E); }
};

// log2(s) for a positive s, in two parts: an integer, and at most 1 with an error of 2^-24
struct TwoLog {
    float hi, lo;
};
__device__ __forceinline__ TwoLog two_log2(float s)
{
    return {(float)__builtin_amdgcn_frexp_expf(s), __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(s))};
}

// exp(x), off by 2^-23 (1 + |x|) relative.  Of log2 e = LOG2E + 1.9e-8 both parts.
__device__ __forceinline__ float exp_of(float x) { return exp2_of(__builtin_fmaf(x, LOG2E, x * 0x1.4ae0cp-26f)); }

// log(1 + x) for x in [0, 1]: 2 atanh(x / (2 + x)), whose series in s = x / (2 + x) <= 1/3 is cut behind s^15 (s^16 / 17 < 2e-9)
__device__ __forceinline__ float log1p_of(float x)
{
    const float s = x * __builtin_amdgcn_rcpf(2.f + x), q = s * s;
    float c = 1.f / 15.f;
    c = __builtin_fmaf(c, q, 1.f / 13.f);
    c = __builtin_fmaf(c, q, 1.f / 11.f);
    c = __builtin_fmaf(c, q, 1.f / 9.f);
    c = __builtin_fmaf(c, q, 1.f / 7.f);
    c = __builtin_fmaf(c, q, 1.f / 5.f);
    c = __builtin_fmaf(c, q, 1.f / 3.f);
    return 2.f * __builtin_fmaf(s * q, c, s);
}

// exp(d) - 1 and exp(d) - 1 - d, to a few roundings where d is small, too: d^2 times a series there
struct Expm1 {
    float em, kl;
    __device__ __forceinline__ explicit Expm1(float d)
    {
        if (fabsf(d) < 0.5f) {
            float c = 1.f / 40320.f;
            c = __builtin_fmaf(c, d, 1.f / 5040.f);
            c = __builtin_fmaf(c, d, 1.f / 720.f);
            c = __builtin_fmaf(c, d, 1.f / 120.f);
            c = __builtin_fmaf(c, d, 1.f / 24.f);
            c = __builtin_fmaf(c, d, 1.f / 6.f);
            c = __builtin_fmaf(c, d, 0.5f);
            kl = d * d * c;
            em = d + kl;
        } else {
            em = exp_of(d) - 1.f;
            kl = em == INFINITY ? INFINITY : em - d;
        }
    }
};

// ---------------------------------------------------------------- what a row comes down to
// part: the row takes part.  One without a choice has lp = lse = 0, one whose logits are all -inf has -inf.
struct RowTerms {
    bool part;
    Under under;             // of the maximum
    float inv_sum, others;   // 1 / s, 1 - p_y
    double lp, lse;          // log-probability, log of the sum of exponentials: off by 1e-7 beside what s is
};

// zy: the chosen logit; top: the maximum; o: the sum over the others under it.
// 64-bit additions, but no function of 64 bits: those would take more registers than the rows do.  The log-probability starts from the
// distance to the maximum, not from lse: beside a large maximum log s would be rounded away.
__device__ __forceinline__ RowTerms finish_row(float zy, float top, float o)
{
    RowTerms t = {false, Under(0.f), 0.f, 0.f, 0.0, 0.0};
    if (top == -INFINITY && o == 0.f && zy == zy) {  // NaN in o or zy: no maximum either, but a row that takes part
        t.lp = t.lse = -INFINITY;
        return t;
    }
    t.part = true;
    t.under = Under(top);
    const float e = t.under.exp(zy), s = o + e;
    const TwoLog l = two_log2(s);
    t.inv_sum = __builtin_amdgcn_rcpf(s);  // off by a rounding
    t.others = o * t.inv_sum;
    const double log2_s = (double)l.hi + (double)l.lo;
    t.lse = (double)t.under.ref + LN2 * log2_s;
    t.lp = LN2 * (((double)zy - (double)t.under.ref) * (double)LOG2E - log2_s);
    if (o < e) t.lp = -(double)log1p_of(o * __builtin_amdgcn_rcpf(e));
    return t;
}

// The gradient of a row: dz_k = scale * exp(z_k - ref) 2^add for k != y and `chosen` for k = y; all zero where both are
struct RowCoef {
    float ref, scale, chosen, add;
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
    int n;
    float *stats;
};

// What is done with a row's terms
enum { HEAD_LOGPROB, HEAD_TERMS, HEAD_POLICY };

// What the kernels that read the logits first are given.  With up to 112 bytes of arguments, and no block size among them, a
// launch takes 2.8 us on the host, with more 3.5 in most processes (a call of hb_logprob_async 3.95 -> 3.24 us, a policy loss of 300 x 7,
// two launches, 5.17 -> 4.84).
struct RowsArgs {
    const void *Z;
    const int32_t *y;
    const float *weight;
    int ldz, B, K;
    unsigned char head, tensor;
    bool past;             // POLICY: of dZ, as in ChoiceGrad
    bool one;              // POLICY, one block: out is the statistics
    union {
        struct {
            float *logp, *lse;  // lse may be null
        } l;
        struct {
            double *row_lp;     // 0 where a row takes no part
            const int32_t *seq; // rows in front of seq[0] and from seq[last] on are not looked at
            RowCoef *coef;      // {maximum, 1 / s, 1 - p_y}; null: none
            int last;
        } t;
        struct {
            const float *old_logp, *ref_logp, *adv;
            float *logp;
            float clip_low, clip_high, kl_coef, uniform;
        } p;
    };
    void *out;             // POLICY: four sums a block, or with one block the statistics
    void *dZ;              // POLICY, whole rows: as in ChoiceGrad
    int lddz, pad;
};
static_assert(sizeof(RowsArgs) == 112, "more arguments cost every launch up to 0.7 us");

__device__ __forceinline__ float logit(const RowsArgs &a, long long row, int k)
{
    const long long i = row * a.ldz + k;
    return a.tensor == TENSOR_BF16 ? (float)static_cast<const __bf16 *>(a.Z)[i] : static_cast<const float *>(a.Z)[i];
}

// What a row has besides its logits, asked for together
struct RowInputs {
    int y;
    float w, old_logp, adv, ref_logp;  // POLICY
    __device__ __forceinline__ RowInputs(const RowsArgs &a, long long row)
        : y(a.y[row]), w(1.f), old_logp(0.f), adv(0.f), ref_logp(0.f)
    {
        if (a.head == HEAD_TERMS && (row < a.t.seq[0] || row >= a.t.seq[a.t.last])) y = -1;
        if (a.head != HEAD_POLICY) return;
        w = a.weight ? a.weight[row] : a.p.uniform;
        old_logp = a.p.old_logp[row];
        adv = a.p.adv[row];
        if (a.p.ref_logp) ref_logp = a.p.ref_logp[row];
    }
    __device__ __forceinline__ bool choice(int K) const { return y >= 0 && y < K && w != 0.f; }
};

__device__ __forceinline__ RowCoef head_row(const RowsArgs &a, const RowInputs &in, long long row, const RowTerms &t, bool write,
                                            Four &sums)
{
    RowCoef c = {0.f, 0.f, 0.f, 0.f};
    if (a.head == HEAD_LOGPROB) {
        if (write) {
            a.l.logp[row] = (float)t.lp;
            if (a.l.lse) a.l.lse[row] = (float)t.lse;
        }
        return c;
    }
    if (a.head == HEAD_TERMS) {
        if (write) {
            a.t.row_lp[row] = t.part ? t.lp : 0.0;
            if (a.t.coef) a.t.coef[row] = RowCoef{t.under.ref, t.inv_sum, t.others, 0.f};
        }
        return c;
    }
    const auto &p = a.p;
    if (t.part) {
        const float A = in.adv;
        float pg = 0.f, g = 0.f, kl = 0.f;
        bool cut = false;
        if (A != 0.f) {  // (NaN too); without an advantage the ratio does not matter, however large
            const float ratio = exp_of((float)(t.lp - (double)in.old_logp));
            const float lo = 1.f - p.clip_low, hi = 1.f + p.clip_high;
            cut = (A > 0.f && ratio > hi) || (A < 0.f && ratio < lo);
            pg = cut ? -(A > 0.f ? hi : lo) * A : -ratio * A;
            g = cut ? 0.f : pg;
        }
        if (p.ref_logp) {
            const Expm1 d((float)((double)in.ref_logp - t.lp));
            kl = d.kl;
            if (p.kl_coef != 0.f) g -= p.kl_coef * d.em;
        }
        const float w = in.w;
        if (write) {
            const double pgw = (double)w * pg, klw = (double)w * kl;
            sums = add_four(sums, Four{{p.kl_coef != 0.f ? pgw + (double)p.kl_coef * klw : pgw, pgw, klw, cut ? (double)w : 0.0}});
        }
        g *= w;
        c.ref = t.under.ref;
        c.scale = -g * t.inv_sum;
        c.chosen = g * t.others;
    }
    if (write && p.logp) p.logp[row] = (float)t.lp;
    return c;
}

// Every G-th lane has something to add.  red: a wavefront each
template <int THREADS, int G = 1>
__device__ __forceinline__ Four sum_block(Four s, Four *red)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int o = 32; o >= G; o >>= 1) s.v[i] += __shfl_xor(s.v[i], o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    s = red[0];
    for (int w = 1; w < THREADS / 64; ++w) s = add_four(s, red[w]);
    return s;
}

__device__ __forceinline__ void store_stats(float *stats, const Four &s)
{
    if (threadIdx.x == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) stats[i] = (float)s.v[i];
}

template <int THREADS>
__device__ __forceinline__ void sum_four(const SumFour &f, Four *red)
{
    Four s = {};
#pragma unroll 8
    for (int i = threadIdx.x; i < f.n; i += THREADS) s = add_four(s, f.partial[i]);
    store_stats(f.stats, sum_block<THREADS>(s, red));
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void sum_four_kernel(SumFour f)
{
    __shared__ Four red[THREADS / 64];
    sum_four<THREADS>(f, red);
}

// One of SUM_SLICES neighbouring parts of the sums a block
__global__ __launch_bounds__(NT) void sum_slices_kernel(const Four *partial, int n, Four *out)
{
    __shared__ Four red[NT / 64];
    const int per = (n + SUM_SLICES - 1) / SUM_SLICES, end = min(n, ((int)blockIdx.x + 1) * per);
    Four s = {};
    for (int i = (int)blockIdx.x * per + threadIdx.x; i < end; i += NT) s = add_four(s, partial[i]);
    s = sum_block<NT>(s, red);
    if (threadIdx.x == 0) out[blockIdx.x] = s;
}

// ---------------------------------------------------------------- whole rows in registers
// What a block leaves of a policy loss
__device__ __forceinline__ void store_sums(const RowsArgs &a, const Four &sums)
{
    if (a.one) store_stats(static_cast<float *>(a.out), sums);
    else if (threadIdx.x == 0) static_cast<Four *>(a.out)[blockIdx.x] = sums;
}

// wavefronts a SIMD that the registers have to leave room for
constexpr int row_waves(int g, int n) { return g <= 4 || n > 4 ? (n > 8 ? 4 : 5) : 6; }

// A row of dZ and its padding
template <int G, typename TO>
__device__ __forceinline__ void zero_row(TO *dz, const RowsArgs &a, int g)
{
    constexpr int V = 16 / sizeof(TO);
    const int n = max(a.K, a.pad), off = (int)((reinterpret_cast<uintptr_t>(dz) & 15) / sizeof(TO));
    const int head = off ? min(V - off, n) : 0, pieces = (n - head) / V;
    const v4u zero = {0u, 0u, 0u, 0u};
    for (int p = g; p < pieces; p += G) reinterpret_cast<v4u *>(dz + head)[p] = zero;
    for (int j = g; j < head; j += G) dz[j] = TO(0.f);
    for (int j = head + pieces * V + g; j < n; j += G) dz[j] = TO(0.f);
}

// The maximum over the G lanes of a row; red: a wavefront each
template <int G, int WAVES>
__device__ __forceinline__ float max_of_row(float top, float *red)
{
#pragma unroll
    for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    if (G > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
        __syncthreads();
        top = red[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, red[w]);
    }
    return top;
}

// G lanes have a row between them, N pieces each and what there is at its ends: it is read once, whole, for the maximum,
// the sum and the gradient.
template <typename T, typename TO, int G, int N, int WAVES>
__device__ __forceinline__ void row_in_registers(const RowsArgs &a, long long row, int g, float *red_top, float *red_sum,
                                                 RowCoef *red_coef, Four &sums)
{
    constexpr int V = Piece<T>::V;
    constexpr int E = G < Row<T>::EDGE ? Row<T>::EDGE / G : 1;
    // The exponentials stay in registers, too, where they take the place of the logits or there is room for them; else they
    // are made again for the gradient.
    constexpr bool KEEP = sizeof(T) == 4 || N <= 4;
    const Row<T> z(a.Z, a.ldz, row, a.K);
    const RowInputs in(a, row);
    const int y = in.y;
    // the choice: its place in the pieces (if it is in one), the lane that has it, and which piece of that lane's it is
    const int ay = y - z.head, py = ay / V, iy = py / G;
    const bool own = ay >= 0 && py < z.pieces && py % G == g;
    TO *dz = static_cast<TO *>(a.dZ) + row * a.lddz;
    if (!in.choice(a.K)) {
        const RowTerms t = {false, Under(0.f), 0.f, 0.f, 0.0, 0.0};
        if (g == 0) head_row(a, in, row, t, true, sums);
        if (a.dZ) zero_row<G>(dz, a, g);
        return;
    }
    const float zy = logit(a, row, y);
    Piece<T> x[N];
    float edge[E];
    const int most = a.K / V;  // pieces of any row; one less is in all of them
    if constexpr (G >= 64) {
        const __amdgpu_buffer_rsrc_t rs = z.buffer();
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * G < most) x[i] = a.past ? Row<T>::template load<PAST>(rs, g, i * G) : Row<T>::template load<0>(rs, g, i * G);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if ((i + 1) * G < most) x[i] = z.load(i * G + g);
            else if (i * G + g < z.pieces) x[i] = z.load(i * G + g);
        }
    }
    float v[KEEP ? N : 1][V];
    float top = zy;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int j = z.edge(i * G + g);
        edge[i] = j == y ? -INFINITY : z.at(j);
        top = fmaxf(top, edge[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i * G >= most) continue;
        if (i == iy) x[i].drop(ay % V, own);
        if ((i + 1) * G >= most && i * G + g >= z.pieces) x[i].set_none();
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float t = x[i].get(e);
            top = fmaxf(top, t);
            if (KEEP) v[i][e] = t;
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    top = max_of_row<G, WAVES>(top, red_top);
    const Under under(top);
    float o4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < E; ++i) o4[i & 3] += edge[i] = under.exp(edge[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i * G >= most) continue;
        if (!KEEP) x[i].forget();
        float t[V];
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = under.exp(KEEP ? v[i][e] : x[i].get(e));
#pragma unroll
        for (int e = 0; e < V; ++e) {
            o4[e & 3] += t[e];
            if (KEEP) v[i][e] = t[e];
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    float others = (o4[0] + o4[1]) + (o4[2] + o4[3]);
#pragma unroll
    for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1) others += __shfl_xor(others, o, 64);
    RowCoef c;
    if (G <= 64) {
        c = head_row(a, in, row, finish_row(zy, top, others), g == 0, sums);
    } else {
        if ((threadIdx.x & 63) == 0) red_sum[threadIdx.x >> 6] = others;
        __syncthreads();
        if (threadIdx.x < 64) {
            others = red_sum[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) others += red_sum[w];
            c = head_row(a, in, row, finish_row(zy, top, others), g == 0, sums);
            if (threadIdx.x == 0) *red_coef = c;
        }
        __syncthreads();
        c = *red_coef;
    }
    if (!a.dZ) return;
    if (c.scale == 0.f && c.chosen == 0.f) {
        zero_row<G>(dz, a, g);
        return;
    }
    TO *to = dz + z.head;
    // whole wavefronts that store at 16-byte boundaries: through a buffer, which leaves out what is behind the row
    const bool through = G >= 64 && (reinterpret_cast<uintptr_t>(to) & (V * sizeof(TO) - 1)) == 0;
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(to, (short)0, z.pieces * V * (int)sizeof(TO), 0x00027000);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i * G >= most) continue;
        if (!KEEP) x[i].forget();
        float out[V];
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = c.scale * (KEEP ? v[i][e] : under.exp(x[i].get(e)));
        if (through && a.past) store_buffer<TO, V, PAST>(rs, g, i * G, out);
        else if (through) store_buffer<TO, V, 0>(rs, g, i * G, out);
        else if (i * G + g < z.pieces) store<TO, V>(to + (i * G + g) * V, out, false);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (own) dz[y] = TO(c.chosen);  // over what this lane has just stored there
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int j = z.edge(i * G + g);
        if (j >= 0) dz[j] = TO(j == y ? c.chosen : c.scale * edge[i]);
    }
    for (int j = a.K + g; j < a.pad; j += G) dz[j] = TO(0.f);
}

template <typename T, typename TO, int G, int N, int THREADS>
__global__ __launch_bounds__(THREADS, row_waves(G, N)) void rows_kernel(RowsArgs a)
{
    constexpr int WAVES = THREADS / 64, ROWS = THREADS / G;
    __shared__ float red_top[WAVES], red_sum[WAVES];
    __shared__ RowCoef red_coef;
    __shared__ Four red_four[WAVES];
    const int g = threadIdx.x % G, sub = G >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G;
    const long long row = (long long)blockIdx.x * ROWS + sub;
    // (a loop over rows would keep registers for the row before)
    Four sums = {};
    if (row < a.B) row_in_registers<T, TO, G, N, WAVES>(a, row, g, red_top, red_sum, &red_coef, sums);
    if (a.head == HEAD_POLICY) {
        if constexpr (G <= 64) sums = sum_block<THREADS, G>(sums, red_four);  // else the first thread's
        store_sums(a, sums);
    }
}

// ---------------------------------------------------------------- rows in chunks
// A running maximum and the sum of exponentials under it.  top = -inf: nothing but -inf so far (sum 0), or NaN (sum NaN)
struct TopSum {
    float top, sum;
};

// What a sum under `from` is multiplied with to be one under `to` >= from
__device__ __forceinline__ float rescale(float from, float to)
{
    return from == to || from == -INFINITY ? 1.f : exp2_of((from - to) * LOG2E);
}

template <bool B>
struct Flag {
    static constexpr bool value = B;
};

// A block a chunk, without the chosen class; the first chunk has the edges.  A row of one chunk is finished here.
// chosen (may be null): the chosen logits, for a gradient that may be written over them.
template <typename T>
__global__ __launch_bounds__(NT) void row_sums_kernel(RowsArgs a, int chunks, int pieces_per_chunk, TopSum *partial, float *chosen)
{
    constexpr int V = Piece<T>::V, U = 4;
    __shared__ float red_top[NT / 64], red_sum[NT / 64];
    const long long row = blockIdx.x / chunks;
    const int c = blockIdx.x % chunks;
    const RowInputs in(a, row);
    if (!in.choice(a.K)) {
        const RowTerms none = {false, Under(0.f), 0.f, 0.f, 0.0, 0.0};
        Four sums = {};
        if (chunks == 1 && a.head != HEAD_POLICY && threadIdx.x == 0) head_row(a, in, row, none, true, sums);
        return;
    }
    const Row<T> z(a.Z, a.ldz, row, a.K);
    const int y = in.y, end = min(z.pieces, (c + 1) * pieces_per_chunk);
    TopSum t = {-INFINITY, 0.f};
    if (c == 0) {
        const int j = z.edge(threadIdx.x);
        const float v = j == y ? -INFINITY : z.at(j);
        t.top = v == v ? v : -INFINITY;
        t.sum = Under(t.top).exp(v);
    }
    // U pieces a lane; guard: not all lanes have that many left, and their loads are sent together all the same
    auto pieces = [&](auto guard, int p) {
        Piece<T> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!decltype(guard)::value || p + u * NT < end) x[u] = z.load(p + u * NT);
            else x[u].set_none();
        }
        float top = t.top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = y - z.first(p + u * NT);
            if ((unsigned)at < (unsigned)V) x[u].drop(at, true);
#pragma unroll
            for (int e = 0; e < V; ++e) top = fmaxf(top, x[u].get(e));
        }
        t.sum *= rescale(t.top, top);
        t.top = top;
        const Under under(top);
        float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u].forget();
#pragma unroll
            for (int e = 0; e < V; ++e) o[e & 3] += under.exp(x[u].get(e));
        }
        t.sum += (o[0] + o[1]) + (o[2] + o[3]);
    };
    int p = c * pieces_per_chunk;
    for (; p + U * NT <= end; p += U * NT) pieces(Flag<false>(), p + (int)threadIdx.x);
    if (p < end) pieces(Flag<true>(), p + (int)threadIdx.x);
    // The maximum first, so that every sum is rescaled once more, not at each step of the way
    const bool whole = chunks == 1 && a.head != HEAD_POLICY;  // (its sums are added up over the rows)
    const float zy = logit(a, row, y);
    float top = max_of_row<NT, NT / 64>(whole ? fmaxf(t.top, zy) : t.top, red_top);
    t.sum *= rescale(t.top, top);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t.sum += __shfl_xor(t.sum, o, 64);
    if ((threadIdx.x & 63) == 0) red_sum[threadIdx.x >> 6] = t.sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < NT / 64; ++w) t.sum += red_sum[w];
        if (whole) {
            Four sums = {};
            head_row(a, in, row, finish_row(zy, top, t.sum), true, sums);
        } else {
            partial[blockIdx.x] = TopSum{top, t.sum};
            if (chosen && c == 0) chosen[row] = zy;
        }
    }
}

// The terms of a row from its chunks, in `lanes` neighbouring lanes (a power of two up to 64), of which this is number g.
__device__ __forceinline__ RowTerms terms_of_chunks(const TopSum *partial, int chunks, float zy, int g, int lanes)
{
    float top = zy, others = 0.f;
    for (int c = g; c < chunks; c += lanes) top = fmaxf(top, partial[c].top);
    for (int o = lanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    for (int c = g; c < chunks; c += lanes) others += partial[c].sum * rescale(partial[c].top, top);
    for (int o = lanes / 2; o > 0; o >>= 1) others += __shfl_xor(others, o, 64);
    return finish_row(zy, top, others);
}

// The rows' terms from their chunks, G lanes a row.  coef (may be null): POLICY, the gradient's coefficients
template <int G>
__global__ __launch_bounds__(NT) void merge_kernel(RowsArgs a, int blocks, int chunks, const TopSum *partial, RowCoef *coef)
{
    __shared__ Four red[NT / 64];
    Four sums = {};
    const int g = threadIdx.x % G;
    const long long per_grid = (long long)blocks * (NT / G);
    for (long long row = (long long)blockIdx.x * (NT / G) + threadIdx.x / G; row < a.B; row += per_grid) {
        RowTerms t = {false, Under(0.f), 0.f, 0.f, 0.0, 0.0};
        const RowInputs in(a, row);
        if (in.choice(a.K)) t = terms_of_chunks(partial + row * chunks, chunks, logit(a, row, in.y), g, G);
        const RowCoef c = head_row(a, in, row, t, g == 0, sums);
        if (coef && g == 0) coef[row] = c;
    }
    if (a.head == HEAD_POLICY) store_sums(a, sum_block<NT>(sums, red));
}

// ---------------------------------------------------------------- pairs of sequences
__device__ __forceinline__ double softplus(double v) { return fmax(v, 0.0) + log1p(exp(-fabs(v))); }
__device__ __forceinline__ double sigma(double v) { return v >= 0.0 ? 1.0 / (1.0 + exp(-v)) : exp(v) / (1.0 + exp(v)); }

// The rows of pair n: at[0] .. at[1] - 1 were preferred over at[1] .. at[2] - 1
struct PairRows {
    long long at[3];
    __device__ __forceinline__ PairRows(const PreferenceTerms &p, long long B, int n)
    {
#pragma unroll
        for (int i = 0; i < 3; ++i) at[i] = min(max((long long)p.seq[2 * n + i], i ? at[i - 1] : 0ll), B);
    }
};

// s_0 and s_1: sums of log-probabilities over the sequences of pair n
struct Pair {
    double up, down;  // what they are above the reference's
    __device__ __forceinline__ Pair(const PreferenceTerms &p, int n, double s0, double s1)
        : up(s0 - (p.ref ? (double)p.ref[2 * n] : 0.0)), down(s1 - (p.ref ? (double)p.ref[2 * n + 1] : 0.0))
    {
    }
    __device__ __forceinline__ Four stats(const PreferenceTerms &p) const
    {
        const double h = up - down, b = p.beta, eps = p.smoothing, mean = 1.0 / (double)p.pairs;
        double loss = (1.0 - eps) * softplus(-b * h);
        if (eps != 0.0) loss += eps * softplus(b * h);
        return Four{{mean * loss, h > 0.0 ? mean : 0.0, mean * b * up, mean * b * down}};
    }
    // the loss' derivative in s_0; in s_1 its negative
    __device__ __forceinline__ double slope(const PreferenceTerms &p) const
    {
        const double h = up - down, b = p.beta, eps = p.smoothing, mean = 1.0 / (double)p.pairs;
        return b * mean * (eps * sigma(b * h) - (1.0 - eps) * sigma(-b * h));
    }
};

__device__ __forceinline__ void store_pair(const PreferenceTerms &p, int n, double s0, double s1)
{
    if (!p.seq_logp) return;
    p.seq_logp[2 * n] = (float)s0;
    p.seq_logp[2 * n + 1] = (float)s1;
}

// From a row's terms to its coefficients, g = the loss' derivative in its log-probability
__device__ __forceinline__ RowCoef slope_of_row(RowCoef c, float g)
{
    if (c.scale == 0.f && c.chosen == 0.f) return c;  // takes no part, whatever the slope
    c.scale *= -g;
    c.chosen *= g;
    return c;
}

// One block per pair.
__global__ __launch_bounds__(NT) void preference_kernel(PreferenceTerms p, long long B, const double *row_lp, RowCoef *coef,
                                                        Four *sums)
{
    __shared__ Four red[NT / 64];
    const int n = blockIdx.x;
    const PairRows rows(p, B, n);
    Four s = {};
#pragma unroll
    for (int q = 0; q < 2; ++q)
        for (long long row = rows.at[q] + threadIdx.x; row < rows.at[q + 1]; row += NT) s.v[q] += row_lp[row];
    s = sum_block<NT>(s, red);
    const Pair pair(p, n, s.v[0], s.v[1]);
    if (threadIdx.x == 0) {
        sums[n] = pair.stats(p);
        store_pair(p, n, s.v[0], s.v[1]);
    }
    if (!coef) return;
    const double slope = pair.slope(p);
#pragma unroll
    for (int q = 0; q < 2; ++q)
        for (long long row = rows.at[q] + threadIdx.x; row < rows.at[q + 1]; row += NT)
            coef[row] = slope_of_row(coef[row], (float)(q ? -slope : slope));
}

// Sums over the sequences of a pair in `lanes` neighbouring lanes, of which this is number g
__device__ __forceinline__ void sums_of_pair(const PairRows &rows, const double *row_lp, int g, int lanes, double (&s)[2])
{
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        s[q] = 0.0;
#pragma unroll 4
        for (long long row = rows.at[q] + g; row < rows.at[q + 1]; row += lanes) s[q] += row_lp[row];
    }
    for (int o = lanes / 2; o > 0; o >>= 1) {
        s[0] += __shfl_xor(s[0], o, 64);
        s[1] += __shfl_xor(s[1], o, 64);
    }
}

// ---------------------------------------------------------------- the gradient in the logits, from the rows' coefficients
// What the coefficients are made from
enum {
    GRAD_ROWS,    // they are there
    GRAD_LOGPROB, // log-probabilities and what these are multiplied with
    GRAD_CHUNKS,  // policy: what row_sums_kernel leaves
    GRAD_PAIRS    // preference: the rows' terms
};
struct GradArgs {
    const void *Z;
    const int32_t *y;
    void *dZ;
    union {
        const RowCoef *coef;  // ROWS, PAIRS
        const float *logp;    // LOGPROB, with:
    };
    const float *lse, *g;
    const int32_t *seq;      // rows [seq[0], seq[last]) only; null: all
    const Four *partial;     // ROWS: what the first block adds up, if there is one
    float *stats;
    int ldz, lddz, B, K, pad;
    int chunks, pieces_per_chunk;  // G = NT
    int last, sums;
    bool first;              // the first block does something else: it adds up the sums (ROWS), or makes them
    bool all_rows, past;     // as in ChoiceGrad
    bool keep;               // LOGPROB: the chosen logits stay where they are, for what else reads them
};
template <int FROM>
struct GradFrom : GradArgs {};
template <>
struct GradFrom<GRAD_CHUNKS> : GradArgs {  // pieces are divided in row_sums_kernel as they are here
    RowsArgs rows;
    const TopSum *partial_rows;
    const float *chosen;
};
template <>
struct GradFrom<GRAD_PAIRS> : GradArgs {
    PreferenceTerms p;
    const double *row_lp;
};
static_assert(sizeof(GradFrom<GRAD_ROWS>) == 112 && sizeof(GradFrom<GRAD_LOGPROB>) == 112, "more arguments cost every launch up to 0.7 us");

// p_k = exp(z_k - lse) from what hb_logprob_async has left.  As fp32 numbers lse and logp are each off by up to 2^-24 of themselves, and
// lse = z_y - logp: the smaller one says more.  With lse alone an offset of the logits goes into every p_k (three classes at 1e7,
// 1e7 + 1 and 1e7 + 2: 1.07 instead of 0.665); with z_y - logp only the distance of the choice does.  Where both are large p_k is
// still at most 1 - p_y.
struct LogprobCoef {
    RowCoef c;
    float others;  // 1 - p_y
};
template <typename T>
__device__ __forceinline__ LogprobCoef coef_of_logprob(const GradArgs &a, const Row<T> &z, long long row, int y)
{
    LogprobCoef k = {{0.f, 0.f, 0.f, 0.f}, 0.f};
    const float lse = a.lse[row], g = a.g[row], lp = a.logp[row];
    const float zy = (float)z.z[min(max(y, 0), a.K - 1)];  // (asked for first: it has a load in front of it)
    if (y < 0 || y >= a.K || lse == -INFINITY || g == 0.f) return k;
    const bool near = 2.f * fabsf(lp) <= fabsf(lse);
    k.others = -expm1f(lp);
    k.c.ref = near ? zy : lse;
    k.c.add = near ? lp * LOG2E : 0.f;
    k.c.scale = -g;
    k.c.chosen = g * k.others;
    return k;
}

// The chosen elements of a gradient in place of the logits whose rows go in several chunks: all of those read them
template <typename T>
__global__ __launch_bounds__(NT) void chosen_grad_kernel(GradArgs a)
{
    const int row = blockIdx.x * NT + threadIdx.x;
    if (row >= a.B) return;
    const int y = a.y[row];
    const float g = a.g[row];
    if (y < 0 || y >= a.K || a.lse[row] == -INFINITY || g == 0.f) return;
    static_cast<T *>(a.dZ)[(long long)row * a.lddz + y] = T(g * -expm1f(a.logp[row]));
}

// What a call on few rows has its first block do instead of one more launch: the statistics and what else is returned
constexpr int FEW = NT;
__device__ __forceinline__ void few_rows(const GradFrom<GRAD_CHUNKS> &a, Four *red)
{
    int lanes = 64;
    while (lanes * a.B > NT) lanes /= 2;
    const int row = threadIdx.x / lanes, g = threadIdx.x % lanes;
    Four sums = {};
    if (row < a.B) {
        RowTerms t = {false, Under(0.f), 0.f, 0.f, 0.0, 0.0};
        const RowInputs in(a.rows, row);
        if (in.choice(a.K)) t = terms_of_chunks(a.partial_rows + row * a.chunks, a.chunks, a.chosen[row], g, lanes);
        head_row(a.rows, in, row, t, g == 0, sums);
    }
    store_stats(a.stats, sum_block<NT>(sums, red));
}
__device__ __forceinline__ void few_pairs(const GradFrom<GRAD_PAIRS> &a, Four *red)
{
    int lanes = 64;
    while (lanes * a.p.pairs > NT) lanes /= 2;
    const int n = threadIdx.x / lanes, g = threadIdx.x % lanes;
    Four sums = {};
    if (n < a.p.pairs) {
        double s[2];
        sums_of_pair(PairRows(a.p, a.B, n), a.row_lp, g, lanes, s);
        if (g == 0) {
            sums = Pair(a.p, n, s[0], s[1]).stats(a.p);
            store_pair(a.p, n, s[0], s[1]);
        }
    }
    store_stats(a.stats, sum_block<NT>(sums, red));
}

// The coefficients of a row of one of the pairs, in `lanes` neighbouring lanes.
__device__ __forceinline__ RowCoef coef_in_pair(const GradFrom<GRAD_PAIRS> &a, long long row, int g, int lanes)
{
    int n = 0;  // pairs that end in front of it
    for (int i = g; i < a.p.pairs; i += lanes) n += a.p.seq[2 * i + 2] <= row;
    for (int o = lanes / 2; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    n = min(n, a.p.pairs - 1);
    const PairRows rows(a.p, a.B, n);
    double s[2];
    sums_of_pair(rows, a.row_lp, g, lanes, s);
    const double slope = Pair(a.p, n, s[0], s[1]).slope(a.p);
    return slope_of_row(a.coef[row], (float)(row < rows.at[1] ? slope : -slope));
}

// G lanes have a row, or a chunk of one, between them.  The last rows come first: they are what the pass over the logits
// before this one has left in the caches.
template <typename T, typename TO, int G, int FROM>
__global__ __launch_bounds__(NT) void logit_grad_kernel(GradFrom<FROM> a)
{
    constexpr int V = Piece<T>::V, U = 4, LANES = G < 64 ? G : 64;
    __shared__ Four red[NT / 64];
    if ((int)blockIdx.x < a.first) {
        if constexpr (FROM == GRAD_CHUNKS) few_rows(a, red);
        else if constexpr (FROM == GRAD_PAIRS) few_pairs(a, red);
        else if constexpr (FROM == GRAD_ROWS) sum_four<NT>(SumFour{a.partial, a.sums, a.stats}, red);
        return;
    }
    const int g = threadIdx.x % G;
    long long row = blockIdx.x - a.first;
    int c = 0;
    if (G == NT) {
        c = (int)(row % a.chunks);
        row /= a.chunks;
    } else {
        row = row * (NT / G) + threadIdx.x / G;
        if (row >= a.B) return;
    }
    row = a.B - 1 - row;
    const bool outside = a.seq && (row < a.seq[0] || row >= a.seq[a.last]);
    if (outside && !a.all_rows) return;
    const Row<T> z(a.Z, a.ldz, row, a.K);
    TO *dz = static_cast<TO *>(a.dZ) + row * a.lddz;
    const int y = a.y[row];
    RowCoef k = {0.f, 0.f, 0.f, 0.f};
    float others = INFINITY;  // at most this of a class that is not chosen
    if constexpr (FROM == GRAD_LOGPROB) {
        const LogprobCoef l = coef_of_logprob(a, z, row, y);
        k = l.c;
        others = l.others;
        if (G == NT && a.Z == a.dZ) {  // all wavefronts have the chosen logit before one of them writes over it
            asm volatile("" : "+v"(k.ref));
            __syncthreads();
        }
    } else if constexpr (FROM == GRAD_CHUNKS) {
        const RowInputs in(a.rows, row);
        Four sums;
        if (in.choice(a.K)) {
            const RowTerms t = terms_of_chunks(a.partial_rows + row * a.chunks, a.chunks, a.chosen[row], g % 64, 64);
            k = head_row(a.rows, in, row, t, false, sums);
        }
    } else if constexpr (FROM == GRAD_PAIRS) {
        if (!outside) k = coef_in_pair(a, row, g % LANES, LANES);
    } else {
        if (!outside) k = a.coef[row];
    }
    const int end = G == NT ? min(z.pieces, (c + 1) * a.pieces_per_chunk) : z.pieces;
    const bool none = k.scale == 0.f && k.chosen == 0.f;
    auto other = [&](float v) {
        const float e = exp2_of(__builtin_fmaf(v - k.ref, LOG2E, k.add));
        return k.scale * (FROM == GRAD_LOGPROB ? fminf(e, others) : e);
    };
    TO *to = dz + z.head;
    const bool past = a.past && (reinterpret_cast<uintptr_t>(to) & (V * sizeof(TO) - 1)) == 0;
    // U pieces a lane; guard: not all lanes have that many left, and their loads are sent together all the same
    auto pieces = [&](auto guard, int p) {
        Piece<T> x[U];
        if (!none)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (!decltype(guard)::value || p + u * G < end) x[u] = z.load(p + u * G);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (decltype(guard)::value && p + u * G >= end) continue;
            float out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = none ? 0.f : other(x[u].get(e));
            TO *const piece = to + (long long)(p + u * G) * V;
            const int at = y - z.first(p + u * G);
            const bool own = (unsigned)at < (unsigned)V;
            if (FROM == GRAD_LOGPROB && own && a.keep && !none) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e != at) piece[e] = TO(out[e]);
                continue;
            }
            store<TO, V>(piece, out, past);
            if (own) dz[y] = TO(k.chosen);  // over what this lane has just stored there
        }
    };
    int p = c * a.pieces_per_chunk;
    for (; p + U * G <= end; p += U * G) pieces(Flag<false>(), p + g);
    if (p < end) pieces(Flag<true>(), p + g);
    if (c == a.chunks - 1) {
        constexpr int E = G < Row<T>::EDGE ? Row<T>::EDGE / G : 1;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int j = z.edge(i * G + g);
            if (j < 0 || (FROM == GRAD_LOGPROB && j == y && a.keep && !none)) continue;
            dz[j] = TO(none ? 0.f : j == y ? k.chosen : other(z.at(j)));
        }
        for (int j = a.K + g; j < a.pad; j += G) dz[j] = TO(0.f);
    }
}

// ---------------------------------------------------------------- launches
struct Workspace {
    Four *sums;      // all of it for a call that leaves a sum a block of rows and nothing else
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
int most_pieces(int K, int tensor) { return K / (tensor == TENSOR_BF16 ? 8 : 4); }  // of a row, wherever it begins
int most_pieces(const ChoiceRows &r) { return most_pieces(r.K, r.tensor); }

// Whether a gradient goes past the caches: up to half of the last one (256 MB) it is left there for who reads it next, and
// storing it past them gains little (classes 32000 in bf16, log-probabilities and their gradient: 65 MB 42.6 -> 43.1 us, 131 MB
// 68.6 -> 68.9 us); a larger one drives out the logits that are still to be read a second time (192 MB 107 -> 97 us, 262 MB 159 ->
// 129 us; the policy loss, which reads them once, 192 MB 87 -> 77 us).
bool past_caches(const ChoiceRows &r, const ChoiceGrad &d)
{
    return (double)r.B * r.K * (d.tensor == TENSOR_BF16 ? 2 : 4) > (double)(128 << 20);
}

struct Split {
    int chunks, pieces_per_chunk;
};

constexpr int ROW_PIECES = 20 * 1024;  // the longest row that rows_kernel has a form for
constexpr int MAX_ROW = 8 * ROW_PIECES;

// Rows go through registers, but for long ones that are few (a workgroup each leaves most of the device idle) or, where they are only
// read, many (one workgroup of 1024 a compute unit waits between its rows), and those too long for a workgroup.
// Chunks are a launch more (but for a gradient of several rows, which has a second one anyway), so the lines are further out where
// logits are only read, or where there is one row.  us a call in a stream, the same input again and again, registers / chunks:
//   policy loss and gradient, bf16: 4 x 24000 11.4 / 12.2, 2 x 28000 12.1 / 11.8, 64 x 28000 12.5 / 11.6, 4 x 32000 12.4 / 11.9, 64 x 32000
//   13.2 / 11.7, 4 x 52000 12.6 / 10.3, 64 x 65000 15.7 / 10.4; fp32: 4 x 33000 11.5 / 12.1, 4 x 40000 11.8 / 12.1, 64 x 40000 12.6 / 11.5,
//   4 x 44000 12.1 / 12.0, 64 x 49000 13.6 / 11.4; one row: bf16 40000 9.4 / 11.3, 52000 10.2 / 10.4, 65000 11.9 / 10.3, fp32 49000 10.1 / 11.3
//   log-probabilities, bf16: 4 x 52000 6.9 / 8.4, 64 x 65000 8.1 / 8.5, 64 x 80000 9.4 / 8.5; policy loss alone 4 x 52000 9.6 / 9.7, 4 x 65000
//   10.5 / 9.7; preference loss and gradient 4 x 52000 12.0 / 12.4, 64 x 65000 15.4 / 14.2; fp32: 4 x 49000 7.9 / 9.6, 10.9 / 11.5, 12.2 / 14.4
// With data from memory the figures on the left are 0 to 3 us higher, those on the right 0 to 2.  More rows (data from memory):
//   policy loss 128 x 65000 bf16 19.8 / 19.6, 128 x 130000 27.1 / 28.1, 256 x 130000 40.2 / 52.7, 128 x 80000 fp32 29.4 / 33.3;
//   log-probabilities 1000 x 65000 bf16 33.2 / 35.8, 1000 x 128000 74.9 / 57.7.
bool rows_in_registers(const ChoiceRows &r, bool grad)
{
    const bool bf16 = r.tensor == TENSOR_BF16;
    const int few = !grad ? (bf16 ? 60000 : MAX_ROW) : r.B == 1 ? 52000 : bf16 ? 27000 : 40000;
    if (r.B <= 64 && r.K > few) return false;
    const int n = most_pieces(r);
    return n <= 12288 || (grad && n <= ROW_PIECES);
}

Split split_for(const ChoiceRows &r)
{
    const int pieces = most_pieces(r);
    int chunks = pieces > 0 ? ceil_div(pieces, 4 * NT) : 1;
    const long long room = r.B < MAX_CHUNKED ? MAX_CHUNKED / (r.B > 0 ? r.B : 1) : 1;
    if (chunks > room) chunks = (int)room;
    return {chunks, ceil_div(pieces, chunks)};
}

// Where the blocks of a policy loss leave their sums
struct Results {
    Four *sums;
    float *stats;
    void of(RowsArgs &a, int blocks) const
    {
        a.one = blocks == 1;
        a.out = a.one ? static_cast<void *>(stats) : static_cast<void *>(sums);
    }
};

template <typename T, typename TO, int G, int N, int THREADS>
hipError_t rows_launch(RowsArgs a, const Results &to, int *blocks_out, hipStream_t stream, const LaunchEvents &ev)
{
    const int blocks = ceil_div(a.B, THREADS / G);
    to.of(a, blocks);
    *blocks_out = blocks;
    return launch_kernel(rows_kernel<T, TO, G, N, THREADS>, dim3((unsigned)blocks), dim3(THREADS), stream, ev, a);
}

// A loss whose rows fit a block of 1024 needs no second launch for its sums: 256 rows of 7 classes 8.8 us a call, 257 rows 11.5 us,
// and 11.1 us for 256 rows in four blocks; 64 rows of 983 classes 8.8 and 11.3 us (one call alone 24.9 and 23.7 us).
template <typename T, typename TO, int G, int N>
hipError_t rows_form(const RowsArgs &a, const Results &to, int *blocks, hipStream_t s, const LaunchEvents &ev)
{
    if constexpr (G < 64)
        if (a.head == HEAD_POLICY && a.B > NT / G && a.B <= 1024 / G) return rows_launch<T, TO, G, N, 1024>(a, to, blocks, s, ev);
    return rows_launch<T, TO, G, N, (G > 64 ? G : NT)>(a, to, blocks, s, ev);
}

template <typename T, typename TO>
hipError_t rows_of_type(const RowsArgs &a, const Results &to, int *blocks, hipStream_t s, const LaunchEvents &ev)
{
    // Four pieces a lane, in as many lanes as that takes, more pieces where a row would need more than 256 lanes.  Fewer lanes
    // with more pieces make fewer wavefronts than it takes to wait for the memory, more lanes compute more of what is the same in all
    // of them (policy loss, data from memory, kernel alone in us: 20000 x 983 fp32 64 lanes x 4 34.4, 16 x 16 48.0; 2047 x 983
    // 10.7, 17.0, 256 x 1 9.2; 8192 x 983 19.6, 22.4, 24.6; 65536 x 100 fp32 8 x 4 20.1, 16 x 2 21.6, 32 x 1 33.0; 8192 x 4000
    // bf16 128 x 4 26.9, 64 x 8 29.6, 256 x 2 29.7; 2048 x 32000 bf16 256 x 16 55.0, 512 x 8 55.4, 1024 x 4 57.7; the whole call:
    // 65536 x 7 fp32 1 x 2 7.9, 2 x 1 10.5, 4 x 1 11.2).  Long rows in blocks that a compute unit has room for two of: 4000 x
    // 83793 bf16 512 x 24 271, 1024 x 12 307.
    const int n = most_pieces(a.K, a.tensor);
    if (n <= 2) return rows_form<T, TO, 1, 2>(a, to, blocks, s, ev);
    if (n <= 4) return rows_form<T, TO, 2, 2>(a, to, blocks, s, ev);
    if (n <= 16) return rows_form<T, TO, 4, 4>(a, to, blocks, s, ev);
    if (n <= 32) return rows_form<T, TO, 8, 4>(a, to, blocks, s, ev);
    if (n <= 64) return rows_form<T, TO, 16, 4>(a, to, blocks, s, ev);
    if (n <= 128) return rows_form<T, TO, 32, 4>(a, to, blocks, s, ev);
    if (n <= 256) return rows_form<T, TO, 64, 4>(a, to, blocks, s, ev);
    if (n <= 512) return rows_form<T, TO, 128, 4>(a, to, blocks, s, ev);
    if (n <= 1024) return rows_form<T, TO, 256, 4>(a, to, blocks, s, ev);
    if (n <= 2048) return rows_form<T, TO, 256, 8>(a, to, blocks, s, ev);
    if (n <= 4096) return rows_form<T, TO, 256, 16>(a, to, blocks, s, ev);
    if (n <= 6656) return rows_form<T, TO, 512, 13>(a, to, blocks, s, ev);
    if (n <= 8192) return rows_form<T, TO, 512, 16>(a, to, blocks, s, ev);
    if (n <= 12288) return rows_form<T, TO, 512, 24>(a, to, blocks, s, ev);
    if (n <= 16384) return rows_form<T, TO, 1024, 16>(a, to, blocks, s, ev);
    return rows_form<T, TO, 1024, 20>(a, to, blocks, s, ev);
}

// dz: the type of the gradient, if there is one
hipError_t rows(const RowsArgs &a, int dz, const Results &to, int *blocks, hipStream_t stream, const LaunchEvents &ev)
{
    if (a.tensor == TENSOR_BF16) return rows_of_type<__bf16, __bf16>(a, to, blocks, stream, ev);
    return a.dZ && dz == TENSOR_BF16 ? rows_of_type<float, __bf16>(a, to, blocks, stream, ev)
                                     : rows_of_type<float, float>(a, to, blocks, stream, ev);
}

RowsArgs rows_args(const ChoiceRows &r, int head)
{
    RowsArgs a = {};
    a.Z = r.Z;
    a.y = r.y;
    a.weight = r.weight;
    a.ldz = (int)r.ldz;
    a.B = (int)r.B;
    a.K = r.K;
    a.tensor = (unsigned char)r.tensor;
    a.head = (unsigned char)head;
    return a;
}

template <int FROM>
GradFrom<FROM> grad_args(const ChoiceRows &r, const ChoiceGrad &d)
{
    GradFrom<FROM> a = {};
    a.Z = r.Z;
    a.y = r.y;
    a.ldz = (int)r.ldz;
    a.B = (int)r.B;
    a.K = r.K;
    a.dZ = d.dZ;
    a.lddz = (int)d.ld;
    a.pad = d.pad;
    a.all_rows = d.all_rows;
    a.past = past_caches(r, d);
    return a;
}

// The heads of rows in chunks.  blocks: those that leave sums
hipError_t row_sums(const RowsArgs &a, const Split &s, TopSum *partial, float *chosen, hipStream_t stream, const LaunchEvents &ev)
{
    const dim3 grid((unsigned)((long long)a.B * s.chunks)), block(NT);
    return a.tensor == TENSOR_BF16
               ? launch_kernel(row_sums_kernel<__bf16>, grid, block, stream, ev, a, s.chunks, s.pieces_per_chunk, partial, chosen)
               : launch_kernel(row_sums_kernel<float>, grid, block, stream, ev, a, s.chunks, s.pieces_per_chunk, partial, chosen);
}

hipError_t chunked_rows(RowsArgs a, const Split &s, TopSum *partial, RowCoef *coef, const Results &to, int *blocks, hipStream_t stream,
                        const PassEvents &ev, double bytes)
{
    const dim3 block(NT);
    const hipError_t e = row_sums(a, s, partial, nullptr, stream, ev(PASS_LOGITS, bytes));
    if (e != hipSuccess || (s.chunks == 1 && a.head != HEAD_POLICY)) return e;
    // One block makes a loss' sums itself, if fewer lanes a row make it one
    const int lanes = s.chunks == 1 ? 1 : a.head != HEAD_POLICY || a.B <= 4 || a.B > 64 ? 64 : a.B <= 16 ? 16 : 4;
    *blocks = ceil_div(a.B, NT / lanes);
    if (*blocks > MAX_SUM_BLOCKS) *blocks = MAX_SUM_BLOCKS;
    to.of(a, *blocks);
    const dim3 merge((unsigned)*blocks);
    const auto kernel = lanes == 64 ? merge_kernel<64> : lanes == 16 ? merge_kernel<16> : lanes == 4 ? merge_kernel<4> : merge_kernel<1>;
    return launch_kernel(kernel, merge, block, stream, ev(PASS_SUMS, (double)sizeof(TopSum) * s.chunks * a.B), a, *blocks, s.chunks,
                         (const TopSum *)partial, coef);
}

// A row in G lanes
template <typename T, typename TO, int G, int FROM>
hipError_t grad_form(const GradFrom<FROM> &a, hipStream_t stream, const LaunchEvents &ev)
{
    const int blocks = ceil_div(a.B, NT / G) + a.first;
    return launch_kernel(logit_grad_kernel<T, TO, G, FROM>, dim3((unsigned)blocks), dim3(NT), stream, ev, a);
}

int grad_lanes(const ChoiceRows &r)
{
    const int n = most_pieces(r);
    return n <= 4 ? 4 : n <= 32 ? 8 : n <= 64 ? 16 : n <= 128 ? 32 : n <= 512 ? 64 : NT;
}

template <typename T, typename TO, int FROM>
hipError_t grad_of_type(const ChoiceRows &r, GradFrom<FROM> a, hipStream_t stream, const LaunchEvents &ev)
{
    a.chunks = 1;
    a.keep = false;
    if constexpr (FROM != GRAD_CHUNKS) {
        switch (grad_lanes(r)) {
        case 4: return grad_form<T, TO, 4, FROM>(a, stream, ev);
        case 8: return grad_form<T, TO, 8, FROM>(a, stream, ev);
        case 16: return grad_form<T, TO, 16, FROM>(a, stream, ev);
        case 32: return grad_form<T, TO, 32, FROM>(a, stream, ev);
        case 64: return grad_form<T, TO, 64, FROM>(a, stream, ev);
        }
    }
    const Split s = split_for(r);
    a.chunks = s.chunks;
    a.pieces_per_chunk = s.pieces_per_chunk;
    a.keep = FROM == GRAD_LOGPROB && a.Z == a.dZ && s.chunks > 1;
    const hipError_t e =
        launch_kernel(logit_grad_kernel<T, TO, NT, FROM>, dim3((unsigned)(r.B * s.chunks + a.first)), dim3(NT), stream, ev, a);
    if (e != hipSuccess || !a.keep) return e;
    return launch_kernel(chosen_grad_kernel<TO>, dim3((unsigned)ceil_div(r.B, NT)), dim3(NT), stream, LaunchEvents(), GradArgs(a));
}

template <int FROM>
hipError_t logit_grad(const ChoiceRows &r, int dz, GradFrom<FROM> a, hipStream_t stream, const LaunchEvents &ev)
{
    a.first = FROM == GRAD_CHUNKS || FROM == GRAD_PAIRS || (FROM == GRAD_ROWS && a.sums > 0);
    if (r.tensor == TENSOR_BF16) return grad_of_type<__bf16, __bf16, FROM>(r, a, stream, ev);
    if constexpr (FROM == GRAD_LOGPROB) return grad_of_type<float, float, FROM>(r, a, stream, ev);
    else return dz == TENSOR_BF16 ? grad_of_type<float, __bf16, FROM>(r, a, stream, ev) : grad_of_type<float, float, FROM>(r, a, stream, ev);
}

// Whether the gradient's kernel sums up the pairs itself, each row those of its own, and its first block all of them: one launch
// less, as long as sums of all rows in a row's lanes, or in a pair's of the first block, stay short (a pair may have all rows).
// In one stream, us, sequences of one length and all rows in the first, with a launch for the pairs and without: 300 x 983 fp32,
// 4 pairs 13.6 / 10.9 and 13.1 / 10.9; 2048 x 983, 16 pairs 18.2 / 15.4 and 20.7 / 17.4; 1024 x 32000 bf16, 16 pairs 53.5 / 50.9 and
// 53.9 / 52.2; beyond the lines 4096 x 983, 16 pairs 22.4 / 20.4 and 29.0 / 30.6, 64 pairs 22.4 / 19.9 and 29.0 / 63.7; 1024 x 7, 64
// pairs 9.3 / 8.2 and 10.0 / 27.1.
bool pairs_in_grad(const ChoiceRows &r, int pairs)
{
    const int lanes = grad_lanes(r) < 64 ? grad_lanes(r) : 64;
    return pairs <= FEW && r.B <= 32 * lanes && r.B * pairs <= 128 * NT;
}

// Up to this many pairs the first block of a gradient's kernel adds up their sums beside the other blocks; one block's reading of more
// outlasts them (us, so and with launches of their own: 16385 pairs of 4 rows x 7 46.9 / 45.8, x 983 152.6 / 156.6; 40000 pairs 102.8 /
// 96.0 and 403 / 408; 262144 pairs x 7 572 / 499; 2^22 pairs 9490 / 7050, the loss alone there 7180 / 5140).
constexpr int FEW_SUMS = 65536;

// more: room for SUM_SLICES
hipError_t add_sums(SumFour f, Four *more, hipStream_t stream, const PassEvents &ev)
{
    if (f.n > 16 * SUM_THREADS) {
        const hipError_t e =
            launch_kernel(sum_slices_kernel, dim3(SUM_SLICES), dim3(NT), stream, ev(PASS_SUMS, (double)sizeof(Four) * f.n), f.partial, f.n, more);
        if (e != hipSuccess) return e;
        f.partial = more;
        f.n = SUM_SLICES;
    }
    const LaunchEvents le = ev(PASS_SUMS, (double)sizeof(Four) * f.n);
    return f.n > NT ? launch_kernel(sum_four_kernel<SUM_THREADS>, dim3(1), dim3(SUM_THREADS), stream, le, f)
                    : launch_kernel(sum_four_kernel<NT>, dim3(1), dim3(NT), stream, le, f);
}

// What a pass over the logits, and one that writes their gradient, cannot do without
double logits_bytes(const ChoiceRows &r) { return ((r.tensor == TENSOR_BF16 ? 2.0 : 4.0) * r.K + 4.0) * (double)r.B; }
double grad_bytes(const ChoiceRows &r, const ChoiceGrad &d) { return d.dZ ? (d.tensor == TENSOR_BF16 ? 2.0 : 4.0) * r.K * (double)r.B : 0.0; }

}  // namespace

size_t choice_workspace(long long B, int pairs)
{
    static_assert(sizeof(RowCoef) + sizeof(double) + sizeof(TopSum) == sizeof(Four) && MAX_SUM_BLOCKS >= SUM_SLICES,
                  "a sum for each row, and SUM_SLICES more");
    static_assert(sizeof(TopSum) * MAX_CHUNKED >= sizeof(Four) * SUM_SLICES, "SUM_SLICES in the place of the chunks");
    return sizeof(Four) * (size_t)(pairs > MAX_SUM_BLOCKS ? pairs : MAX_SUM_BLOCKS) + (sizeof(RowCoef) + sizeof(double)) * (size_t)B +
           sizeof(TopSum) * (size_t)(B > MAX_CHUNKED ? B : MAX_CHUNKED);
}

hipError_t launch_logprob(const ChoiceRows &r, float *logp, float *lse, void *ws, hipStream_t stream, const PassEvents &ev)
{
    if (r.B == 0) return hipSuccess;
    RowsArgs a = rows_args(r, HEAD_LOGPROB);
    a.l.logp = logp;
    a.l.lse = lse;
    int blocks = 0;
    if (rows_in_registers(r, false)) return rows(a, 0, Results{}, &blocks, stream, ev(PASS_LOGITS, logits_bytes(r)));
    return chunked_rows(a, split_for(r), Workspace(ws, r.B, 0).partial, nullptr, Results{}, &blocks, stream, ev, logits_bytes(r));
}

hipError_t launch_logprob_grad(const ChoiceRows &r, const float *logp, const float *lse, const float *g, const ChoiceGrad &d,
                               hipStream_t stream, const PassEvents &ev)
{
    if (r.B == 0) return hipSuccess;
    auto a = grad_args<GRAD_LOGPROB>(r, d);
    a.logp = logp;
    a.lse = lse;
    a.g = g;
    return logit_grad(r, d.tensor, a, stream, ev(PASS_GRAD, logits_bytes(r) + grad_bytes(r, d)));
}

hipError_t launch_policy(const ChoiceRows &r, const PolicyTerms &t, const ChoiceGrad &d, void *ws, hipStream_t stream,
                         const PassEvents &ev)
{
    const Workspace w(ws, r.B, 0);
    const Results to = {w.sums, t.stats};
    SumFour fin = {w.sums, 0, t.stats};
    Four *const more = w.sums + r.B;  // (rows_kernel leaves a sum a row at most, in all of the workspace)
    if (r.B == 0) return add_sums(fin, more, stream, ev);
    RowsArgs a = rows_args(r, HEAD_POLICY);
    a.p.old_logp = t.old_logp;
    a.p.ref_logp = t.ref_logp;
    a.p.adv = t.adv;
    a.p.logp = t.logp;
    a.p.clip_low = t.clip_low;
    a.p.clip_high = t.clip_high;
    a.p.kl_coef = t.kl_coef;
    a.p.uniform = t.uniform;
    if (rows_in_registers(r, d.dZ != nullptr)) {
        a.dZ = d.dZ;
        a.lddz = (int)d.ld;
        a.pad = d.pad;
        a.past = past_caches(r, d);
        const hipError_t e = rows(a, d.tensor, to, &fin.n, stream, ev(PASS_LOGITS, logits_bytes(r) + grad_bytes(r, d)));
        return e != hipSuccess || fin.n == 1 ? e : add_sums(fin, more, stream, ev);
    }
    const Split s = split_for(r);
    // Chunks of few rows: their gradient's kernel joins them itself, and one block of it makes the sums (in one stream, with a launch
    // for that and without, us: 24 x 131072 fp32 19.1 / 16.1, 1 x 131072 10.3 / 9.3, 64 x 500000 bf16 54.9 / 51.9).
    if (d.dZ && r.B <= FEW) {
        float *const chosen = reinterpret_cast<float *>(w.coef);
        const hipError_t e = row_sums(a, s, w.partial, chosen, stream, ev(PASS_LOGITS, logits_bytes(r)));
        if (e != hipSuccess) return e;
        auto g = grad_args<GRAD_CHUNKS>(r, d);
        g.rows = a;
        g.partial_rows = w.partial;
        g.chosen = chosen;
        g.stats = t.stats;
        return logit_grad(r, d.tensor, g, stream, ev(PASS_GRAD, logits_bytes(r) + grad_bytes(r, d)));
    }
    const hipError_t e = chunked_rows(a, s, w.partial, d.dZ ? w.coef : nullptr, to, &fin.n, stream, ev, logits_bytes(r));
    if (e != hipSuccess) return e;
    if (fin.n == 1) fin.n = 0;
    if (!d.dZ) return fin.n ? add_sums(fin, nullptr, stream, ev) : hipSuccess;
    auto g = grad_args<GRAD_ROWS>(r, d);
    g.coef = w.coef;
    g.partial = fin.partial;
    g.sums = fin.n;
    g.stats = t.stats;
    return logit_grad(r, d.tensor, g, stream, ev(PASS_GRAD, logits_bytes(r) + grad_bytes(r, d)));
}

template <int FROM>
static GradFrom<FROM> grad_of_pairs(const ChoiceRows &r, const PreferenceTerms &t, const ChoiceGrad &d, const Workspace &w)
{
    auto g = grad_args<FROM>(r, d);
    g.coef = w.coef;
    g.seq = t.seq;
    g.last = 2 * t.pairs;
    g.stats = t.stats;
    return g;
}

hipError_t launch_preference(const ChoiceRows &r, const PreferenceTerms &t, const ChoiceGrad &d, void *ws, hipStream_t stream,
                             const PassEvents &ev)
{
    const Workspace w(ws, r.B, t.pairs);
    hipError_t e = hipSuccess;
    if (r.B > 0) {
        RowsArgs a = rows_args(r, HEAD_TERMS);
        a.t.row_lp = w.row_lp;
        a.t.coef = d.dZ ? w.coef : nullptr;
        a.t.seq = t.seq;
        a.t.last = 2 * t.pairs;
        int blocks = 0;
        e = rows_in_registers(r, false) ? rows(a, 0, Results{}, &blocks, stream, ev(PASS_LOGITS, logits_bytes(r)))
                                        : chunked_rows(a, split_for(r), w.partial, nullptr, Results{}, &blocks, stream, ev, logits_bytes(r));
        if (e != hipSuccess) return e;
    }
    if (d.dZ && r.B > 0 && pairs_in_grad(r, t.pairs)) {
        auto g = grad_of_pairs<GRAD_PAIRS>(r, t, d, w);
        g.p = t;
        g.row_lp = w.row_lp;
        return logit_grad(r, d.tensor, g, stream, ev(PASS_GRAD, logits_bytes(r) + grad_bytes(r, d)));
    }
    e = launch_kernel(preference_kernel, dim3((unsigned)t.pairs), dim3(NT), stream,
                      ev(PASS_SUMS, (sizeof(double) + (d.dZ ? 2.0 * sizeof(RowCoef) : 0.0)) * (double)r.B), t, r.B, (const double *)w.row_lp,
                      d.dZ ? w.coef : nullptr, w.sums);
    if (e != hipSuccess) return e;
    const SumFour fin = {w.sums, t.pairs, t.stats};
    const bool apart = !d.dZ || r.B == 0 || t.pairs > FEW_SUMS;
    if (apart) e = add_sums(fin, reinterpret_cast<Four *>(w.partial), stream, ev);  // (what was in chunks has been joined)
    if (e != hipSuccess || !d.dZ || r.B == 0) return e;
    auto g = grad_of_pairs<GRAD_ROWS>(r, t, d, w);
    g.partial = w.sums;
    g.sums = apart ? 0 : t.pairs;
    return logit_grad(r, d.tensor, g, stream, ev(PASS_GRAD, logits_bytes(r) + grad_bytes(r, d)));
}

}  // namespace hb
