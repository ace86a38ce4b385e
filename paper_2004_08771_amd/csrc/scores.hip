// Scores of rows of logits: the log-probability of a given class, the normaliser, the entropy and the most likely classes, and the gradient in the
// logits of a weighted sum of log-probabilities and entropies.
//
// Row z of K logits.  With w the class of the largest logit m (the lowest of several), u_k = (z_k - m) log2 e, e_k = 2^u_k,
// o = sum over k != w of e_k, h = sum over k != w of e_k u_k (e_w = 1, u_w = 0), s = 1 + o:
//     log p_k = (u_k - log2 s) ln 2,   lse = m + ln s,   entropy = -sum p log p = (log2 s - h / s) ln 2,
//     d log p_y / d z_k = [k = y] - p_k,   d entropy / d z_k = -p_k (log p_k + entropy) = -p_k (u_k - h / s) ln 2.
// The largest logit is kept out of the sums, so that the log-probability of a class that is all but certain and the entropy of such a row
// keep their digits; both terms of the entropy are positive.  Exponentials and sums are fp32, what is made of them once a row is put
// together in 64 bits.
//
// The most likely classes.  Each of 64 groups of lanes has a largest logit; the top-th largest of these is a lower bound T of the top-th largest of
// the row, and what is at least T (for logits without an order little more than top values) goes to a list in LDS, where a value's rank is the number of
// those before it in the order (value, then the lowest class).  Where the list is too short (many equal values, values in order), the classes are found
// one after the other.  The order of the list does not matter, so results are the same every time.
#include "operators.h"
#include "rows_device.h"

namespace hb {
namespace {

constexpr int NT = 256;
constexpr int NO_CLASS = 0x7fffffff;
constexpr float LN2F = 0x1.62e43p-1f;
constexpr float LOWEST = -3.402823466e38f;
typedef unsigned long long u64;

enum { ROW_SCORES, ROW_GRAD, ROW_CHUNK };

// a value and its class as one number: the larger value first, of equal ones (-0 is 0) the lower class.  0: none
__device__ __forceinline__ u64 key_of(float v, int k)
{
    const unsigned b = __float_as_uint(v + 0.f);
    return ((u64)((b & 0x80000000u) ? ~b : b | 0x80000000u) << 32) | (0xffffffffu - (unsigned)k);
}
__device__ __forceinline__ int class_of(u64 key) { return (int)(0xffffffffu - (unsigned)key); }
__device__ __forceinline__ float value_of(u64 key)
{
    const unsigned b = (unsigned)(key >> 32);
    return __uint_as_float((b & 0x80000000u) ? b & 0x7fffffffu : ~b);
}

// a part of a row that a block has summed up; `top` keys follow behind all parts
struct Part {
    float top, o, h;  // top = -inf: nothing, or NaN in o
    int w;            // its largest logit's class
};

struct ScoreArgs {
    const void *Z;
    const int32_t *y;      // may be null
    int ldz, B, K;
    unsigned char tensor, top;
    bool past;             // GRAD: stored past the caches
    union {
        struct {
            float *logp, *lse, *entropy;  // each may be null
            int32_t *top_class;
            float *top_logp;              // may be null
        } s;
        struct {
            const float *g_logp, *g_entropy;  // one may be null
            void *dZ;
            int lddz;
        } g;
        struct {
            Part *parts;   // chunks a row, from row0 on
            u64 *keys;     // top a part
            int chunks, pieces, row0;
        } c;
    };
};
static_assert(sizeof(ScoreArgs) <= 112, "more arguments cost every launch up to 0.7 us");

// What a row comes down to
struct RowNumbers {
    bool none;      // no class is allowed
    float ref;      // the largest logit, 0 if there is none
    float o, h, inv_s;
    double log2_s;
    __device__ __forceinline__ RowNumbers(float top, float o_, float h_) : none(top == -INFINITY && o_ == 0.f), ref(Under(top).ref), o(o_), h(h_)
    {
        if (top == INFINITY) o = __builtin_nanf("");
        const float s = 1.f + o;
        inv_s = __builtin_amdgcn_rcpf(s);
        const TwoLog l = two_log2(s);
        log2_s = o <= 1.f ? (double)log1p_of(o) * 1.44269504088896341 : (double)l.hi + (double)l.lo;
    }
    __device__ __forceinline__ float lse() const { return none ? -INFINITY : (float)((double)ref + LN2 * log2_s); }
    __device__ __forceinline__ float entropy() const { return none ? 0.f : (float)(LN2 * (log2_s - (double)(h * inv_s))); }
    __device__ __forceinline__ float logp(float z) const
    {
        // the distance from the maximum with the factor that the exponentials have, but where it is all of the result
        const double d = (double)z - (double)ref;
        return none ? -INFINITY : (float)((d < -64.0 ? d : LN2 * (double)LOG2E * d) - LN2 * log2_s);
    }
};

__device__ __forceinline__ float logit(const ScoreArgs &a, long long row, int k)
{
    const long long i = row * a.ldz + k;
    return a.tensor == TENSOR_BF16 ? (float)static_cast<const __bf16 *>(a.Z)[i] : static_cast<const float *>(a.Z)[i];
}

// the class of a row, -1 where it has none to be found; false: the row takes no part
__device__ __forceinline__ bool takes_part(const ScoreArgs &a, long long row, int &y)
{
    y = -1;
    if (!a.y) return true;
    y = a.y[row];
    return y >= 0 && y < a.K;
}

// a place among a row's alternatives
__device__ __forceinline__ void put(const ScoreArgs &a, long long row, int slot, u64 key, const RowNumbers &r)
{
    const long long at = row * a.top + slot;
    a.s.top_class[at] = key ? class_of(key) : -1;
    if (a.s.top_logp) a.s.top_logp[at] = key ? r.logp(value_of(key)) : -INFINITY;
}

__device__ __forceinline__ void put_numbers(const ScoreArgs &a, long long row, int y, float zy, const RowNumbers &r)
{
    if (a.s.lse) a.s.lse[row] = r.lse();
    if (a.s.entropy) a.s.entropy[row] = r.entropy();
    if (a.s.logp) a.s.logp[row] = r.logp(zy);
}

// a row that takes no part
__device__ __forceinline__ void put_nothing(const ScoreArgs &a, long long row, int g, int lanes)
{
    if (g == 0) {
        if (a.s.lse) a.s.lse[row] = 0.f;
        if (a.s.entropy) a.s.entropy[row] = 0.f;
        if (a.s.logp) a.s.logp[row] = 0.f;
    }
    for (int i = g; i < a.top; i += lanes) {
        a.s.top_class[row * a.top + i] = -1;
        if (a.s.top_logp) a.s.top_logp[row * a.top + i] = 0.f;
    }
}

// The value of lane ^ J, without the trip through the LDS unit that a general shuffle is (100 cycles; what a row waits for between its passes is a few
// dozen of these): permutations within sixteen lanes are part of an instruction, those between sixteens and halves are swaps of gfx950.
template <int CTRL>
__device__ __forceinline__ float within(float v)
{
    const int x = __float_as_int(v);
    return __int_as_float(__builtin_amdgcn_update_dpp(x, x, CTRL, 0xf, 0xf, true));
}
template <int J>
__device__ __forceinline__ float across(float v)
{
    if constexpr (J == 1) return within<0xb1>(v);                      // 1 0 3 2 of four
    else if constexpr (J == 2) return within<0x4e>(v);                 // 2 3 0 1
    else if constexpr (J == 4) return within<0x1b>(within<0x141>(v));  // eight lanes mirrored, then each four
    else if constexpr (J == 8) return within<0x141>(within<0x140>(v)); // sixteen mirrored, then each eight
    else {
        typedef unsigned two __attribute__((ext_vector_type(2)));
        const unsigned x = __float_as_uint(v);
        two r;
        if constexpr (J == 16) r = __builtin_bit_cast(two, __builtin_amdgcn_permlane16_swap(x, x, false, false));
        else r = __builtin_bit_cast(two, __builtin_amdgcn_permlane32_swap(x, x, false, false));
        return __uint_as_float((threadIdx.x & J) ? r[0] : r[1]);
    }
}
template <typename F>
__device__ __forceinline__ float over_wave(float v, F f)
{
    v = f(v, across<32>(v));
    v = f(v, across<16>(v));
    v = f(v, across<8>(v));
    v = f(v, across<4>(v));
    v = f(v, across<2>(v));
    return f(v, across<1>(v));
}
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }

// the values of a wavefront's lanes in descending order
template <int K, int J>
__device__ __forceinline__ float exchanged(float v)
{
    const int lane = threadIdx.x & 63;
    const float w = across<J>(v);
    v = ((lane & J) == 0) == ((lane & K) == 0) ? fmaxf(v, w) : fminf(v, w);
    if constexpr (J > 1) v = exchanged<K, J / 2>(v);
    return v;
}
__device__ __forceinline__ float sorted(float v)
{
    v = exchanged<2, 1>(v);
    v = exchanged<4, 2>(v);
    v = exchanged<8, 4>(v);
    v = exchanged<16, 8>(v);
    v = exchanged<32, 16>(v);
    return exchanged<64, 32>(v);
}

// The maximum over the lanes of a row; red: a wavefront each
template <int WAVES>
__device__ __forceinline__ float max_of_lanes(float top, float *red)
{
    top = over_wave(top, max_of);
    if (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
        __syncthreads();
        top = red[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, red[w]);
    }
    return top;
}

__device__ __forceinline__ u64 max_of_wave(u64 v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const u64 w = __shfl_xor(v, o, 64);
        v = w > v ? w : v;
    }
    return v;
}

// what the lanes of a wavefront have written to LDS is there for the others
__device__ __forceinline__ void wave_meets()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int G>
__device__ __forceinline__ void row_meets()
{
    if (G > 64) __syncthreads();
    else wave_meets();
}

template <int G>
struct Shared {
    static constexpr int WAVES = G / 64, LIST = G == 64 ? 512 : 1024;
    float top[WAVES], o[WAVES], h[WAVES], lane_top[G > 64 ? G : 1];
    u64 best[2][WAVES];
    int w, count;
    float bound;
    u64 list[LIST];
};

template <typename T>
__device__ __forceinline__ void zero_row(T *dz, int K, int g, int lanes)
{
    constexpr int V = 16 / sizeof(T);
    const int off = (int)((reinterpret_cast<uintptr_t>(dz) & 15) / sizeof(T)), head = off ? min(V - off, K) : 0, pieces = (K - head) / V;
    const v4u zero = {0u, 0u, 0u, 0u};
    for (int p = g; p < pieces; p += lanes) reinterpret_cast<v4u *>(dz + head)[p] = zero;
    for (int j = g; j < head; j += lanes) dz[j] = T(0.f);
    for (int j = head + pieces * V + g; j < K; j += lanes) dz[j] = T(0.f);
}

// The gradient of a row: dz_k = -e_k inv_s (base + slope u_k), but for the class itself
struct GradRow {
    float ref, inv_s, base, slope, gl;
    float rest;  // 1 - p of the row's largest logit
    __device__ __forceinline__ GradRow(const RowNumbers &r, float gl_, float gh)
        : ref(r.ref), inv_s(r.inv_s), base(gl_ - gh * LN2F * r.h * r.inv_s), slope(gh * LN2F), gl(gl_), rest(r.o * r.inv_s)
    {
    }
    __device__ __forceinline__ float of(float z) const
    {
        const float u = fmaxf((z - ref) * LOG2E, -300.f);  // e u of a class that is not allowed is 0, not NaN (a NaN is in inv_s)
        return -(exp2_of(u) * inv_s) * __builtin_fmaf(slope, u, base);
    }
    // of the row's class
    __device__ __forceinline__ float chosen(float z, bool largest) const
    {
        const float u = fmaxf((z - ref) * LOG2E, -300.f), p = exp2_of(u) * inv_s;
        return gl * (largest ? rest : 1.f - p) - p * __builtin_fmaf(slope, u, base - gl);
    }
};

// G lanes have a row, or a chunk of one, between them, N pieces each and what there is at its ends: read once, whole.
template <typename T, int G, int N, int MODE>
__device__ __forceinline__ void row_in_registers(const ScoreArgs &a, long long row, int chunk, int g, Shared<G> &sh)
{
    constexpr int V = Piece<T>::V, WAVES = G / 64;
    const int lane = threadIdx.x & 63, wave = WAVES > 1 ? (int)threadIdx.x >> 6 : 0;
    int y;
    const bool part = takes_part(a, row, y);
    float gl = 0.f, gh = 0.f;
    T *dz = nullptr;
    if (MODE == ROW_GRAD) {
        dz = static_cast<T *>(a.g.dZ) + row * a.g.lddz;
        gl = a.g.g_logp ? a.g.g_logp[row] : 0.f;
        gh = a.g.g_entropy ? a.g.g_entropy[row] : 0.f;
        if (!part || (gl == 0.f && gh == 0.f)) {
            zero_row<T>(dz, a.K, g, G);
            return;
        }
    } else if (!part) {
        if (MODE == ROW_SCORES) put_nothing(a, row, g, G);
        return;
    }
    const Row<T> z(a.Z, a.ldz, row, a.K);
    const float zy = MODE != ROW_CHUNK && y >= 0 ? logit(a, row, y) : 0.f;
    const int p0 = MODE == ROW_CHUNK ? chunk * a.c.pieces : 0;
    const int count = MODE == ROW_CHUNK ? max(0, min(z.pieces - p0, a.c.pieces)) : z.pieces;
    const int most = MODE == ROW_CHUNK ? a.c.pieces : a.K / V;
    const int first = z.first(p0);
    if (g == 0) {
        sh.w = NO_CLASS;
        sh.count = 0;
    }
    Piece<T> x[N];
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(z.z + (count > 0 ? first : 0)), (short)0, count * 16, 0x00027000);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i * G < most) x[i] = Row<T>::template load<0>(rs, g, i * G);
    const int ej = MODE == ROW_CHUNK && chunk > 0 ? -1 : z.edge(g);
    float edge = z.at(ej);
    float lane_top = edge == edge ? edge : -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i * G >= most) continue;
        if ((i + 1) * G > count && i * G + g >= count) x[i].set_none();
#pragma unroll
        for (int e = 0; e < V; ++e) lane_top = fmaxf(lane_top, x[i].get(e));
        __builtin_amdgcn_sched_barrier(0);
    }
    const int top_n = MODE == ROW_GRAD ? 0 : a.top;
    if (WAVES > 1 && top_n > 1) sh.lane_top[g] = lane_top;
    const float top = max_of_lanes<WAVES>(lane_top, sh.top);

    // ---- the class of the largest logit, which leaves the sums
    int w = NO_CLASS;
    if (lane_top == top && top > -INFINITY) {
#pragma unroll
        for (int i = N - 1; i >= 0; --i) {
            if (i * G >= most) continue;
#pragma unroll
            for (int e = V - 1; e >= 0; --e) w = x[i].get(e) == top ? first + (i * G + g) * V + e : w;
        }
        if (edge == top) w = min(w, ej);
        if (WAVES > 1) atomicMin(&sh.w, w);
    }
    if (WAVES > 1) {
        __syncthreads();
        w = sh.w;
    } else {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) w = min(w, __shfl_xor(w, o, 64));
    }
    const int aw = w - first, pw = aw / V, iw = pw / G;
    const bool own = w != NO_CLASS && aw >= 0 && pw < count && pw % G == g, own_edge = w == ej;  // (no class: ej is never that)
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i * G < most && i == iw) x[i].drop(aw % V, own);
    if (own_edge) edge = -INFINITY;

    // ---- the bound of the alternatives
    if (top_n > 1 && (WAVES == 1 || wave == 0)) {
        float t = lane_top;
        if (WAVES > 1) {
#pragma unroll
            for (int i = 0; i < WAVES; ++i) t = fmaxf(t, sh.lane_top[i * 64 + lane]);
        }
        t = __shfl(sorted(t), top_n - 1, 64);
        if (g == 0) sh.bound = t;
    }

    // ---- the sums
    const Under under(top);
    float o4[4] = {0.f, 0.f, 0.f, 0.f}, h4[4] = {0.f, 0.f, 0.f, 0.f};
    {
        const float u = (edge - under.ref) * LOG2E, e = exp2_of(u);
        o4[0] = e;
        h4[0] = e * fmaxf(u, -300.f);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i * G >= most) continue;
        x[i].forget();
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float u = (x[i].get(e) - under.ref) * LOG2E, p = exp2_of(u);
            o4[e & 3] += p;
            h4[e & 3] = __builtin_fmaf(p, fmaxf(u, -300.f), h4[e & 3]);  // 0 for a class that is not allowed
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    float o = (o4[0] + o4[1]) + (o4[2] + o4[3]), h = (h4[0] + h4[1]) + (h4[2] + h4[3]);
    o = over_wave(o, sum_of);
    h = over_wave(h, sum_of);
    if (WAVES > 1) {
        if (lane == 0) {
            sh.o[wave] = o;
            sh.h[wave] = h;
        }
        __syncthreads();
        o = sh.o[0];
        h = sh.h[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) {
            o += sh.o[i];
            h += sh.h[i];
        }
    } else {
        wave_meets();
    }

    if (MODE == ROW_GRAD) {
        const RowNumbers r(top, o, h);
        if (r.none) {
            zero_row<T>(dz, a.K, g, G);
            return;
        }
        const GradRow d(r, gl, gh);
        T *to = dz + z.head;
        const bool through = (reinterpret_cast<uintptr_t>(to) & 15) == 0;
        const __amdgpu_buffer_rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(to, (short)0, z.pieces * 16, 0x00027000);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i * G >= most) continue;
            x[i].forget();
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = d.of(x[i].get(e));
            if (through && a.past) store_buffer<T, V, PAST>(out, g, i * G, v);
            else if (through) store_buffer<T, V, 0>(out, g, i * G, v);
            else if (i * G + g < count) store<T, V>(to + (i * G + g) * V, v, false);
            __builtin_amdgcn_sched_barrier(0);
        }
        // over what this lane has just stored there
        if (ej >= 0) dz[ej] = T(d.of(edge));
        if (own || own_edge) dz[w] = T(w == y ? d.chosen(top, true) : d.of(top));
        const int ay = y - z.head, py = ay / V;
        const bool has_y = y >= 0 && y != w && (y == ej || (ay >= 0 && py < count && py % G == g));
        if (has_y) dz[y] = T(d.chosen(zy, false));
        return;
    }

    const RowNumbers r(top, o, h);
    const u64 w_key = w == NO_CLASS ? 0 : key_of(top, w);
    Part *const mine = MODE == ROW_CHUNK ? a.c.parts + (row - a.c.row0) * a.c.chunks + chunk : nullptr;
    u64 *const keys = MODE == ROW_CHUNK ? a.c.keys + ((row - a.c.row0) * a.c.chunks + chunk) * a.top : nullptr;
    auto place = [&](int slot, u64 key) {
        if (MODE == ROW_CHUNK) keys[slot] = key;
        else put(a, row, slot, key, r);
    };
    if (g == 0) {
        if (MODE == ROW_CHUNK) *mine = Part{top, o, h, w};
        else put_numbers(a, row, y, zy, r);
        if (top_n > 0) place(0, w_key);
    }
    if (top_n < 2) return;

    // ---- the alternatives behind the first
    const float bound = fmaxf(sh.bound, LOWEST);  // (a class that is not allowed is none)
    if (lane_top >= bound) {
        auto add = [&](float v, int k) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < Shared<G>::LIST) sh.list[at] = key_of(v, k);
        };
        if (edge >= bound) add(edge, ej);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i * G >= most) continue;
            x[i].forget();
            unsigned in = 0u;
#pragma unroll
            for (int e = 0; e < V; ++e) in |= x[i].get(e) >= bound ? 1u << e : 0u;
            while (in) {
                const int e = __builtin_ctz(in);
                in &= in - 1;
                const int word = V == 4 ? e : e >> 1;
                const unsigned b = word & 2 ? (word & 1 ? x[i].w[3] : x[i].w[2]) : (word & 1 ? x[i].w[1] : x[i].w[0]);
                add(__uint_as_float(V == 4 ? b : (e & 1) ? b & 0xffff0000u : b << 16), first + (i * G + g) * V + e);
            }
        }
    }
    row_meets<G>();
    const int n = sh.count;
    if (n <= Shared<G>::LIST) {
        for (int t = g; t < n; t += G) {
            const u64 key = sh.list[t];
            int rank = 1;
#pragma unroll 8
            for (int j = 0; j < n; ++j) rank += sh.list[j] > key ? 1 : 0;
            if (rank < top_n) place(rank, key);
        }
        for (int t = n + 1 + g; t < top_n; t += G) place(t, 0);
        return;
    }
    // more than the list holds: one after the other, from memory again (in registers the keys of this would push the row out of them)
    u64 before = w_key;
    for (int slot = 1; slot < top_n; ++slot) {
        u64 best = 0;
        auto see = [&](float v, int k) {
            const u64 key = key_of(v, k);
            if (v >= LOWEST && key < before && key > best) best = key;
        };
        if (ej >= 0) see(z.at(ej), ej);
#pragma unroll 1
        for (int p = g; p < count; p += G) {
            const Piece<T> t = z.load(p0 + p);
#pragma unroll
            for (int e = 0; e < V; ++e) see(t.get(e), first + p * V + e);
        }
        best = max_of_wave(best);
        if (WAVES > 1) {
            if (lane == 0) sh.best[slot & 1][wave] = best;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) best = sh.best[slot & 1][i] > best ? sh.best[slot & 1][i] : best;
        }
        if (g == 0) place(slot, best);
        before = best;
    }
}

// wavefronts a SIMD that the registers have to leave room for
constexpr int score_waves(int n) { return n > 8 ? 4 : n > 4 ? 5 : 6; }

template <typename T, int G, int N, int MODE>
__global__ __launch_bounds__(G == 64 ? NT : G, score_waves(N)) void scores_kernel(ScoreArgs a)
{
    __shared__ Shared<G> sh[G == 64 ? NT / 64 : 1];
    if constexpr (MODE == ROW_CHUNK) {
        const int row = (int)blockIdx.x / a.c.chunks;
        row_in_registers<T, G, N, MODE>(a, a.c.row0 + row, (int)blockIdx.x - row * a.c.chunks, threadIdx.x, sh[0]);
    } else if constexpr (G == 64) {
        const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const long long row = (long long)blockIdx.x * (NT / 64) + sub;
        if (row < a.B) row_in_registers<T, G, N, MODE>(a, row, 0, threadIdx.x & 63, sh[sub]);
    } else {
        row_in_registers<T, G, N, MODE>(a, blockIdx.x, 0, threadIdx.x, sh[0]);
    }
}

// ---------------------------------------------------------------- rows in chunks
// A row's sums from those of its parts, by a block: every thread has them.  The largest logits of the other parts come back into them.
__device__ __forceinline__ Part merged(const Part *parts, int chunks, Part *red)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Part m = {-INFINITY, 0.f, 0.f, NO_CLASS};
    for (int c = threadIdx.x; c < chunks; c += NT) {
        const Part p = parts[c];
        if (p.top > m.top || (p.top == m.top && p.w < m.w)) {
            m.top = p.top;
            m.w = p.w;
        }
    }
    auto further = [&](float t, int w) {
        if (t > m.top || (t == m.top && w < m.w)) {
            m.top = t;
            m.w = w;
        }
    };
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) further(__shfl_xor(m.top, i, 64), __shfl_xor(m.w, i, 64));
    if (lane == 0) red[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) further(red[i].top, red[i].w);
    __syncthreads();
    for (int c = threadIdx.x; c < chunks; c += NT) {
        const Part p = parts[c];
        if (p.top == -INFINITY) {
            m.o += p.o;  // 0, or NaN
            continue;
        }
        const float all = p.w == m.w ? p.o : p.o + 1.f, down = fmaxf((p.top - m.top) * LOG2E, -300.f), r = exp2_of(down);
        m.o = __builtin_fmaf(r, all, m.o);
        m.h = __builtin_fmaf(r, __builtin_fmaf(down, all, p.h), m.h);
    }
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) {
        m.o += __shfl_xor(m.o, i, 64);
        m.h += __shfl_xor(m.h, i, 64);
    }
    if (lane == 0) {
        red[wave].o = m.o;
        red[wave].h = m.h;
    }
    __syncthreads();
    m.o = (red[0].o + red[1].o) + (red[2].o + red[3].o);
    m.h = (red[0].h + red[1].h) + (red[2].h + red[3].h);
    return m;
}

__global__ __launch_bounds__(NT) void merge_scores_kernel(ScoreArgs a, const Part *parts, const u64 *keys, int chunks, int row0)
{
    constexpr int LIST = 1024, MINE = 4;
    __shared__ Part red[NT / 64];
    __shared__ u64 red_key[2][NT / 64], list[LIST];
    __shared__ int count;
    const long long row = row0 + (long long)blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int y;
    if (!takes_part(a, row, y)) {
        put_nothing(a, row, threadIdx.x, NT);
        return;
    }
    if (threadIdx.x == 0) count = 0;
    const u64 *const k0 = keys + (long long)blockIdx.x * chunks * a.top;
    const int n = chunks * a.top;
    u64 mine[MINE];  // asked for before the sums are waited for
#pragma unroll
    for (int u = 0; u < MINE; ++u) mine[u] = threadIdx.x + u * NT < n ? k0[threadIdx.x + u * NT] : 0;
    const Part m = merged(parts + (long long)blockIdx.x * chunks, chunks, red);
    const RowNumbers r(m.top, m.o, m.h);
    if (threadIdx.x == 0) put_numbers(a, row, y, y >= 0 ? logit(a, row, y) : 0.f, r);
    if (a.top == 0) return;
    // Two lower bounds of the last key that is looked for: the largest of the parts' last ones, and the top-th largest first one (of 64 groups of parts)
    u64 bound = 1;
    for (int c = threadIdx.x; c < chunks; c += NT) {
        const u64 k = k0[(long long)c * a.top + a.top - 1];
        bound = k > bound ? k : bound;
    }
    if (wave == 0) {
        float first = -INFINITY;
        for (int c = lane; c < chunks; c += 64) first = fmaxf(first, parts[(long long)blockIdx.x * chunks + c].top);
        first = __shfl(sorted(first), a.top - 1, 64);
        const u64 k = first >= LOWEST ? key_of(first, -1) & ~0xffffffffull : 0;
        bound = k > bound ? k : bound;
    }
    bound = max_of_wave(bound);
    if (lane == 0) red_key[0][wave] = bound;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) bound = red_key[0][i] > bound ? red_key[0][i] : bound;
    auto see = [&](u64 k) {
        if (k < bound) return;
        const int at = atomicAdd(&count, 1);
        if (at < LIST) list[at] = k;
    };
#pragma unroll
    for (int u = 0; u < MINE; ++u) see(mine[u]);
    for (int i = threadIdx.x + MINE * NT; i < n; i += NT) see(k0[i]);
    __syncthreads();
    const int found = count;
    if (found <= LIST) {
        for (int t = threadIdx.x; t < found; t += NT) {
            const u64 key = list[t];
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < found; ++j) rank += list[j] > key ? 1 : 0;
            if (rank < a.top) put(a, row, rank, key, r);
        }
        for (int t = found + threadIdx.x; t < a.top; t += NT) put(a, row, t, 0, r);
        return;
    }
    u64 before = ~0ull;
    for (int slot = 0; slot < a.top; ++slot) {
        u64 best = 0;
        for (int i = threadIdx.x; i < n; i += NT) {
            const u64 k = k0[i];
            if (k < before && k > best) best = k;
        }
        best = max_of_wave(best);
        if (lane == 0) red_key[(slot + 1) & 1][wave] = best;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) best = red_key[(slot + 1) & 1][i] > best ? red_key[(slot + 1) & 1][i] : best;
        if (threadIdx.x == 0) put(a, row, slot, best, r);
        before = best;
    }
}

// A block a chunk: the row's sums from its parts, then the gradient of the chunk's pieces; the first chunk has the edges
template <typename T>
__global__ __launch_bounds__(NT) void chunk_grad_kernel(ScoreArgs a, const Part *parts, int chunks, int pieces, int row0)
{
    constexpr int V = Piece<T>::V;
    __shared__ Part red[NT / 64];
    const int at = (int)blockIdx.x / chunks, c = (int)blockIdx.x - at * chunks, g = threadIdx.x;
    const long long row = row0 + at;
    T *const dz = static_cast<T *>(a.g.dZ) + row * a.g.lddz;
    const Row<T> z(a.Z, a.ldz, row, a.K);
    const int end = min(z.pieces, (c + 1) * pieces);
    int y;
    const bool part = takes_part(a, row, y);
    const float gl = a.g.g_logp ? a.g.g_logp[row] : 0.f, gh = a.g.g_entropy ? a.g.g_entropy[row] : 0.f;
    bool zero = !part || (gl == 0.f && gh == 0.f);
    Part m = {-INFINITY, 0.f, 0.f, NO_CLASS};
    if (!zero) m = merged(parts + (long long)at * chunks, chunks, red);
    const RowNumbers r(m.top, m.o, m.h);
    zero = zero || r.none;
    const GradRow d(r, gl, gh);
    auto one = [&](float v, int k) { return zero ? 0.f : k == y ? d.chosen(v, k == m.w) : d.of(v); };
    T *const to = dz + z.head;
    for (int p = c * pieces + g; p < end; p += NT) {
        const Piece<T> x = z.load(p);
        float v[V];
        const int k = z.first(p);
        const bool has_y = (unsigned)(y - k) < (unsigned)V;
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = has_y ? one(x.get(e), k + e) : zero ? 0.f : d.of(x.get(e));
        store<T, V>(to + p * V, v, a.past);
    }
    const int ej = c == 0 ? z.edge(g) : -1;
    if (ej >= 0) dz[ej] = T(one(z.at(ej), ej));
}

// ---------------------------------------------------------------- launches
int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
int most_pieces(const ChoiceRows &r) { return r.K / (r.tensor == TENSOR_BF16 ? 8 : 4); }

constexpr int ROW_PIECES = 20 * 1024;   // the longest row that a block has room for
constexpr int CHUNK_PIECES = 4 * NT, LONG_CHUNK = 16 * NT;
constexpr int MAX_PAIRS = 8192;         // (row, chunk) pairs at a time

// Chunks are two launches: up to 64 rows they pay from 8192 pieces on (fp32 32768 classes, 64 rows, scores 11.0 us in chunks, 8.0 in registers; 65536
// 12.0 in chunks, 12.2), for gradients in bf16 from 4096 on (40000 classes 11.6, 12.4).
bool in_registers(const ChoiceRows &r, bool grad)
{
    const int n = most_pieces(r);
    return n <= (r.B > 64 ? ROW_PIECES : grad && r.tensor == TENSOR_BF16 ? 4096 : 8192);
}

struct Chunks {
    int count, pieces, rows;  // of a row; pieces of each; rows at a time
};
Chunks chunks_for(long long B, int pieces)
{
    Chunks c;
    c.count = ceil_div(pieces, CHUNK_PIECES);
    if (c.count * (B < 4 ? B : 4) > 512) c.count = ceil_div(pieces, LONG_CHUNK);
    if (c.count < 1) c.count = 1;
    c.pieces = ceil_div(pieces, c.count);
    c.rows = MAX_PAIRS / c.count;
    if (c.rows > B) c.rows = (int)B;
    return c;
}

// Lanes and pieces a lane.  A row's phases follow one another, so more lanes with less each are faster until a compute unit has rows enough to fill the
// waits of one with the work of others (us, scores with five alternatives / gradients):
//     bf16 16384 classes, 64 rows     256 x 8  8.7 /  8.5, 512 x 4  6.7 / 6.4;   4096 rows 34.5 / 49.1, 36.4 / 47.8
//     bf16 32768          64          256 x 16 13.9 / 14.7, 512 x 8 9.7 / 10.1;  4096      62.5 / 98.1, 57.3 / 93.9
//     bf16 50257          64          512 x 13 13.5 / 14.8, 1024 x 8 11.1 / 13.6; 4096     96.2 / 165, 105 / 164
//     bf16 65536        1024          512 x 16 41.3 / 51.7, 1024 x 8 36.3 / 50.2; 4096     139 / 205, 120 / 198
//     fp32 32768         256          512 x 16 10.1 / 16.5, 1024 x 8 8.7 / 16.2;  4096     99.8 / 192, 149 / 191
template <typename T, int MODE>
hipError_t rows_of_type(const ScoreArgs &a, int n, hipStream_t s, const LaunchEvents &ev)
{
    auto one = [&](auto kernel, int G) {
        const int rows = G == 64 ? NT / 64 : 1;
        return launch_kernel(kernel, dim3((unsigned)ceil_div(a.B, rows)), dim3(G == 64 ? NT : G), s, ev, a);
    };
    if (n <= 64) return one(scores_kernel<T, 64, 1, MODE>, 64);
    if (n <= 256) return one(scores_kernel<T, 64, 4, MODE>, 64);
    if (n <= 512) return one(scores_kernel<T, 128, 4, MODE>, 128);
    if (n <= 1024) return one(scores_kernel<T, 256, 4, MODE>, 256);
    if constexpr (MODE == ROW_SCORES)
        if (n <= 2048 && a.B > 1024) return one(scores_kernel<T, 256, 8, MODE>, 256);
    if (n <= 2048) return one(scores_kernel<T, 512, 4, MODE>, 512);
    if (n <= 4096) return one(scores_kernel<T, 512, 8, MODE>, 512);
    if (n <= 8192 && (a.B <= 256 || (sizeof(T) == 2 && n > 6656))) return one(scores_kernel<T, 1024, 8, MODE>, 1024);
    if (n <= 6656) return one(scores_kernel<T, 512, 13, MODE>, 512);
    if constexpr (sizeof(T) == 4)
        if (n <= 8192) return one(scores_kernel<T, 512, 16, MODE>, 512);
    if constexpr (sizeof(T) == 2 || MODE == ROW_GRAD)  // (fp32 scores would leave registers)
        if (n <= 12288) return one(scores_kernel<T, 512, 24, MODE>, 512);
    if (n <= 16384) return one(scores_kernel<T, 1024, 16, MODE>, 1024);
    return one(scores_kernel<T, 1024, 20, MODE>, 1024);
}

template <typename T>
hipError_t parts_of_type(const ScoreArgs &a, int blocks, hipStream_t s, const LaunchEvents &ev)
{
    if (a.c.pieces <= CHUNK_PIECES) return launch_kernel(scores_kernel<T, NT, 4, ROW_CHUNK>, dim3(blocks), dim3(NT), s, ev, a);
    return launch_kernel(scores_kernel<T, NT, 16, ROW_CHUNK>, dim3(blocks), dim3(NT), s, ev, a);
}

ScoreArgs args_of(const ChoiceRows &r, int top)
{
    ScoreArgs a = {};
    a.Z = r.Z;
    a.y = r.y;
    a.ldz = (int)r.ldz;
    a.B = (int)r.B;
    a.K = r.K;
    a.tensor = (unsigned char)r.tensor;
    a.top = (unsigned char)top;
    return a;
}

}  // namespace

// of either type, in registers or in chunks: what the larger needs
size_t scores_workspace(long long B, int K, int top)
{
    const long long need = B * (K / (4 * CHUNK_PIECES) + 1);
    return 256 + (size_t)(need < MAX_PAIRS ? need : MAX_PAIRS) * (sizeof(Part) + sizeof(u64) * (size_t)top);
}

// Launches of parts and of what is made of them, for as many rows at a time as the workspace takes
template <typename F>
static hipError_t in_chunks(const ChoiceRows &r, int top, void *ws, hipStream_t stream, const PassEvents &ev, F then)
{
    const int size = r.tensor == TENSOR_BF16 ? 2 : 4;
    const Chunks c = chunks_for(r.B, most_pieces(r));
    Part *const parts = static_cast<Part *>(ws);
    u64 *const keys = reinterpret_cast<u64 *>(parts + (long long)c.rows * c.count);
    hipError_t e = hipSuccess;
    for (long long row0 = 0; row0 < r.B && e == hipSuccess; row0 += c.rows) {
        const int rows = (int)(r.B - row0 < c.rows ? r.B - row0 : c.rows);
        ScoreArgs a = args_of(r, top);
        a.c.parts = parts;
        a.c.keys = keys;
        a.c.chunks = c.count;
        a.c.pieces = c.pieces;
        a.c.row0 = (int)row0;
        const LaunchEvents pass = ev(PASS_LOGITS, (double)size * rows * r.K);
        e = r.tensor == TENSOR_BF16 ? parts_of_type<__bf16>(a, rows * c.count, stream, pass) : parts_of_type<float>(a, rows * c.count, stream, pass);
        if (e == hipSuccess) e = then(parts, keys, c, rows, (int)row0);
    }
    return e;
}

hipError_t launch_scores(const ChoiceRows &r, const ScoreOut &out, int top, void *ws, hipStream_t stream, const PassEvents &ev)
{
    if (r.B == 0) return hipSuccess;
    const int size = r.tensor == TENSOR_BF16 ? 2 : 4;
    ScoreArgs a = args_of(r, top);
    a.s.logp = out.logp;
    a.s.lse = out.lse;
    a.s.entropy = out.entropy;
    a.s.top_class = out.top_class;
    a.s.top_logp = out.top_logp;
    if (in_registers(r, false)) {
        const LaunchEvents pass = ev(PASS_LOGITS, (double)size * r.B * r.K);
        return r.tensor == TENSOR_BF16 ? rows_of_type<__bf16, ROW_SCORES>(a, most_pieces(r), stream, pass)
                                       : rows_of_type<float, ROW_SCORES>(a, most_pieces(r), stream, pass);
    }
    return in_chunks(r, top, ws, stream, ev, [&](const Part *parts, const u64 *keys, const Chunks &c, int rows, int row0) {
        return launch_kernel(merge_scores_kernel, dim3((unsigned)rows), dim3(NT), stream, ev(PASS_SUMS, 0.0), a, parts, keys, c.count, row0);
    });
}

hipError_t launch_scores_grad(const ChoiceRows &r, const float *g_logp, const float *g_entropy, const ChoiceGrad &d, void *ws,
                              hipStream_t stream, const PassEvents &ev)
{
    if (r.B == 0) return hipSuccess;
    const int size = r.tensor == TENSOR_BF16 ? 2 : 4;
    ScoreArgs a = args_of(r, 0);
    a.past = (double)size * r.B * r.K > 128e6;
    a.g.g_logp = g_logp;
    a.g.g_entropy = g_entropy;
    a.g.dZ = d.dZ;
    a.g.lddz = (int)d.ld;
    if (in_registers(r, true)) {
        const LaunchEvents pass = ev(PASS_GRAD, 2.0 * size * r.B * r.K);
        return r.tensor == TENSOR_BF16 ? rows_of_type<__bf16, ROW_GRAD>(a, most_pieces(r), stream, pass)
                                       : rows_of_type<float, ROW_GRAD>(a, most_pieces(r), stream, pass);
    }
    // (the pieces of the gradient lie as those of the logits do)
    a.past = a.past && ((reinterpret_cast<uintptr_t>(d.dZ) - reinterpret_cast<uintptr_t>(r.Z)) & 15) == 0 && (d.ld - r.ldz) * size % 16 == 0;
    return in_chunks(r, 0, ws, stream, ev, [&](const Part *parts, const u64 *, const Chunks &c, int rows, int row0) {
        const LaunchEvents pass = ev(PASS_GRAD, 2.0 * size * rows * r.K);
        if (r.tensor == TENSOR_BF16)
            return launch_kernel(chunk_grad_kernel<__bf16>, dim3((unsigned)(rows * c.count)), dim3(NT), stream, pass, a, parts, c.count, c.pieces, row0);
        return launch_kernel(chunk_grad_kernel<float>, dim3((unsigned)(rows * c.count)), dim3(NT), stream, pass, a, parts, c.count, c.pieces, row0);
    });
}

}  // namespace hb
