// Rows of logits, as the kernels of log-probabilities, losses and scores read and write them, and the exponentials and logarithms that
// these share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hb {
namespace {

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

}  // namespace
}  // namespace hb
