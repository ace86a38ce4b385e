// Dropout with a mask that is made again wherever it is needed, never stored: a counter-based generator (Philox4x32-10,
// J. Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", SC 2011) gives element (row, col) its 16 random bits
// from (seed, offset, row, col / 8), so the forward pass and the gradient's are one kernel on other data.
#include "operators.h"

namespace hb {
namespace {

constexpr int NT = 256;
struct Words {
    unsigned w[4];
};

// a ^ b ^ c
__device__ __forceinline__ unsigned xor3(unsigned a, unsigned b, unsigned c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

__device__ __forceinline__ Words philox10(unsigned c0, unsigned c1, unsigned c2, unsigned c3, unsigned k0, unsigned k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long p0 = 0xD2511F53ull * c0, p1 = 0xCD9E8D57ull * c2;
        c0 = xor3((unsigned)(p1 >> 32), c1, k0);
        c2 = xor3((unsigned)(p0 >> 32), c3, k1);
        c1 = (unsigned)p1;
        c3 = (unsigned)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

// Eight neighbouring elements of a row, as they are stored
template <typename T>
struct Group {
    unsigned w[8 * sizeof(T) / 4];
};

__device__ __forceinline__ bool kept(const Words &r, int e, unsigned threshold)
{
    return ((e & 1) ? r.w[e >> 1] >> 16 : r.w[e >> 1] & 0xffffu) >= threshold;
}

__device__ __forceinline__ void apply(Group<float> &x, const Words &r, unsigned threshold, float scale)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) x.w[e] = kept(r, e, threshold) ? __float_as_uint(__uint_as_float(x.w[e]) * scale) : 0u;
}
__device__ __forceinline__ void apply(Group<__bf16> &x, const Words &r, unsigned threshold, float scale)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
        v2bf t;
        t[0] = (__bf16)(__uint_as_float(x.w[i] << 16) * scale);
        t[1] = (__bf16)(__uint_as_float(x.w[i] & 0xffff0000u) * scale);
        const unsigned u = __builtin_bit_cast(unsigned, t);
        x.w[i] = u & ((kept(r, 2 * i, threshold) ? 0xffffu : 0u) | (kept(r, 2 * i + 1, threshold) ? 0xffff0000u : 0u));
    }
}

// A group a thread: one counter, half a word for each element.  The load is on its way while the counter goes through its rounds
// (20 products of 32 x 32 -> 64 bits; the compiler keeps the key's additions scalar).
// Bound: memory.  16384 x 4096 bf16 38.0 us, a copy of as many bytes 37.7 us (7.1 TB/s: twice 134 MB, from the last
// cache); 65536 x 4096 172 us (6.2 TB/s).  Two or four groups a thread are slower (40.8 and 42.0 us), as is waiting for the
// load in front of the rounds (53 us); stores past the caches change nothing at 134 MB and lose at 32-bit elements (40 -> 52 us).
template <typename T>
__global__ __launch_bounds__(NT) void dropout_kernel(DropoutArgs a)
{
    const unsigned q = blockIdx.x * (unsigned)NT + threadIdx.x;
    if (q >= a.total) return;
    const unsigned row = (unsigned)(((unsigned long long)q * a.magic) >> a.shift);
    const unsigned g = q - row * a.groups;
    const T *x = static_cast<const T *>(a.x) + (long long)row * a.ldx + 8ll * g;
    T *out = static_cast<T *>(a.out) + (long long)row * a.ldo + 8ll * g;
    const int left = a.cols - 8 * (int)g;
    Group<T> v;
    T single[7];
    if (left >= 8) {
        __builtin_memcpy(&v, x, sizeof(v));
    } else {  // the row ends inside it
#pragma unroll
        for (int e = 0; e < 7; ++e) single[e] = x[min(e, left - 1)];
    }
    const Words r = philox10(g, a.row0 + row, a.c2, a.c3, a.k0, a.k1);
    if (left >= 8) {
        apply(v, r, a.threshold, a.scale);
        __builtin_memcpy(out, &v, sizeof(v));
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left) out[e] = kept(r, e, a.threshold) ? T((float)single[e] * a.scale) : T(0.f);
    }
}

}  // namespace

unsigned dropout_threshold(float p) { return (unsigned)(65536.0 * (double)p + 0.5); }

hipError_t launch_dropout(int tensor, const void *x, long long ldx, void *out, long long ldo, long long rows, long long cols,
                          unsigned threshold, uint64_t seed, uint64_t offset, hipStream_t stream, const LaunchEvents &ev)
{
    if (rows <= 0 || cols <= 0) return hipSuccess;
    DropoutArgs a = {};
    a.ldx = ldx;
    a.ldo = ldo;
    a.cols = (int)cols;
    a.groups = (unsigned)((cols + 7) / 8);
    // q / groups as a product and a shift, for q < 2^31: shift = 31 + ceil(log2 groups), magic = ceil(2^shift / groups)
    int bits = 0;
    while ((1ull << bits) < a.groups) ++bits;
    a.shift = 31 + bits;
    a.magic = (unsigned)(((1ull << a.shift) + a.groups - 1) / a.groups);
    a.threshold = threshold;
    a.scale = (float)(65536.0 / (double)(65536u - threshold));
    a.k0 = (unsigned)seed;
    a.k1 = (unsigned)(seed >> 32);
    a.c2 = (unsigned)offset;
    a.c3 = (unsigned)(offset >> 32);
    const size_t size = tensor == TENSOR_BF16 ? 2 : 4;
    const long long most = 0x7fffffffll / a.groups;  // rows of a launch (groups <= 2^28)
    for (long long r = 0; r < rows; r += most) {
        const long long n = rows - r < most ? rows - r : most;
        a.row0 = (unsigned)r;
        a.total = (unsigned)(n * a.groups);
        a.x = static_cast<const char *>(x) + (size_t)r * (size_t)ldx * size;
        a.out = static_cast<char *>(out) + (size_t)r * (size_t)ldo * size;
        const dim3 grid((a.total - 1) / NT + 1), block(NT);
        const hipError_t e = tensor == TENSOR_BF16 ? launch_kernel(dropout_kernel<__bf16>, grid, block, stream, ev, a)
                                                   : launch_kernel(dropout_kernel<float>, grid, block, stream, ev, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace hb
