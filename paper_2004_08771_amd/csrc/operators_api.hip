// C ABI of the operators on device tensors (see include/hb.h): argument checks, then the launches.
#include "../../include/hb.h"
#include "operators.h"

#include <cmath>

using namespace hb;

namespace {

constexpr int64_t MAX_ROWS = 0x7fffffff, MAX_COLS = 0x7fffffff;
constexpr int64_t MAX_CHOICE_ROWS = 1 << 22, MAX_CLASSES = 1 << 24;

size_t size_of(int tensor) { return tensor == HB_TENSOR_BF16 ? 2 : 4; }

int check_type(int tensor)
{
    if (tensor != HB_TENSOR_F32 && tensor != HB_TENSOR_BF16) return set_error(HB_ERR_INVALID, "unknown tensor type %d", tensor);
    return HB_OK;
}

bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// in place (the same rows), or apart
int check_out(const void *in, int64_t ldi, const void *out, int64_t ldo, int64_t rows, int64_t cols, size_t size, const char *what)
{
    if (in == out && ldi == ldo) return HB_OK;
    if (Block(in, rows, cols, ldi, size).meets(Block(out, rows, cols, ldo, size)))
        return set_error(HB_ERR_INVALID, "%s overlaps the input without being the same rows", what);
    return HB_OK;
}

// The launches go to the current device: what they read and write has to be there.
struct Pointer {
    const void *p;
    const char *name;
};
template <int N>
int check_device(const Pointer (&list)[N], hipStream_t stream)
{
    int device = -1;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return set_error(HB_ERR_DEVICE, "hipGetDevice failed: %s", hipGetErrorString(e));
    for (const Pointer &q : list) {
        if (!q.p) continue;
        hipPointerAttribute_t at = {};
        e = hipPointerGetAttributes(&at, q.p);
        if (e != hipSuccess || (at.type != hipMemoryTypeDevice && at.type != hipMemoryTypeManaged)) {
            (void)hipGetLastError();
            return set_error(HB_ERR_INVALID, "%s is not a device pointer", q.name);
        }
        if (at.type == hipMemoryTypeDevice && at.device != device)
            return set_error(HB_ERR_INVALID, "%s is on device %d, the current device is %d", q.name, at.device, device);
    }
    if (stream) {
        hipDevice_t of = -1;
        e = hipStreamGetDevice(stream, &of);
        if (e != hipSuccess) return set_error(HB_ERR_DEVICE, "hipStreamGetDevice failed: %s", hipGetErrorString(e));
        if (of != device) return set_error(HB_ERR_INVALID, "the stream is of device %d, the current device is %d", (int)of, device);
    }
    return HB_OK;
}

int launched(hipError_t e, const char *what)
{
    if (e != hipSuccess) return set_error(HB_ERR_DEVICE, "%s failed: %s", what, hipGetErrorString(e));
    return HB_OK;
}

int check_rows(const void *Z, int64_t ldz, int tensor, const int32_t *y, int64_t B, int64_t K)
{
    const int rc = check_type(tensor);
    if (rc != HB_OK) return rc;
    if (B < 0 || B > MAX_CHOICE_ROWS)
        return set_error(HB_ERR_INVALID, "B = %lld is outside [0, %lld]", (long long)B, (long long)MAX_CHOICE_ROWS);
    if (K < 1 || K > MAX_CLASSES) return set_error(HB_ERR_INVALID, "K = %lld is outside [1, %lld]", (long long)K, (long long)MAX_CLASSES);
    if (ldz < K) return set_error(HB_ERR_INVALID, "ldz = %lld is less than K = %lld", (long long)ldz, (long long)K);
    if (ldz > MAX_COLS) return set_error(HB_ERR_INVALID, "ldz = %lld is more than %lld", (long long)ldz, (long long)MAX_COLS);
    if (B > 0 && !Z) return set_error(HB_ERR_INVALID, "d_Z is NULL");
    if (B > 0 && !y) return set_error(HB_ERR_INVALID, "d_y is NULL");
    if (!aligned_to(Z, size_of(tensor))) return set_error(HB_ERR_INVALID, "d_Z is not aligned to its elements");
    return HB_OK;
}

int check_grad(const void *Z, int64_t ldz, int tensor, int64_t B, int64_t K, const void *dZ, int64_t lddz)
{
    if (lddz < K) return set_error(HB_ERR_INVALID, "lddz = %lld is less than K = %lld", (long long)lddz, (long long)K);
    if (lddz > MAX_COLS) return set_error(HB_ERR_INVALID, "lddz = %lld is more than %lld", (long long)lddz, (long long)MAX_COLS);
    if (!aligned_to(dZ, size_of(tensor))) return set_error(HB_ERR_INVALID, "d_dZ is not aligned to its elements");
    return check_out(Z, ldz, dZ, lddz, B, K, size_of(tensor), "d_dZ");
}

int check_workspace(const void *ws, size_t ws_bytes, int64_t B, int32_t pairs)
{
    if (!ws) return set_error(HB_ERR_INVALID, "d_ws is NULL");
    if (!aligned_to(ws, 16)) return set_error(HB_ERR_INVALID, "d_ws must be 16-byte aligned");
    const size_t need = choice_workspace(B, pairs);
    if (ws_bytes < need)
        return set_error(HB_ERR_INVALID, "the workspace has %zu bytes, %zu are needed (hb_choice_workspace_bytes)", ws_bytes, need);
    return HB_OK;
}

// What they write apart from what they read, but for d_dZ and d_Z
int check_policy_apart(const hb_policy *p, const int32_t *y, int64_t B, const float *stats, const float *logp, const void *Z,
                       int64_t ldz, const void *dZ, int64_t lddz, int64_t K, int tensor, const void *ws, size_t ws_bytes)
{
    const size_t n = sizeof(float) * (size_t)B, size = size_of(tensor);
    return check_apart<4, 6>({{dZ, B, K, lddz, size, "d_dZ"}, {stats, 4 * sizeof(float), "d_stats"}, {logp, n, "d_logp"}, {ws, ws_bytes, "d_ws"}},
                             {{Z, B, K, ldz, size, "d_Z"}, {y, n, "d_y"}, {p->d_old_logp, n, "d_old_logp"}, {p->d_ref_logp, n, "d_ref_logp"},
                              {p->d_adv, n, "d_adv"}, {p->d_weight, n, "d_weight"}}, 1);
}

int check_preference_apart(const hb_preference *p, const int32_t *y, int64_t B, const float *stats, const float *seq_logp,
                           const void *Z, int64_t ldz, const void *dZ, int64_t lddz, int64_t K, int tensor, const void *ws,
                           size_t ws_bytes)
{
    const size_t n = sizeof(float) * (size_t)B, pairs = 2 * sizeof(float) * (size_t)p->pairs, size = size_of(tensor);
    return check_apart<4, 4>({{dZ, B, K, lddz, size, "d_dZ"}, {stats, 4 * sizeof(float), "d_stats"}, {seq_logp, pairs, "d_seq_logp"},
                              {ws, ws_bytes, "d_ws"}},
                             {{Z, B, K, ldz, size, "d_Z"}, {y, n, "d_y"}, {p->d_seq, pairs + sizeof(int32_t), "d_seq"},
                              {p->d_ref_logp, pairs, "d_ref_logp"}}, 1);
}

ChoiceRows rows_of(const void *Z, int64_t ldz, int tensor, const int32_t *y, const float *weight, int64_t B, int32_t K)
{
    ChoiceRows r = {};
    r.Z = Z;
    r.ldz = ldz;
    r.tensor = tensor;
    r.y = y;
    r.weight = weight;
    r.B = B;
    r.K = K;
    return r;
}

ChoiceGrad grad_of(void *dZ, int64_t lddz, int tensor)
{
    ChoiceGrad d = {};
    d.dZ = dZ;
    d.ld = lddz;
    d.tensor = tensor;
    return d;
}

}  // namespace

namespace hb {

// Sum over i = 0 .. n - 1 of floor((a i + b) / m), a, b >= 0: the lattice points under a line.  What a and b hold of whole m is
// counted at once, the rest with the axes exchanged, as in Euclid's algorithm.
static __int128 floor_sum(__int128 n, __int128 m, __int128 a, __int128 b)
{
    __int128 sum = 0;
    for (;;) {
        sum += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m;
        b %= m;
        const __int128 top = a * n + b;
        if (top < m) return sum;
        n = top / m;
        b = top % m;
        const __int128 t = m;
        m = a;
        a = t;
    }
}

// Row i of this block begins s = c + i pitch behind the other one and meets row j of it if j o.pitch < s + row and j o.pitch + o.row > s:
// floor((s + row - 1) / o.pitch) - floor((s - o.row) / o.pitch) whole numbers j.  Of the rows that are within the other one's range, one that
// meets a row in front of its first or behind its last meets that one, too, so the sum of these is 0 if they are apart.
bool Block::rows_meet(const Block &o) const
{
    const __int128 c = (__int128)(begin - o.begin), range = o.end - o.begin;
    __int128 i0 = 0, i1 = rows - 1;
    if (c <= -row) i0 = (-row - c) / pitch + 1;                                   // the first with s > -row
    if (c + i1 * pitch >= range) i1 = c >= range ? -1 : (range - 1 - c) / pitch;  // the last with s < range
    if (i0 > i1) return false;
    const __int128 shift = ((__int128)row + o.row) / o.pitch + 1;                 // whole pitches, so that nothing below is negative
    const __int128 first = c + i0 * pitch + shift * o.pitch;
    return floor_sum(i1 - i0 + 1, o.pitch, pitch, first + row - 1) > floor_sum(i1 - i0 + 1, o.pitch, pitch, first - o.row);
}

int check_dropout_p(float p, unsigned *threshold)
{
    if (!(p >= 0.f && p < 1.f)) return set_error(HB_ERR_INVALID, "p = %g is outside [0, 1)", (double)p);
    *threshold = dropout_threshold(p);
    if (*threshold >= 65536u) return set_error(HB_ERR_INVALID, "p = %g rounds to 1 (it is taken in steps of 2^-16)", (double)p);
    return HB_OK;
}

int check_policy(const hb_policy *p)
{
    if (!p) return set_error(HB_ERR_INVALID, "the policy's arguments are NULL");
    if (!(p->clip_low >= 0.f && p->clip_low <= 1.f)) return set_error(HB_ERR_INVALID, "clip_low = %g is outside [0, 1]", (double)p->clip_low);
    if (!(p->clip_high >= 0.f) || !std::isfinite(p->clip_high))
        return set_error(HB_ERR_INVALID, "clip_high = %g is negative or not finite", (double)p->clip_high);
    if (!(p->kl_coef >= 0.f) || !std::isfinite(p->kl_coef))
        return set_error(HB_ERR_INVALID, "kl_coef = %g is negative or not finite", (double)p->kl_coef);
    if (p->kl_coef != 0.f && !p->d_ref_logp) return set_error(HB_ERR_INVALID, "kl_coef = %g without d_ref_logp", (double)p->kl_coef);
    return HB_OK;
}

int check_preference(const hb_preference *p)
{
    if (!p) return set_error(HB_ERR_INVALID, "the preference's arguments are NULL");
    if (p->pairs < 1 || p->pairs > (1 << 22)) return set_error(HB_ERR_INVALID, "pairs = %d is outside [1, %d]", p->pairs, 1 << 22);
    if (!p->d_seq) return set_error(HB_ERR_INVALID, "d_seq is NULL");
    if (!std::isfinite(p->beta) || !(p->beta > 0.f)) return set_error(HB_ERR_INVALID, "beta = %g is not positive and finite", (double)p->beta);
    if (!(p->smoothing >= 0.f && p->smoothing <= 0.5f))
        return set_error(HB_ERR_INVALID, "smoothing = %g is outside [0, 0.5]", (double)p->smoothing);
    return HB_OK;
}

PolicyTerms policy_terms(const hb_policy *p, int64_t B, float *d_stats, float *d_logp)
{
    PolicyTerms t = {};
    t.old_logp = p->d_old_logp;
    t.ref_logp = p->d_ref_logp;
    t.adv = p->d_adv;
    t.clip_low = p->clip_low;
    t.clip_high = p->clip_high;
    t.kl_coef = p->kl_coef;
    t.uniform = B > 0 ? 1.f / (float)B : 0.f;
    t.stats = d_stats;
    t.logp = d_logp;
    return t;
}

PreferenceTerms preference_terms(const hb_preference *p, float *d_stats, float *d_seq_logp)
{
    PreferenceTerms t = {};
    t.seq = p->d_seq;
    t.pairs = p->pairs;
    t.ref = p->d_ref_logp;
    t.beta = p->beta;
    t.smoothing = p->smoothing;
    t.stats = d_stats;
    t.seq_logp = d_seq_logp;
    return t;
}

}  // namespace hb

extern "C" {

int hb_dropout_async(const void *d_x, int64_t ldx, void *d_out, int64_t ldo, int tensor, int64_t rows, int64_t cols, float p,
                     uint64_t seed, uint64_t offset, void *hip_stream)
{
    int rc = check_type(tensor);
    if (rc != HB_OK) return rc;
    unsigned threshold = 0;
    rc = check_dropout_p(p, &threshold);
    if (rc != HB_OK) return rc;
    if (rows < 0 || rows > MAX_ROWS) return set_error(HB_ERR_INVALID, "rows = %lld is outside [0, 2^31)", (long long)rows);
    if (cols < 0 || cols > MAX_COLS) return set_error(HB_ERR_INVALID, "cols = %lld is outside [0, 2^31)", (long long)cols);
    if (rows == 0 || cols == 0) return HB_OK;
    if (ldx < cols || ldo < cols || ldx > MAX_COLS || ldo > MAX_COLS)
        return set_error(HB_ERR_INVALID, "ldx = %lld or ldo = %lld is outside [cols = %lld, 2^31)", (long long)ldx, (long long)ldo,
                         (long long)cols);
    if (!d_x || !d_out) return set_error(HB_ERR_INVALID, "d_x or d_out is NULL");
    if (!aligned_to(d_x, size_of(tensor)) || !aligned_to(d_out, size_of(tensor)))
        return set_error(HB_ERR_INVALID, "d_x or d_out is not aligned to its elements");
    rc = check_out(d_x, ldx, d_out, ldo, rows, cols, size_of(tensor), "d_out");
    if (rc != HB_OK) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    rc = check_device({{d_x, "d_x"}, {d_out, "d_out"}}, stream);
    if (rc != HB_OK) return rc;
    return launched(launch_dropout(tensor, d_x, ldx, d_out, ldo, rows, cols, threshold, seed, offset, stream), "hb_dropout_async");
}

size_t hb_choice_workspace_bytes(int64_t B, int32_t pairs)
{
    if (B < 0 || B > MAX_CHOICE_ROWS || pairs < 0 || pairs > (1 << 22)) return 0;
    return choice_workspace(B, pairs);
}

int hb_logprob_async(const void *d_Z, int64_t ldz, int tensor, const int32_t *d_y, int64_t B, int32_t K, float *d_logp,
                     float *d_lse, void *d_ws, size_t ws_bytes, void *hip_stream)
{
    int rc = check_rows(d_Z, ldz, tensor, d_y, B, K);
    if (rc == HB_OK) rc = check_workspace(d_ws, ws_bytes, B, 0);
    if (rc != HB_OK) return rc;
    if (B == 0) return HB_OK;
    if (!d_logp) return set_error(HB_ERR_INVALID, "d_logp is NULL");
    const size_t n = sizeof(float) * (size_t)B;
    rc = check_apart<3, 2>({{d_logp, n, "d_logp"}, {d_lse, n, "d_lse"}, {d_ws, choice_workspace(B, 0), "d_ws"}},
                           {{d_Z, B, K, ldz, size_of(tensor), "d_Z"}, {d_y, n, "d_y"}});
    if (rc != HB_OK) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    rc = check_device({{d_Z, "d_Z"}, {d_y, "d_y"}, {d_logp, "d_logp"}, {d_lse, "d_lse"}, {d_ws, "d_ws"}}, stream);
    if (rc != HB_OK) return rc;
    return launched(launch_logprob(rows_of(d_Z, ldz, tensor, d_y, nullptr, B, K), d_logp, d_lse, d_ws, stream), "hb_logprob_async");
}

int hb_logprob_grad_async(const void *d_Z, int64_t ldz, int tensor, const int32_t *d_y, int64_t B, int32_t K, const float *d_logp,
                          const float *d_lse, const float *d_g, void *d_dZ, int64_t lddz, void *hip_stream)
{
    int rc = check_rows(d_Z, ldz, tensor, d_y, B, K);
    if (rc == HB_OK) rc = check_grad(d_Z, ldz, tensor, B, K, d_dZ, lddz);
    if (rc != HB_OK) return rc;
    if (B == 0) return HB_OK;
    if (!d_logp || !d_lse || !d_g || !d_dZ) return set_error(HB_ERR_INVALID, "d_logp, d_lse, d_g or d_dZ is NULL");
    const size_t n = sizeof(float) * (size_t)B;
    rc = check_apart<1, 4>({{d_dZ, B, K, lddz, size_of(tensor), "d_dZ"}},
                           {{d_y, n, "d_y"}, {d_logp, n, "d_logp"}, {d_lse, n, "d_lse"}, {d_g, n, "d_g"}});
    if (rc != HB_OK) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    rc = check_device({{d_Z, "d_Z"}, {d_y, "d_y"}, {d_logp, "d_logp"}, {d_lse, "d_lse"}, {d_g, "d_g"}, {d_dZ, "d_dZ"}}, stream);
    if (rc != HB_OK) return rc;
    return launched(launch_logprob_grad(rows_of(d_Z, ldz, tensor, d_y, nullptr, B, K), d_logp, d_lse, d_g,
                                        grad_of(d_dZ, lddz, tensor), stream),
                    "hb_logprob_grad_async");
}

int hb_policy_loss_async(const void *d_Z, int64_t ldz, int tensor, const int32_t *d_y, int64_t B, int32_t K,
                         const hb_policy *policy, float *d_stats, float *d_logp, void *d_dZ, int64_t lddz, void *d_ws,
                         size_t ws_bytes, void *hip_stream)
{
    int rc = check_rows(d_Z, ldz, tensor, d_y, B, K);
    if (rc == HB_OK) rc = check_policy(policy);
    if (rc == HB_OK && d_dZ) rc = check_grad(d_Z, ldz, tensor, B, K, d_dZ, lddz);
    if (rc == HB_OK) rc = check_workspace(d_ws, ws_bytes, B, 0);
    if (rc != HB_OK) return rc;
    if (!d_stats) return set_error(HB_ERR_INVALID, "d_stats is NULL");
    if (B > 0 && (!policy->d_old_logp || !policy->d_adv)) return set_error(HB_ERR_INVALID, "d_old_logp or d_adv is NULL");
    rc = check_policy_apart(policy, d_y, B, d_stats, d_logp, d_Z, ldz, d_dZ, lddz, K, tensor, d_ws, choice_workspace(B, 0));
    if (rc != HB_OK) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    rc = check_device({{d_Z, "d_Z"}, {d_y, "d_y"}, {policy->d_old_logp, "d_old_logp"}, {policy->d_ref_logp, "d_ref_logp"},
                       {policy->d_adv, "d_adv"}, {policy->d_weight, "d_weight"}, {d_stats, "d_stats"}, {d_logp, "d_logp"},
                       {d_dZ, "d_dZ"}, {d_ws, "d_ws"}},
                      stream);
    if (rc != HB_OK) return rc;
    return launched(launch_policy(rows_of(d_Z, ldz, tensor, d_y, policy->d_weight, B, K), policy_terms(policy, B, d_stats, d_logp),
                                  grad_of(d_dZ, lddz, tensor), d_ws, stream),
                    "hb_policy_loss_async");
}

int hb_preference_loss_async(const void *d_Z, int64_t ldz, int tensor, const int32_t *d_y, int64_t B, int32_t K,
                             const hb_preference *preference, float *d_stats, float *d_seq_logp, void *d_dZ, int64_t lddz,
                             void *d_ws, size_t ws_bytes, void *hip_stream)
{
    int rc = check_rows(d_Z, ldz, tensor, d_y, B, K);
    if (rc == HB_OK) rc = check_preference(preference);
    if (rc == HB_OK && d_dZ) rc = check_grad(d_Z, ldz, tensor, B, K, d_dZ, lddz);
    if (rc == HB_OK) rc = check_workspace(d_ws, ws_bytes, B, preference->pairs);
    if (rc != HB_OK) return rc;
    if (!d_stats) return set_error(HB_ERR_INVALID, "d_stats is NULL");
    rc = check_preference_apart(preference, d_y, B, d_stats, d_seq_logp, d_Z, ldz, d_dZ, lddz, K, tensor, d_ws,
                                choice_workspace(B, preference->pairs));
    if (rc != HB_OK) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    rc = check_device({{d_Z, "d_Z"}, {d_y, "d_y"}, {preference->d_seq, "d_seq"}, {preference->d_ref_logp, "d_ref_logp"},
                       {d_stats, "d_stats"}, {d_seq_logp, "d_seq_logp"}, {d_dZ, "d_dZ"}, {d_ws, "d_ws"}},
                      stream);
    if (rc != HB_OK) return rc;
    return launched(launch_preference(rows_of(d_Z, ldz, tensor, d_y, nullptr, B, K),
                                      preference_terms(preference, d_stats, d_seq_logp), grad_of(d_dZ, lddz, tensor), d_ws, stream),
                    "hb_preference_loss_async");
}

}  // extern "C"
