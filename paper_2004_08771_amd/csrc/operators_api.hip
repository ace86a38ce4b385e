// C ABI of the operators on device tensors (see include/hb.h): argument checks, then the launches.
#include "../../include/hb.h"
#include "operators.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

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

int check_rows(const void *Z, int64_t ldz, int tensor, const int32_t *y, int64_t B, int64_t K, bool needs_y = true)
{
    const int rc = check_type(tensor);
    if (rc != HB_OK) return rc;
    if (B < 0 || B > MAX_CHOICE_ROWS)
        return set_error(HB_ERR_INVALID, "B = %lld is outside [0, %lld]", (long long)B, (long long)MAX_CHOICE_ROWS);
    if (K < 1 || K > MAX_CLASSES) return set_error(HB_ERR_INVALID, "K = %lld is outside [1, %lld]", (long long)K, (long long)MAX_CLASSES);
    if (ldz < K) return set_error(HB_ERR_INVALID, "ldz = %lld is less than K = %lld", (long long)ldz, (long long)K);
    if (ldz > MAX_COLS) return set_error(HB_ERR_INVALID, "ldz = %lld is more than %lld", (long long)ldz, (long long)MAX_COLS);
    if (B > 0 && !Z) return set_error(HB_ERR_INVALID, "d_Z is NULL");
    if (B > 0 && needs_y && !y) return set_error(HB_ERR_INVALID, "d_y is NULL");
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

constexpr int32_t MAX_TOP = 64;

int check_scores_workspace(const void *ws, size_t ws_bytes, int64_t B, int32_t K, int32_t top)
{
    if (!ws) return set_error(HB_ERR_INVALID, "d_ws is NULL");
    if (!aligned_to(ws, 16)) return set_error(HB_ERR_INVALID, "d_ws must be 16-byte aligned");
    const size_t need = scores_workspace(B, K, top);
    if (ws_bytes < need)
        return set_error(HB_ERR_INVALID, "the workspace has %zu bytes, %zu are needed (hb_scores_workspace_bytes)", ws_bytes, need);
    return HB_OK;
}

constexpr int64_t MAX_ORTHO_DIM = 32768, MAX_ORTHO_SIZE = 1 << 30;
constexpr int MAX_ORTHO_LIST = 4096, MAX_ORTHO_STEPS = ORTHO_STEPS;
const float USUAL_COEF[3] = {3.4445f, -4.7750f, 2.0315f};

int check_ortho_operand(const void *p, int64_t ld, int64_t cols, size_t size, const char *name, int k)
{
    if (!p) return set_error(HB_ERR_INVALID, "%s of matrix %d is NULL", name, k);
    if (ld < cols || ld > MAX_COLS)
        return set_error(HB_ERR_INVALID, "the pitch of %s of matrix %d, %lld, is outside [cols = %lld, 2^31)", name, k, (long long)ld, (long long)cols);
    if (!aligned_to(p, size)) return set_error(HB_ERR_INVALID, "%s of matrix %d is not aligned to its elements", name, k);
    return HB_OK;
}

// What a list writes, and the workspace, apart from everything else in it.  Sorted by where they begin, so that only those that begin within another are compared
int check_list_apart(std::vector<Block> &outs, std::vector<Block> &ins, const void *ws, size_t ws_bytes)
{
    struct Part {
        const Block *b;
        bool out;
    };
    std::vector<Part> all;
    const Block work(ws, ws_bytes, "d_ws");
    all.reserve(outs.size() + ins.size() + 1);
    for (const Block &b : outs) all.push_back({&b, true});
    for (const Block &b : ins) all.push_back({&b, false});
    all.push_back({&work, true});
    std::sort(all.begin(), all.end(), [](const Part &x, const Part &y) { return x.b->begin < y.b->begin; });
    for (size_t i = 0; i < all.size(); ++i)
        for (size_t j = i + 1; j < all.size() && all[j].b->begin < all[i].b->end; ++j)
            if ((all[i].out || all[j].out) && all[i].b->meets(*all[j].b))
                return set_error(HB_ERR_INVALID, "%s overlaps %s", all[i].b->name, all[j].b->name);
    return HB_OK;
}

int check_ortho_workspace(const void *ws, size_t ws_bytes, const std::vector<OrthoShape> &shapes, int products, size_t *need)
{
    if (!ws) return set_error(HB_ERR_INVALID, "d_ws is NULL");
    if (!aligned_to(ws, 16)) return set_error(HB_ERR_INVALID, "d_ws must be 16-byte aligned");
    *need = ortho_workspace(shapes.data(), (int)shapes.size(), products);
    if (ws_bytes < *need)
        return set_error(HB_ERR_INVALID, "the workspace has %zu bytes, %zu are needed (hb_ortho_workspace_bytes)", ws_bytes, *need);
    return HB_OK;
}

// of a list
int check_pointers(const std::vector<Pointer> &list, hipStream_t stream)
{
    for (const Pointer &p : list) {
        const int rc = check_device<1>({p}, nullptr);
        if (rc != HB_OK) return rc;
    }
    return check_device<1>({{nullptr, ""}}, stream);
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

int check_ortho_shape(int64_t rows, int64_t cols, int k)
{
    if (rows < 0 || rows > MAX_ORTHO_DIM || cols < 0 || cols > MAX_ORTHO_DIM || rows * cols > MAX_ORTHO_SIZE)
        return set_error(HB_ERR_INVALID, "matrix %d is %lld x %lld: at most %lld rows and columns and %lld elements are supported", k, (long long)rows,
                         (long long)cols, (long long)MAX_ORTHO_DIM, (long long)MAX_ORTHO_SIZE);
    return HB_OK;
}

int check_top(int32_t top)
{
    if (top < 0 || top > MAX_TOP) return set_error(HB_ERR_INVALID, "top = %d is outside [0, %d]", top, MAX_TOP);
    return HB_OK;
}

int check_ortho(const hb_ortho *o)
{
    if (!o) return set_error(HB_ERR_INVALID, "the arguments of the steps are NULL");
    if (o->steps < 1 || o->steps > MAX_ORTHO_STEPS) return set_error(HB_ERR_INVALID, "steps = %d is outside [1, %d]", o->steps, MAX_ORTHO_STEPS);
    if (o->coef ? (o->n_coef != 1 && o->n_coef != o->steps) : o->n_coef != 0)
        return set_error(HB_ERR_INVALID, "n_coef = %d: 1 or steps = %d are needed with coef, 0 without", o->n_coef, o->steps);
    for (int i = 0; o->coef && i < 3 * o->n_coef; ++i)
        if (!(std::fabs(o->coef[i]) <= 32.f)) return set_error(HB_ERR_INVALID, "coefficient %d, %g, is outside [-32, 32]", i, (double)o->coef[i]);
    if (!(o->eps >= 0.f) || !std::isfinite(o->eps)) return set_error(HB_ERR_INVALID, "eps = %g is negative or not finite", (double)o->eps);
    return check_type(o->products);
}

int check_muon(const hb_muon *h)
{
    if (!h) return set_error(HB_ERR_INVALID, "the arguments of the update are NULL");
    if (!(h->lr >= 0.f) || !std::isfinite(h->lr)) return set_error(HB_ERR_INVALID, "lr = %g is negative or not finite", (double)h->lr);
    if (!(h->momentum >= 0.f && h->momentum < 1.f)) return set_error(HB_ERR_INVALID, "momentum = %g is outside [0, 1)", (double)h->momentum);
    if (!(h->weight_decay >= 0.f) || !std::isfinite(h->weight_decay) || !std::isfinite(h->lr * h->weight_decay))
        return set_error(HB_ERR_INVALID, "weight_decay = %g is negative or not finite", (double)h->weight_decay);
    return check_ortho(&h->ortho);
}

OrthoSteps ortho_steps(const hb_ortho *o)
{
    OrthoSteps s = {};
    s.products = o->products;
    s.steps = o->steps;
    s.n_coef = o->coef ? o->n_coef : 1;
    s.coef = o->coef ? o->coef : USUAL_COEF;
    s.eps = o->eps;
    return s;
}

OrthoSteps muon_steps(const hb_muon *h, int g_tensor)
{
    OrthoSteps s = ortho_steps(&h->ortho);
    s.g_tensor = g_tensor;
    s.muon = true;
    s.nesterov = h->nesterov != 0;
    s.lr = h->lr;
    s.momentum = h->momentum;
    s.weight_decay = h->weight_decay;
    return s;
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

size_t hb_scores_workspace_bytes(int64_t B, int32_t K, int32_t top)
{
    if (B < 0 || B > MAX_CHOICE_ROWS || K < 1 || K > MAX_CLASSES || top < 0 || top > MAX_TOP) return 0;
    return scores_workspace(B, K, top);
}

int hb_scores_async(const void *d_Z, int64_t ldz, int tensor, const int32_t *d_y, int64_t B, int32_t K, int32_t top, float *d_logp,
                    float *d_lse, float *d_entropy, int32_t *d_top_class, float *d_top_logp, void *d_ws, size_t ws_bytes,
                    void *hip_stream)
{
    int rc = check_rows(d_Z, ldz, tensor, d_y, B, K, d_logp != nullptr);
    if (rc != HB_OK) return rc;
    rc = check_top(top);
    if (rc != HB_OK) return rc;
    rc = check_scores_workspace(d_ws, ws_bytes, B, K, top);
    if (rc != HB_OK) return rc;
    if (B == 0) return HB_OK;
    if (top > 0 && !d_top_class) return set_error(HB_ERR_INVALID, "d_top_class is NULL");
    if (top == 0) {
        d_top_class = nullptr;
        d_top_logp = nullptr;
    }
    const size_t n = sizeof(float) * (size_t)B, t = n * (size_t)top;
    rc = check_apart<6, 2>({{d_logp, n, "d_logp"}, {d_lse, n, "d_lse"}, {d_entropy, n, "d_entropy"}, {d_top_class, t, "d_top_class"},
                            {d_top_logp, t, "d_top_logp"}, {d_ws, scores_workspace(B, K, top), "d_ws"}},
                           {{d_Z, B, K, ldz, size_of(tensor), "d_Z"}, {d_y, n, "d_y"}});
    if (rc != HB_OK) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    rc = check_device({{d_Z, "d_Z"}, {d_y, "d_y"}, {d_logp, "d_logp"}, {d_lse, "d_lse"}, {d_entropy, "d_entropy"},
                       {d_top_class, "d_top_class"}, {d_top_logp, "d_top_logp"}, {d_ws, "d_ws"}},
                      stream);
    if (rc != HB_OK) return rc;
    return launched(launch_scores(rows_of(d_Z, ldz, tensor, d_y, nullptr, B, K), {d_logp, d_lse, d_entropy, d_top_class, d_top_logp}, top,
                                  d_ws, stream),
                    "hb_scores_async");
}

int hb_scores_grad_async(const void *d_Z, int64_t ldz, int tensor, const int32_t *d_y, int64_t B, int32_t K, const float *d_g_logp,
                         const float *d_g_entropy, void *d_dZ, int64_t lddz, void *d_ws, size_t ws_bytes, void *hip_stream)
{
    int rc = check_rows(d_Z, ldz, tensor, d_y, B, K, d_g_logp != nullptr);
    if (rc == HB_OK) rc = check_grad(d_Z, ldz, tensor, B, K, d_dZ, lddz);
    if (rc == HB_OK) rc = check_scores_workspace(d_ws, ws_bytes, B, K, 0);
    if (rc != HB_OK) return rc;
    if (B == 0) return HB_OK;
    if (!d_dZ) return set_error(HB_ERR_INVALID, "d_dZ is NULL");
    if (!d_g_logp && !d_g_entropy) return set_error(HB_ERR_INVALID, "d_g_logp and d_g_entropy are NULL");
    const size_t n = sizeof(float) * (size_t)B;
    rc = check_apart<2, 4>({{d_dZ, B, K, lddz, size_of(tensor), "d_dZ"}, {d_ws, scores_workspace(B, K, 0), "d_ws"}},
                           {{d_Z, B, K, ldz, size_of(tensor), "d_Z"}, {d_y, n, "d_y"}, {d_g_logp, n, "d_g_logp"}, {d_g_entropy, n, "d_g_entropy"}},
                           1);
    if (rc != HB_OK) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    rc = check_device({{d_Z, "d_Z"}, {d_y, "d_y"}, {d_g_logp, "d_g_logp"}, {d_g_entropy, "d_g_entropy"}, {d_dZ, "d_dZ"}, {d_ws, "d_ws"}}, stream);
    if (rc != HB_OK) return rc;
    return launched(launch_scores_grad(rows_of(d_Z, ldz, tensor, d_y, nullptr, B, K), d_g_logp, d_g_entropy, grad_of(d_dZ, lddz, tensor),
                                       d_ws, stream),
                    "hb_scores_grad_async");
}

size_t hb_ortho_workspace_bytes(const int64_t *rows, const int64_t *cols, int32_t n, int products)
{
    if (n < 0 || n > MAX_ORTHO_LIST || check_type(products) != HB_OK || (n > 0 && (!rows || !cols))) return 0;
    try {
        std::vector<OrthoShape> shapes;
        for (int k = 0; k < n; ++k) {
            if (check_ortho_shape(rows[k], cols[k], k) != HB_OK) return 0;
            if (rows[k] > 0 && cols[k] > 0) shapes.push_back({(int)rows[k], (int)cols[k]});
        }
        return std::max<size_t>(16, ortho_workspace(shapes.data(), (int)shapes.size(), products));
    } catch (const std::bad_alloc &) {
        return 0;
    }
}

int hb_orthogonalize_async(const hb_ortho_matrix *list, int32_t n, int g_tensor, int out_tensor, const hb_ortho *how, void *d_ws,
                           size_t ws_bytes, void *hip_stream)
{
    int rc = check_type(g_tensor);
    if (rc == HB_OK) rc = check_type(out_tensor);
    if (rc == HB_OK) rc = check_ortho(how);
    if (rc != HB_OK) return rc;
    if (n < 0 || n > MAX_ORTHO_LIST) return set_error(HB_ERR_INVALID, "n = %d is outside [0, %d]", n, MAX_ORTHO_LIST);
    if (n > 0 && !list) return set_error(HB_ERR_INVALID, "the list is NULL");
    try {
        std::vector<OrthoMatrix> mats;
        std::vector<OrthoShape> shapes;
        std::vector<Block> outs, ins;
        std::vector<Pointer> pointers;
        for (int k = 0; k < n; ++k) {
            const hb_ortho_matrix &a = list[k];
            rc = check_ortho_shape(a.rows, a.cols, k);
            if (rc != HB_OK) return rc;
            if (a.rows == 0 || a.cols == 0) continue;
            rc = check_ortho_operand(a.d_g, a.ldg, a.cols, size_of(g_tensor), "d_g", k);
            if (rc == HB_OK) rc = check_ortho_operand(a.d_out, a.ldo, a.cols, size_of(out_tensor), "d_out", k);
            if (rc != HB_OK) return rc;
            outs.emplace_back(a.d_out, a.rows, a.cols, a.ldo, size_of(out_tensor), "d_out");
            // in place: all of G has been read when the first of the result is written
            if (a.d_g != a.d_out || a.ldg != a.ldo || g_tensor != out_tensor) ins.emplace_back(a.d_g, a.rows, a.cols, a.ldg, size_of(g_tensor), "d_g");
            pointers.push_back({a.d_g, "d_g"});
            pointers.push_back({a.d_out, "d_out"});
            OrthoMatrix m = {};
            m.g = a.d_g;
            m.ldg = a.ldg;
            m.out = a.d_out;
            m.ldo = a.ldo;
            mats.push_back(m);
            shapes.push_back({(int)a.rows, (int)a.cols});
        }
        if (mats.empty()) return HB_OK;
        size_t need = 0;
        rc = check_ortho_workspace(d_ws, ws_bytes, shapes, how->products, &need);
        if (rc == HB_OK) rc = check_list_apart(outs, ins, d_ws, need);
        if (rc != HB_OK) return rc;
        pointers.push_back({d_ws, "d_ws"});
        hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        rc = check_pointers(pointers, stream);
        if (rc != HB_OK) return rc;
        OrthoSteps steps = ortho_steps(how);
        steps.g_tensor = g_tensor;
        steps.out_tensor = out_tensor;
        return launched(launch_ortho(mats.data(), shapes.data(), (int)mats.size(), steps, d_ws, stream), "hb_orthogonalize_async");
    } catch (const std::bad_alloc &) {
        return set_error(HB_ERR_ALLOC, "out of host memory");
    }
}

int hb_muon_async(const hb_muon_matrix *list, int32_t n, int g_tensor, const hb_muon *how, void *d_ws, size_t ws_bytes,
                  void *hip_stream)
{
    int rc = check_type(g_tensor);
    if (rc == HB_OK) rc = check_muon(how);
    if (rc != HB_OK) return rc;
    if (n < 0 || n > MAX_ORTHO_LIST) return set_error(HB_ERR_INVALID, "n = %d is outside [0, %d]", n, MAX_ORTHO_LIST);
    if (n > 0 && !list) return set_error(HB_ERR_INVALID, "the list is NULL");
    try {
        std::vector<OrthoMatrix> mats;
        std::vector<OrthoShape> shapes;
        std::vector<Block> outs, ins;
        std::vector<Pointer> pointers;
        for (int k = 0; k < n; ++k) {
            const hb_muon_matrix &a = list[k];
            rc = check_ortho_shape(a.rows, a.cols, k);
            if (rc == HB_OK && !(std::isfinite(a.scale) && std::isfinite(how->lr * a.scale)))
                rc = set_error(HB_ERR_INVALID, "scale = %g of matrix %d is not finite", (double)a.scale, k);
            if (rc != HB_OK) return rc;
            if (a.rows == 0 || a.cols == 0) continue;
            rc = check_ortho_operand(a.d_g, a.ldg, a.cols, size_of(g_tensor), "d_g", k);
            if (rc == HB_OK) rc = check_ortho_operand(a.d_m, a.ldm, a.cols, sizeof(float), "d_m", k);
            if (rc == HB_OK) rc = check_ortho_operand(a.d_w, a.ldw, a.cols, sizeof(float), "d_w", k);
            if (rc != HB_OK) return rc;
            outs.emplace_back(a.d_m, a.rows, a.cols, a.ldm, sizeof(float), "d_m");
            outs.emplace_back(a.d_w, a.rows, a.cols, a.ldw, sizeof(float), "d_w");
            ins.emplace_back(a.d_g, a.rows, a.cols, a.ldg, size_of(g_tensor), "d_g");
            pointers.push_back({a.d_g, "d_g"});
            pointers.push_back({a.d_m, "d_m"});
            pointers.push_back({a.d_w, "d_w"});
            OrthoMatrix m = {};
            m.g = a.d_g;
            m.ldg = a.ldg;
            m.out = a.d_w;
            m.ldo = a.ldw;
            m.momentum = a.d_m;
            m.ldm = a.ldm;
            m.scale = a.scale;
            mats.push_back(m);
            shapes.push_back({(int)a.rows, (int)a.cols});
        }
        if (mats.empty()) return HB_OK;
        size_t need = 0;
        rc = check_ortho_workspace(d_ws, ws_bytes, shapes, how->ortho.products, &need);
        if (rc == HB_OK) rc = check_list_apart(outs, ins, d_ws, need);
        if (rc != HB_OK) return rc;
        pointers.push_back({d_ws, "d_ws"});
        hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        rc = check_pointers(pointers, stream);
        if (rc != HB_OK) return rc;
        return launched(launch_ortho(mats.data(), shapes.data(), (int)mats.size(), muon_steps(how, g_tensor), d_ws, stream), "hb_muon_async");
    } catch (const std::bad_alloc &) {
        return set_error(HB_ERR_ALLOC, "out of host memory");
    }
}

}  // extern "C"
