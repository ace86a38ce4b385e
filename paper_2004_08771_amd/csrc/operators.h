// Internal declarations of the operators on device tensors: dropout, log-probabilities of chosen classes, the policy and the
// preference loss.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/hb.h"
#include "hb_internal.h"

namespace hb {

enum { TENSOR_F32 = 0, TENSOR_BF16 = 1 };  // HB_TENSOR_*

// ---------------------------------------------------------------- dropout
struct DropoutArgs {
    const void *x;
    void *out;
    long long ldx, ldo;
    int cols;
    unsigned row0, total, groups;  // first row, groups of eight elements in this launch and in a row
    unsigned magic;
    int shift;
    unsigned threshold;            // of 65536: halves below it drop their element
    float scale;
    unsigned k0, k1, c2, c3;       // seed and offset
};
unsigned dropout_threshold(float p);  // 65536: p rounds to 1
// out (may be x, with ldo = ldx) = x scaled where it is kept, else 0
hipError_t launch_dropout(int tensor, const void *x, long long ldx, void *out, long long ldo, long long rows, long long cols,
                          unsigned threshold, uint64_t seed, uint64_t offset, hipStream_t stream,
                          const LaunchEvents &ev = LaunchEvents());

// ---------------------------------------------------------------- chosen classes
// B rows of K logits with a chosen class each.  A row takes part if its class is in [0, K), its weight (where there are any)
// is not 0 and some logit is above -inf.
struct ChoiceRows {
    const void *Z;
    long long ldz;
    int tensor;            // of Z
    const int32_t *y;
    const float *weight;   // B entries, or null
    long long B;
    int K;
};
// Where the gradient in the logits goes; columns K .. pad - 1 of every row written are zeros (pad <= K: none)
struct ChoiceGrad {
    void *dZ;              // null: none
    long long ld;
    int tensor;
    int pad;
    bool all_rows;         // rows outside of all sequences are written, too: zeros
    bool past;             // set by the launchers: stored past the caches
};
struct PolicyTerms {
    const float *old_logp, *ref_logp, *adv;  // B entries; ref_logp may be null
    float clip_low, clip_high, kl_coef;
    float uniform;                           // weight of every row where ChoiceRows::weight is null
    float *stats;                            // 4
    float *logp;                             // B, may be null
};
struct PreferenceTerms {
    const int32_t *seq;    // 2 pairs + 1 offsets into the rows
    int pairs;
    const float *ref;      // 2 pairs, may be null
    float beta, smoothing;
    float *stats;          // 4
    float *seq_logp;       // 2 pairs, may be null
};
// Who asks for the times of a call's launches: events for each, as it is made
enum { PASS_LOGITS = 0, PASS_SUMS = 1, PASS_GRAD = 2 };  // over the logits; over rows and pairs; over the logits again, for the gradient
struct PassEvents {
    void *who = nullptr;
    LaunchEvents (*events)(void *who, int pass, double bytes) = nullptr;
    LaunchEvents operator()(int pass, double bytes) const { return events ? events(who, pass, bytes) : LaunchEvents(); }
};
size_t choice_workspace(long long B, int pairs);  // bytes, for all of the calls below
hipError_t launch_logprob(const ChoiceRows &r, float *logp, float *lse, void *ws, hipStream_t stream,
                          const PassEvents &ev = PassEvents());
hipError_t launch_logprob_grad(const ChoiceRows &r, const float *logp, const float *lse, const float *g, const ChoiceGrad &d,
                               hipStream_t stream, const PassEvents &ev = PassEvents());
hipError_t launch_policy(const ChoiceRows &r, const PolicyTerms &t, const ChoiceGrad &d, void *ws, hipStream_t stream,
                         const PassEvents &ev = PassEvents());
hipError_t launch_preference(const ChoiceRows &r, const PreferenceTerms &t, const ChoiceGrad &d, void *ws, hipStream_t stream,
                             const PassEvents &ev = PassEvents());

// rows x cols elements of `size` bytes from p on, `ld` apart; or n bytes.  A null pointer has none.
struct Block {
    const char *begin, *end;
    const char *name;
    int64_t rows, row, pitch;  // bytes of a row, and from one to the next
    Block(const void *p, int64_t rows_, int64_t cols, int64_t ld, size_t size, const char *name_ = "")
        : begin(static_cast<const char *>(p)), end(begin), name(name_), rows(rows_), row(cols * (int64_t)size), pitch(ld * (int64_t)size)
    {
        if (p && rows > 0 && cols > 0) end = begin + (size_t)(rows - 1) * (size_t)pitch + (size_t)row;
        if (rows == 1 || pitch == row) {  // one piece
            row = pitch = end - begin;
            rows = 1;
        }
    }
    Block(const void *p, size_t bytes, const char *name_)
        : begin(static_cast<const char *>(p)), end(begin + (p ? bytes : 0)), name(name_), rows(1), row(end - begin), pitch(row)
    {
    }
    bool meets(const Block &o) const
    {
        if (begin >= end || o.begin >= o.end || begin >= o.end || o.begin >= end) return false;
        return (rows == 1 && o.rows == 1) || rows_meet(o);
    }
    bool rows_meet(const Block &o) const;  // what of the two ranges is between rows is not counted
};

// What a call writes has to be apart from what it reads, and from what else it writes.  (A block of the launch may have written
// where another still has to read.)  skip: that many of either list may be the same memory
template <int N, int M>
int check_apart(const Block (&outs)[N], const Block (&ins)[M], int skip = 0)
{
    for (int i = 0; i < N; ++i) {
        for (int j = 0; j < i; ++j)
            if (outs[i].meets(outs[j])) return set_error(HB_ERR_INVALID, "%s overlaps %s", outs[i].name, outs[j].name);
        for (int j = 0; j < M; ++j)
            if ((i >= skip || j >= skip) && outs[i].meets(ins[j]))
                return set_error(HB_ERR_INVALID, "%s overlaps %s", outs[i].name, ins[j].name);
    }
    return HB_OK;
}

// what the entry points check and pass on of their arguments (operators_api.hip)
int check_dropout_p(float p, unsigned *threshold);
int check_policy(const hb_policy *p);
int check_preference(const hb_preference *p);
PolicyTerms policy_terms(const hb_policy *p, int64_t B, float *d_stats, float *d_logp);
PreferenceTerms preference_terms(const hb_preference *p, float *d_stats, float *d_seq_logp);

}  // namespace hb
