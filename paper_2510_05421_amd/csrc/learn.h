// Internal interface between the C entry points (engine.hip) and the learning operators' kernels
// (learn.hip): token log-probabilities, the clipped policy loss with its gradient, and AdamW.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace dvi {

// What the kernels keep of a part of a row: with x = (z - M) log2(e) / T and y = (ref - Mq) log2(e) / Tr,
// s = sum 2^x, t = sum 2^x x, k = sum 2^x (x - y), sq = sum 2^y; za: the token's logit, where the part
// holds it; top: 1 where s leaves the largest logit itself out.  M and Mq start at the lowest finite number,
// so s == 0 (and top == 0) says that there is no logit above -inf.
struct RowStats {
    float M, s, t, k, Mq, sq, za, top;
};

struct RowArgs {
    const void *z;           // logits [N][V], row stride ldz
    long ldz;
    const void *q;           // reference logits [N][V] or nullptr
    long ldq;
    const int32_t *tok;      // [N]
    long N;
    int V;
    double it, iq;           // 1 / T, 1 / Tr
    float kz, kq;            // log2(e) / T, log2(e) / Tr (set by launch_rows)
    float *logp, *entropy;   // [N] out, or nullptr
    // policy loss (policy != 0)
    int policy;
    const float *adv, *old, *weights, *ref_logp;  // [N]; old, weights, ref_logp may be nullptr
    const int8_t *on_policy; // [N] or nullptr: rows whose ratio is 1; with it a NaN in old says the same
    const int8_t *reward;    // [N] or nullptr: advantages reward_scale (reward - baseline) instead of adv
    float reward_scale, baseline;
    float w0;                // weight of every row where weights == nullptr
    double lo, hi;           // 1 - clip_low, 1 + clip_high
    double c_kl, c_ent;
    void *dz;                // gradient [N][V], row stride lddz, or nullptr
    long lddz;
    float *terms;            // [5]: loss, policy, kl, entropy, clipped
    // workspace
    RowStats *part;          // [N][S]
    double *row_terms;       // [N][4]
};

// Workspace of launch_rows in bytes (any dtype, with or without reference).
size_t rows_workspace(long N, int V, bool policy);
// The same for N rows or any smaller number of them (fewer rows may take more: they are split).
size_t rows_workspace_up_to(long N, int V, bool policy);
void launch_rows(DType t, RowArgs a, void *workspace, hipStream_t s);

// ---- AdamW ----
constexpr int kStateBlock = 256;   // elements of a tensor that share the scales of 8-bit states
constexpr int kAdamTensors = 48;   // tensors of one launch: their table is a kernel argument (4 KiB)
constexpr int kAdamChunk = 1024;   // elements of a tensor that a workgroup takes at least
constexpr int kNormChunk = 8192;   // elements that a workgroup of the norm takes at a time
constexpr int kNormGrid = 2048;    // workgroups, and so partial sums, of a launch of the norm
constexpr int kNormDirect = 256;   // up to so many partial sums every workgroup of the step adds itself

struct AdamTensor {
    long n;
    void *p;          // parameter
    float *master;    // 32-bit copy of a bf16 parameter, or nullptr
    const void *g;
    void *m, *v;      // 32 bits: fp32 m and v; 8 bits: e4m3 codes of m and sqrt(v)
    float *ms, *vs;   // 8 bits: a scale per block of kStateBlock
    long base;        // 8 bits: number of the first element's random bits
};
struct AdamArgs {
    float b1, one_b1, b2, one_b2, decay, rate, root, eps;
    double max_norm;
    uint32_t key0, key1;
    const double *norm_part;  // partial sums of squares, n_part of them, or nullptr
    int n_part;
    float *norm;              // out, or nullptr
};
// Partial sums for a table of tensors, kNormGrid of them at most from part on; returns how many.
int adam_norm_parts(const AdamTensor *t, int n);
void launch_adam_norm(DType gt, const AdamTensor *t, int n, double *part, hipStream_t s);
// One launch for up to kAdamTensors tensors.
void launch_adamw(DType pt, bool master, DType gt, int bits, const AdamTensor *t, int n, const AdamArgs &a, hipStream_t s);
// One partial sum, part[0], for n_part of them.
void launch_adam_norm_join(double *part, int n_part, hipStream_t s);
// The norm alone, for a call without any element.
void launch_adam_norm_out(const double *part, int n_part, float *norm, hipStream_t s);

}  // namespace dvi
