// gfx950 kernels of the learning operators: log-probabilities of tokens, the clipped policy loss with its
// gradient, and AdamW over many tensors with states in 32 or 8 bits.
//
// All of them are bound by memory (by launches where the tensors are small), so each reads its inputs as
// few times as the caches allow, 16 bytes a lane, and keeps everything else in registers.
#include "learn.h"

#include <algorithm>
#include <type_traits>

#include "device.h"

namespace dvi {

// ------------------------------------------------------------------------------------------
// Rows of logits
// ------------------------------------------------------------------------------------------
// 16, 8 and 4 bytes at any address, each one access: the target allows it.  (As vectors: the compiler takes a
// copied array apart.)
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef v4u v4u_any __attribute__((aligned(1)));
typedef v2u v2u_any __attribute__((aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));
__device__ __forceinline__ uint4 ld16(const void *p) {
    const v4u v = *(const v4u_any *)p;
    return uint4{v.x, v.y, v.z, v.w};
}
// Read once, or written and not read again: past the caches (rows of 32000 in bf16 read at 6.1 TB/s so, at
// 5.3 with ordinary loads; the loss with its gradient, 4096 rows, 112 -> 108 us with such stores).
__device__ __forceinline__ uint4 ld16_once(const void *p) {
    const v4u v = __builtin_nontemporal_load((const v4u_any *)p);
    return uint4{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ void st16(void *p, const uint4 &r) { *(v4u_any *)p = v4u{r.x, r.y, r.z, r.w}; }
__device__ __forceinline__ void st16_once(void *p, const uint4 &r) {
    __builtin_nontemporal_store(v4u{r.x, r.y, r.z, r.w}, (v4u_any *)p);
}

// A row is cut into chunks of 16 bytes from its own start; the last may be partial, and is filled up with
// -inf, which adds nothing to any sum.
template <DType T> struct Chunk {
    typedef typename St<T>::type E;
    static constexpr int N = 16 / (int)sizeof(E);
    static constexpr uint32_t kNegInf = T == DType::BF16 ? 0xff80ff80u : 0xff800000u;

    // The last V % N elements (V % N > 0) and -inf behind them: the row's last 16 bytes moved down, or one by
    // one where the row is shorter than that.  V is the same for the whole launch.
    static __device__ __forceinline__ uint4 tail(const E *row, int V) {
        const int n = V % N;
        uint32_t w[4] = {kNegInf, kNegInf, kNegInf, kNegInf};
        if (V >= N) {
            const uint4 t = ld16((const uint8_t *)row + (uint32_t)(V - N) * (uint32_t)sizeof(E));
            w[0] = t.x, w[1] = t.y, w[2] = t.z, w[3] = t.w;
            int drop = N - n;
            if (T == DType::BF16) {
                if (drop & 1) {
                    w[0] = __builtin_amdgcn_alignbyte(w[1], w[0], 2);
                    w[1] = __builtin_amdgcn_alignbyte(w[2], w[1], 2);
                    w[2] = __builtin_amdgcn_alignbyte(w[3], w[2], 2);
                    w[3] = __builtin_amdgcn_alignbyte(kNegInf, w[3], 2);
                }
                drop >>= 1;
            }
            for (; drop > 0; --drop) {
                w[0] = w[1];
                w[1] = w[2];
                w[2] = w[3];
                w[3] = kNegInf;
            }
        } else if (T == DType::BF16) {
#pragma unroll
            for (int k = 0; k < 7; ++k)
                if (k < n) {
                    const uint32_t b = ((const uint16_t *)row)[k];
                    w[k / 2] = (k & 1) ? (w[k / 2] & 0xffffu) | (b << 16) : (w[k / 2] & 0xffff0000u) | b;
                }
        } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (k < n) w[k] = ((const uint32_t *)row)[k];
        }
        return uint4{w[0], w[1], w[2], w[3]};
    }
    static __device__ __forceinline__ void store_tail(E *row, int V, const uint4 &r) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
        const int first = V / N * N;
#pragma unroll
        for (int k = 0; k < N - 1; ++k)
            if (k < V % N) {
                if (T == DType::BF16)
                    ((uint16_t *)row)[first + k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
                else
                    ((uint32_t *)row)[first + k] = w[k];
            }
    }
    // all but the first element
    static __device__ __forceinline__ void store_first(uint16_t *row, const uint4 &r) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int k = 1; k < 8; ++k) row[k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
    }
};

constexpr float kLowest = -3.402823466e38f;

// What is one number a row, read at the start (beside the logits on their way); and whether the row takes
// part: a weight other than 0 and a token of the vocabulary.
struct RowIn {
    int tok;
    float w, adv, old, ref;
    bool on, counts;
};
__device__ __forceinline__ RowIn row_in(const RowArgs &a, long i) {
    RowIn r = {a.tok[i], 1.f, 0.f, 0.f, 0.f, true, false};
    if (a.policy) {
        r.w = a.weights != nullptr ? a.weights[i] : a.w0;
        r.adv = a.reward != nullptr ? a.reward_scale * ((float)a.reward[i] - a.baseline) : a.adv[i];
        if (a.old != nullptr) {
            r.old = a.old[i];
            r.on = a.on_policy != nullptr && (a.on_policy[i] != 0 || isnan(r.old));
        }
        if (a.ref_logp != nullptr) r.ref = a.ref_logp[i];
    }
    r.counts = (uint32_t)r.tok < (uint32_t)a.V && r.w != 0.f;
    return r;
}

// Where a row lies.  A bf16 row that starts between two 32-bit words counts from one element earlier
// (lead = 1), so that its chunks start on words: 16 bytes at an odd element load at three quarters of the
// rate (1024 rows of 65521 entries 73 -> 61 us), at any word at the full one, and stores at either.  Chunk 0
// then holds -inf in front.
template <DType T> struct Row {
    typedef typename St<T>::type E;
    const E *z, *q;  // less the lead
    E *dz;
    int lead, V, at, nfull, nch;  // entries and token with the lead; whole chunks, all chunks
    __device__ __forceinline__ Row(const RowArgs &a, long i, int tok, bool ref) {
        constexpr int N = Chunk<T>::N;
        z = (const E *)a.z + i * a.ldz;
        lead = T == DType::BF16 && a.V >= N ? (int)(((uintptr_t)z >> 1) & 1) : 0;
        z -= lead;
        q = ref ? (const E *)a.q + i * a.ldq - lead : nullptr;
        dz = (E *)a.dz + i * a.lddz - lead;
        V = a.V + lead;
        at = tok + lead;
        nfull = V / N;
        nch = (V + N - 1) / N;
    }
    // Whole chunk c as it lies in memory; chunk 0 of a row with a lead needs first() then.
    template <bool ONCE>
    __device__ __forceinline__ uint4 load(const E *row, int c) const {
        const uint32_t off = T == DType::BF16 ? max((uint32_t)c * 16u, (uint32_t)lead * 2u) : (uint32_t)c * 16u;
        return ONCE ? ld16_once((const uint8_t *)row + off) : ld16((const uint8_t *)row + off);
    }
    __device__ __forceinline__ void first(uint4 &r) const {
        r.w = __builtin_amdgcn_alignbyte(r.w, r.z, 2);
        r.z = __builtin_amdgcn_alignbyte(r.z, r.y, 2);
        r.y = __builtin_amdgcn_alignbyte(r.y, r.x, 2);
        r.x = __builtin_amdgcn_alignbyte(r.x, 0xff80ff80u, 2);
    }
    // Any chunk of the row (slow where the row begins or ends in it).
    __device__ __forceinline__ uint4 any(const E *row, int c) const {
        if (c >= nfull) return Chunk<T>::tail(row, V);
        uint4 r = load<false>(row, c);
        if (T == DType::BF16 && lead && c == 0) first(r);
        return r;
    }
    __device__ __forceinline__ void store(int c, const uint4 &r) const {
        if (c >= nfull)
            Chunk<T>::store_tail(dz, V, r);
        else if (T == DType::BF16 && lead && c == 0)
            Chunk<T>::store_first((uint16_t *)dz, r);
        else
            st16_once((uint8_t *)dz + (uint32_t)c * 16u, r);
    }
};

// a * b with 0 * anything == 0: a probability of 0 takes no part, whatever it is multiplied with.
// (The compiler has to know the instruction: it keeps a product that follows an exponential of its wave at
// the distance the hardware needs.)
__device__ float fmul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float mul0(float a, float b) { return fmul_legacy(a, b); }

// x = z k - b is a logit in base-2 units relative to its row's maximum M: k = log2(e) / T, b = M k as rounded,
// so that every exponential of a row is off by the same factor 2^(M k - b), which the row's numbers take out
// again.  That factor grows with |M k|.  From 2^31 on (rows that are masked with large negative numbers as
// a whole), logits that differ at all differ by more than any exponential can show: a power of two near k, by
// which M k is exact, serves as well, and one 2^60 times smaller where M k would leave fp32's range.
struct Scale {
    float k, b;
    __device__ __forceinline__ float of(float z) const { return fmaf(z, k, -b); }
};
__device__ __forceinline__ Scale scale_of(float M, float k) {
#pragma clang fp contract(off)  // b is the rounded product wherever it goes
    Scale s = {k, M * k};
    const bool large = !(fabsf(s.b) < 0x1p31f);
    if (__builtin_amdgcn_ballot_w64(large) != 0) {  // hardly ever: a branch, not its instructions
        const float two = __uint_as_float(__float_as_uint(k) & 0x7f800000u);
        const float kl = fabsf(s.b) < 0x1p100f ? two : two * 0x1p-60f;
        s.k = large ? kl : k;
        s.b = large ? M * kl : s.b;
    }
    return s;
}

// The sums of one more chunk, x of the logits and y of the reference's: s = sum 2^x, t = sum 2^x x and, for the
// KL divergence, k = sum 2^x (x - y): differences of logits that are already relative to their maxima, so
// nothing large cancels.  A -inf (2^x == 0) adds nothing even where x or y is infinite; a NaN makes the
// sums NaN.
template <DType T, bool REF>
__device__ __forceinline__ void add_chunk(RowStats &r, const uint4 &zc, const uint4 &qc, Scale sz, Scale sq) {
    constexpr int N = Chunk<T>::N;
    float z[N], q[N];
    unpack_frag<T>(zc, z);
    if (REF) unpack_frag<T>(qc, q);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float x = sz.of(z[k]), e = __builtin_amdgcn_exp2f(x);
        r.s += e;
        r.t += mul0(e, x);
        if (REF) {
            const float y = sq.of(q[k]);
            r.sq += __builtin_amdgcn_exp2f(y);
            r.k += mul0(e, x - y);
        }
    }
}

// A thread's sums and the scales that they are relative to.
struct Sums {
    RowStats r;
    Scale z, q;
};
__device__ __forceinline__ Sums no_sums(float za, float kz, float kq) {
    return {{kLowest, 0.f, 0.f, 0.f, kLowest, 0.f, za, 0.f}, scale_of(kLowest, kz), scale_of(kLowest, kq)};
}

// Sums relative to new maxima M, Mq (at least the old ones).
template <bool REF>
__device__ __forceinline__ void rebase(Sums &s, float M, float Mq, float kz, float kq) {
    RowStats &r = s.r;
    const Scale nz = scale_of(M, kz);
    const float dx = s.z.b - nz.b, f = __builtin_amdgcn_exp2f(dx);
    if (REF) {
        // a reference masked by the lowest number: dy is as large as that, and counts only where f s does
        const Scale nq = scale_of(Mq, kq);
        const float dy = s.q.b - nq.b;
        r.k = mul0(f, r.k + mul0(r.s, dx - dy));
        r.sq *= __builtin_amdgcn_exp2f(dy);
        r.Mq = Mq;
        s.q = nq;
    }
    r.t = mul0(f, r.t + mul0(r.s, dx));
    r.s *= f;
    r.M = M;
    s.z = nz;
}

template <DType T>
__device__ __forceinline__ float chunk_max(const uint4 &c) {
    constexpr int N = Chunk<T>::N;
    float v[N];
    unpack_frag<T>(c, v);
    float m = v[0];
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, v[k]);
    return m;
}

// The sums of U more chunks, their maxima first; chunk u counts where used[u].
template <DType T, bool REF, int U>
__device__ __forceinline__ void add_chunks(Sums &s, const uint4 *zc, const uint4 *qc, const bool *used, float kz, float kq) {
    float M = s.r.M, Mq = s.r.Mq;
#pragma unroll
    for (int u = 0; u < U; ++u) {  // a thread's maximum is one of its own chunks'
        M = fmaxf(M, used[u] ? chunk_max<T>(zc[u]) : kLowest);
        if (REF) Mq = fmaxf(Mq, used[u] ? chunk_max<T>(qc[u]) : kLowest);
    }
    rebase<REF>(s, M, Mq, kz, kq);
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (used[u]) add_chunk<T, REF>(s.r, zc[u], REF ? qc[u] : zc[u], s.z, s.q);
}

// What the gradient of a row needs: dz = 2^x (A x - C y + B), plus `at` at the token.
struct RowCoef {
    Scale z, q;
    float A, B, C, at, dead, pad;
};

// exp and log of a row's numbers in 64 bits, by a Taylor and an atanh series: accurate to a few 1e-15, and short
// enough that the rows the waves hold stay in their registers beside them.
__device__ __forceinline__ double exp64(double x) {
    x = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;  // a NaN stays one
    const double k = rint(x * 1.4426950408889634074);
    const double r = fma(k, -1.9082149292705877e-10, fma(k, -0.69314718036912381649, x));
    double p = 1.0 / 39916800.0;
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return ldexp(p, (int)k);
}
__device__ __forceinline__ double log64(double s) {  // s > 0 and normal
    int k;
    double m = frexp(s, &k);  // [0.5, 1)
    if (m < 0.70710678118654752) {
        m *= 2.0;
        --k;
    }
    const double t = (m - 1.0) / (m + 1.0), t2 = t * t;
    double p = 1.0 / 17.0;
    p = fma(p, t2, 1.0 / 15.0);
    p = fma(p, t2, 1.0 / 13.0);
    p = fma(p, t2, 1.0 / 11.0);
    p = fma(p, t2, 1.0 / 9.0);
    p = fma(p, t2, 1.0 / 7.0);
    p = fma(p, t2, 1.0 / 5.0);
    p = fma(p, t2, 1.0 / 3.0);
    p = fma(p, t2, 1.0);
    return fma((double)k, 0.693147180559945309417, 2.0 * t * p);
}

__device__ __forceinline__ float uniform(float v) {
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}
__device__ __forceinline__ RowCoef uniform(const RowCoef &c) {
    return {{uniform(c.z.k), uniform(c.z.b)}, {uniform(c.q.k), uniform(c.q.b)}, uniform(c.A), uniform(c.B), uniform(c.C),
            uniform(c.at), uniform(c.dead), 0.f};
}

// The row's numbers from its sums, in 64 bits: differences of logits and their logarithms decide on which
// side of the clipping border a ratio falls.
__device__ __forceinline__ RowCoef row_numbers(const RowArgs &a, const RowIn &in, const RowStats &r, float &logp,
                                               float &entropy, double (&terms)[4]) {
    constexpr double ln2 = 0.693147180559945309417;
    RowCoef c = {scale_of(r.M, a.kz), scale_of(r.Mq, a.kq), 0.f, 0.f, 0.f, 0.f, 1.f, 0.f};
    logp = entropy = 0.f;
    terms[0] = terms[1] = terms[2] = terms[3] = 0.0;
    if ((r.s == 0.f && r.top == 0.f) || (a.q != nullptr && r.sq == 0.f)) return c;
    // the factor that all of the row's exponentials share; the token's logit goes by the exact temperature
    const double rest = ln2 * ((double)r.M * (double)c.z.k - (double)c.z.b);
    const double s = (double)r.s + (r.top != 0.f ? (double)r.top * exp64(rest) : 0.0), lns = log64(s);
    const double lp = ((double)r.za - (double)r.M) * a.it + rest - lns;
    const double H = lns - ln2 * (double)r.t / s;
    logp = (float)lp;
    entropy = (float)H;
    c.dead = 0.f;
    if (!a.policy) return c;
    const double w = (double)in.w, adv = (double)in.adv;
    const double ratio = in.on ? 1.0 : exp64(lp - (double)in.old);
    const double plain = ratio * adv, held = fmin(fmax(ratio, a.lo), a.hi) * adv;
    const bool cut = held < plain;
    const double pol = cut ? -held : -plain;
    double by_lp = cut ? 0.0 : -plain, kl = 0.0, k0 = a.c_ent * (H - lns);
    if (a.q != nullptr) {
        const double lnq = log64((double)r.sq);
        kl = ln2 * (double)r.k / s - lns + lnq;
        if (a.c_kl != 0.0) k0 += a.c_kl * (lnq - lns - kl);
    } else if (a.ref_logp != nullptr) {
        const double d = (double)in.ref - lp, ed = exp64(d);
        kl = ed - d - 1.0;
        if (a.c_kl != 0.0) by_lp += a.c_kl * (1.0 - ed);
    }
    const double scale = w * a.it;
    c.A = (float)(scale / s * ln2 * (a.q != nullptr ? a.c_ent + a.c_kl : a.c_ent));
    c.B = (float)(scale / s * (k0 - by_lp));
    c.C = (float)(scale / s * ln2 * a.c_kl);
    c.at = (float)(scale * by_lp);
    terms[0] = w * pol;
    terms[1] = w * kl;
    terms[2] = w * H;
    terms[3] = cut ? w : 0.0;
    return c;
}

// The gradient of one chunk, without the token's own term.
template <DType T, bool REF>
__device__ __forceinline__ void grad_chunk(const RowCoef &r, const uint4 &zc, const uint4 &qc, float *g) {
    constexpr int N = Chunk<T>::N;
    float z[N], q[N];
    unpack_frag<T>(zc, z);
    if (REF) unpack_frag<T>(qc, q);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float x = r.z.of(z[k]), e = __builtin_amdgcn_exp2f(x);
        float in = fmaf(r.A, x, r.B);
        if (REF) in = fmaf(-r.C, r.q.of(q[k]), in);
        g[k] = mul0(e, in);
    }
}
template <DType T>
__device__ __forceinline__ void add_token(float *g, int k0, float v) {
#pragma unroll
    for (int k = 0; k < Chunk<T>::N; ++k) g[k] += k == k0 ? v : 0.f;
}

template <bool REF>
__device__ __forceinline__ void sum_lanes(RowStats &r) {
    r.s = wave_sum(r.s);
    r.t = wave_sum(r.t);
    if (REF) {
        r.k = wave_sum(r.k);
        r.sq = wave_sum(r.sq);
    }
}

// The workgroup's threads' sums as one, in a fixed order, in every lane of wave 0 (other waves: anything).
// A row whose largest probability is close to 1 has its logarithm in what the other tokens add, which a sum
// that holds the largest itself would round away: where the whole is below 1.5 times that (so that one thread alone
// has the maximum, once), that thread's chunks are read again and added without it; s is then the sum of the
// others, and top 1.  Thread t's chunks are first + t, first + t + NT, ... below last.
template <DType T, bool REF, int NT>
__device__ __forceinline__ RowStats join_threads(Sums s, const RowArgs &a, const Row<T> &row, int first, int last) {
    constexpr int NW = NT / 64, N = Chunk<T>::N;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    RowStats &r = s.r;
    const float M = wave_max(r.M), Mq = REF ? wave_max(r.Mq) : kLowest;
    const bool mine = r.M == M;
    rebase<REF>(s, M, Mq, a.kz, a.kq);
    float other = wave_sum(mine ? 0.f : r.s), who = wave_max(mine ? (float)threadIdx.x : -1.f);
    sum_lanes<REF>(r);
    if (NW > 1) {
        __shared__ RowStats waves[NW];
        __shared__ float others[NW], whos[NW];
        if (lane == 0) {
            waves[w] = r;
            others[w] = other;
            whos[w] = who;
        }
        __syncthreads();
        if (w != 0) return r;
        const int l = lane & (NW - 1);
        const bool in = lane < NW;
        const float za = r.za;
        r = waves[l];
        r.za = za;
        s.z = scale_of(r.M, a.kz);
        s.q = scale_of(r.Mq, a.kq);
        const float Mw = wave_max(r.M), Mqw = REF ? wave_max(r.Mq) : kLowest;
        const bool has = r.M == Mw;
        rebase<REF>(s, Mw, Mqw, a.kz, a.kq);
        other = wave_sum(in ? (has ? others[l] : r.s) : 0.f);
        who = wave_max(in && has ? whos[l] : -1.f);
        if (!in) r.s = r.t = r.k = r.sq = 0.f;
        sum_lanes<REF>(r);
    }
    const Scale sz = s.z;
    if (r.s < 1.5f * __builtin_amdgcn_exp2f(sz.of(r.M)) && r.s > 0.f) {
        float own = 0.f;
        for (int c = first + (int)who + lane * NT; c < last; c += 64 * NT) {
            float v[N];
            unpack_frag<T>(row.any(row.z, c), v);
#pragma unroll
            for (int k = 0; k < N; ++k) own += v[k] == r.M ? 0.f : __builtin_amdgcn_exp2f(sz.of(v[k]));
        }
        r.s = other + wave_sum(own);
        r.top = 1.f;
    }
    return r;
}

// Wave 0 of a row's workgroup: its numbers out of its sums, and the outputs that are one a row.
__device__ __forceinline__ RowCoef finish_row(const RowArgs &a, long i, const RowIn &in, const RowStats &r, bool out) {
    float logp, entropy;
    double terms[4];
    const RowCoef c = row_numbers(a, in, r, logp, entropy, terms);
    if (out && threadIdx.x == 0) {
        if (a.logp != nullptr) a.logp[i] = logp;
        if (a.entropy != nullptr) a.entropy[i] = entropy;
        if (a.policy)
#pragma unroll
            for (int k = 0; k < 4; ++k) a.row_terms[i * 4 + k] = terms[k];
    }
    return c;
}
__device__ __forceinline__ void mask_row(const RowArgs &a, long i) {
    if (threadIdx.x != 0) return;
    if (a.logp != nullptr) a.logp[i] = 0.f;
    if (a.entropy != nullptr) a.entropy[i] = 0.f;
    if (a.policy)
        for (int k = 0; k < 4; ++k) a.row_terms[i * 4 + k] = 0.0;
}

// The gradient of chunk c of a row.
template <DType T, bool REF>
__device__ __forceinline__ uint4 grad_of(const RowCoef &r, int c, int at, const uint4 &zc, const uint4 &qc) {
    constexpr int N = Chunk<T>::N;
    if (r.dead != 0.f) return uint4{0u, 0u, 0u, 0u};
    float g[N];
    if (REF && r.C != 0.f)
        grad_chunk<T, REF>(r, zc, qc, g);
    else
        grad_chunk<T, false>(r, zc, zc, g);
    if (c == at / N) add_token<T>(g, at % N, r.at);
    return pack_frag_cvt<T>(g);
}

// One workgroup a row, read once: thread t holds chunks t, t + NT, ... from the first look to the gradient,
// NC of them in registers and the next SL in LDS.  With BIG there are more, which are read twice: last for the
// sums and first for the gradient, when the L2 may still hold them (2048 rows of 131072 in bf16 with a
// reference, a quarter of it read twice: 384 -> 342 us).  The sums run with each thread's own maximum, as the
// loads arrive, so a row needs two barriers.  NC = 0: no gradient is wanted, and nothing is held.
// Bound by memory where rows share a compute unit, one loading while another computes: 4096 rows of 32000 in
// bf16, a quarter of them masked, 85 us (5.4 TB/s; a device copy reaches 5.0), log-probabilities of 8192
// rows 77 us (6.1 TB/s read).  A reference makes it 30 vector operations an entry, which a row that fills the
// unit hides only in part: 256 rows of 32000 in fp32 19.4 us (5.1 TB/s), 2048 of 131072 in bf16 342 (4.7).
template <DType T, bool REF, int NT, int NC, int SL, bool BIG>
__global__ void __launch_bounds__(NT) row_kernel(RowArgs a) {
    typedef typename St<T>::type E;
    constexpr int N = Chunk<T>::N, R = NC > 0 ? NC : 1, P = REF ? 2 : 1;
    __shared__ RowCoef coef;
    extern __shared__ uint4 kept[];  // [SL][P][NT]
    const long i = blockIdx.x;
    const int tid = threadIdx.x;
    const RowIn in = row_in(a, i);
    const Row<T> row(a, i, in.tok, REF);
    const int nfull = row.nfull, nch = row.nch;
    if (!in.counts) {
        if (NC > 0)
            for (int c = tid; c < nch; c += NT) row.store(c, uint4{0u, 0u, 0u, 0u});
        mask_row(a, i);
        return;
    }
    const uint4 none = uint4{Chunk<T>::kNegInf, Chunk<T>::kNegInf, Chunk<T>::kNegInf, Chunk<T>::kNegInf};
    uint4 zr[R], qr[R];
#pragma unroll
    for (int c = 0; c < NC; ++c) {  // all loads in flight; past the whole chunks the last one again
        zr[c] = none;
        if (REF) qr[c] = none;
        if (c * NT < nfull) {
            const int cc = min(tid + c * NT, nfull - 1);
            zr[c] = row.template load<true>(row.z, cc);
            if (REF) qr[c] = row.template load<true>(row.q, cc);
        }
    }
    Sums s = no_sums(St<T>::load(row.z, row.at), a.kz, a.kq);
    if (NC > 0 && T == DType::BF16 && row.lead && tid == 0) {
        row.first(zr[0]);
        if (REF) row.first(qr[0]);
    }
    constexpr int G = 2;  // chunks between two looks at the maximum
    static_assert(NC % G == 0, "whole groups");
#pragma unroll
    for (int c = 0; c < NC; c += G)
        if (c * NT < nfull) {
            bool used[G];
#pragma unroll
            for (int u = 0; u < G; ++u) used[u] = tid + (c + u) * NT < nfull;
            // the second of a group may lie wholly past the row and hold -inf, which adds nothing
            add_chunks<T, REF, G>(s, zr + c, REF ? qr + c : zr + c, used, a.kz, a.kq);
        }
    if (BIG) {
        constexpr int U = REF ? 2 : 4;
        static_assert(SL % U == 0, "a round of loads is kept whole or not at all");
        // chunks c, c + NT, ...: U of them, kept from the given slot on (or not: -1), read once or twice
        auto round = [&](int c, int slot, auto once) __attribute__((always_inline)) {
            constexpr bool ONCE = decltype(once)::value;
            uint4 zc[U], qc[U];
            bool used[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                used[u] = c + u * NT < nfull;
                const int cc = min(c + u * NT, nfull - 1);
                zc[u] = row.template load<ONCE>(row.z, cc);
                if (REF) qc[u] = row.template load<ONCE>(row.q, cc);
            }
            if (NC == 0 && T == DType::BF16 && row.lead && c == 0) {
                row.first(zc[0]);
                if (REF) row.first(qc[0]);
            }
            if (slot >= 0) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    kept[((slot + u) * P) * NT + tid] = zc[u];
                    if (REF) kept[((slot + u) * P + 1) * NT + tid] = qc[u];
                }
            }
            add_chunks<T, REF, U>(s, zc, REF ? qc : zc, used, a.kz, a.kq);
        };
        int c = NC * NT + tid;
#pragma unroll 1
        for (int slot = 0; slot < SL && c < nfull; slot += U, c += NT * U) round(c, slot, std::true_type{});
#pragma unroll 1
        for (; c < nfull; c += NT * U) round(c, -1, std::integral_constant<bool, NC == 0>{});
    }
    const bool ends = nfull < nch && tid == nfull % NT;  // the row's last elements are this thread's
    if (ends) {
        const uint4 zt = Chunk<T>::tail(row.z, row.V), qt = REF ? Chunk<T>::tail(row.q, row.V) : none;
        const bool used = true;
        add_chunks<T, REF, 1>(s, &zt, &qt, &used, a.kz, a.kq);
    }
    const RowStats r = join_threads<T, REF, NT>(s, a, row, 0, nch);
    if (tid < 64) {
        const RowCoef c = finish_row(a, i, in, r, true);
        if (tid == 0) coef = c;
    }
    if (NC == 0) return;
    __syncthreads();
    const RowCoef rc = uniform(coef);
    if (BIG) {  // what has to be read again first: it was read last, and the L2 may still hold it
        for (int c = (NC + SL) * NT + tid; c < nfull; c += NT) {
            const uint4 zc = row.template load<false>(row.z, c), qc = REF ? row.template load<false>(row.q, c) : zc;
            st16_once((uint8_t *)row.dz + (uint32_t)c * 16u, grad_of<T, REF>(rc, c, row.at, zc, qc));
        }
        for (int slot = 0, c = NC * NT + tid; slot < SL && c < nfull; ++slot, c += NT)
            st16_once((uint8_t *)row.dz + (uint32_t)c * 16u,
                      grad_of<T, REF>(rc, c, row.at, kept[slot * P * NT + tid], kept[(slot * P + P - 1) * NT + tid]));
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int cc = tid + c * NT;
        if (cc < nfull) {
            const uint4 g = grad_of<T, REF>(rc, cc, row.at, zr[c], REF ? qr[c] : zr[c]);
            if (c == 0)
                row.store(cc, g);
            else
                st16_once((uint8_t *)row.dz + (uint32_t)cc * 16u, g);
        }
    }
    if (ends) {
        const uint4 zt = Chunk<T>::tail(row.z, row.V), qt = REF ? Chunk<T>::tail(row.q, row.V) : none;
        Chunk<T>::store_tail(row.dz, row.V, grad_of<T, REF>(rc, nfull, row.at, zt, qt));
    }
}

// Few rows: each split over S workgroups (S <= 64), two launches.  The first leaves the sums of every part, the
// second joins a row's parts in each of its workgroups (wave 0, a lane a part) and writes their gradients.
// The first's loads stay in the caches for the second.
constexpr int kPartThreads = 256;

template <DType T, bool REF>
__global__ void __launch_bounds__(kPartThreads) row_part_kernel(RowArgs a, int S, int per) {
    typedef typename St<T>::type E;
    constexpr int N = Chunk<T>::N, NT = kPartThreads, U = 2;
    const long i = blockIdx.x / S;
    const int p = (int)(blockIdx.x - i * S), tid = threadIdx.x;
    const RowIn in = row_in(a, i);
    if (!in.counts) return;
    const Row<T> row(a, i, in.tok, REF);
    const int first = p * per, last = min(row.nch, first + per), whole = min(row.nfull, last);
    const int own = row.at / N;
    Sums s = no_sums(own >= first && own < last ? St<T>::load(row.z, row.at) : 0.f, a.kz, a.kq);
    for (int c = first + tid; c < whole; c += NT * U) {
        uint4 zc[U], qc[U];
        bool used[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            used[u] = c + u * NT < whole;
            const int cc = min(c + u * NT, whole - 1);
            zc[u] = row.template load<false>(row.z, cc);
            if (REF) qc[u] = row.template load<false>(row.q, cc);
        }
        if (T == DType::BF16 && row.lead && c == 0) {
            row.first(zc[0]);
            if (REF) row.first(qc[0]);
        }
        add_chunks<T, REF, U>(s, zc, REF ? qc : zc, used, a.kz, a.kq);
    }
    if (last > row.nfull && first <= row.nfull && tid == (row.nfull - first) % NT) {  // the row's end is in this part
        const uint4 zt = Chunk<T>::tail(row.z, row.V), qt = REF ? Chunk<T>::tail(row.q, row.V) : zt;
        const bool used = true;
        add_chunks<T, REF, 1>(s, &zt, &qt, &used, a.kz, a.kq);
    }
    const RowStats r = join_threads<T, REF, NT>(s, a, row, first, last);
    if (tid == 0) a.part[i * S + p] = r;
}

// The parts of row i as one, a lane of the wave a part.  What is left out of a part's s (its top) stays out
// only where it is the row's maximum.
template <bool REF>
__device__ __forceinline__ RowStats join_parts(const RowArgs &a, long i, int S, int own) {
    const int lane = threadIdx.x & 63;
    const bool in = lane < S;
    Sums s;
    RowStats &r = s.r;
    r = a.part[i * S + min(lane, S - 1)];
    s.z = scale_of(r.M, a.kz);
    s.q = scale_of(r.Mq, a.kq);
    const float M = wave_max(r.M), Mq = REF ? wave_max(r.Mq) : kLowest;
    const float top = r.top * __builtin_amdgcn_exp2f(s.z.of(r.M));
    if (r.M != M) {
        r.s += top;
        r.top = 0.f;
    } else if (REF) {  // its maximum stays, but the reference's may lie in another part
        r.k -= mul0(top, s.q.b - scale_of(Mq, a.kq).b);
    }
    rebase<REF>(s, M, Mq, a.kz, a.kq);
    if (!in) r.s = r.t = r.k = r.sq = r.top = 0.f;
    sum_lanes<REF>(r);
    r.top = wave_sum(r.top);
    r.za = lane_f32(r.za, __builtin_amdgcn_readfirstlane(own));
    return r;
}

template <DType T, bool REF, bool GRAD>
__global__ void __launch_bounds__(kPartThreads) row_rest_kernel(RowArgs a, int S, int per) {
    typedef typename St<T>::type E;
    constexpr int N = Chunk<T>::N, NT = kPartThreads;
    __shared__ RowCoef coef;
    const long i = GRAD ? blockIdx.x / S : blockIdx.x;
    const int p = (int)(blockIdx.x - i * S), tid = threadIdx.x;
    const RowIn in = row_in(a, i);
    const Row<T> row(a, i, in.tok, REF);
    const int first = p * per, last = min(row.nch, first + per);
    if (!in.counts) {
        if (GRAD)
            for (int c = first + tid; c < last; c += NT) row.store(c, uint4{0u, 0u, 0u, 0u});
        if (!GRAD || p == 0) mask_row(a, i);
        return;
    }
    if (tid < 64) {
        const RowCoef c = finish_row(a, i, in, join_parts<REF>(a, i, S, row.at / N / per), !GRAD || p == 0);
        if (tid == 0) coef = c;
    }
    if (!GRAD) return;
    __syncthreads();
    const RowCoef rc = uniform(coef);
    for (int c = first + tid; c < last; c += NT) {
        const uint4 zc = row.any(row.z, c), qc = REF ? row.any(row.q, c) : zc;
        row.store(c, grad_of<T, REF>(rc, c, row.at, zc, qc));
    }
}

// The loss and its terms, the rows in a fixed order: each thread its rows, the waves' lanes, the waves.
template <int NT>
__global__ void __launch_bounds__(NT) row_terms_kernel(RowArgs a) {
    constexpr int NW = NT / 64;
    __shared__ double red[4][NW];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (long i = threadIdx.x; i < a.N; i += NT)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += a.row_terms[i * 4 + k];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += __shfl_xor(s[k], o);
    if (NW > 1) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < 4; ++k) red[k][threadIdx.x >> 6] = s[k];
        __syncthreads();
        if (threadIdx.x >= 64) return;
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] = (int)threadIdx.x < NW ? red[k][threadIdx.x & (NW - 1)] : 0.0;
#pragma unroll
        for (int o = NW / 2; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] += __shfl_xor(s[k], o);
    }
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) a.terms[1 + k] = (float)s[k];
    // a divergence that is only reported may be infinite
    a.terms[0] = (float)(s[0] + (a.c_kl != 0.0 ? a.c_kl * s[1] : 0.0) - a.c_ent * s[2]);
}

static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Parts of a row: 1 where its workgroup does the whole row.  A workgroup takes longer for a longer row, and few
// rows leave most of the chip idle; splitting costs another launch, 2.5 to 3 us of the host's time (3.7 where
// it also needs the workspace that whole rows do not).  So a row is split where the chip gains more than
// the host loses: by its entries, which count twice with a reference (a unit is busy with their
// arithmetic: both types take as long), and by the rows, up to an eighth or a quarter of the units.
// Whole and split, in us, on the chip alone (and a call by itself where the host is the longer):
//   with reference, 8 rows of 16000 10.2 and 9.0 (17.2, 19.3), of 32000 13.3 and 9.1 (17.6, 19.8), of 65536 20.8 and
//   9.6; 48 of 32000 13.8 and 12.2 (17.6, 20.6); 64 of 65536 23.0 and 18.9;
//   without, 8 rows of 32000 10.4 and 8.1 (16.2, 18.5), of 65536 13.8 and 8.6 (16.4, 18.7), of 131072 21.9 and 9.0;
//   64 of 65536 14.2 and 12.2 (16.5, 19.1), of 131072 22.0 and 14.8;
//   log-probabilities, 8 rows of 65536 7.0 and 5.5 (7.7, 11.6), of 131072 10.7 and 5.6 (10.9, 11.7).
static int row_parts(long N, int V, int nch, bool grad, bool ref, int &per) {
    const int cu = compute_units();
    per = nch;
    const long work = (long)V * (ref ? 2 : 1);
    if (N <= 0 || 4 * N > cu || work < (grad && 8 * N <= cu ? 49152 : 98304)) return 1;
    const long want = std::min<long>(64, std::min<long>(2L * cu / N, (nch + kPartThreads - 1) / kPartThreads));
    per = (int)((nch + want - 1) / want);
    per = (per + kPartThreads - 1) / kPartThreads * kPartThreads;
    return (nch + per - 1) / per;
}

size_t rows_workspace(long N, int V, bool policy) {
    int per;
    const int S = row_parts(N, V, (V + 3) / 4, policy, policy, per);  // as many chunks as any type has
    return (S > 1 ? up256((size_t)N * 64 * sizeof(RowStats)) : 0) + (policy ? up256((size_t)N * 32) : 0);
}

size_t rows_workspace_up_to(long N, int V, bool policy) {
    int per;
    const bool split = N > 0 && row_parts(1, V, (V + 3) / 4, policy, policy, per) > 1;  // as one row is, if any number is
    const long few = std::min<long>(N, compute_units() / 4);                 // more are not
    return (split ? up256((size_t)few * 64 * sizeof(RowStats)) : 0) + (policy ? up256((size_t)N * 32) : 0);
}

template <DType T, bool REF, int NT, int NC, int SL = 0, bool BIG = false>
static void launch_row_shape(const RowArgs &a, hipStream_t s) {
    constexpr int lds = SL * (REF ? 2 : 1) * NT * 16;
    if (lds > 0)  // for the current device, each time; a refusal shows at the launch
        (void)hipFuncSetAttribute((const void *)row_kernel<T, REF, NT, NC, SL, BIG>,
                                  hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    row_kernel<T, REF, NT, NC, SL, BIG><<<(unsigned)a.N, NT, lds, s>>>(a);
}

// The workgroup that holds a row of nch chunks: as few threads as hold it with eight chunks each (four where that
// is enough), so that several rows share a compute unit, one loading while another computes.  Longer rows
// without a reference have room for sixteen chunks a thread (65521 entries in bf16: 512 threads with sixteen
// 59.6 us for 1024 rows, 1024 with eight 77), and keep eight more in LDS where even that is short.  With a
// reference a chunk is two, so eight and four in LDS (2048 rows of 131072 in bf16: 407 us with the LDS part,
// 432 without).  Without a gradient a row is only streamed: by 256 threads where there are rows enough to
// fill the chip, by 1024 else.
template <DType T, bool REF>
static void launch_row(const RowArgs &a, int nch, hipStream_t s) {
    if (a.dz == nullptr) {
        if (nch <= 64 * 8)
            launch_row_shape<T, REF, 64, 0, 0, true>(a, s);
        else if (a.N >= 512)
            launch_row_shape<T, REF, 256, 0, 0, true>(a, s);
        else
            launch_row_shape<T, REF, 1024, 0, 0, true>(a, s);
    } else if (nch <= 64 * 4) {
        launch_row_shape<T, REF, 64, 4>(a, s);
    } else if (nch <= 256 * 4) {
        launch_row_shape<T, REF, 256, 4>(a, s);
    } else if (nch <= 256 * 8) {
        launch_row_shape<T, REF, 256, 8>(a, s);
    } else if (nch <= 512 * 8) {
        launch_row_shape<T, REF, 512, 8>(a, s);
    } else if constexpr (REF) {
        if (nch <= 1024 * 8)
            launch_row_shape<T, REF, 1024, 8>(a, s);
        else
            launch_row_shape<T, REF, 1024, 8, 4, true>(a, s);
    } else {
        if (nch <= 512 * 16)
            launch_row_shape<T, REF, 512, 16>(a, s);
        else if (nch <= 1024 * 16)
            launch_row_shape<T, REF, 1024, 16>(a, s);
        else
            launch_row_shape<T, REF, 1024, 16, 8, true>(a, s);
    }
}

template <DType T, bool REF>
static void launch_rows_t(RowArgs a, void *workspace, hipStream_t s) {
    const int nch = (a.V + (T == DType::BF16 ? 1 : 0) + Chunk<T>::N - 1) / Chunk<T>::N;  // with a lead
    int per;
    const int S = row_parts(a.N, a.V, nch, a.dz != nullptr, REF, per);
    a.row_terms = (double *)workspace;
    a.part = (RowStats *)((uint8_t *)workspace + (a.policy ? up256((size_t)a.N * 32) : 0));
    if (a.N > 0 && S == 1) {
        launch_row<T, REF>(a, nch, s);
    } else if (a.N > 0) {
        row_part_kernel<T, REF><<<(unsigned)(a.N * S), kPartThreads, 0, s>>>(a, S, per);
        if (a.dz != nullptr)
            row_rest_kernel<T, REF, true><<<(unsigned)(a.N * S), kPartThreads, 0, s>>>(a, S, per);
        else
            row_rest_kernel<T, REF, false><<<(unsigned)a.N, 64, 0, s>>>(a, S, per);
    }
    if (a.policy) {
        if (a.N <= 256)  // one wave has no barrier to wait at: 16 rows 11.4 -> 9.4 us for both launches
            row_terms_kernel<64><<<1, 64, 0, s>>>(a);
        else
            row_terms_kernel<1024><<<1, 1024, 0, s>>>(a);
    }
}

void launch_rows(DType t, RowArgs a, void *workspace, hipStream_t s) {
    constexpr double log2e = 1.44269504088896340736;
    a.kz = (float)(a.it * log2e);
    a.kq = (float)(a.iq * log2e);
    if (t == DType::BF16)
        a.q != nullptr ? launch_rows_t<DType::BF16, true>(a, workspace, s) : launch_rows_t<DType::BF16, false>(a, workspace, s);
    else
        a.q != nullptr ? launch_rows_t<DType::F32, true>(a, workspace, s) : launch_rows_t<DType::F32, false>(a, workspace, s);
}

// ------------------------------------------------------------------------------------------
// AdamW over many tensors
// ------------------------------------------------------------------------------------------
// A launch takes a table of tensors as its argument: no copy to the device, and a captured launch keeps
// it.  Chunk c of the launch belongs to the tensor t with first[t] <= c < first[t + 1].
struct AdamTable {
    int n, chunks;
    uint32_t first[kAdamTensors];
    AdamTensor t[kAdamTensors];
};
struct NormTable {
    int n, chunks;
    uint32_t first[kAdamTensors];
    const void *g[kAdamTensors];
    long len[kAdamTensors];
};
template <class Table>
__device__ __forceinline__ int tensor_of(const Table &t, uint32_t c) {
    int lo = 0, hi = t.n;  // first[lo] <= c < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid; else hi = mid;
    }
    return lo;
}

// Four consecutive elements from i on; those at n and past it are 0.  ONCE: past the caches.
template <DType T, bool ONCE>
__device__ __forceinline__ void load4(const void *p, long i, long n, float *v) {
    typedef typename St<T>::type E;
    const E *e = (const E *)p + i;
    if (i + 4 <= n) {
        if (T == DType::F32) {
            unpack_frag<DType::F32>(ONCE ? ld16_once(e) : ld16(e), v);
        } else {
            const v2u w = ONCE ? __builtin_nontemporal_load((const v2u_any *)e) : *(const v2u_any *)e;
            v[0] = __uint_as_float(w.x << 16);
            v[1] = __uint_as_float(w.x & 0xffff0000u);
            v[2] = __uint_as_float(w.y << 16);
            v[3] = __uint_as_float(w.y & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = i + k < n ? St<T>::load(e, k) : 0.f;
    }
}
template <DType T, bool ONCE>
__device__ __forceinline__ void store4(void *p, long i, long n, const float *v) {
    typedef typename St<T>::type E;
    E *e = (E *)p + i;
    if (i + 4 <= n) {
        const v2u w = {pack2bf(v[0], v[1]), pack2bf(v[2], v[3])};
        if (T == DType::F32) {
            if (ONCE) st16_once(e, pack_frag_cvt<DType::F32>(v)); else st16(e, pack_frag_cvt<DType::F32>(v));
        } else {
            if (ONCE) __builtin_nontemporal_store(w, (v2u_any *)e); else *(v2u_any *)e = w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) St<T>::store(e, k, v[k]);
    }
}
template <bool ONCE>
__device__ __forceinline__ uint32_t load4_codes(const void *p, long i, long n) {
    const uint8_t *b = (const uint8_t *)p + i;
    uint32_t w = 0;
    if (i + 4 <= n) {
        w = ONCE ? __builtin_nontemporal_load((const u32_any *)b) : *(const u32_any *)b;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) w |= (uint32_t)b[k] << (8 * k);
    }
    return w;
}
template <bool ONCE>
__device__ __forceinline__ void store4_codes(void *p, long i, long n, uint32_t w) {
    uint8_t *b = (uint8_t *)p + i;
    if (i + 4 <= n) {
        if (ONCE) __builtin_nontemporal_store(w, (u32_any *)b); else *(u32_any *)b = w;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) b[k] = (uint8_t)(w >> (8 * k));
    }
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Sums of squares of the gradients, in 64 bits (the square of any fp32 gradient is finite there, and the
// scale that follows from the sum is the same whatever the order); workgroup b takes chunks b, b + grid, ...
// of kNormChunk elements, all of a chunk's loads in flight together.  134M bf16 gradients 47 us (5.7 TB/s).
template <DType GT>
__global__ void __launch_bounds__(256) adam_norm_kernel(NormTable tab, double *part) {
    typedef typename St<GT>::type E;
    constexpr int N = Chunk<GT>::N, U = kNormChunk / (256 * N);
    __shared__ double red[4];
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < (uint32_t)tab.chunks; c += gridDim.x) {
        const int t = tensor_of(tab, c);
        const long at = (long)(c - tab.first[t]) * kNormChunk;
        const E *g = (const E *)tab.g[t] + at;
        const int n = (int)min(tab.len[t] - at, (long)kNormChunk), whole = n / N;
        uint4 r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            r[u] = uint4{0u, 0u, 0u, 0u};
            const int i = threadIdx.x + 256 * u;
            if (i < whole) r[u] = ld16((const uint8_t *)g + (uint32_t)i * 16u);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[N];
            unpack_frag<GT>(r[u], v);
#pragma unroll
            for (int k = 0; k < N; ++k) s += (double)v[k] * (double)v[k];
        }
        if ((int)threadIdx.x < n - whole * N) {  // the tensor's last elements
            const double v = (double)St<GT>::load(g, whole * N + threadIdx.x);
            s += v * v;
        }
    }
    s = wave_sum_f64(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = ((red[0] + red[1]) + red[2]) + red[3];
}

// The sum of the partial sums, the same in every workgroup.
__device__ __forceinline__ double sum_parts(const double *part, int n, double *red4) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) s += part[i];
    s = wave_sum_f64(s);
    if ((threadIdx.x & 63) == 0) red4[threadIdx.x >> 6] = s;
    __syncthreads();
    return ((red4[0] + red4[1]) + red4[2]) + red4[3];
}

// Many partial sums become one, in the place of the first (which every thread has read by then), before the
// step's workgroups all read them: 4.5 us for 2048 of them, and with clipping and 8-bit states 1000 tensors of
// 200000 bf16 elements 3451 -> 1154 us, 48 of 4.2M 773 -> 748.
__global__ void __launch_bounds__(256) adam_norm_join_kernel(double *part, int n) {
    __shared__ double red[4];
    const double s = sum_parts(part, n, red);
    if (threadIdx.x == 0) part[0] = s;
}

__global__ void __launch_bounds__(256) adam_norm_out_kernel(const double *part, int n, float *norm) {
    __shared__ double red[4];
    const double v = sum_parts(part, n, red);
    if (threadIdx.x == 0) norm[0] = (float)sqrt(v);
}

// 32 random bits for element number `at` of the step with these keys: xorshifts and multiplications whose
// constants come from a published search for mixes of low bias, and one more round with the second key.
__device__ __forceinline__ uint32_t random_bits(uint64_t at, uint32_t key0, uint32_t key1) {
    uint32_t h = (uint32_t)at ^ (key0 + (uint32_t)(at >> 32) * 0x85ebca6bu);
    h = (h ^ (h >> 16)) * 0x7feb352du;
    h = (h ^ (h >> 15)) * 0x846ca68bu;
    h = ((h ^ (h >> 16)) + key1) * 0x9e3779b1u;
    return h ^ (h >> 15);
}

// x in [0, 448] to a value of e4m3, up or down by 16 random bits: they are added below the three kept bits
// of the mantissa.  Below 2^-6 the spacing of e4m3 is that of the binade above, where x is moved for this.
__device__ __forceinline__ float round_e4m3(float x, uint32_t bits16) {
    const bool small = x < 0.015625f;
    const float t = small ? x + 0.015625f : x;
    const float r = __uint_as_float((__float_as_uint(t) + (bits16 << 4)) & 0xfff00000u);
    return small ? r - 0.015625f : r;
}

template <int BITS> struct State;   // four elements' m and v, with the block's scales for 8 bits
template <> struct State<32> {
    float m[4], v[4];
};
template <> struct State<8> {
    uint32_t m, r;
    float ms, rs;
};

// One AdamW step, a wave per 256 elements (the block of an 8-bit state), four consecutive ones a lane; a wave takes
// U blocks, whose loads are all in flight together.  Bound by memory: 134M elements in bf16 with 32-bit states
// and masters 600 to 615 us (6.1 to 6.3 TB/s), 202M with 8-bit states 570 to 645 (5.0 to 5.7).
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p (1 - lr wd) - rate m / (sqrt(v) root + eps)
// 8-bit states hold m and sqrt(v) as e4m3 times a scale per block (its largest / 448), rounded up or down
// at random so that the mean is right: v moves by 1 - b2 of itself a step, far less than half a spacing of
// e4m3, and would stay where it is under rounding to nearest.  The step itself uses m and v before that
// rounding.  A root that is not zero is kept from rounding to zero, which would blow the next step up.
// Every operation rounds by itself (no fused multiply-add): near the border of a random rounding the codes
// then are those of the same formulas in any other IEEE arithmetic of 32 bits.
template <DType PT, bool MASTER, DType GT, int BITS, int U, bool ONCE>
__global__ void __launch_bounds__(256) adamw_kernel(AdamTable tab, AdamArgs a) {
#pragma clang fp contract(off)
    __shared__ double red[4];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t c = blockIdx.x;
    const int ti = tensor_of(tab, c);
    const AdamTensor t = tab.t[ti];
    const long n = t.n, i0 = (long)(c - tab.first[ti]) * (1024 * U) + kStateBlock * U * w + 4 * lane;
    float p[U][4], g[U][4];
    State<BITS> st[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long i = i0 + kStateBlock * u;
        if (i - 4 * lane >= n) continue;  // uniform: the block is past the tensor
        load4<MASTER ? DType::F32 : PT, ONCE>(MASTER ? (const void *)t.master : (const void *)t.p, i, n, p[u]);
        load4<GT, ONCE>(t.g, i, n, g[u]);
        if constexpr (BITS == 32) {
            load4<DType::F32, ONCE>(t.m, i, n, st[u].m);
            load4<DType::F32, ONCE>(t.v, i, n, st[u].v);
        } else {
            st[u].m = load4_codes<ONCE>(t.m, i, n);
            st[u].r = load4_codes<ONCE>(t.v, i, n);
            st[u].ms = t.ms[(i - 4 * lane) / kStateBlock];
            st[u].rs = t.vs[(i - 4 * lane) / kStateBlock];
        }
    }
    float clip = 1.f;
    if (a.norm_part != nullptr) {  // while the loads are on their way
        const double norm = sqrt(sum_parts(a.norm_part, a.n_part, red));
        if (a.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) a.norm[0] = (float)norm;
        if (!(norm <= 1.7e308)) return;  // a gradient that is not finite: no step
        if (norm > a.max_norm) clip = (float)(a.max_norm / norm);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long i = i0 + kStateBlock * u;
        if (i - 4 * lane >= n) continue;
        float m[4], v[4], r[4];
        if constexpr (BITS == 32) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                m[k] = st[u].m[k];
                v[k] = st[u].v[k];
            }
        } else {
            m[0] = __builtin_amdgcn_cvt_f32_fp8(st[u].m, 0) * st[u].ms;
            m[1] = __builtin_amdgcn_cvt_f32_fp8(st[u].m, 1) * st[u].ms;
            m[2] = __builtin_amdgcn_cvt_f32_fp8(st[u].m, 2) * st[u].ms;
            m[3] = __builtin_amdgcn_cvt_f32_fp8(st[u].m, 3) * st[u].ms;
            v[0] = __builtin_amdgcn_cvt_f32_fp8(st[u].r, 0) * st[u].rs;
            v[1] = __builtin_amdgcn_cvt_f32_fp8(st[u].r, 1) * st[u].rs;
            v[2] = __builtin_amdgcn_cvt_f32_fp8(st[u].r, 2) * st[u].rs;
            v[3] = __builtin_amdgcn_cvt_f32_fp8(st[u].r, 3) * st[u].rs;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] *= v[k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float gk = g[u][k] * clip;
            m[k] = a.b1 * m[k] + a.one_b1 * gk;
            v[k] = a.b2 * v[k] + a.one_b2 * gk * gk;
            r[k] = sqrtf(v[k]);
            p[u][k] = p[u][k] * a.decay - a.rate * m[k] / (r[k] * a.root + a.eps);
        }
        if (MASTER) store4<DType::F32, ONCE>(t.master, i, n, p[u]);
        store4<PT, ONCE>(t.p, i, n, p[u]);
        if constexpr (BITS == 32) {
            store4<DType::F32, ONCE>(t.m, i, n, m);
            store4<DType::F32, ONCE>(t.v, i, n, v);
        } else {
            // lanes past the tensor hold m = v = 0
            float mm = fmaxf(fmaxf(fabsf(m[0]), fabsf(m[1])), fmaxf(fabsf(m[2]), fabsf(m[3])));
            float rm = fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3]));
            mm = wave_max(mm);
            rm = wave_max(rm);
            constexpr float kTiny = 0x1p-100f;  // blocks whose largest is below are held as zeros
            const float im = mm < kTiny ? 0.f : 1.f / mm * 448.f, ir = rm < kTiny ? 0.f : 1.f / rm * 448.f;
            float mc[4], rc[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t bits = random_bits((uint64_t)(t.base + i + k), a.key0, a.key1);
                mc[k] = copysignf(round_e4m3(fminf(fabsf(m[k]) * im, 448.f), bits & 0xffffu), m[k]);
                const float y = fminf(r[k] * ir, 448.f), q = round_e4m3(y, bits >> 16);
                rc[k] = y > 0.f ? fmaxf(q, 0x1p-9f) : q;
            }
            int mw = __builtin_amdgcn_cvt_pk_fp8_f32(mc[0], mc[1], 0, false);
            mw = __builtin_amdgcn_cvt_pk_fp8_f32(mc[2], mc[3], mw, true);
            int rw = __builtin_amdgcn_cvt_pk_fp8_f32(rc[0], rc[1], 0, false);
            rw = __builtin_amdgcn_cvt_pk_fp8_f32(rc[2], rc[3], rw, true);
            store4_codes<ONCE>(t.m, i, n, (uint32_t)mw);
            store4_codes<ONCE>(t.v, i, n, (uint32_t)rw);
            if (lane == 0) {
                t.ms[i / kStateBlock] = mm < kTiny ? 0.f : mm * (1.f / 448.f);
                t.vs[i / kStateBlock] = rm < kTiny ? 0.f : rm * (1.f / 448.f);
            }
        }
    }
}

static uint32_t chunks_of(long n, long chunk) { return (uint32_t)((n + chunk - 1) / chunk); }

int adam_norm_parts(const AdamTensor *t, int n) {
    long c = 0;
    for (int i = 0; i < n; ++i) c += chunks_of(t[i].n, kNormChunk);
    return (int)(c < kNormGrid ? c : kNormGrid);
}

void launch_adam_norm(DType gt, const AdamTensor *t, int n, double *part, hipStream_t s) {
    NormTable tab;
    tab.n = n;
    uint32_t c = 0;
    for (int i = 0; i < n; ++i) {
        tab.first[i] = c;
        tab.g[i] = t[i].g;
        tab.len[i] = t[i].n;
        c += chunks_of(t[i].n, kNormChunk);
    }
    tab.chunks = (int)c;
    const int grid = adam_norm_parts(t, n);
    if (gt == DType::BF16)
        adam_norm_kernel<DType::BF16><<<grid, 256, 0, s>>>(tab, part);
    else
        adam_norm_kernel<DType::F32><<<grid, 256, 0, s>>>(tab, part);
}

void launch_adam_norm_join(double *part, int n_part, hipStream_t s) {
    adam_norm_join_kernel<<<1, 256, 0, s>>>(part, n_part);
}

void launch_adam_norm_out(const double *part, int n_part, float *norm, hipStream_t s) {
    adam_norm_out_kernel<<<1, 256, 0, s>>>(part, n_part, norm);
}

template <DType PT, bool MASTER, DType GT, int BITS>
static void launch_adamw_t(const AdamTable &tab, bool large, const AdamArgs &a, hipStream_t s) {
    if (large)
        adamw_kernel<PT, MASTER, GT, BITS, 4, true><<<tab.chunks, 256, 0, s>>>(tab, a);
    else
        adamw_kernel<PT, MASTER, GT, BITS, 1, false><<<tab.chunks, 256, 0, s>>>(tab, a);
}

void launch_adamw(DType pt, bool master, DType gt, int bits, const AdamTensor *t, int n, const AdamArgs &a, hipStream_t s) {
    AdamTable tab;
    tab.n = n;
    long all = 0;
    for (int i = 0; i < n; ++i) {
        tab.t[i] = t[i];
        all += t[i].n;
    }
    // A step that moves more than the last-level cache (256 MiB) goes past it, four blocks a wave: 134M elements
    // in bf16 with 32-bit states 773 -> 663 us, 202M with 8-bit ones 630 -> 597; with fewer bytes the
    // caches may hold what the next step reads (8M fp32 elements: 34 us, past the caches 46), and one block a
    // wave spreads small tensors over more of the chip (570000 elements 8.9 -> 7.3 us, 8M the same).
    const long bytes = all * (2 * (bits / 4) + (gt == DType::BF16 ? 2 : 4) + (pt == DType::F32 ? 8 : master ? 10 : 4));
    const bool large = bytes > (256L << 20);
    const long blocks = large ? 4 : 1;
    uint32_t c = 0;
    for (int i = 0; i < n; ++i) {
        tab.first[i] = c;
        c += chunks_of(t[i].n, 1024L * blocks);
    }
    tab.chunks = (int)c;
    auto go = [&](auto b) {
        constexpr int B = decltype(b)::value;
        const bool gb = gt == DType::BF16;
        constexpr DType F = DType::F32, H = DType::BF16;
        if (pt == F)
            gb ? launch_adamw_t<F, false, H, B>(tab, large, a, s) : launch_adamw_t<F, false, F, B>(tab, large, a, s);
        else if (master)
            gb ? launch_adamw_t<H, true, H, B>(tab, large, a, s) : launch_adamw_t<H, true, F, B>(tab, large, a, s);
        else
            gb ? launch_adamw_t<H, false, H, B>(tab, large, a, s) : launch_adamw_t<H, false, F, B>(tab, large, a, s);
    };
    if (bits == 8)
        go(std::integral_constant<int, 8>{});
    else
        go(std::integral_constant<int, 32>{});
}

}  // namespace dvi
