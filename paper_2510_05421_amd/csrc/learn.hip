// gfx950 kernels of the learning operators: log-probabilities of tokens, the clipped policy loss with its
// gradient, and AdamW over many tensors with states in 32 or 8 bits.
//
// All of them are bound by memory (by launches where the tensors are small), so each reads its inputs as
// few times as the caches allow, 16 bytes a lane, and keeps everything else in registers.
#include "learn.h"

#include "device.h"

namespace dvi {

// ------------------------------------------------------------------------------------------
// Rows of logits
// ------------------------------------------------------------------------------------------
// A row is cut into 16-byte chunks from its own start.  Rows of an odd vocabulary or stride start at any
// element, so the 16 bytes are loaded without an alignment (one global load all the same: the target
// allows it); the last chunk may be partial and is filled up with -inf, which adds nothing to any sum.
// 16, 8 and 4 bytes at any address, each one access (as vectors: the compiler takes a copied array apart)
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef v4u v4u_any __attribute__((aligned(1)));
typedef v2u v2u_any __attribute__((aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));
__device__ __forceinline__ uint4 ld16(const void *p) {
    const v4u v = *(const v4u_any *)p;
    return uint4{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ void st16(void *p, const uint4 &r) { *(v4u_any *)p = v4u{r.x, r.y, r.z, r.w}; }

template <DType T> struct Chunk {
    typedef typename St<T>::type E;
    static constexpr int N = 16 / (int)sizeof(E);
    static constexpr uint32_t kNegInf = T == DType::BF16 ? 0xff80ff80u : 0xff800000u;
    static __device__ __forceinline__ uint4 load(const E *row, int c, int V) {
        uint4 r;
        if ((c + 1) * N <= V) {
            r = ld16(row + (size_t)c * N);
        } else {
            E e[N];
#pragma unroll
            for (int k = 0; k < N; ++k) e[k] = c * N + k < V ? row[(size_t)c * N + k] : (E)0;
            __builtin_memcpy(&r, e, 16);
            uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (c * N + k >= V) {
                    if (T == DType::BF16)
                        w[k / 2] = (k & 1) ? (w[k / 2] & 0xffffu) | 0xff800000u : (w[k / 2] & 0xffff0000u) | 0xff80u;
                    else
                        w[k] = kNegInf;
                }
            r = uint4{w[0], w[1], w[2], w[3]};
        }
        return r;
    }
    static __device__ __forceinline__ void store(E *row, int c, int V, const float *v) {
        const uint4 r = pack_frag_cvt<T>(v);
        if ((c + 1) * N <= V) {
            st16(row + (size_t)c * N, r);
        } else {
            E e[N];
            __builtin_memcpy(e, &r, 16);
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (c * N + k < V) row[(size_t)c * N + k] = e[k];
        }
    }
};
template <> struct Chunk<DType::F32> {
    typedef float E;
    static constexpr int N = 4;
    static constexpr uint32_t kNegInf = 0xff800000u;
    static __device__ __forceinline__ uint4 load(const float *row, int c, int V) {
        uint4 r;
        if ((c + 1) * 4 <= V) {
            r = ld16(row + (size_t)c * 4);
        } else {
            float e[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) e[k] = c * 4 + k < V ? row[(size_t)c * 4 + k] : -INFINITY;
            __builtin_memcpy(&r, e, 16);
        }
        return r;
    }
    static __device__ __forceinline__ void store(float *row, int c, int V, const float *v) {
        if ((c + 1) * 4 <= V) {
            st16(row + (size_t)c * 4, pack_frag_cvt<DType::F32>(v));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (c * 4 + k < V) row[(size_t)c * 4 + k] = v[k];
        }
    }
};

constexpr float kLowest = -3.402823466e38f;

// Whether row i takes part: a weight other than 0 and a token of the vocabulary.
__device__ __forceinline__ bool row_counts(const RowArgs &a, long i) {
    const uint32_t t = (uint32_t)a.tok[i];
    return t < (uint32_t)a.V && !(a.weights != nullptr && a.weights[i] == 0.f);
}

// a * b with 0 * anything == 0: a probability of 0 takes no part, whatever it is multiplied with.
// (The compiler has to know the instruction: it keeps a product that follows an exponential of its wave at
// the distance the hardware needs.)
__device__ float fmul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float mul0(float a, float b) { return fmul_legacy(a, b); }

// The sums of one more chunk.  x = (z - M) log2(e) / T and y of the reference likewise (kz, kq: log2(e) over
// the temperature); the terms are 2^x, 2^x x and, for the KL divergence, 2^x (x - y): differences of logits
// that are already relative to their maxima, so nothing large cancels.  A -inf (2^x == 0) adds nothing even
// where x or y is infinite; a NaN makes the sums NaN.
template <DType T, bool REF>
__device__ __forceinline__ void add_chunk(RowStats &r, const uint4 &zc, const uint4 &qc, float kz, float kq) {
    constexpr int N = Chunk<T>::N;
    float z[N], q[N];
    unpack_frag<T>(zc, z);
    if (REF) unpack_frag<T>(qc, q);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float x = (z[k] - r.M) * kz, e = __builtin_amdgcn_exp2f(x);
        r.s += e;
        r.t += mul0(e, x);
        if (REF) {
            const float y = (q[k] - r.Mq) * kq;
            r.sq += __builtin_amdgcn_exp2f(y);
            r.k += mul0(e, x - y);
        }
    }
}

// Sums relative to new maxima M, Mq (at least the old ones).
template <bool REF>
__device__ __forceinline__ void rebase(RowStats &r, float M, float Mq, float kz, float kq) {
    const float dx = (r.M - M) * kz, f = __builtin_amdgcn_exp2f(dx);
    if (REF) {
        // a reference masked by the lowest number: dy is as large as that, and counts only where f s does
        const float dy = (r.Mq - Mq) * kq;
        r.k = mul0(f, r.k + mul0(r.s, dx - dy));
        r.sq *= __builtin_amdgcn_exp2f(dy);
        r.Mq = Mq;
    }
    r.t = mul0(f, r.t + mul0(r.s, dx));
    r.s *= f;
    r.M = M;
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

constexpr int kRowThreads = 256;
constexpr int kRowUnroll = 4;  // chunks that a thread has in flight

// Stats of part blockIdx.x % S of row blockIdx.x / S: one pass with running maxima, four chunks a thread
// between two looks at the maximum, then the workgroup's threads in a fixed order.
template <DType T, bool REF>
__global__ void __launch_bounds__(kRowThreads) row_stats_kernel(RowArgs a, int S, int per) {
    typedef typename St<T>::type E;
    __shared__ float red[4];
    const long i = blockIdx.x / S;
    const int p = (int)(blockIdx.x - i * S);
    if (!row_counts(a, i)) return;
    const E *z = (const E *)a.z + i * a.ldz;
    const E *q = REF ? (const E *)a.q + i * a.ldq : nullptr;
    const int nch = (a.V + Chunk<T>::N - 1) / Chunk<T>::N;
    const int c1 = min(nch, (p + 1) * per);
    const float kz = a.kz, kq = a.kq;
    RowStats r = {kLowest, 0.f, 0.f, 0.f, kLowest, 0.f, 0.f, 0.f};
    for (int c = p * per + threadIdx.x; c < c1; c += kRowThreads * kRowUnroll) {
        uint4 zc[kRowUnroll], qc[kRowUnroll];
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u) {
            // past the part: the first chunk again, which is not added
            const int cc = c + u * kRowThreads < c1 ? c + u * kRowThreads : c;
            zc[u] = Chunk<T>::load(z, cc, a.V);
            if (REF) qc[u] = Chunk<T>::load(q, cc, a.V);
        }
        float M = r.M, Mq = r.Mq;
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u) {
            M = fmaxf(M, chunk_max<T>(zc[u]));
            if (REF) Mq = fmaxf(Mq, chunk_max<T>(qc[u]));
        }
        rebase<REF>(r, M, Mq, kz, kq);
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u)
            if (c + u * kRowThreads < c1) add_chunk<T, REF>(r, zc[u], REF ? qc[u] : zc[u], kz, kq);
    }
    rebase<REF>(r, block_max256(r.M, red), REF ? block_max256(r.Mq, red) : kLowest, kz, kq);
    r.s = block_sum256(r.s, red);
    r.t = block_sum256(r.t, red);
    if (REF) {
        r.k = block_sum256(r.k, red);
        r.sq = block_sum256(r.sq, red);
    }
    if (threadIdx.x == 0) {
        const int at = a.tok[i];
        if (at / Chunk<T>::N >= p * per && at / Chunk<T>::N < c1) r.za = St<T>::load(z, at);
        a.part[i * S + p] = r;
    }
}

// What the gradient of a row needs: dz = 2^x (A x + C (x - y) + B), x and y relative to M and Mq, plus `at`
// at the token.
struct RowCoef {
    float M, Mq, A, B, C, at, dead, pad;
};

// The row's numbers from its sums, in 64 bits: differences of logits and their logarithms decide on which
// side of the clipping border a ratio falls.
__device__ __forceinline__ RowCoef row_numbers(const RowArgs &a, long i, const RowStats &r, float &logp, float &entropy,
                                               double (&terms)[4]) {
    constexpr double ln2 = 0.693147180559945309417;
    RowCoef c = {r.M, r.Mq, 0.f, 0.f, 0.f, 0.f, 1.f, 0.f};
    logp = entropy = 0.f;
    terms[0] = terms[1] = terms[2] = terms[3] = 0.0;
    if (!row_counts(a, i) || r.s == 0.f || (a.q != nullptr && r.sq == 0.f)) return c;
    const double s = (double)r.s, lns = log(s), lp = ((double)r.za - (double)r.M) * a.it - lns;
    const double H = lns - ln2 * (double)r.t / s;
    logp = (float)lp;
    entropy = (float)H;
    c.dead = 0.f;
    if (!a.policy) return c;
    const double w = a.weights != nullptr ? (double)a.weights[i] : (double)a.w0, adv = (double)a.adv[i];
    const bool on = a.old == nullptr || (a.on_policy != nullptr && a.on_policy[i] != 0);
    const double ratio = on ? 1.0 : exp(lp - (double)a.old[i]);
    const double plain = ratio * adv, held = fmin(fmax(ratio, a.lo), a.hi) * adv;
    const bool cut = held < plain;
    const double pol = cut ? -held : -plain;
    double by_lp = cut ? 0.0 : -plain, kl = 0.0, k0 = a.c_ent * (H - lns);
    if (a.q != nullptr) {
        const double lnq = log((double)r.sq);
        kl = ln2 * (double)r.k / s - lns + lnq;
        if (a.c_kl != 0.0) k0 += a.c_kl * (lnq - lns - kl);
    } else if (a.ref_logp != nullptr) {
        const double d = (double)a.ref_logp[i] - lp, ed = exp(d);
        kl = ed - d - 1.0;
        if (a.c_kl != 0.0) by_lp += a.c_kl * (1.0 - ed);
    }
    const double scale = w * a.it;
    c.A = (float)(scale / s * ln2 * a.c_ent);
    c.B = (float)(scale / s * (k0 - by_lp));
    c.C = (float)(scale / s * ln2 * a.c_kl);
    c.at = (float)(scale * by_lp);
    terms[0] = w * pol;
    terms[1] = w * kl;
    terms[2] = w * H;
    terms[3] = cut ? w : 0.0;
    return c;
}

// The S parts of row i as one, in order.
template <bool REF>
__device__ __forceinline__ RowStats join_parts(const RowArgs &a, long i, int S, int per, int chunk) {
    const RowStats *part = a.part + i * S;
    RowStats r = part[0];
    for (int p = 1; p < S; ++p) {
        RowStats o = part[p];
        const float M = fmaxf(r.M, o.M), Mq = fmaxf(r.Mq, o.Mq);
        rebase<REF>(r, M, Mq, a.kz, a.kq);
        rebase<REF>(o, M, Mq, a.kz, a.kq);
        r.s += o.s;
        r.t += o.t;
        if (REF) {
            r.k += o.k;
            r.sq += o.sq;
        }
    }
    r.za = part[a.tok[i] / chunk / per].za;
    return r;
}

// One thread a row: its numbers out of the parts' sums.
template <DType T, bool REF>
__global__ void __launch_bounds__(64) row_finish_kernel(RowArgs a, RowCoef *coef, int S, int per) {
    const long i = (long)blockIdx.x * 64 + threadIdx.x;
    if (i >= a.N) return;
    RowStats r = {};
    if (row_counts(a, i)) r = join_parts<REF>(a, i, S, per, Chunk<T>::N);
    float logp, entropy;
    double terms[4];
    const RowCoef c = row_numbers(a, i, r, logp, entropy, terms);
    if (a.logp != nullptr) a.logp[i] = logp;
    if (a.entropy != nullptr) a.entropy[i] = entropy;
    if (!a.policy) return;
    coef[i] = c;
#pragma unroll
    for (int k = 0; k < 4; ++k) a.row_terms[i * 4 + k] = terms[k];
}

// The gradient of one chunk, without the token's own term.
template <DType T, bool REF>
__device__ __forceinline__ void grad_chunk(const RowCoef &r, const uint4 &zc, const uint4 &qc, float kz, float kq, float *g) {
    constexpr int N = Chunk<T>::N;
    float z[N], q[N];
    unpack_frag<T>(zc, z);
    if (REF) unpack_frag<T>(qc, q);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float x = (z[k] - r.M) * kz, e = __builtin_amdgcn_exp2f(x);
        float in = r.A * x + r.B;
        if (REF) in += r.C * (x - (q[k] - r.Mq) * kq);
        g[k] = mul0(e, in);
    }
}
template <DType T>
__device__ __forceinline__ void add_token(float *g, int k0, float v) {
#pragma unroll
    for (int k = 0; k < Chunk<T>::N; ++k) g[k] += k == k0 ? v : 0.f;
}

template <DType T, bool REF>
__global__ void __launch_bounds__(kRowThreads) row_grad_kernel(RowArgs a, const RowCoef *coef, int S, int per) {
    typedef typename St<T>::type E;
    const long i = blockIdx.x / S;
    const int p = (int)(blockIdx.x - i * S);
    const E *z = (const E *)a.z + i * a.ldz;
    const E *q = REF ? (const E *)a.q + i * a.ldq : nullptr;
    E *dz = (E *)a.dz + i * a.lddz;
    const int nch = (a.V + Chunk<T>::N - 1) / Chunk<T>::N;
    const int c1 = min(nch, (p + 1) * per);
    const RowCoef r = coef[i];
    const int at = a.tok[i];
    for (int c = p * per + threadIdx.x; c < c1; c += kRowThreads) {
        float g[Chunk<T>::N];
        if (r.dead != 0.f) {
#pragma unroll
            for (int k = 0; k < Chunk<T>::N; ++k) g[k] = 0.f;
        } else {
            const uint4 zc = Chunk<T>::load(z, c, a.V), qc = REF ? Chunk<T>::load(q, c, a.V) : zc;
            grad_chunk<T, REF>(r, zc, qc, a.kz, a.kq, g);
            if (c == at / Chunk<T>::N) add_token<T>(g, at % Chunk<T>::N, r.at);
        }
        Chunk<T>::store(dz, c, a.V, g);
    }
}

// One workgroup a row, the row in registers: read once, its maximum, its sums, its numbers, its gradient
// written.  Thread t holds chunks t, t + NT, ...; NT NC of them at most, and with BIG those past that are
// read twice, once for the sums with running maxima and once (from the last-level cache) for the gradient.
template <DType T, bool REF, int NT, int NC, bool BIG>
__global__ void __launch_bounds__(NT) row_fused_kernel(RowArgs a) {
    typedef typename St<T>::type E;
    constexpr int N = Chunk<T>::N, NW = NT / 64;
    __shared__ float redm[2][NW], reds[4][NW];
    __shared__ RowCoef coef;
    const long i = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int nfull = a.V / N, nch = (a.V + N - 1) / N;
    E *dz = (E *)a.dz + i * a.lddz;
    if (!row_counts(a, i)) {
        if (a.dz != nullptr) {
            const float zero[N] = {};
            for (int c = tid; c < nch; c += NT) Chunk<T>::store(dz, c, a.V, zero);
        }
        if (tid == 0) {
            if (a.logp != nullptr) a.logp[i] = 0.f;
            if (a.entropy != nullptr) a.entropy[i] = 0.f;
            if (a.policy)
                for (int k = 0; k < 4; ++k) a.row_terms[i * 4 + k] = 0.0;
        }
        return;
    }
    const E *z = (const E *)a.z + i * a.ldz;
    const E *q = REF ? (const E *)a.q + i * a.ldq : nullptr;
    const float kz = a.kz, kq = a.kq;
    const uint4 none = uint4{Chunk<T>::kNegInf, Chunk<T>::kNegInf, Chunk<T>::kNegInf, Chunk<T>::kNegInf};
    uint4 zr[NC], qr[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {  // all loads in flight; past the row the last whole chunk again, replaced below
        zr[c] = none;
        if (REF) qr[c] = none;
        if (c * NT < nfull) {
            const size_t at = (size_t)min(tid + c * NT, nfull - 1) * N;
            zr[c] = ld16(z + at);
            if (REF) qr[c] = ld16(q + at);
        }
    }
    const int at = a.tok[i];
    const float za = St<T>::load(z, at);
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (c * NT < nch && (c + 1) * NT > nfull) {  // where the row ends
            const int cc = tid + c * NT;
            if (cc >= nfull) {
                zr[c] = none;
                if (REF) qr[c] = none;
                if (cc < nch) {
                    zr[c] = Chunk<T>::load(z, cc, a.V);
                    if (REF) qr[c] = Chunk<T>::load(q, cc, a.V);
                }
            }
        }
    RowStats r = {kLowest, 0.f, 0.f, 0.f, kLowest, 0.f, za, 0.f};
    if (BIG) {
        constexpr int U = REF ? 2 : 4;
        for (int c = NC * NT + tid; c < nch; c += NT * U) {
            uint4 zc[U], qc[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int cc = c + u * NT < nch ? c + u * NT : c;
                zc[u] = Chunk<T>::load(z, cc, a.V);
                if (REF) qc[u] = Chunk<T>::load(q, cc, a.V);
            }
            float M = r.M, Mq = r.Mq;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                M = fmaxf(M, chunk_max<T>(zc[u]));
                if (REF) Mq = fmaxf(Mq, chunk_max<T>(qc[u]));
            }
            rebase<REF>(r, M, Mq, kz, kq);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c + u * NT < nch) add_chunk<T, REF>(r, zc[u], REF ? qc[u] : zc[u], kz, kq);
        }
    }
    float M = r.M, Mq = r.Mq;
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (c * NT < nch) {
            M = fmaxf(M, chunk_max<T>(zr[c]));
            if (REF) Mq = fmaxf(Mq, chunk_max<T>(qr[c]));
        }
    M = wave_max(M);
    if (REF) Mq = wave_max(Mq);
    if (NW > 1) {
        if (lane == 0) {
            redm[0][w] = M;
            if (REF) redm[1][w] = Mq;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            M = fmaxf(M, redm[0][k]);
            if (REF) Mq = fmaxf(Mq, redm[1][k]);
        }
    }
    if (BIG) {
        rebase<REF>(r, M, Mq, kz, kq);
    } else {
        r.M = M;
        r.Mq = Mq;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (c * NT < nch) add_chunk<T, REF>(r, zr[c], REF ? qr[c] : zr[c], kz, kq);
    r.s = wave_sum(r.s);
    r.t = wave_sum(r.t);
    if (REF) {
        r.k = wave_sum(r.k);
        r.sq = wave_sum(r.sq);
    }
    if (NW > 1) {
        if (lane == 0) {
            reds[0][w] = r.s;
            reds[1][w] = r.t;
            if (REF) {
                reds[2][w] = r.k;
                reds[3][w] = r.sq;
            }
        }
        __syncthreads();
    }
    if (w == 0) {
        if (NW > 1) {
            r.s = wave_sum(lane < NW ? reds[0][lane & (NW - 1)] : 0.f);
            r.t = wave_sum(lane < NW ? reds[1][lane & (NW - 1)] : 0.f);
            if (REF) {
                r.k = wave_sum(lane < NW ? reds[2][lane & (NW - 1)] : 0.f);
                r.sq = wave_sum(lane < NW ? reds[3][lane & (NW - 1)] : 0.f);
            }
        }
        float logp, entropy;
        double terms[4];
        const RowCoef c = row_numbers(a, i, r, logp, entropy, terms);
        if (lane == 0) {
            coef = c;
            if (a.logp != nullptr) a.logp[i] = logp;
            if (a.entropy != nullptr) a.entropy[i] = entropy;
            if (a.policy)
#pragma unroll
                for (int k = 0; k < 4; ++k) a.row_terms[i * 4 + k] = terms[k];
        }
    }
    if (a.dz == nullptr) return;
    __syncthreads();
    const RowCoef rc = coef;
    const bool dead = rc.dead != 0.f, kl = REF && rc.C != 0.f;
    auto put = [&](int c, const uint4 &zc, const uint4 &qc) {  // chunk c of the row
        float g[N];
        if (dead) {
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] = 0.f;
        } else {
            if (kl)
                grad_chunk<T, REF>(rc, zc, qc, kz, kq, g);
            else
                grad_chunk<T, false>(rc, zc, zc, kz, kq, g);
            if (c == at / N) add_token<T>(g, at % N, rc.at);
        }
        Chunk<T>::store(dz, c, a.V, g);
    };
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (tid + c * NT < nch) put(tid + c * NT, zr[c], REF ? qr[c] : zr[c]);
    if (BIG)
        for (int c = NC * NT + tid; c < nch; c += NT)
            put(c, Chunk<T>::load(z, c, a.V), REF ? Chunk<T>::load(q, c, a.V) : none);
}

// The loss and its terms, the rows in a fixed order.
__global__ void __launch_bounds__(1024) row_terms_kernel(RowArgs a) {
    __shared__ double red[4][16];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (long i = threadIdx.x; i < a.N; i += 1024)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += a.row_terms[i * 4 + k];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s[k] += __shfl_xor(s[k], o);
        if ((threadIdx.x & 63) == 0) red[k][threadIdx.x >> 6] = s[k];
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        s[k] = 0.0;
        for (int w = 0; w < 16; ++w) s[k] += red[k][w];
        a.terms[1 + k] = (float)s[k];
    }
    // a divergence that is only reported may be infinite
    a.terms[0] = (float)(s[0] + (a.c_kl != 0.0 ? a.c_kl * s[1] : 0.0) - a.c_ent * s[2]);
}

// Parts of a row: enough workgroups for the chip where there are few rows, but at least one round of
// loads (kRowThreads * kRowUnroll chunks) each.
static int row_parts(long N, int nch, int &per) {
    const int most = (nch + kRowThreads * kRowUnroll - 1) / (kRowThreads * kRowUnroll);
    const long want = (4L * compute_units() + N - 1) / N;
    int S = (int)(want < most ? want : most);
    per = (nch + S - 1) / S;
    return (nch + per - 1) / per;
}

static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

size_t rows_workspace(long N, int V, bool policy) {
    int per;
    const int S = row_parts(N > 0 ? N : 1, (V + 3) / 4, per);
    return up256((size_t)N * S * sizeof(RowStats)) + (policy ? up256((size_t)N * 32) + up256((size_t)N * sizeof(RowCoef)) : 0);
}

// Whether a row is one workgroup's (row_fused_kernel) or is split over several.
static bool row_whole(long N, int V) { return true; }

template <DType T, bool REF>
static void launch_fused(const RowArgs &a, int nch, hipStream_t s) {
    const unsigned n = (unsigned)a.N;
    if (nch <= 64 * 4)
        row_fused_kernel<T, REF, 64, 4, false><<<n, 64, 0, s>>>(a);
    else if (nch <= 256 * 4)
        row_fused_kernel<T, REF, 256, 4, false><<<n, 256, 0, s>>>(a);
    else if (nch <= 256 * 8)
        row_fused_kernel<T, REF, 256, 8, false><<<n, 256, 0, s>>>(a);
    else if (nch <= 512 * 8)
        row_fused_kernel<T, REF, 512, 8, false><<<n, 512, 0, s>>>(a);
    else if (nch <= 1024 * 8)
        row_fused_kernel<T, REF, 1024, 8, false><<<n, 1024, 0, s>>>(a);
    else
        row_fused_kernel<T, REF, 1024, 8, true><<<n, 1024, 0, s>>>(a);
}

template <DType T, bool REF>
static void launch_rows_t(RowArgs a, void *workspace, hipStream_t s) {
    const int nch = (a.V + Chunk<T>::N - 1) / Chunk<T>::N;
    if (a.N > 0 && row_whole(a.N, a.V)) {
        a.row_terms = (double *)workspace;
        launch_fused<T, REF>(a, nch, s);
        if (a.policy) row_terms_kernel<<<1, 1024, 0, s>>>(a);
        return;
    }
    int per;
    const int S = row_parts(a.N > 0 ? a.N : 1, nch, per);
    uint8_t *w = (uint8_t *)workspace;
    a.part = (RowStats *)w;
    w += up256((size_t)a.N * S * sizeof(RowStats));
    a.row_terms = (double *)w;
    RowCoef *coef = (RowCoef *)(w + up256((size_t)a.N * 32));
    if (a.N == 0) {  // no rows: the terms are 0
        row_terms_kernel<<<1, 1024, 0, s>>>(a);
        return;
    }
    row_stats_kernel<T, REF><<<(unsigned)(a.N * S), kRowThreads, 0, s>>>(a, S, per);
    row_finish_kernel<T, REF><<<(unsigned)((a.N + 63) / 64), 64, 0, s>>>(a, coef, S, per);
    if (!a.policy) return;
    if (a.dz != nullptr) {
        if (REF && a.c_kl != 0.0)
            row_grad_kernel<T, REF><<<(unsigned)(a.N * S), kRowThreads, 0, s>>>(a, coef, S, per);
        else
            row_grad_kernel<T, false><<<(unsigned)(a.N * S), kRowThreads, 0, s>>>(a, coef, S, per);
    }
    row_terms_kernel<<<1, 1024, 0, s>>>(a);
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

// Four consecutive elements from i on; those at n and past it are 0.
template <DType T>
__device__ __forceinline__ void load4(const void *p, long i, long n, float *v) {
    typedef typename St<T>::type E;
    const E *e = (const E *)p + i;
    if (i + 4 <= n) {
        if (T == DType::F32) {
            unpack_frag<DType::F32>(ld16(e), v);
        } else {
            const v2u w = *(const v2u_any *)e;
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
template <DType T>
__device__ __forceinline__ void store4(void *p, long i, long n, const float *v) {
    typedef typename St<T>::type E;
    E *e = (E *)p + i;
    if (i + 4 <= n) {
        if (T == DType::F32)
            st16(e, pack_frag_cvt<DType::F32>(v));
        else
            *(v2u_any *)e = v2u{pack2bf(v[0], v[1]), pack2bf(v[2], v[3])};
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) St<T>::store(e, k, v[k]);
    }
}
__device__ __forceinline__ uint32_t load4_codes(const void *p, long i, long n) {
    const uint8_t *b = (const uint8_t *)p + i;
    uint32_t w = 0;
    if (i + 4 <= n) {
        w = *(const u32_any *)b;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) w |= (uint32_t)b[k] << (8 * k);
    }
    return w;
}
__device__ __forceinline__ void store4_codes(void *p, long i, long n, uint32_t w) {
    uint8_t *b = (uint8_t *)p + i;
    if (i + 4 <= n) {
        *(u32_any *)b = w;
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
template <DType GT>
__global__ void __launch_bounds__(256) adam_norm_kernel(NormTable tab, double *part) {
    __shared__ double red[4];
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < (uint32_t)tab.chunks; c += gridDim.x) {
        const int t = tensor_of(tab, c);
        const long n = tab.len[t], i0 = (long)(c - tab.first[t]) * kAdamChunk + 4 * threadIdx.x;
        float g[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i0 + 1024 * u < n) {
                load4<GT>(tab.g[t], i0 + 1024 * u, n, g[u]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) g[u][k] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) s += (double)g[u][k] * (double)g[u][k];
    }
    s = wave_sum_f64(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = ((red[0] + red[1]) + red[2]) + red[3];
}

// The norm out of the partial sums, the same in every workgroup.
__device__ __forceinline__ double norm_of(const double *part, int n, double *red4) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) s += part[i];
    s = wave_sum_f64(s);
    if ((threadIdx.x & 63) == 0) red4[threadIdx.x >> 6] = s;
    __syncthreads();
    return sqrt(((red4[0] + red4[1]) + red4[2]) + red4[3]);
}

__global__ void __launch_bounds__(256) adam_norm_out_kernel(const double *part, int n, float *norm) {
    __shared__ double red[4];
    const double v = norm_of(part, n, red);
    if (threadIdx.x == 0) norm[0] = (float)v;
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

// One AdamW step, a wave per 256 elements (the block of an 8-bit state), four consecutive ones a lane; a
// workgroup takes a chunk of 4096, each wave four blocks whose loads are all in flight together.
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p (1 - lr wd) - rate m / (sqrt(v) root + eps)
// 8-bit states hold m and sqrt(v) as e4m3 times a scale per block (its largest / 448), rounded up or down
// at random so that the mean is right: v moves by 1 - b2 of itself a step, far less than half a spacing of
// e4m3, and would stay where it is under rounding to nearest.  The step itself uses m and v before that
// rounding.  A root that is not zero is kept from rounding to zero, which would blow the next step up.
// Every operation rounds by itself (no fused multiply-add): near the border of a random rounding the codes
// then are those of the same formulas in any other IEEE arithmetic of 32 bits.
template <DType PT, bool MASTER, DType GT, int BITS>
__global__ void __launch_bounds__(256) adamw_kernel(AdamTable tab, AdamArgs a) {
#pragma clang fp contract(off)
    __shared__ double red[4];
    float clip = 1.f;
    if (a.norm_part != nullptr) {
        const double norm = norm_of(a.norm_part, a.n_part, red);
        if (a.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) a.norm[0] = (float)norm;
        if (!(norm <= 1.7e308)) return;  // a gradient that is not finite: no step
        if (norm > (double)a.max_norm) clip = (float)((double)a.max_norm / norm);
    }
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t c = blockIdx.x;
    const int ti = tensor_of(tab, c);
    const AdamTensor t = tab.t[ti];
    const long n = t.n, i0 = (long)(c - tab.first[ti]) * kAdamChunk + 1024 * w + 4 * lane;
    constexpr int U = 4;
    float p[U][4], g[U][4];
    State<BITS> st[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long i = i0 + kStateBlock * u;
        if (i - 4 * lane >= n) continue;  // uniform: the block is past the tensor
        load4<MASTER ? DType::F32 : PT>(MASTER ? (const void *)t.master : (const void *)t.p, i, n, p[u]);
        load4<GT>(t.g, i, n, g[u]);
        if constexpr (BITS == 32) {
            load4<DType::F32>(t.m, i, n, st[u].m);
            load4<DType::F32>(t.v, i, n, st[u].v);
        } else {
            st[u].m = load4_codes(t.m, i, n);
            st[u].r = load4_codes(t.v, i, n);
            st[u].ms = t.ms[(i - 4 * lane) / kStateBlock];
            st[u].rs = t.vs[(i - 4 * lane) / kStateBlock];
        }
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
        if (MASTER) store4<DType::F32>(t.master, i, n, p[u]);
        store4<PT>(t.p, i, n, p[u]);
        if constexpr (BITS == 32) {
            store4<DType::F32>(t.m, i, n, m);
            store4<DType::F32>(t.v, i, n, v);
        } else {
            // lanes past the tensor hold m = v = 0
            float mm = fmaxf(fmaxf(fabsf(m[0]), fabsf(m[1])), fmaxf(fabsf(m[2]), fabsf(m[3])));
            float rm = fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3]));
            mm = wave_max(mm);
            rm = wave_max(rm);
            constexpr float kTiny = 0x1p-100f;  // blocks whose largest is below are held as zeros
            const float im = mm < kTiny ? 0.f : 448.f / mm, ir = rm < kTiny ? 0.f : 448.f / rm;
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
            store4_codes(t.m, i, n, (uint32_t)mw);
            store4_codes(t.v, i, n, (uint32_t)rw);
            if (lane == 0) {
                t.ms[i / kStateBlock] = mm < kTiny ? 0.f : mm / 448.f;
                t.vs[i / kStateBlock] = rm < kTiny ? 0.f : rm / 448.f;
            }
        }
    }
}

static uint32_t chunks_of(long n) { return (uint32_t)((n + kAdamChunk - 1) / kAdamChunk); }

int adam_norm_parts(const AdamTensor *t, int n) {
    long c = 0;
    for (int i = 0; i < n; ++i) c += chunks_of(t[i].n);
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
        c += chunks_of(t[i].n);
    }
    tab.chunks = (int)c;
    const int grid = adam_norm_parts(t, n);
    if (gt == DType::BF16)
        adam_norm_kernel<DType::BF16><<<grid, 256, 0, s>>>(tab, part);
    else
        adam_norm_kernel<DType::F32><<<grid, 256, 0, s>>>(tab, part);
}

void launch_adam_norm_out(const double *part, int n_part, float *norm, hipStream_t s) {
    adam_norm_out_kernel<<<1, 256, 0, s>>>(part, n_part, norm);
}

template <DType PT, bool MASTER, DType GT>
static void launch_adamw_t(int bits, const AdamTable &tab, const AdamArgs &a, hipStream_t s) {
    if (bits == 8)
        adamw_kernel<PT, MASTER, GT, 8><<<tab.chunks, 256, 0, s>>>(tab, a);
    else
        adamw_kernel<PT, MASTER, GT, 32><<<tab.chunks, 256, 0, s>>>(tab, a);
}

void launch_adamw(DType pt, bool master, DType gt, int bits, const AdamTensor *t, int n, const AdamArgs &a, hipStream_t s) {
    AdamTable tab;
    tab.n = n;
    uint32_t c = 0;
    for (int i = 0; i < n; ++i) {
        tab.first[i] = c;
        tab.t[i] = t[i];
        c += chunks_of(t[i].n);
    }
    tab.chunks = (int)c;
    const bool gb = gt == DType::BF16;
    if (pt == DType::F32)
        gb ? launch_adamw_t<DType::F32, false, DType::BF16>(bits, tab, a, s) : launch_adamw_t<DType::F32, false, DType::F32>(bits, tab, a, s);
    else if (master)
        gb ? launch_adamw_t<DType::BF16, true, DType::BF16>(bits, tab, a, s) : launch_adamw_t<DType::BF16, true, DType::F32>(bits, tab, a, s);
    else
        gb ? launch_adamw_t<DType::BF16, false, DType::BF16>(bits, tab, a, s) : launch_adamw_t<DType::BF16, false, DType::F32>(bits, tab, a, s);
}

}  // namespace dvi
