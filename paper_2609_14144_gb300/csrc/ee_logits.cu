// Operators over rows of logits [rows, vocab]: log probabilities of given
// tokens with entropy and the best alternatives (ee_token_logprobs), and the
// distillation of a teacher's best tokens into the row with its gradient
// (ee_distill_topk, ee_distill_topk_backward).
//
// All of them are bound by reading (and, for the gradient, writing) the logits
// once.  A row is streamed by one CTA, or by a cluster of up to 8 CTAs when
// there are few rows, each thread with a running maximum m and the sum of
// 2^((x - m) c), c = log2(e) / T, in 32 bits; the threads' pairs join in the
// warp, the CTA and the cluster.  x - m is formed before the product with c, so
// that rows masked with the type's lowest value do not overflow.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>

#include <algorithm>

#include "ee_internal.h"

namespace cg = cooperative_groups;

namespace ee {
namespace {

constexpr int kLT = 256;      // threads per CTA
constexpr int kLU = 4;        // 16-byte vectors per thread and batch
constexpr int kCand = 2048;   // candidates a CTA collects for the best tokens
constexpr int kMaxList = EE_MAX_TOP;
constexpr int kMaxCluster = 8;
constexpr int kMaxBits = (EE_MAX_VOCAB / kMaxCluster) / 8 + 256;  // shared bytes of a slice's listed bits
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kInf = __builtin_huge_valf();
constexpr unsigned kFull = 0xffffffffu;

__device__ __forceinline__ float ex2(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
// The same without flushing powers below 2^-126 to zero, for results.
__device__ __forceinline__ float ex2_full(float t) {
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// ---------------------------------------------------------------- element types
template <int DT>
struct El;
template <>
struct El<EE_BF16> {
    using T = uint16_t;
    static constexpr int E = 8;
    static constexpr uint32_t ninf = 0xff80ff80u;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ float vmax(const uint4& v) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        const __nv_bfloat162 a = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        return max_nan(__low2float(a), __high2float(a));
    }
    static __device__ __forceinline__ float one(T v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ T put(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
};
template <>
struct El<EE_FP16> {
    using T = uint16_t;
    static constexpr int E = 8;
    static constexpr uint32_t ninf = 0xfc00fc00u;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(h[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float vmax(const uint4& v) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
        const __half2 a = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        return max_nan(__low2float(a), __high2float(a));
    }
    static __device__ __forceinline__ float one(T v) { return __half2float(__ushort_as_half(v)); }
    static __device__ __forceinline__ T put(float f) { return __half_as_ushort(__float2half_rn(f)); }
};
template <>
struct El<EE_FP32> {
    using T = uint32_t;
    static constexpr int E = 4;
    static constexpr uint32_t ninf = 0xff800000u;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x);
        x[1] = __uint_as_float(v.y);
        x[2] = __uint_as_float(v.z);
        x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ float vmax(const uint4& v) {
        return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)),
                       max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float one(T v) { return __uint_as_float(v); }
    static __device__ __forceinline__ T put(float f) { return __float_as_uint(f); }
};

// A row as 16-byte vectors: vector v holds elements [v E - mis, v E - mis + E)
// of the row, mis being how many elements lie between a 16-byte boundary and
// the row's start.  Elements outside the row read as -inf.
template <int DT>
struct Row {
    using T = typename El<DT>::T;
    const T* p;
    int V, mis, nv;
    __device__ Row(const void* logits, int64_t ld, int64_t row, int vocab) {
        p = reinterpret_cast<const T*>(logits) + row * ld;
        V = vocab;
        mis = (int)(((uintptr_t)p & 15) / sizeof(T));
        nv = (int)(((int64_t)V + mis + El<DT>::E - 1) / El<DT>::E);
    }
    __device__ __forceinline__ uint4 load(int v) const {
        const int64_t b = (int64_t)v * El<DT>::E - mis;
        if (b >= 0 && b + El<DT>::E <= V) return *reinterpret_cast<const uint4*>(p + b);
        return load_edge(b);
    }
    __device__ __noinline__ uint4 load_edge(int64_t b) const {
        uint4 r = make_uint4(El<DT>::ninf, El<DT>::ninf, El<DT>::ninf, El<DT>::ninf);
        T* e = reinterpret_cast<T*>(&r);
        for (int i = 0; i < El<DT>::E; ++i)
            if (b + i >= 0 && b + i < V) e[i] = p[b + i];
        return r;
    }
    __device__ __forceinline__ uint4 load_if(int v, int end) const {
        if (v < end) return load(v);
        return make_uint4(El<DT>::ninf, El<DT>::ninf, El<DT>::ninf, El<DT>::ninf);
    }
};

// ---------------------------------------------------------------- running softmax
// m: largest value so far (-inf: none); s: sum of 2^((x - m) c); a: sum of
// t 2^t, t = (x - m) c, from which the entropy follows.
struct Run {
    float m, s, a;
};
// Rescale to the larger maximum m2.
__device__ __forceinline__ void run_to(Run& r, float m2, float c) {
    const float d = (r.m - m2) * c, f = ex2(d);
    const bool none = r.m == -kInf || f == 0.f;  // (0 times an infinite d would be NaN)
    r.a = none ? 0.f : f * (r.a + d * r.s);
    r.s = none && r.s == r.s ? 0.f : f * r.s;
    r.m = m2;
}
__device__ __forceinline__ void run_join(Run& r, Run o, float c) {
    if (o.m > r.m) {
        const Run t = r;
        r = o;
        o = t;
    }
    if (o.m == -kInf) {  // nothing in o, but a NaN stays one
        r.s += o.s;
        return;
    }
    run_to(o, r.m, c);
    r.s += o.s;
    r.a += o.a;
}
__device__ __forceinline__ Run run_shfl(const Run& r, int off) {
    return Run{__shfl_xor_sync(kFull, r.m, off), __shfl_xor_sync(kFull, r.s, off), __shfl_xor_sync(kFull, r.a, off)};
}

// The CTA's joined state, then the cluster's; every thread returns it.
struct RunShared {
    Run warp[kLT / 32];
    Run cta;
};
__device__ Run run_reduce(Run r, RunShared& sh, float c, int cs) {
#pragma unroll
    for (int o = 16; o; o >>= 1) run_join(r, run_shfl(r, o), c);
    if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5] = r;
    __syncthreads();
    r = sh.warp[0];
    for (int i = 1; i < kLT / 32; ++i) run_join(r, sh.warp[i], c);
    if (cs > 1) {
        cg::cluster_group cl = cg::this_cluster();
        if (threadIdx.x == 0) sh.cta = r;
        cl.sync();
        r = *cl.map_shared_rank(&sh.cta, 0);
        for (int i = 1; i < cs; ++i) run_join(r, *cl.map_shared_rank(&sh.cta, i), c);
    }
    return r;
}

// ---------------------------------------------------------------- best tokens
// A candidate is one 64-bit key: the value's order in the high half (NaN above
// +inf, both zeros alike), the complement of its index in the low half, so that
// of equal values the lowest index is the largest key.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ (uint32_t)((int)u >> 31 | (int)0x80000000);
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ unsigned long long key_of(float x, int idx) {
    return (unsigned long long)order_of(x) << 32 | (0xffffffffu - (uint32_t)idx);
}

struct TopShared {
    unsigned long long keys[kCand];
    unsigned long long best[kMaxList];
    unsigned long long surv[2 * kMaxList + 128];
    unsigned hist[256];
    int n;         // candidates pushed (may pass kCand: the surplus was dropped)
    int n_surv;
    int sum[3];    // rotating counters of block_sum, zero between uses
    unsigned long long prefix;
    int done;
};

// Sum over the CTA with one barrier: a slot is cleared two calls before it is
// used again.
__device__ __forceinline__ int block_sum(int v, TopShared& sh, int& turn) {
    v = __reduce_add_sync(kFull, v);
    const int slot = turn % 3;
    if ((threadIdx.x & 31) == 0 && v) atomicAdd(&sh.sum[slot], v);
    __syncthreads();
    const int r = sh.sum[slot];
    if (threadIdx.x == 0) sh.sum[(turn + 2) % 3] = 0;
    ++turn;
    return r;
}

// Of the n keys, the largest prefix (over the bits from 63 down to `last`) that
// at least `want` keys reach; stops early once at most `enough` do.  Every
// thread returns it.
__device__ unsigned long long key_prefix(const unsigned long long* keys, int n, int want, int enough, int last,
                                         TopShared& sh, int& turn) {
    unsigned long long P = 0;
    for (int bit = 63; bit >= last; --bit) {
        const unsigned long long cand = P | 1ull << bit;
        int c = 0;
        for (int i = threadIdx.x; i < n; i += kLT) c += keys[i] >= cand;
        c = block_sum(c, sh, turn);
        if (c >= want) {
            P = cand;
            if (c <= enough) break;
        }
    }
    return P;
}

// The value a later candidate has to reach, given a prefix of 16 bits.
__device__ __forceinline__ float prefix_value(unsigned long long P) {
    const uint32_t o = (uint32_t)(P >> 32);
    if (o <= 0x007fffffu) return -FLT_MAX;  // -inf is never a candidate
    if (o > 0xff800000u) return kInf;
    return value_of(o);
}

__device__ __forceinline__ void push(float x, int idx, TopShared& sh) {
    const int at = atomicAdd(&sh.n, 1);
    if (at < kCand) sh.keys[at] = key_of(x, idx);
}

// sh.best = the largest min(n, k) of sh.keys[0..n), in order; returns how many.
__device__ int select_best(int n, int k, TopShared& sh, int& turn) {
    const int want = n < k ? n : k;
    if (threadIdx.x == 0) sh.n_surv = 0;
    if (want == 0) {
        __syncthreads();
        return 0;
    }
    constexpr int room = 2 * kMaxList + 128;
    const int enough = 2 * want + 64;  // <= room
    const unsigned long long P = n > enough ? key_prefix(sh.keys, n, want, enough, 0, sh, turn) : 0ull;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kLT)
        if (sh.keys[i] >= P) {
            const int at = atomicAdd(&sh.n_surv, 1);
            if (at < room) sh.surv[at] = sh.keys[i];
        }
    __syncthreads();
    const int ns = sh.n_surv;  // the keys differ, so that at most `enough` reach the prefix
    for (int i = threadIdx.x; i < ns; i += kLT) {
        const unsigned long long me = sh.surv[i];
        int above = 0;
        for (int j = 0; j < ns; ++j) above += sh.surv[j] > me;
        if (above < want) sh.best[above] = me;
    }
    __syncthreads();
    return want;
}

// More candidates than the buffer holds (ascending rows, thousands of equal
// values): the prefix is found digit by digit over the slice itself, eight bits
// a pass, until at most kCand keys reach it; then they are collected again.
template <int DT>
__device__ int recollect(const Row<DT>& row, int v0, int v1, int k, TopShared& sh) {
    constexpr int E = El<DT>::E;
    unsigned long long prefix = 0;
    int above = 0;  // keys known to lie above the prefix
    for (int shift = 56;; shift -= 8) {
        sh.hist[threadIdx.x] = 0;
        __syncthreads();
        for (int vb = v0; vb < v1; vb += kLT) {
            const int v = vb + threadIdx.x;
            float x[E];
            El<DT>::unpack(row.load_if(v, v1), x);
#pragma unroll 1
            for (int e = 0; e < E; ++e) {
                const unsigned long long key = key_of(x[e], (int)((int64_t)v * E - row.mis + e));
                const bool in = x[e] != -kInf && (shift == 56 || (key >> (shift + 8)) == prefix);
                const int d = in ? (int)(key >> shift & 255) : 256;
                int same;
                __match_all_sync(kFull, d, &same);
                if (d < 256) {
                    if (!same) atomicAdd(&sh.hist[d], 1u);
                    else if ((threadIdx.x & 31) == 0) atomicAdd(&sh.hist[d], 32u);
                }
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int got = above, d = 255;
            while (d > 0 && got + (int)sh.hist[d] < k) got += (int)sh.hist[d--];
            sh.prefix = prefix << 8 | (unsigned)d;
            sh.done = got + (int)sh.hist[d] <= kCand;
            sh.n_surv = got;
            sh.n = 0;
        }
        __syncthreads();
        prefix = sh.prefix;
        above = sh.n_surv;
        if (sh.done || shift == 0) {
            prefix <<= shift;
            break;
        }
        __syncthreads();
    }
    for (int v = v0 + threadIdx.x; v < v1; v += kLT) {
        float x[E];
        El<DT>::unpack(row.load(v), x);
#pragma unroll 1
        for (int e = 0; e < E; ++e) {
            const int idx = (int)((int64_t)v * E - row.mis + e);
            if (x[e] != -kInf && key_of(x[e], idx) >= prefix) push(x[e], idx, sh);
        }
    }
    __syncthreads();
    return sh.n;
}

struct LogprobArgs {
    const void* logits;
    int64_t ld;
    int vocab, k;
    const int32_t* ids;
    float temperature;
    float *logprob, *entropy, *lse, *top_logprob;
    int32_t* top_id;
};

// One row per cluster of `cs` CTAs.  Which elements can be among the k best is
// decided with one comparison per vector: after the first batch the k-th
// largest of the threads' maxima bounds the k-th best from below, and the bound
// is raised from the collected candidates while they are many.  Per element the
// pass spends about eight instructions; what bounds it is the read.
template <int DT, bool TOP>
__global__ void __launch_bounds__(kLT) k_logprobs(LogprobArgs a, int cs) {
    constexpr int E = El<DT>::E;
    __shared__ RunShared rs;
    __shared__ TopShared ts;
    const int64_t r = blockIdx.x / cs;
    const int rank = (int)(blockIdx.x % cs), tid = threadIdx.x;
    const Row<DT> row(a.logits, a.ld, r, a.vocab);
    const int v0 = (int)((int64_t)row.nv * rank / cs), v1 = (int)((int64_t)row.nv * (rank + 1) / cs);
    const float c = 1.4426950408889634f / a.temperature;
    Run run{-kInf, 0.f, 0.f};
    float thr = -FLT_MAX;
    int turn = 0;
    if (TOP) {
        if (tid < 3) ts.sum[tid] = 0;
        if (tid == 3) ts.n = 0;
        __syncthreads();
    }
    uint4 nxt[kLU];
#pragma unroll
    for (int u = 0; u < kLU; ++u) nxt[u] = row.load_if(v0 + tid + u * kLT, v1);
    int it = 0;
    for (int vb = v0; vb < v1; vb += kLT * kLU, ++it) {
        uint4 cur[kLU];
#pragma unroll
        for (int u = 0; u < kLU; ++u) {
            cur[u] = nxt[u];
            nxt[u] = row.load_if(vb + tid + (kLU + u) * kLT, v1);
        }
        float vm[kLU];
#pragma unroll
        for (int u = 0; u < kLU; ++u) vm[u] = El<DT>::vmax(cur[u]);
        if (TOP) {
            if (it == 0) {
                float t = vm[0];
#pragma unroll
                for (int u = 1; u < kLU; ++u) t = max_nan(t, vm[u]);
                ts.keys[tid] = (unsigned long long)order_of(t) << 32;
                __syncthreads();
                thr = a.k <= kLT ? prefix_value(key_prefix(ts.keys, kLT, a.k, a.k, 48, ts, turn)) : -FLT_MAX;
                __syncthreads();
            } else if ((it & (it - 1)) == 0) {
                __syncthreads();
                const int n = ts.n;
                __syncthreads();  // nobody pushes before all have read it
                if (n > 512 && n <= kCand) {
                    thr = fmaxf(thr, prefix_value(key_prefix(ts.keys, n, a.k, a.k, 48, ts, turn)));
                    __syncthreads();
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kLU; ++u) {
            float x[E];
            El<DT>::unpack(cur[u], x);
            if (vm[u] > run.m) run_to(run, vm[u], c);
            const float m = run.m == -kInf ? 0.f : run.m;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float t = (x[e] - m) * c, p = ex2(t);
                run.s += p;
                run.a = fmaf(p, fmaxf(t, -1e6f), run.a);  // (0 times -inf would be NaN)
            }
            if (TOP && !(vm[u] < thr)) {
                const int base = (int)((int64_t)(vb + tid + u * kLT) * E - row.mis);
#pragma unroll 1
                for (int e = 0; e < E; ++e) {
                    float y[E];
                    El<DT>::unpack(cur[u], y);
                    float xe = y[0];
#pragma unroll
                    for (int j = 1; j < E; ++j) xe = e == j ? y[j] : xe;
                    if (!(xe < thr)) push(xe, base + e, ts);
                }
            }
        }
    }
    run = run_reduce(run, rs, c, cs);
    const float lns = logf(run.s), inv_t = 1.f / a.temperature;
    const bool none = run.m == -kInf && run.s == 0.f;
    if (rank == 0 && tid == 0) {
        const float lse = none ? -kInf : fmaf(run.m, inv_t, lns);
        if (a.lse) a.lse[r] = lse;
        if (a.entropy) a.entropy[r] = none ? 0.f : lns - run.a / run.s * kLn2;
        if (a.logprob) {
            const int32_t id = a.ids[r];
            float lp = 0.f;
            if (id >= a.vocab) lp = __int_as_float(0x7fffffff);
            else if (id >= 0) lp = none ? -kInf : (El<DT>::one(row.p[id]) - run.m) * inv_t - lns;
            a.logprob[r] = lp;
        }
    }
    if constexpr (!TOP) {
        if (cs > 1) cg::this_cluster().sync();  // the others may still read this CTA's state
    } else {
        __syncthreads();
        int n = ts.n;
        __syncthreads();
        if (n > kCand) n = recollect<DT>(row, v0, v1, a.k, ts);
        int nb = select_best(n, a.k, ts, turn);
        if (cs > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (tid == 0) ts.n = nb;
            cl.sync();
            if (rank == 0) {
                int at = 0;
                for (int i = 0; i < cs; ++i) {
                    const TopShared* o = cl.map_shared_rank(&ts, i);
                    const int ni = o->n;
                    for (int j = tid; j < ni; j += kLT) ts.keys[at + j] = o->best[j];
                    at += ni;
                }
                n = at;
            }
            cl.sync();  // the others' lists have been read
            if (rank != 0) return;
            nb = select_best(n, a.k, ts, turn);
        }
        float* tl = a.top_logprob + r * a.k;
        int32_t* ti = a.top_id + r * a.k;
        for (int i = tid; i < nb; i += kLT) {
            const unsigned long long key = ts.best[i];
            const float x = value_of((uint32_t)(key >> 32));
            ti[i] = (int32_t)(0xffffffffu - (uint32_t)key);
            tl[i] = (x - run.m) * inv_t - lns;
        }
        if (nb < a.k && tid < 32) {  // fewer than k above -inf: the masked ones follow by index
            int at = nb;
            for (int b = 0; b < a.vocab && at < a.k; b += 32) {
                const bool is = b + tid < a.vocab && El<DT>::one(row.p[b + tid]) == -kInf;
                const unsigned vote = __ballot_sync(kFull, is);
                const int mine = at + __popc(vote & ((1u << tid) - 1));
                if (is && mine < a.k) {
                    ti[mine] = b + tid;
                    tl[mine] = none ? -kInf : (-kInf - run.m) * inv_t - lns;
                }
                at += __popc(vote);
            }
        }
    }
}

// ---------------------------------------------------------------- distillation
// With u = x / T, p = softmax(u), the teacher's list S with weights q (over S
// alone, or with the rest q0 = 1 - sum q of the vocabulary as one bucket):
//   loss = T^2 [ sum_S q (log q - log p) + q0 (log q0 - log p0) ]
//   d loss / d x_v = T (Q p_v - q_v)                               v in S
//                  = T (Q p_v - q0 2^((x_v - mo) c) / So)          otherwise
// (mo, So) is the running softmax of the unlisted elements alone, so p0 is
// their sum and not what is left of 1, and with Q = sum q + q0 both terms of an
// unlisted element share one power: alpha 2^((x_v - mo) c).  A bit per element
// of the slice tells which are listed.
struct DistillArgs {
    const void* logits;
    int64_t ld;
    int vocab, k, tail;
    const int32_t* ids;
    int64_t ld_ids;
    const float* teacher;
    int64_t ld_teacher;
    float temperature;
    const float* weight;  // per-row factor of the gradient (null: 1)
    float* loss;
    float4* stats;
    void* grad;
    int64_t ld_grad;
};

struct ListShared {
    int id[kMaxList];     // -1: absent
    float x[kMaxList];    // the row's value there
    float t[kMaxList];    // the teacher's value
    double lq[kMaxList];  // log q
    float q[kMaxList];
    bool first[kMaxList]; // no earlier entry names this token
    float4 coef;          // mo, alpha, M, Q / S
    float loss;
};

// The teacher's list of a row; an entry is absent if its token is outside the
// vocabulary or its value is -inf.
template <int DT>
__device__ void list_load(const DistillArgs& a, const Row<DT>& row, int64_t r, ListShared& ls) {
    for (int i = threadIdx.x; i < a.k; i += blockDim.x) {
        const int id = a.ids[r * a.ld_ids + i];
        const float t = a.teacher[r * a.ld_teacher + i];
        const bool in = id >= 0 && id < a.vocab && t != -kInf;
        ls.id[i] = in ? id : -1;
        ls.t[i] = in ? t : -kInf;
        ls.x[i] = in ? El<DT>::one(row.p[id]) : -kInf;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.k; i += blockDim.x) {
        bool first = ls.id[i] >= 0;
        for (int j = 0; j < i && first; ++j) first = ls.id[j] != ls.id[i];
        ls.first[i] = first;
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}

// q and log q of the list (one warp); returns sum q.  In 64 bits, as the loss
// below: it is a small difference of terms q log q and q log p, and q0 one of 1
// and the sum.
__device__ double list_weights(const DistillArgs& a, ListShared& ls) {
    const int lane = threadIdx.x & 31;
    double shift = 0.0;
    if (!a.tail) {  // softmax over the list
        float tm = -kInf;
        for (int i = lane; i < a.k; i += 32) tm = fmaxf(tm, ls.t[i]);
        tm = warp_max(tm);
        if (tm == -kInf) tm = 0.f;
        double z = 0.0;
        for (int i = lane; i < a.k; i += 32) z += exp((double)ls.t[i] - tm);
        z = warp_sum(z);
        shift = tm + (z > 0.0 || z != z ? log(z) : 0.0);
    }
    double q = 0.0;
    for (int i = lane; i < a.k; i += 32) {
        ls.lq[i] = ls.t[i] - shift;
        const double e = exp(ls.lq[i]);
        ls.q[i] = (float)e;
        q += e;
    }
    return warp_sum(q);
}

// Loss and gradient coefficients of a row from the unlisted elements' joined
// softmax (one warp).
__device__ void list_finish(const DistillArgs& a, const Run& o, float c, ListShared& ls) {
    const int lane = threadIdx.x & 31;
    int listed = 0;
    for (int i = lane; i < a.k; i += 32) listed += ls.first[i];
    listed = __reduce_add_sync(kFull, listed);
    const double Q = list_weights(a, ls), inv_t = 1.0 / a.temperature;
    double q0 = a.tail ? fmax(0.0, 1.0 - Q) : 0.0;
    if (Q != Q) q0 = Q;  // a NaN in the list stays one
    // nothing can be left over where the list covers the vocabulary; and where
    // the rest is masked out, what rounding leaves of 1 - Q is nothing either
    if (listed == a.vocab || (o.s == 0.f && q0 < a.k * 0x1p-22)) q0 = 0.0;
    float M = o.m;
    for (int i = lane; i < a.k; i += 32)
        if (ls.id[i] >= 0) M = max_nan(M, ls.x[i]);
#pragma unroll
    for (int w = 16; w; w >>= 1) M = max_nan(M, __shfl_xor_sync(kFull, M, w));
    const float ref = M == -kInf ? 0.f : M, mo = o.m == -kInf ? 0.f : o.m;
    float in = 0.f;
    for (int i = lane; i < a.k; i += 32)
        if (ls.first[i]) in += ex2((ls.x[i] - ref) * c);
    const float shrink = o.m == -kInf ? 0.f : ex2_full((o.m - ref) * c);  // unlisted powers relative to M
    const float S = fmaf(o.s, shrink, warp_sum(in));
    const bool none = S == 0.f;  // no finite logit in the row
    const double lns = none ? 0.0 : log((double)S);
    double loss = 0.0;
    for (int i = lane; i < a.k; i += 32) {
        const double q = exp(ls.lq[i]), lp = none ? -kInf : ((double)ls.x[i] - ref) * inv_t - lns;
        if (q > 0.0 || q != q) loss += q * (ls.lq[i] - lp);
    }
    loss = warp_sum(loss);
    if (lane == 0) {
        if (q0 > 0.0 || q0 != q0)
            loss += q0 * (log(q0) - (o.s == 0.f ? -kInf : ((double)o.m - ref) * inv_t + (log((double)o.s) - lns)));
        ls.loss = (float)(loss * a.temperature * a.temperature);
        const double Qt = Q + q0, k = none ? 0.0 : Qt / S;
        ls.coef = make_float4(mo, o.s == 0.f ? 0.f : (float)(k * shrink - q0 / o.s), ref, (float)k);
    }
}

// Writes the gradient of vectors [v0, v1) of the row, then the listed elements
// among them.  f: the row's factor (weight times T).
template <int DT>
__device__ void write_grad(const DistillArgs& a, const Row<DT>& row, int64_t r, int v0, int v1, float c, float f,
                           const ListShared& ls) {
    using T = typename El<DT>::T;
    constexpr int E = El<DT>::E;
    T* g = reinterpret_cast<T*>(a.grad) + r * a.ld_grad;
    const bool aligned = (int)(((uintptr_t)g & 15) / sizeof(T)) == row.mis;
    const float mo = ls.coef.x, alpha = ls.coef.y * f;
    const bool zero = f == 0.f;  // rows outside the batch: zeros, whatever they hold
    for (int vb = v0; vb < v1; vb += kLT * kLU) {
        uint4 cur[kLU];
#pragma unroll
        for (int u = 0; u < kLU; ++u)
            if (!zero) cur[u] = row.load_if(vb + threadIdx.x + u * kLT, v1);
#pragma unroll
        for (int u = 0; u < kLU; ++u) {
            const int v = vb + threadIdx.x + u * kLT;
            if (v >= v1) continue;
            float x[E];
            uint4 out = make_uint4(0, 0, 0, 0);
            T* o = reinterpret_cast<T*>(&out);
            if (!zero) {
                El<DT>::unpack(cur[u], x);
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = El<DT>::put(alpha * ex2_full((x[e] - mo) * c));
            }
            const int64_t b = (int64_t)v * E - row.mis;
            if (aligned && b >= 0 && b + E <= row.V) *reinterpret_cast<uint4*>(g + b) = out;
            else
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (b + e >= 0 && b + e < row.V) g[b + e] = o[e];
        }
    }
    if (zero) return;
    __syncthreads();
    for (int i = threadIdx.x; i < a.k; i += kLT) {
        const int id = ls.id[i], v = (id + row.mis) / E;
        if (!ls.first[i] || v < v0 || v >= v1) continue;
        float q = 0.f;
        for (int j = i; j < a.k; ++j)
            if (ls.id[j] == id) q += ls.q[j];
        // (a row without a finite logit has no softmax: no gradient)
        g[id] = El<DT>::put(ls.coef.w == 0.f ? 0.f : f * (ls.coef.w * ex2_full((ls.x[i] - ls.coef.z) * c) - q));
    }
}

// Loss, statistics for a later backward pass and (GRAD) the gradient of one row
// per cluster.  The gradient's second read of the row comes from L2.
template <int DT, bool GRAD>
__global__ void __launch_bounds__(kLT) k_distill(DistillArgs a, int cs) {
    constexpr int E = El<DT>::E;
    extern __shared__ uint32_t d_bits[];  // a bit per element of the slice: listed
    __shared__ RunShared rs;
    __shared__ ListShared ls;
    const int64_t r = blockIdx.x / cs;
    const int rank = (int)(blockIdx.x % cs), tid = threadIdx.x;
    const Row<DT> row(a.logits, a.ld, r, a.vocab);
    const int v0 = (int)((int64_t)row.nv * rank / cs), v1 = (int)((int64_t)row.nv * (rank + 1) / cs);
    const float c = 1.4426950408889634f / a.temperature;
    const int words = ((v1 - v0) * E + 31) / 32;
    for (int i = tid; i < words; i += kLT) d_bits[i] = 0;
    list_load<DT>(a, row, r, ls);
    __syncthreads();
    for (int i = tid; i < a.k; i += kLT) {
        const int v = (ls.id[i] + row.mis) / E - v0;
        if (ls.first[i] && v >= 0 && v < v1 - v0) {
            const int b = v * E + (ls.id[i] + row.mis) % E;
            atomicOr(&d_bits[b >> 5], 1u << (b & 31));
        }
    }
    __syncthreads();
    Run run{-kInf, 0.f, 0.f};
    uint4 nxt[kLU];
#pragma unroll
    for (int u = 0; u < kLU; ++u) nxt[u] = row.load_if(v0 + tid + u * kLT, v1);
    for (int vb = v0; vb < v1; vb += kLT * kLU) {
        uint4 cur[kLU];
#pragma unroll
        for (int u = 0; u < kLU; ++u) {
            cur[u] = nxt[u];
            nxt[u] = row.load_if(vb + tid + (kLU + u) * kLT, v1);
        }
#pragma unroll
        for (int u = 0; u < kLU; ++u) {
            const int v = vb + tid + u * kLT - v0;
            uint32_t m = 0;
            if (v < v1 - v0) m = d_bits[(v * E) >> 5] >> ((v * E) & 31) & ((1u << E) - 1);
            float x[E];
            El<DT>::unpack(cur[u], x);
            float vm = El<DT>::vmax(cur[u]);
            if (m) {
                vm = -kInf;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (m >> e & 1) x[e] = -kInf;
                    vm = max_nan(vm, x[e]);
                }
            }
            if (vm > run.m) run_to(run, vm, c);
            const float ref = run.m == -kInf ? 0.f : run.m;
#pragma unroll
            for (int e = 0; e < E; ++e) run.s += ex2((x[e] - ref) * c);
        }
    }
    run = run_reduce(run, rs, c, cs);
    if (tid < 32) list_finish(a, run, c, ls);
    __syncthreads();
    if (rank == 0 && tid == 0) {
        a.loss[r] = ls.loss;
        if (a.stats) a.stats[r] = ls.coef;
    }
    if constexpr (GRAD) {
        const float f = (a.weight ? a.weight[r] : 1.f) * a.temperature;
        write_grad<DT>(a, row, r, v0, v1, c, f, ls);
    }
    if (cs > 1) cg::this_cluster().sync();  // the others may still read this CTA's state
}

// The gradient alone, from the forward pass's statistics: a CTA per chunk of a
// row.
template <int DT>
__global__ void __launch_bounds__(kLT) k_distill_backward(DistillArgs a, int chunks) {
    __shared__ ListShared ls;
    const int64_t r = blockIdx.x / chunks;
    const int ch = (int)(blockIdx.x % chunks);
    const Row<DT> row(a.logits, a.ld, r, a.vocab);
    const int v0 = (int)((int64_t)row.nv * ch / chunks), v1 = (int)((int64_t)row.nv * (ch + 1) / chunks);
    const float c = 1.4426950408889634f / a.temperature;
    list_load<DT>(a, row, r, ls);
    if (threadIdx.x == 0) ls.coef = a.stats[r];
    __syncthreads();
    if (threadIdx.x < 32) list_weights(a, ls);
    __syncthreads();
    write_grad<DT>(a, row, r, v0, v1, c, a.weight[r] * a.temperature, ls);
}

// ---------------------------------------------------------------- host side
int fail(int code, const char* msg) { return set_last_error(code, msg); }

int cuda_status(cudaError_t e) { return e == cudaSuccess ? EE_OK : fail(EE_ECUDA, cudaGetErrorString(e)); }

int sm_count(int* n) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
    return cuda_status(e);
}

size_t elem_bytes(int type) { return type == EE_FP32 ? 4 : 2; }

int check_logits(const void* p, int type, int64_t rows, int vocab, int64_t ld, float temperature) {
    if (type != EE_BF16 && type != EE_FP16 && type != EE_FP32) return fail(EE_EINVAL, "unknown element type");
    if (rows < 0 || vocab < 1 || vocab > EE_MAX_VOCAB) return fail(EE_EINVAL, "bad number of rows or vocabulary");
    if (ld < vocab) return fail(EE_EINVAL, "rows overlap: the row stride is below the vocabulary");
    if (!(temperature >= 1e-6f && temperature <= 1e6f)) return fail(EE_EINVAL, "temperature must lie in 1e-6 to 1e6");
    if (rows > 0x7fffffff / kMaxCluster) return fail(EE_EINVAL, "too many rows");
    if (rows && !p) return fail(EE_EINVAL, "NULL argument");
    if ((uintptr_t)p % elem_bytes(type)) return fail(EE_EINVAL, "logits are not aligned to their type");
    return EE_OK;
}

// CTAs per row: with fewer rows than two waves of one CTA per SM a row is shared
// by a cluster, as long as every CTA keeps a batch of vectors.
int cluster_size(int64_t rows, int vocab, int type, int n_sm) {
    const int64_t vecs = (int64_t)vocab * (int64_t)elem_bytes(type) / 16;
    int cs = 1;
    while (cs < kMaxCluster && rows * cs < 2 * n_sm && vecs / (2 * cs) >= kLT * kLU) cs *= 2;
    return cs;
}

template <class K, class A>
int launch_rows(K kern, int64_t rows, int cs, size_t smem, cudaStream_t s, const A& args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(rows * cs));
    cfg.blockDim = dim3(kLT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cs;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cs > 1 ? 1 : 0;
    if (smem > 40 * 1024) {  // (one limit for every size: calls of other threads may set it too)
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxBits);
        if (e != cudaSuccess) return cuda_status(e);
    }
    return cuda_status(cudaLaunchKernelEx(&cfg, kern, args, cs));
}

template <int DT>
int run_logprobs(const LogprobArgs& a, int64_t rows, int cs, cudaStream_t s) {
    return a.k ? launch_rows(k_logprobs<DT, true>, rows, cs, 0, s, a)
               : launch_rows(k_logprobs<DT, false>, rows, cs, 0, s, a);
}

template <int DT>
int run_distill(const DistillArgs& a, int64_t rows, int cs, size_t smem, cudaStream_t s) {
    return a.grad ? launch_rows(k_distill<DT, true>, rows, cs, smem, s, a)
                  : launch_rows(k_distill<DT, false>, rows, cs, smem, s, a);
}

int check_list(const int32_t* ids, int64_t ld_ids, const float* teacher, int64_t ld_teacher, int k, int64_t rows) {
    if (k < 1 || k > EE_MAX_TOP) return fail(EE_EINVAL, "the list must have 1 to EE_MAX_TOP entries");
    if (rows && (!ids || !teacher)) return fail(EE_EINVAL, "NULL argument");
    if (ld_ids < k || ld_teacher < k) return fail(EE_EINVAL, "list rows overlap");
    return EE_OK;
}

int check_grad(const void* grad, int type, int vocab, int64_t ld_grad) {
    if (ld_grad < vocab) return fail(EE_EINVAL, "gradient rows overlap");
    if ((uintptr_t)grad % elem_bytes(type)) return fail(EE_EINVAL, "the gradient is not aligned to its type");
    return EE_OK;
}

}  // namespace
}  // namespace ee

using namespace ee;

extern "C" {

int ee_token_logprobs(const void* logits, int type, int64_t rows, int vocab, int64_t ld, const int32_t* ids, int k,
                      float temperature, float* logprob, float* entropy, float* lse, float* top_logprob,
                      int32_t* top_id, void* stream) {
    int rc = check_logits(logits, type, rows, vocab, ld, temperature);
    if (rc != EE_OK) return rc;
    if (k < 0 || k > EE_MAX_TOP || k > vocab) return fail(EE_EINVAL, "k must lie in 0..min(EE_MAX_TOP, vocab)");
    if (!rows) return EE_OK;
    if ((logprob && !ids) || (k && (!top_logprob || !top_id))) return fail(EE_EINVAL, "NULL argument");
    int n_sm = 0;
    if ((rc = sm_count(&n_sm)) != EE_OK) return rc;
    const LogprobArgs a{logits, ld, vocab, k, ids, temperature, logprob, entropy, lse, top_logprob, top_id};
    const int cs = cluster_size(rows, vocab, type, n_sm);
    cudaStream_t s = (cudaStream_t)stream;
    if (type == EE_BF16) return run_logprobs<EE_BF16>(a, rows, cs, s);
    if (type == EE_FP16) return run_logprobs<EE_FP16>(a, rows, cs, s);
    return run_logprobs<EE_FP32>(a, rows, cs, s);
}

int ee_distill_topk(const void* logits, int type, int64_t rows, int vocab, int64_t ld, const int32_t* ids,
                    int64_t ld_ids, const float* teacher, int64_t ld_teacher, int k, float temperature, int tail,
                    float* loss, float* stats, const float* weight, void* grad, int64_t ld_grad, void* stream) {
    int rc = check_logits(logits, type, rows, vocab, ld, temperature);
    if (rc == EE_OK) rc = check_list(ids, ld_ids, teacher, ld_teacher, k, rows);
    if (rc == EE_OK && grad) rc = check_grad(grad, type, vocab, ld_grad);
    if (rc != EE_OK) return rc;
    if (!rows) return EE_OK;
    if (!loss) return fail(EE_EINVAL, "NULL argument");
    if ((uintptr_t)stats % 16) return fail(EE_EINVAL, "stats must be 16-byte aligned");
    int n_sm = 0;
    if ((rc = sm_count(&n_sm)) != EE_OK) return rc;
    int cs = cluster_size(rows, vocab, type, n_sm);
    // a bit per element of a slice, 128 KB at most
    while (vocab / cs > EE_MAX_VOCAB / kMaxCluster) cs *= 2;
    const int E = type == EE_FP32 ? 4 : 8;
    const size_t smem = ((size_t)(vocab / E + 2) / cs + 1) * E / 8 + 8;
    const DistillArgs a{logits, ld, vocab, k, tail ? 1 : 0, ids, ld_ids, teacher, ld_teacher, temperature, weight, loss,
                        reinterpret_cast<float4*>(stats), grad, ld_grad};
    cudaStream_t s = (cudaStream_t)stream;
    if (type == EE_BF16) return run_distill<EE_BF16>(a, rows, cs, smem, s);
    if (type == EE_FP16) return run_distill<EE_FP16>(a, rows, cs, smem, s);
    return run_distill<EE_FP32>(a, rows, cs, smem, s);
}

int ee_distill_topk_backward(const float* dloss, const void* logits, int type, int64_t rows, int vocab, int64_t ld,
                             const int32_t* ids, int64_t ld_ids, const float* teacher, int64_t ld_teacher, int k,
                             float temperature, int tail, const float* stats, void* grad, int64_t ld_grad,
                             void* stream) {
    int rc = check_logits(logits, type, rows, vocab, ld, temperature);
    if (rc == EE_OK) rc = check_list(ids, ld_ids, teacher, ld_teacher, k, rows);
    if (rc == EE_OK) rc = check_grad(grad, type, vocab, ld_grad);
    if (rc != EE_OK) return rc;
    if (!rows) return EE_OK;
    if (!dloss || !stats || !grad) return fail(EE_EINVAL, "NULL argument");
    if ((uintptr_t)stats % 16) return fail(EE_EINVAL, "stats must be 16-byte aligned");
    const DistillArgs a{logits, ld, vocab, k, tail ? 1 : 0, ids, ld_ids, teacher, ld_teacher, temperature, dloss, nullptr,
                        reinterpret_cast<float4*>(const_cast<float*>(stats)), grad, ld_grad};
    // four batches of vectors per CTA
    const int64_t vecs = (int64_t)vocab * (int64_t)elem_bytes(type) / 16;
    const int64_t chunks = std::max<int64_t>(1, vecs / (4 * kLT * kLU));
    if (rows * chunks > 0x7fffffff) return fail(EE_EINVAL, "too many rows");
    const unsigned grid = (unsigned)(rows * chunks);
    cudaStream_t s = (cudaStream_t)stream;
    if (type == EE_BF16) k_distill_backward<EE_BF16><<<grid, kLT, 0, s>>>(a, (int)chunks);
    else if (type == EE_FP16) k_distill_backward<EE_FP16><<<grid, kLT, 0, s>>>(a, (int)chunks);
    else k_distill_backward<EE_FP32><<<grid, kLT, 0, s>>>(a, (int)chunks);
    return cuda_status(cudaGetLastError());
}

}  // extern "C"
