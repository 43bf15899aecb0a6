// Log probabilities of given tokens, entropy and the most likely alternatives of rows of logits, and the gradient.
//
//   forward   m = max x, s = sum e^(x - m), t = sum (x - m) e^(x - m):  lse = m + log s, entropy = log s - t / s
//   backward  dx = dlogp (1[target] - p) - dentropy p (log p + entropy),  p = e^(x - lse)
//
// HBM bounds both: the logits are read once.  A thread carries the running (m, s, t) of its elements and rescales them when its maximum
// rises; the threads' triples are joined at the end by the same rule.  In bf16 the instructions per logit bound it next to HBM (one
// exponential, a conversion, half a maximum), so sums and products go two at a time (f32x2).  With few rows a row is split over the CTAs of a cluster, which
// join through distributed shared memory: no workspace, no second launch.
// The k most likely tokens: every warp keeps a sorted list of its own, one entry per lane, of keys (logit, then the lower index) as 64-bit
// integers.  A logit is looked at again only if it reaches the largest k-th entry of any list of the CTA, which after the first few hundred
// is rare in any order but an ascending one (n elements in random order change a list k ln(n / k) times); a list begins as the sorted maxima of
// the warp's 32 lanes.  Leaving out what no list needs changes no result.  Lists are joined pairwise by a bitonic merge.
// Rows need not be aligned: elements in front of the first 32-byte boundary and behind the last are read one by one.
#include "token.cuh"
#include <math.h>

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct LogpArgs {
    const void *x;
    const int32_t *targets;
    const float *lse_in, *ent_in, *dlogp, *dent;
    float *logp, *ent, *lse, *top_logp;
    int32_t *top_index;
    void *dx;
    int64_t rows, ld;
    int vocab, k, chunk;             // chunk: logits per CTA of a cluster (forward), per CTA (backward)
    FastDiv chunks;                  // CTAs per row (backward)
    int *status;
};

// A row's running sums: m the maximum, s = sum 2^d, t = sum d 2^d with d a logit's distance from the maximum in units of log 2.
// Up to kFar in magnitude d is one fused operation, x log2 e - M with M = m log2 e rounded: what the rounding takes, at most 1/16, s gains.  Beyond,
// it would grow past what 2^d holds (at 5e9 it is 220) and M overflow, so there d = (x - m) log2 e, exact where it is small.  m is kept as M / 2 below
// kFar and as the logit itself beyond: so the value tells which it is, and the order is the logits'.
struct Sums { float m, s, t; };
constexpr float kFar = 1048576.f;
__device__ __forceinline__ bool far(float m) { return fabsf(m) > kFar; }         // (-inf, of no logit yet, among them)
__device__ __forceinline__ float level(float x) { return far(x) ? x : x * (0.5f * kLog2e); }
__device__ __forceinline__ float distance(float a, float b) {                    // from level b to a
    if (far(a)) return far(b) ? (a - b) * kLog2e : fmaf(a, kLog2e, -2.f * b);
    return far(b) ? fmaf(-b, kLog2e, 2.f * a) : 2.f * (a - b);
}
// a's sums as they are for the maximum m >= a.m; an empty or all -inf one (m = -inf) is zero for any m
__device__ __forceinline__ void rescale(Sums &a, float m) {
    if (a.m == -INFINITY || a.m == m) { a.m = m; return; }
    const float d = distance(a.m, m), e = exp2_ftz(d);
    a.t = (a.t + d * a.s) * e;
    a.s *= e;
    if (e == 0.f) a.t = 0.f;         // d may be -inf (m +inf: the row's sums are NaN through its own element)
    a.m = m;
}
// the warp's sums, in every lane
__device__ __forceinline__ Sums join(Sums a) {
    float m = a.m;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    rescale(a, m);
#pragma unroll
    for (int o = 16; o; o >>= 1) { a.s += __shfl_xor_sync(0xffffffffu, a.s, o); a.t += __shfl_xor_sync(0xffffffffu, a.t, o); }
    return a;
}
// two float32 operations in one instruction
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 two(float lo, float hi) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ void parts(f32x2 v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float both(f32x2 v) { float lo, hi; parts(v, lo, hi); return lo + hi; }

// N logits, N a multiple of 4 or 1, top the largest of them
template <int N> __device__ __forceinline__ void add(Sums &a, const float (&x)[N], float top) {
    top = level(top);
    if (top > a.m) rescale(a, top);
    if (far(a.m)) {                  // one logit at a time; -inf adds nothing, also where there is nothing else yet
#pragma unroll
        for (int i = 0; i < N; i++) {
            if (x[i] == -INFINITY) continue;
            const float d = (x[i] - a.m) * kLog2e, e = exp2_ftz(d);
            a.s += e;
            a.t = fmaf(fmaxf(d, -200.f), e, a.t);                // (0 log 0 = 0)
        }
        return;
    }
    const float m = 2.f * a.m;
    float s, t;
    if constexpr (N == 1) {
        const float d = fmaf(x[0], kLog2e, -m);
        s = exp2_ftz(d);
        t = d * s;
    } else {
        const f32x2 l = two(kLog2e, kLog2e), mm = two(-m, -m);
        f32x2 ss[2] = {0ull, 0ull}, tt[2] = {0ull, 0ull};
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const f32x2 d = fma2(two(x[i], x[i + 1]), l, mm);
            float d0, d1;
            parts(d, d0, d1);
            const f32x2 e = two(exp2_ftz(d0), exp2_ftz(d1));
            ss[(i / 2) & 1] = add2(ss[(i / 2) & 1], e);
            tt[(i / 2) & 1] = fma2(d, e, tt[(i / 2) & 1]);
        }
        s = both(add2(ss[0], ss[1]));
        t = both(add2(tt[0], tt[1]));
    }
    if (t != t && s == s) {
        // 0 log 0 = 0: -inf among them (e is 0 far before -200; fmaxf would drop a NaN, but s has none)
        t = 0.f;
#pragma unroll
        for (int i = 0; i < N; i++) { const float d = fmaf(x[i], kLog2e, -m); t = fmaf(fmaxf(d, -200.f), exp2_ftz(d), t); }
    }
    a.s += s;
    a.t += t;
}
__device__ __forceinline__ float top_of(const Raw16<float> &r) {
    float t = __uint_as_float(r.w[0]);
#pragma unroll
    for (int i = 1; i < 16; i++) t = fmaxf(t, __uint_as_float(r.w[i]));
    return t;
}
__device__ __forceinline__ float top_of(const Raw16<bf16> &r) {
    __nv_bfloat162 t = *reinterpret_cast<const __nv_bfloat162 *>(&r.w[0]);
#pragma unroll
    for (int i = 1; i < 8; i++) t = __hmax2(t, *reinterpret_cast<const __nv_bfloat162 *>(&r.w[i]));
    return fmaxf(__low2float(t), __high2float(t));
}

// ---- most likely tokens
// bits in the logits' order, NaN above all, never 0
__device__ __forceinline__ uint32_t order_of(float x) {
    x += 0.f;                                        // -0 -> 0: equal logits are equal keys
    const uint32_t b = __float_as_uint(x);
    return x != x ? 0xffffffffu : (b & 0x80000000u ? ~b : b | 0x80000000u);
}
__device__ __forceinline__ unsigned long long key_of(float x, int index) { return (unsigned long long)order_of(x) << 32 | (uint32_t)~index; }
__device__ __forceinline__ float value_of(unsigned long long key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return b == 0xffffffffu ? NAN : __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
typedef unsigned long long Key;
__device__ __forceinline__ Key larger(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key smaller(Key a, Key b) { return a < b ? a : b; }
// descending lists of a warp, one key per lane: sort 32 keys; the 32 largest of two lists
__device__ __forceinline__ Key sorted(Key v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size <= 32; size *= 2)
#pragma unroll
        for (int stride = size / 2; stride; stride /= 2) {
            const Key o = __shfl_xor_sync(0xffffffffu, v, stride);
            v = ((lane & stride) == 0) == ((lane & size) == 0) ? larger(v, o) : smaller(v, o);
        }
    return v;
}
__device__ __forceinline__ Key merged(Key a, Key b) {
    const int lane = threadIdx.x & 31;
    Key v = larger(a, __shfl_sync(0xffffffffu, b, 31 - lane));           // one list up, the other down: a bitonic sequence
#pragma unroll
    for (int stride = 16; stride; stride /= 2) {
        const Key o = __shfl_xor_sync(0xffffffffu, v, stride);
        v = (lane & stride) == 0 ? larger(v, o) : smaller(v, o);
    }
    return v;
}
struct TopList {                     // lane i: the i-th largest key so far, 0 for none; least: keys up to this one are not needed
    Key mine, least;
    int k;
    __device__ __forceinline__ void raise() { least = larger(least, __shfl_sync(0xffffffffu, mine, k - 1)); }
    __device__ __forceinline__ void offer(Key key) {                     // one key per lane; the whole warp calls
        unsigned todo = __ballot_sync(0xffffffffu, key > least);
        const int lane = threadIdx.x & 31;
        if (__popc(todo) > 6) {      // a sort and a merge are 20 exchanges, an insertion about three
            mine = merged(mine, sorted(key > least ? key : 0ull));
            raise();
            return;
        }
        while (todo) {
            const int src = __ffs(todo) - 1;
            todo &= todo - 1;
            const Key c = __shfl_sync(0xffffffffu, key, src);
            if (c <= least) continue;
            const int at = __popc(__ballot_sync(0xffffffffu, mine > c));
            const Key up = __shfl_up_sync(0xffffffffu, mine, 1);
            mine = lane < at ? mine : (lane == at ? c : up);
            raise();
        }
    }
};

__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() { __syncwarp(); asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// the same shared-memory location in CTA `rank` of the cluster
template <class T> __device__ __forceinline__ T remote(const T *p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    T v;
    if constexpr (sizeof(T) == 8) { unsigned long long u; asm volatile("ld.shared::cluster.b64 %0, [%1];" : "=l"(u) : "r"(a) : "memory"); v = (T)u; }
    else { uint32_t u; asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(u) : "r"(a) : "memory"); v = __uint_as_float(u); }
    return v;
}

// x - base - logs, not above 0, which rounding could otherwise reach; beside a base of 1e38 the sum base + logs has no room for logs
__device__ __forceinline__ float log_prob(float x, double base, double logs, bool none) {
    const float v = (float)(((double)x - base) - logs);
    return none ? -INFINITY : (v > 0.f ? 0.f : v);
}

constexpr int kVec = 16;             // logits per step of a thread

// CLUSTER: the row's CTAs are a cluster along x; else one CTA per row
template <class T, bool TOP, bool CLUSTER>
__global__ void __launch_bounds__(512, 2) logprobs_fwd_kernel(const LogpArgs p) {
    __shared__ float sm_m[16], sm_s[16], sm_t[16];
    __shared__ Key lists[TOP ? 16 * 32 : 1], best;        // best: the largest k-th key of a warp's list
    pdl_enter();
    const uint32_t rank = CLUSTER ? cluster_rank() : 0, ctas = CLUSTER ? cluster_size() : 1;
    const size_t row = blockIdx.x / ctas;
    const T *x = (const T *)p.x + row * p.ld;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int begin = (int)rank * p.chunk, end = min(p.vocab, begin + p.chunk);
    const int len = end > begin ? end - begin : 0;
    // head: up to the first 32-byte boundary; body: vectors; tail
    const T *xb = x + begin;
    const int head = min(len, (int)((32 - ((uintptr_t)xb & 31)) & 31) / (int)sizeof(T));
    const int vecs = (len - head) / kVec, tail0 = head + vecs * kVec;
    Sums sum{-INFINITY, 0.f, 0.f};
    TopList list{0ull, 0ull, p.k};
    if (TOP) {
        if (threadIdx.x == 0) best = 0ull;
        __syncthreads();
    }

    // whole warps go round the loop: the list's shuffles need all lanes.  The next vector is on its way while one is worked on.
    Raw16<T> raw, next;
    float bar = -INFINITY;           // the bound as a logit, and the largest index that still reaches it
    unsigned bar_index = 0xffffffffu;
    bool started = false;
    if ((int)threadIdx.x < vecs) load_raw<kPieces>(xb + head + (int)threadIdx.x * kVec, 0, kVec, true, next);
    for (int v0 = warp * 32; v0 < vecs; v0 += blockDim.x) {
        const int v = v0 + lane;
        const bool ok = v < vecs;
        raw = next;
        if (v + (int)blockDim.x < vecs) load_raw<kPieces>(xb + head + (v + (int)blockDim.x) * kVec, 0, kVec, true, next);
        float f[kVec];
        const float top = top_of(raw);
        unpack(raw, f);
        if (ok) add(sum, f, top);
        if constexpr (TOP) {
            const int i0 = begin + head + v * kVec;
            const bool nan = sum.s != sum.s;                             // (one of this thread's logits so far)
            if (__any_sync(0xffffffffu, ok && (nan || top > bar || (top == bar && (unsigned)i0 <= bar_index)))) {
                list.least = larger(list.least, __shfl_sync(0xffffffffu, *(volatile Key *)&best, 0));
                uint32_t taken = 0;                                      // of this lane's vector: the logit that is in the list already
                if (!started) {
                    started = true;
                    if (ok && !nan) {
#pragma unroll
                        for (int i = kVec - 1; i >= 0; i--) taken = f[i] == top ? 1u << i : taken;
                    }
                    list.mine = sorted(taken ? key_of(top, i0 + __ffs(taken) - 1) : 0ull);
                    list.raise();
                }
                bar = list.least ? value_of(list.least) : -INFINITY;
                uint32_t todo = 0;
                if (ok && (nan || top >= bar)) {
#pragma unroll
                    for (int i = 0; i < kVec; i++) todo |= !(f[i] < bar) ? 1u << i : 0u;
                }
                todo &= ~taken;
                while (__any_sync(0xffffffffu, todo != 0)) {
                    const int i = i0 + (todo ? __ffs(todo) - 1 : 0);
                    list.offer(todo ? key_of(to_f(x[i]), i) : 0ull);
                    todo &= todo - 1;
                }
                if (lane == p.k - 1 && list.mine > 0ull) atomicMax(&best, list.mine);
                bar = list.least ? value_of(list.least) : -INFINITY;
                bar_index = ~(unsigned)list.least;
            }
        }
    }
    for (int e0 = warp * 32; e0 < head + len - tail0; e0 += blockDim.x) {
        const int e = e0 + lane;
        const bool ok = e < head + len - tail0;
        const int i = e < head ? e : tail0 + e - head;
        const float f[1] = {ok ? to_f(xb[i]) : -INFINITY};
        if (ok) add(sum, f, f[0]);
        if constexpr (TOP) list.offer(ok ? key_of(f[0], begin + i) : 0ull);
    }
    sum = join(sum);
    if (lane == 0) { sm_m[warp] = sum.m; sm_s[warp] = sum.s; sm_t[warp] = sum.t; }
    if constexpr (TOP) lists[warp * 32 + lane] = list.mine;
    __syncthreads();
    if constexpr (TOP)
        for (int off = warps / 2; off; off /= 2) {
            if (warp < off) lists[warp * 32 + lane] = list.mine = merged(list.mine, lists[(warp + off) * 32 + lane]);
            __syncthreads();
        }
    if (warp == 0) {
        // lane w: the sums of warp w
        sum = lane < warps ? Sums{sm_m[lane], sm_s[lane], sm_t[lane]} : Sums{-INFINITY, 0.f, 0.f};
        sum = join(sum);
        if (CLUSTER && lane == 0) { sm_m[0] = sum.m; sm_s[0] = sum.s; sm_t[0] = sum.t; }
    }
    if (CLUSTER) {
        cluster_sync();
        if (rank == 0 && warp == 0) {
            sum = lane < (int)ctas ? Sums{remote(&sm_m[0], lane), remote(&sm_s[0], lane), remote(&sm_t[0], lane)} : Sums{-INFINITY, 0.f, 0.f};
            sum = join(sum);
            if constexpr (TOP) {
                Key others[8];
#pragma unroll
                for (uint32_t c = 1; c < 8; c++) others[c] = c < ctas ? remote(&lists[lane], c) : 0ull;
#pragma unroll
                for (uint32_t c = 1; c < 8; c++)
                    if (c < ctas) list.mine = merged(list.mine, others[c]);
            }
        }
        cluster_sync();              // nobody leaves while rank 0 reads
        if (rank != 0) return;
    }
    if (warp != 0) return;
    // once per row, in double.  The level stands for M / log2 e, with the float kLog2e that M was formed with, not quite the largest logit: s makes up for that
    const bool none = sum.m == -INFINITY && sum.s == 0.f;
    const double logs = (double)logf(sum.s), base = far(sum.m) ? (double)sum.m : 2.0 * sum.m / (double)kLog2e;
    if (lane == 0) {
        if (p.lse) p.lse[row] = none ? -INFINITY : (float)(base + logs);
        if (p.ent) { const float h = (float)(logs - (double)kLn2 * ((double)sum.t / sum.s)); p.ent[row] = none || h < 0.f ? 0.f : h; }
        if (p.logp) {
            const int tgt = p.targets[row];
            float v = 0.f;
            if (tgt >= 0 && tgt < p.vocab) v = log_prob(to_f(x[tgt]), base, logs, none);
            else if (tgt != -1) { v = NAN; atomicExch(p.status, (int)REVNET_E_INVALID_ARG); }
            p.logp[row] = v;
        }
    }
    if constexpr (TOP)
        if (lane < p.k) {
            p.top_index[row * p.k + lane] = (int)~(uint32_t)list.mine;
            p.top_logp[row * p.k + lane] = log_prob(value_of(list.mine), base, logs, none);
        }
}

// one logit's gradient; off: what lse lacks, in units of log 2.  (Roundings spelled out: every copy of this has the same bits)
__device__ __forceinline__ float grad(float x, float lse, float off, float g, float ge, float ent2) {
    const float l = __fmaf_rn(x - lse, kLog2e, -off), q = exp2_ftz(l);
    // ge log p in natural units: ge (l + ent2) ln 2, the factor folded into ge by the caller
    return q == 0.f ? 0.f : __fmul_rn(-q, __fmaf_rn(ge, __fadd_rn(l, ent2), g));
}
// Beyond this float32 holds lse to no better than 2^-12, and p from it likewise; far beyond it has no room for log s at all (all logits -1e9).
constexpr float kCoarse = 4096.f;
// Such a row, by one warp alone (so that it may be overwritten, and without shared memory, of which the kernel asks for none): its maximum and sum once
// more.  They are taken if lse is theirs to float32's resolution; else (lse of more logits than these: parts of a vocabulary) lse is, as it is.
// 4096 x 50000 bf16: 143 us without such rows, 287 with every tenth one.
template <class T> __device__ __noinline__ void coarse_row(const T *x, T *dx, int vocab, int tgt, float lse, float g, float ge, float ent2) {
    const int lane = threadIdx.x, head = min(vocab, (int)((32 - ((uintptr_t)x & 31)) & 31) / (int)sizeof(T)), vecs = (vocab - head) / kVec, tail0 = head + vecs * kVec;
    const bool same = (((uintptr_t)x ^ (uintptr_t)dx) & 31) == 0;
    // every logit, 16 at a time; f(logits, how many, index of the first) -> whether they are gradients now
    auto all = [&](auto f) {
        for (int v = lane; v < vecs; v += 32) {
            float t[kVec];
            const int i = head + v * kVec;
            load16<kPieces>(x + i, 0, kVec, true, t);
            if (!f(t, kVec, i)) continue;
            if (same) store16<kPieces>(dx + i, 0, kVec, true, t);
            else {
#pragma unroll
                for (int j = 0; j < kVec; j++) put(dx[i + j], t[j]);
            }
        }
        for (int e = lane; e < vocab - vecs * kVec; e += 32) {
            const int i = e < head ? e : tail0 + e - head;
            float t[kVec] = {to_f(x[i])};
            if (f(t, 1, i)) put(dx[i], t[0]);
        }
    };
    float m = -INFINITY, s = 0.f;
    all([&](float (&t)[kVec], int n, int) {
#pragma unroll
        for (int j = 0; j < kVec; j++) if (j < n) m = fmaxf(m, t[j]);
        return false;
    });
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    all([&](float (&t)[kVec], int n, int) {
#pragma unroll
        for (int j = 0; j < kVec; j++) if (j < n) s += exp2_ftz((t[j] - m) * kLog2e);
        return false;
    });
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const bool own = fabsf((m - lse) + logf(s)) <= fabsf(lse) * 0x1p-23f;
    const float base = own ? m : lse, off = own ? log2f(s) : 0.f;
    all([&](float (&t)[kVec], int n, int i) {
#pragma unroll
        for (int j = 0; j < kVec; j++) if (j < n) { t[j] = grad(t[j], base, off, g, ge, ent2); if (i + j == tgt) t[j] += g; }
        return true;
    });
}
template <class T>
__global__ void __launch_bounds__(256, 8) logprobs_bwd_kernel(const LogpArgs p) {
    pdl_enter();
    uint32_t r, c;
    p.chunks.divmod(blockIdx.x, r, c);
    const size_t row = r;
    const T *x = (const T *)p.x + row * p.ld + (size_t)c * p.chunk;
    T *dx = (T *)p.dx + row * p.ld + (size_t)c * p.chunk;
    const int begin = (int)c * p.chunk, len = min(p.chunk, p.vocab - begin);
    const float lse = p.lse_in[row];
    int tgt = -1;
    float g = 0.f, ge = 0.f, ent2 = 0.f;
    if (p.dlogp) {
        tgt = p.targets[row];
        if (tgt != -1) g = p.dlogp[row];
        if (tgt < -1 || tgt >= p.vocab) {
            g = NAN;
            if (threadIdx.x == 0) atomicExch(p.status, (int)REVNET_E_INVALID_ARG);
        }
    }
    if (p.dent) { ge = p.dent[row] * kLn2; ent2 = p.ent_in[row] * kLog2e; }
    if (fabsf(lse) > kCoarse && fabsf(lse) < INFINITY && !(g == 0.f && ge == 0.f)) {
        if (c == 0 && threadIdx.x < 32) coarse_row(x, dx, p.vocab, tgt, lse, g, ge, ent2);
        return;
    }
    const bool none = lse == -INFINITY;
    // vectors where both rows have their 32-byte boundaries at the same elements
    const bool same = (((uintptr_t)x ^ (uintptr_t)dx) & 31) == 0;
    const int head = same ? min(len, (int)((32 - ((uintptr_t)x & 31)) & 31) / (int)sizeof(T)) : len;
    const int vecs = (len - head) / kVec, tail0 = head + vecs * kVec;
    for (int v = threadIdx.x; v < vecs; v += blockDim.x) {
        float f[kVec];
        load16<kPieces>(x + head + v * kVec, 0, kVec, true, f);
        const int at = tgt - (begin + head + v * kVec);
#pragma unroll
        for (int i = 0; i < kVec; i++) {
            const float d = none ? 0.f : grad(f[i], lse, 0.f, g, ge, ent2);
            f[i] = at == i && !none ? d + g : d;
        }
        store16<kPieces>(dx + head + v * kVec, 0, kVec, true, f);
    }
    for (int e = threadIdx.x; e < head + len - tail0; e += blockDim.x) {
        const int i = e < head ? e : tail0 + e - head;
        float d = none ? 0.f : grad(to_f(x[i]), lse, 0.f, g, ge, ent2);
        if (begin + i == tgt && !none) d += g;
        put(dx[i], d);
    }
}

template <class T> void fwd_t(Exec &ex, const LogpArgs &p, int cluster, unsigned threads) {
    const unsigned rows = (unsigned)p.rows;
    if (cluster == 1) {
        if (p.k) launch(ex, logprobs_fwd_kernel<T, true, false>, rows, threads, 0, p);
        else launch(ex, logprobs_fwd_kernel<T, false, false>, rows, threads, 0, p);
    } else {
        if (p.k) launch_cluster(ex, logprobs_fwd_kernel<T, true, true>, rows * cluster, threads, 0, cluster, p);
        else launch_cluster(ex, logprobs_fwd_kernel<T, false, true>, rows * cluster, threads, 0, cluster, p);
    }
}

}  // namespace

void logprobs_fwd(Exec &ex, const revnet_logprob_desc &d, const void *logits, const int32_t *targets, float *logp, float *entropy, float *lse,
                  float *top_logp, int32_t *top_index) {
    if (d.rows == 0) return;
    LogpArgs p{};
    p.x = logits; p.targets = targets; p.logp = logp; p.ent = entropy; p.lse = lse; p.top_logp = top_logp; p.top_index = top_index;
    p.rows = d.rows; p.ld = d.ld; p.vocab = d.vocab; p.k = d.k; p.status = ex.ctx->dev_status;
    // 1024 threads per SM (64 registers each): small CTAs where there are rows for all of them, since every CTA has its own start and end (4096 rows
    // of 50000: 97 us with 512 threads, 79 with 128); few rows take large CTAs, and more than one where their parts stay longer than one step
    const int64_t sms = ex.ctx->sm_count;
    const unsigned most = d.rows <= 2 * sms ? 512 : (d.rows <= 6 * sms ? 256 : 128);
    unsigned threads = 32;
    while (threads < most && (int)threads * kVec < d.vocab) threads *= 2;
    int cluster = 1;
    while (cluster < 8 && d.rows * cluster * 2 * threads <= sms * 1280 && d.vocab / (cluster * 2) >= (int)threads * kVec) cluster *= 2;
    p.chunk = (d.vocab + cluster - 1) / cluster;
    const double bytes = (double)d.rows * d.vocab * (d.dtype == REVNET_F32 ? 4 : 2);
    if (d.dtype == REVNET_F32) fwd_t<float>(ex, p, cluster, threads);
    else fwd_t<bf16>(ex, p, cluster, threads);
    ex.check("logprobs_fwd", bytes);
}

void logprobs_bwd(Exec &ex, const revnet_logprob_desc &d, const void *logits, const int32_t *targets, const float *lse, const float *entropy,
                  const float *dlogp, const float *dentropy, void *dlogits) {
    if (d.rows == 0) return;
    LogpArgs p{};
    p.x = logits; p.targets = targets; p.lse_in = lse; p.ent_in = entropy; p.dlogp = dlogp; p.dent = dentropy; p.dx = dlogits;
    p.rows = d.rows; p.ld = d.ld; p.vocab = d.vocab; p.status = ex.ctx->dev_status;
    unsigned threads = 32;
    while (threads < 256 && (int)threads * kVec < d.vocab) threads *= 2;
    // about four vectors per thread (two: 4 % slower, one: 25 %), rows cut into equal parts (of whole vectors, so that they stay aligned)
    const int per = (int)threads * kVec * 4;
    int64_t chunks = (d.vocab + per - 1) / per;
    while (chunks > 1 && d.rows * chunks >= (int64_t(1) << 31)) chunks = (chunks + 1) / 2;
    p.chunk = (int)(((d.vocab + chunks - 1) / chunks + kVec - 1) / kVec * kVec);
    chunks = (d.vocab + p.chunk - 1) / p.chunk;
    p.chunks = fast_div((uint32_t)chunks);
    const double bytes = (double)d.rows * d.vocab * (d.dtype == REVNET_F32 ? 8 : 4);
    const unsigned grid = (unsigned)(d.rows * chunks);
    if (d.dtype == REVNET_F32) launch_stream(ex, bytes, 0, logprobs_bwd_kernel<float>, grid, threads, 0, p);
    else launch_stream(ex, bytes, 0, logprobs_bwd_kernel<bf16>, grid, threads, 0, p);
    ex.check("logprobs_bwd", bytes);
}
