// Root-mean-square norm behind the residual's addition, with an output in 8 bits, and its backward pass.
//
//   forward   h = x + r,  rstd = 1 / sqrt(mean(h^2) + eps),  xh = h rstd,  n = xh gamma,  checkpoint of xh (or n)
//   backward  dx = dh + rstd (gamma dn - xh mean(gamma dn xh)),  dgamma = sum over rows of dn xh
//
// HBM bounds both.  A row stays in the registers of the threads that own it, so every tensor is read and written once: the sum of squares
// (backward: that and the sum of gamma dn h) is one reduction over the row, and everything else is local to a thread's 16 channels
// (token.cuh).  A row belongs to `tpr` threads, a power of two: up to 32 of them reduce by shuffles, more through shared memory.  Short
// rows share a CTA.  CTAs are resident and walk over the rows; while one row is reduced and written, the next ones are on their way into
// shared memory (up to 8192 channels of rows in 16-byte pieces; others are loaded when they are needed).
#include "token.cuh"
#include <algorithm>
#include <type_traits>

namespace {

struct NormArgs {
    const void *x, *r, *dn, *dh;
    const float *gamma, *rstd_in;
    void *h, *n, *dx, *dr;
    float *rstd, *partial, *dgamma;
    Checkpoint ck;
    int64_t rows, ld_s, ld_b;
    int channels;
    int tpr_log;                     // threads per row
    int ck_scaled;
    bool wide;                       // 32-byte accesses (token.cuh)
    float eps, inv_c;
};

// gamma of a thread's channels (ones where there is none, zeros behind the row's end)
template <bool SPREAD> __device__ __forceinline__ void load_gamma(const NormArgs &p, int ch, float (&g)[16]) {
    if (p.gamma) { load16<SPREAD>(p.gamma + ch, p.channels - ch, p.wide, g); return; }
#pragma unroll
    for (int i = 0; i < 16; i++) g[i] = ch + step_of<SPREAD>(i) < p.channels ? 1.f : 0.f;
}

// sums over the tpr threads of a row, given to all of them; red: N floats per warp.  Every thread of the CTA calls it.
template <int N> __device__ __forceinline__ void row_sum(float (&v)[N], int tpr_log, float (*red)[N]) {
    const int tpr = 1 << tpr_log;
#pragma unroll
    for (int o = 16; o; o >>= 1)
        if (o < tpr) {
#pragma unroll
            for (int i = 0; i < N; i++) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        }
    if (tpr <= 32) return;
    const int warp = threadIdx.x >> 5, warps = tpr >> 5, first = warp & ~(warps - 1);
    __syncthreads();                 // the last call's sums have been read
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < N; i++) red[warp][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = red[first][i];
#pragma unroll
    for (int w = 1; w < 16; w++)
        if (w < warps) {
#pragma unroll
            for (int i = 0; i < N; i++) v[i] += red[first + w][i];
        }
}

// How many rows of a CTA lie in shared memory (the one that is worked on among them), and how many CTAs an SM holds, by the chunks of 16 bytes
// that a row takes per thread.  More of either only makes the reads and writes that HBM sees at a time more scattered: forward, bf16, 16384 x 4096,
// 2 CTAs x 2 rows 98 us, 3 x 2 101, 2 x 3 112, 4 x 3 105, 3 x 4 117; float32 stream of 200704 x 512, 3 x 2 223, 2 x 2 233, 4 x 2 263;
// its backward pass, 2 x 2 172, 2 x 3 190.  A CTA of 512 threads is alone on its SM: 8192 x 8192, 3 rows 94, 2 103.
__host__ __device__ constexpr int fwd_stages(int threads) { return threads == 512 ? 3 : 2; }
__host__ __device__ constexpr int fwd_per_sm(int threads, int chunks) { return threads == 512 ? 1 : (chunks <= 4 ? 2 : 3); }
__host__ __device__ constexpr int bwd_stages(int chunks) { return chunks <= 5 ? 3 : 2; }
__host__ __device__ constexpr int bwd_per_sm(int threads) { return threads == 512 ? 1 : 2; }

// SLOTS times 16 channels per thread
template <bool SPREAD, class TS, class TB, int CODE, int SLOTS, int THREADS>
__global__ void __launch_bounds__(THREADS, fwd_per_sm(THREADS, kChunks<TS> + kChunks<TB>)) rmsnorm_fwd_kernel(const __grid_constant__ NormArgs p) {
    extern __shared__ uint4 stages[];
    __shared__ float red[THREADS / 32][1];
    constexpr int kX = kChunks<TS>, kPer = kX + kChunks<TB>, kStages = fwd_stages(THREADS);      // chunks: of x; of a row, r behind x
    constexpr bool kAsync = !SPREAD && SLOTS == 1;       // (longer rows have no room for stages)
    const int tpr = 1 << p.tpr_log, t = threadIdx.x & (tpr - 1), at_once = THREADS >> p.tpr_log;
    const int64_t step = (int64_t)gridDim.x * at_once;
    int64_t row = (int64_t)blockIdx.x * at_once + (threadIdx.x >> p.tpr_log);
    const int ch0 = first_channel<SPREAD>(t);
    float gamma[16];
    pdl_enter();
    load_gamma<SPREAD>(p, ch0, gamma);
    // the lanes of this warp that share the row, their first channel, and where their chunks lie in a part of a stage (THREADS threads' worth)
    const int lanes = tpr < 32 ? tpr : 32, lane = t & (lanes - 1), chw = (t - lane) * kGroup, mine = (int)threadIdx.x - lane;
    auto fetch = [&](int stage, int64_t at) {
        uint4 *to = stages + stage * kPer * THREADS;
        const int left = at < p.rows ? p.channels - chw : 0;
        fetch_row(to + mine * kX, lanes, lane, (const TS *)p.x + (at * p.ld_s + chw), left);
        if (p.r) fetch_row(to + kX * THREADS + mine * kChunks<TB>, lanes, lane, (const TB *)p.r + (at * p.ld_b + chw), left);
    };
    if constexpr (kAsync) {
#pragma unroll
        for (int i = 0; i < kStages - 1; i++) { fetch(i, row + i * step); copies_commit(); }
    }
    int stage = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * at_once; row0 < p.rows; row0 += step, row += step) {
        const bool row_ok = row < p.rows;
        const int64_t at_s = row * p.ld_s, at_b = row * p.ld_b;
        float h[SLOTS][16], sum[1] = {0.f};
        if constexpr (kAsync) { copies_wait<kStages - 2>(); __syncwarp(); }
        const uint4 *from = stages + stage * kPer * THREADS;
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = first_channel<SPREAD>(s * tpr + t), left = row_ok ? p.channels - ch : 0;
            Raw16<TS> x;
            Raw16<TB> r;
            if constexpr (kAsync) {
                fetched(from + mine * kX, lane, x);
                if (p.r) fetched(from + kX * THREADS + mine * kChunks<TB>, lane, r);
            } else {
                load_raw<SPREAD>((const TS *)p.x + (at_s + ch), left, p.wide, x);
                if (p.r) load_raw<SPREAD>((const TB *)p.r + (at_b + ch), left, p.wide, r);
            }
            unpack(x, h[s]);
            if (p.r) {
                float add[16];
                unpack(r, add);
#pragma unroll
                for (int i = 0; i < 16; i++) h[s][i] += add[i];
                pack(h[s], x);                       // the norm is of h as it is stored, so that the backward pass sees the same h
                unpack(x, h[s]);
                if (p.h) store_raw<SPREAD>((TS *)p.h + (at_s + ch), left, p.wide, x);
            }
#pragma unroll
            for (int i = 0; i < 16; i++) sum[0] = fmaf(h[s][i], h[s][i], sum[0]);
        }
        if constexpr (kAsync) {
            // into the stage that the row before this one has left
            fetch(stage == 0 ? kStages - 1 : stage - 1, row + (kStages - 1) * step);
            copies_commit();
            if (++stage == kStages) stage = 0;
        }
        row_sum(sum, p.tpr_log, red);
        const float rstd = rsqrtf(sum[0] * p.inv_c + p.eps);
        if (p.rstd && row_ok && t == 0) p.rstd[row] = rstd;
        if (!p.n && !p.ck.codes) continue;
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = first_channel<SPREAD>(s * tpr + t), left = row_ok ? p.channels - ch : 0;
            float n[16];
            if (s > 0) load_gamma<SPREAD>(p, ch, gamma);
#pragma unroll
            for (int i = 0; i < 16; i++) { h[s][i] *= rstd; n[i] = h[s][i] * gamma[i]; }
            if (p.n) store16<SPREAD>((TB *)p.n + (at_b + ch), left, p.wide, n);
            if (p.ck.codes) {
                if (p.ck_scaled) keep16<SPREAD, CODE>(p.ck, row, ch, row_ok, n);
                else keep16<SPREAD, CODE>(p.ck, row, ch, row_ok, h[s]);
            }
        }
        if (SLOTS > 1) load_gamma<SPREAD>(p, ch0, gamma);
    }
    if constexpr (kAsync) copies_wait<0>();
}

// FROM_H: from h; else from a checkpoint of xh with CODE.  A thread keeps its channels for all rows it works on, and their dgamma in registers.
template <bool SPREAD, class TS, class TB, bool FROM_H, int CODE, int SLOTS, int THREADS>
__global__ void __launch_bounds__(THREADS, bwd_per_sm(THREADS)) rmsnorm_bwd_kernel(const __grid_constant__ NormArgs p) {
    extern __shared__ uint4 stages[];
    constexpr int kSums = FROM_H ? 2 : 1;                // gamma dn x, and the squares
    __shared__ float red[THREADS / 32][kSums];
    constexpr int kS = kChunks<TS>, kB = kChunks<TB>, kX = FROM_H ? kS : 1, kPer = kS + kB + kX, kStages = bwd_stages(kPer);      // chunks of a row: dh, dn, h or codes
    constexpr bool kAsync = !SPREAD && SLOTS == 1;       // (longer rows have no room for stages)
    const int tpr = 1 << p.tpr_log, t = threadIdx.x & (tpr - 1), at_once = THREADS >> p.tpr_log;
    const int64_t step = (int64_t)gridDim.x * at_once;
    int64_t row = (int64_t)blockIdx.x * at_once + (threadIdx.x >> p.tpr_log);
    const int ch0 = first_channel<SPREAD>(t);
    float dg[SLOTS][16], gamma[16];
#pragma unroll
    for (int s = 0; s < SLOTS; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) dg[s][i] = 0.f;
    pdl_enter();
    load_gamma<SPREAD>(p, ch0, gamma);
    // the lanes of this warp that share the row, their first channel, and where their chunks lie in a part of a stage (THREADS threads' worth)
    const int lanes = tpr < 32 ? tpr : 32, lane = t & (lanes - 1), chw = (t - lane) * kGroup, mine = (int)threadIdx.x - lane;
    auto fetch = [&](int stage, int64_t at) {
        uint4 *to = stages + stage * kPer * THREADS;
        const int left = at < p.rows ? p.channels - chw : 0;
        if (p.dh) fetch_row(to + mine * kS, lanes, lane, (const TS *)p.dh + (at * p.ld_s + chw), left);
        fetch_row(to + kS * THREADS + mine * kB, lanes, lane, (const TB *)p.dn + (at * p.ld_b + chw), left);
        if constexpr (FROM_H) fetch_row(to + (kS + kB) * THREADS + mine * kS, lanes, lane, (const TS *)p.x + (at * p.ld_s + chw), left);
        else copy16(to + (kS + kB) * THREADS + threadIdx.x, p.ck.codes + (at * p.ck.pitch + ch0), lane * kGroup < left);
    };
    if constexpr (kAsync) {
#pragma unroll
        for (int i = 0; i < kStages - 1; i++) { fetch(i, row + i * step); copies_commit(); }
    }
    int stage = 0;
    // what a row has besides its channels is loaded a row ahead too
    float rstd_next = 0.f;
    uint32_t byte_next = 0;
    auto ahead = [&](int64_t at) {
        if (FROM_H) return;
        rstd_next = at < p.rows ? p.rstd_in[at] : 0.f;
        if (kAsync) byte_next = at < p.rows && ch0 < p.channels ? byte_of(p.ck.scales + scale_index(p.ck, at, ch0)) : 0u;
    };
    ahead(row);
    for (int64_t row0 = (int64_t)blockIdx.x * at_once; row0 < p.rows; row0 += step, row += step) {
        const bool row_ok = row < p.rows;
        const int64_t at_s = row * p.ld_s, at_b = row * p.ld_b;
        float x[SLOTS][16], dn[SLOTS][16], rstd = rstd_next, sum[kSums];
#pragma unroll
        for (int i = 0; i < kSums; i++) sum[i] = 0.f;
        if constexpr (kAsync) { copies_wait<kStages - 2>(); __syncwarp(); }
        const uint4 *from = stages + stage * kPer * THREADS;
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = first_channel<SPREAD>(s * tpr + t), left = row_ok ? p.channels - ch : 0;
            if constexpr (kAsync) {
                Raw16<TB> rn;
                fetched(from + kS * THREADS + mine * kB, lane, rn);
                unpack(rn, dn[s]);
                if constexpr (FROM_H) {
                    Raw16<TS> rx;
                    fetched(from + (kS + kB) * THREADS + mine * kS, lane, rx);
                    unpack(rx, x[s]);
                } else decode16<CODE>(from[(kS + kB) * THREADS + threadIdx.x], byte_next, x[s]);
            } else {
                load16<SPREAD>((const TB *)p.dn + (at_b + ch), left, p.wide, dn[s]);
                if constexpr (FROM_H) load16<SPREAD>((const TS *)p.x + (at_s + ch), left, p.wide, x[s]);
                else read16<SPREAD, CODE>(p.ck, row, ch, left, x[s]);
                if (s > 0) load_gamma<SPREAD>(p, ch, gamma);
            }
#pragma unroll
            for (int i = 0; i < 16; i++) {
                if constexpr (FROM_H) {
                    sum[0] = fmaf(dn[s][i] * gamma[i], x[s][i], sum[0]);
                    sum[1] = fmaf(x[s][i], x[s][i], sum[1]);
                } else {
                    dg[s][i] = fmaf(dn[s][i], x[s][i], dg[s][i]);         // (zeros where there is no row)
                    dn[s][i] *= gamma[i];
                    sum[0] = fmaf(dn[s][i], x[s][i], sum[0]);
                }
            }
        }
        ahead(row + step);
        if constexpr (kAsync) {
            // into the stage that the row before this one has left
            fetch(stage == 0 ? kStages - 1 : stage - 1, row + (kStages - 1) * step);
            copies_commit();
            if (++stage == kStages) stage = 0;
        }
        row_sum(sum, p.tpr_log, red);
        if constexpr (FROM_H) rstd = rsqrtf(sum[1] * p.inv_c + p.eps);
        // dx = dh + rstd gamma dn - xh (rstd mean(gamma dn xh)); from h: xh = h rstd, and the mean is rstd times that of gamma dn h
        const float back = -sum[0] * p.inv_c * rstd * (FROM_H ? rstd * rstd : 1.f);
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = first_channel<SPREAD>(s * tpr + t), left = row_ok ? p.channels - ch : 0;
            float d[16];
            if (p.dh) {
                Raw16<TS> rh;
                if constexpr (kAsync) fetched(from + mine * kS, lane, rh);
                else load_raw<SPREAD>((const TS *)p.dh + (at_s + ch), left, p.wide, rh);
                unpack(rh, d);
            } else {
#pragma unroll
                for (int i = 0; i < 16; i++) d[i] = 0.f;
            }
            if (SLOTS > 1 && FROM_H) load_gamma<SPREAD>(p, ch, gamma);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                float w = dn[s][i] * rstd;
                if constexpr (FROM_H) {
                    dg[s][i] = fmaf(w, x[s][i], dg[s][i]);
                    w *= gamma[i];
                }
                d[i] = fmaf(x[s][i], back, d[i] + w);
            }
            store16<SPREAD>((TS *)p.dx + (at_s + ch), left, p.wide, d);
            if (p.dr) store16<SPREAD>((TB *)p.dr + (at_b + ch), left, p.wide, d);
        }
        if (SLOTS > 1) load_gamma<SPREAD>(p, ch0, gamma);
    }
    if constexpr (kAsync) copies_wait<0>();
    if (!p.dgamma) return;
    float *out = gridDim.x == 1 ? p.dgamma : p.partial + (size_t)blockIdx.x * p.channels;
    if (THREADS == 256 && at_once > 1) {
        // the CTA's rows first, in a fixed order, through the stages' memory
        float *sums = reinterpret_cast<float *>(stages);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; i++) sums[(threadIdx.x - t) * 16 + ch0 + step_of<SPREAD>(i)] = dg[0][i];
        __syncthreads();
        for (int c = threadIdx.x; c < p.channels; c += THREADS) {
            float v = 0.f;
            for (int k = 0; k < at_once; k++) v += sums[(k << p.tpr_log) * 16 + c];
            out[c] = v;
        }
        return;
    }
#pragma unroll
    for (int s = 0; s < SLOTS; s++) {
        const int ch = first_channel<SPREAD>(s * tpr + t);
#pragma unroll
        for (int i = 0; i < 16; i++) if (ch + step_of<SPREAD>(i) < p.channels) out[ch + step_of<SPREAD>(i)] = dg[s][i];
    }
}

// dgamma = sum of the CTAs' sums: 32 channels per CTA, 32 threads add every 32nd record of a channel, in a fixed order
__global__ void __launch_bounds__(1024) rmsnorm_dgamma_kernel(const float *partial, int parts, int channels, float *dgamma) {
    pdl_enter();
    __shared__ float sm[32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), k0 = threadIdx.x >> 5;
    float v = 0.f;
    if (c < channels)
        for (int k = k0; k < parts; k += 32) v += partial[(size_t)k * channels + c];
    sm[k0][threadIdx.x & 31] = v;
    __syncthreads();
    v = sm[threadIdx.x & 31][k0];    // warp w: channel w, lane l: its sum l
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0 && blockIdx.x * 32 + k0 < channels) dgamma[blockIdx.x * 32 + k0] = v;
}

// 16-channel groups of a row -> threads per row (log2), groups per thread and threads per CTA
struct Shape { int tpr_log, slots, threads; };
Shape shape_of(int channels, bool spread) {
    const int groups = ck_pitch(channels) / kGroup;
    Shape s{spread ? 5 : 1, 1, groups > 256 ? 512 : 256};       // at least the two lanes of a block of 32, or a warp
    while ((1 << s.tpr_log) < groups && (1 << s.tpr_log) < s.threads) s.tpr_log++;
    while ((s.slots << s.tpr_log) < groups) s.slots *= 2;
    return s;
}
// resident CTAs, no more than there are rows for
int grid_of(const revnet_ctx *ctx, int64_t rows, const Shape &s, int per_sm) {
    const int64_t at_once = s.threads >> s.tpr_log, need = (rows + at_once - 1) / at_once, most = (int64_t)ctx->sm_count * per_sm;
    return (int)(need < most ? need : most);
}
template <class K> bool with_shared(Exec &ex, OncePerDevice &once, K kernel, size_t bytes) {
    if (!once.first(ex.ctx->device)) return true;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}
// records of dgamma: by the larger grid of the two forms, whose choice also depends on addresses
int parts_of(const revnet_ctx *ctx, const revnet_norm_desc &d) {
    const Shape a = shape_of(d.channels, false), b = shape_of(d.channels, true);
    const int ga = grid_of(ctx, d.rows, a, bwd_per_sm(a.threads)), gb = grid_of(ctx, d.rows, b, bwd_per_sm(b.threads));
    return ga > gb ? ga : gb;
}

template <bool SPREAD, class TS, class TB, int CODE, int SLOTS, int THREADS> void fwd_k(Exec &ex, const NormArgs &p, unsigned grid, double bytes) {
    static OncePerDevice once;
    constexpr int chunks = kChunks<TS> + kChunks<TB>;
    const size_t smem = SPREAD || SLOTS > 1 ? 0 : (size_t)fwd_stages(THREADS) * chunks * THREADS * 16;
    if (!with_shared(ex, once, rmsnorm_fwd_kernel<SPREAD, TS, TB, CODE, SLOTS, THREADS>, smem)) return;
    launch_stream(ex, bytes, smem ? 100 : 0, rmsnorm_fwd_kernel<SPREAD, TS, TB, CODE, SLOTS, THREADS>, grid, THREADS, smem, p);
}
template <bool SPREAD, class TS, class TB, int CODE> void fwd_t(Exec &ex, const NormArgs &p, const Shape &s, unsigned grid, double bytes) {
    if (s.slots == 2) fwd_k<SPREAD, TS, TB, CODE, 2, 512>(ex, p, grid, bytes);
    else if (s.threads == 512) fwd_k<SPREAD, TS, TB, CODE, 1, 512>(ex, p, grid, bytes);
    else fwd_k<SPREAD, TS, TB, CODE, 1, 256>(ex, p, grid, bytes);
}
template <bool SPREAD, class TS, class TB, bool FROM_H, int CODE, int SLOTS, int THREADS> void bwd_k(Exec &ex, const NormArgs &p, unsigned grid, double bytes) {
    static OncePerDevice once;
    constexpr int chunks = kChunks<TS> + kChunks<TB> + (FROM_H ? kChunks<TS> : 1);
    const size_t rows = SPREAD || SLOTS > 1 ? 0 : (size_t)bwd_stages(chunks) * chunks * THREADS * 16;
    const size_t least = THREADS == 256 ? THREADS * 16 * sizeof(float) : 0, smem = rows > least ? rows : least;
    if (!with_shared(ex, once, rmsnorm_bwd_kernel<SPREAD, TS, TB, FROM_H, CODE, SLOTS, THREADS>, smem)) return;
    launch_stream(ex, bytes, SPREAD || SLOTS > 1 ? 15 : 100, rmsnorm_bwd_kernel<SPREAD, TS, TB, FROM_H, CODE, SLOTS, THREADS>, grid, THREADS, smem, p);
}
template <bool SPREAD, class TS, class TB, bool FROM_H, int CODE> void bwd_t(Exec &ex, const NormArgs &p, const Shape &s, unsigned grid, double bytes) {
    if (s.slots == 2) bwd_k<SPREAD, TS, TB, FROM_H, CODE, 2, 512>(ex, p, grid, bytes);
    else if (s.threads == 512) bwd_k<SPREAD, TS, TB, FROM_H, CODE, 1, 512>(ex, p, grid, bytes);
    else bwd_k<SPREAD, TS, TB, FROM_H, CODE, 1, 256>(ex, p, grid, bytes);
}
template <class F> void by_types(const revnet_norm_desc &d, bool spread, F &&f) {
    auto types = [&](auto s) {
        if (d.stream_dtype == REVNET_BF16) f(s, bf16(), bf16());
        else if (d.branch_dtype == REVNET_BF16) f(s, float(), bf16());
        else f(s, float(), float());
    };
    if (spread) types(std::true_type()); else types(std::false_type());
}
NormArgs args_of(const revnet_norm_desc &d) {
    NormArgs p{};
    p.rows = d.rows; p.ld_s = d.ld_stream; p.ld_b = d.ld_branch;
    p.channels = d.channels;
    p.eps = d.eps; p.inv_c = 1.f / (float)d.channels; p.ck_scaled = d.ck_scaled;
    return p;
}

}  // namespace

void rmsnorm_fwd(Exec &ex, const revnet_norm_desc &d, const void *x, const void *r, const float *gamma, void *h, void *n, void *ck, float *rstd) {
    if (d.rows == 0) return;
    const int ss = d.stream_dtype == REVNET_F32 ? 4 : 2, sb = d.branch_dtype == REVNET_F32 ? 4 : 2;
    NormArgs p = args_of(d);
    p.x = x; p.r = r; p.gamma = gamma; p.h = h; p.n = n; p.rstd = rstd; p.ck = ck_view(ck, d.rows, d.channels);
    const int access = std::min({row_access(x, d.ld_stream, ss, d.channels), row_access(h, d.ld_stream, ss, d.channels), row_access(r, d.ld_branch, sb, d.channels),
                                 row_access(n, d.ld_branch, sb, d.channels), row_access(gamma, 0, 4, d.channels)});
    const bool spread = access == 0;
    p.wide = access == 2;
    const Shape s = shape_of(d.channels, spread);
    p.tpr_log = s.tpr_log;
    const double bytes = (double)d.rows * d.channels * (ss + (r ? sb : 0) + (h ? ss : 0) + (n ? sb : 0) + (ck ? 1 : 0));
    const unsigned grid = (unsigned)grid_of(ex.ctx, d.rows, s, fwd_per_sm(s.threads, ss + sb));
    by_types(d, spread, [&](auto sp, auto ts, auto tb) {
        if (d.code == REVNET_INT8) fwd_t<decltype(sp)::value, decltype(ts), decltype(tb), REVNET_INT8>(ex, p, s, grid, bytes);
        else fwd_t<decltype(sp)::value, decltype(ts), decltype(tb), REVNET_E4M3>(ex, p, s, grid, bytes);
    });
    ex.check("rmsnorm_fwd", bytes);
}

size_t rmsnorm_bwd_workspace(const revnet_ctx *ctx, const revnet_norm_desc &d) { return (size_t)parts_of(ctx, d) * d.channels * sizeof(float) + 256; }

void rmsnorm_bwd(Exec &ex, const revnet_norm_desc &d, const void *dn, const void *dh, const void *h, const void *ck, const float *rstd,
                 const float *gamma, void *dx, void *dr, float *dgamma, float *partial) {
    const int ss = d.stream_dtype == REVNET_F32 ? 4 : 2, sb = d.branch_dtype == REVNET_F32 ? 4 : 2;
    NormArgs p = args_of(d);
    p.x = h; p.dn = dn; p.dh = dh; p.rstd_in = rstd; p.gamma = gamma; p.dx = dx; p.dr = dr; p.dgamma = dgamma; p.partial = partial;
    p.ck = ck_view(ck, d.rows, d.channels);
    const int access = std::min({row_access(h, d.ld_stream, ss, d.channels), row_access(dh, d.ld_stream, ss, d.channels), row_access(dx, d.ld_stream, ss, d.channels),
                                 row_access(dn, d.ld_branch, sb, d.channels), row_access(dr, d.ld_branch, sb, d.channels), row_access(gamma, 0, 4, d.channels)});
    const bool spread = access == 0;
    p.wide = access == 2;
    const Shape s = shape_of(d.channels, spread);
    p.tpr_log = s.tpr_log;
    const int grid = grid_of(ex.ctx, d.rows, s, bwd_per_sm(s.threads));
    if (grid > 0) {
        const double bytes = (double)d.rows * d.channels * (sb + (dh ? ss : 0) + (h ? ss : 1) + ss + (dr ? sb : 0));
        by_types(d, spread, [&](auto sp, auto ts, auto tb) {
            if (h) bwd_t<decltype(sp)::value, decltype(ts), decltype(tb), true, 0>(ex, p, s, grid, bytes);
            else if (d.code == REVNET_INT8) bwd_t<decltype(sp)::value, decltype(ts), decltype(tb), false, REVNET_INT8>(ex, p, s, grid, bytes);
            else bwd_t<decltype(sp)::value, decltype(ts), decltype(tb), false, REVNET_E4M3>(ex, p, s, grid, bytes);
        });
        ex.check("rmsnorm_bwd", bytes);
    }
    if (dgamma && grid != 1) {
        launch(ex, rmsnorm_dgamma_kernel, (unsigned)((d.channels + 31) / 32), 1024, 0, (const float *)partial, grid, d.channels, dgamma);
        ex.check("rmsnorm_dgamma", (double)grid * d.channels * 4);
    }
}
