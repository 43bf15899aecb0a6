// Root-mean-square norm behind the residual's addition, with an output in 8 bits, and its backward pass.
//
//   forward   h = x + r,  rstd = 1 / sqrt(mean(h^2) + eps),  xh = h rstd,  n = xh gamma,  checkpoint of xh (or n)
//   backward  dx = dh + rstd (gamma dn - xh mean(gamma dn xh)),  dgamma = sum over rows of dn xh
//
// HBM bounds both.  A row stays in the registers of the threads that own it, so every tensor is read and written once: the sum of squares
// (backward: that and the sum of gamma dn h) is one reduction over the row, and everything else is local to a group of 16 channels
// (token.cuh).  A row belongs to `tpr` threads, a power of two: up to 32 of them reduce by shuffles, more through shared memory.  Short
// rows share a CTA.
#include "token.cuh"
#include <type_traits>

namespace {

struct NormArgs {
    const void *x, *r, *dn, *dh;
    const float *gamma, *rstd_in;
    void *h, *n, *dx, *dr;
    float *rstd, *partial, *dgamma;
    Checkpoint ck;
    int64_t rows, ld_s, ld_b;
    int channels, groups;            // groups of 16, the padding of the last block of 32 included
    int tpr_log;                     // threads per row
    int ck_scaled;
    int lv_x, lv_r, lv_h, lv_n, lv_dn, lv_dh, lv_dx, lv_dr, lv_g;
    float eps, inv_c;
};

// gamma of a group (ones where there is none, zeros behind the row's end)
__device__ __forceinline__ void load_gamma(const NormArgs &p, int ch, float (&g)[16]) {
    if (p.gamma) { load16(p.gamma + ch, p.channels - ch, p.lv_g, g); return; }
#pragma unroll
    for (int i = 0; i < 16; i++) g[i] = ch + i < p.channels ? 1.f : 0.f;
}

// sum over the tpr threads of a row, given to all of them; red: a float2 per warp.  Every thread of the CTA calls it.
__device__ __forceinline__ float2 row_sum(float2 v, int tpr_log, float2 *red) {
    const int tpr = 1 << tpr_log, within = tpr < 32 ? tpr : 32;
    for (int o = within >> 1; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if (tpr <= 32) return v;
    const int warp = threadIdx.x >> 5, warps = tpr >> 5, first = warp & ~(warps - 1);
    __syncthreads();                 // the last call's sums have been read
    if ((threadIdx.x & 31) == 0) red[warp] = v;
    __syncthreads();
    float2 s = red[first];
    for (int w = 1; w < warps; w++) { const float2 t = red[first + w]; s.x += t.x; s.y += t.y; }
    return s;
}

// SLOTS groups per thread
template <class TS, class TB, int CODE, int SLOTS, int THREADS>
__global__ void __launch_bounds__(THREADS) rmsnorm_fwd_kernel(const NormArgs p) {
    __shared__ float2 red[THREADS / 32];
    pdl_enter();
    const int tpr = 1 << p.tpr_log, t = threadIdx.x & (tpr - 1);
    const size_t row = (size_t)blockIdx.x * (THREADS >> p.tpr_log) + (threadIdx.x >> p.tpr_log);
    const bool row_ok = row < (size_t)p.rows;
    float h[SLOTS][16];
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int s = 0; s < SLOTS; s++) {
        const int ch = (s * tpr + t) * kGroup, n = row_ok ? p.channels - ch : 0;
        load16((const TS *)p.x + row * p.ld_s + ch, n, p.lv_x, h[s]);
    }
    if (p.r) {
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = (s * tpr + t) * kGroup, n = row_ok ? p.channels - ch : 0;
            float r[16];
            load16((const TB *)p.r + row * p.ld_b + ch, n, p.lv_r, r);
            Raw16<TS> raw;
#pragma unroll
            for (int i = 0; i < 16; i++) h[s][i] += r[i];
            pack(h[s], raw);                         // the norm is of h as it is stored, so that the backward pass sees the same h
            unpack(raw, h[s]);
            if (p.h) store_raw((TS *)p.h + row * p.ld_s + ch, n, p.lv_h, raw);
        }
    }
#pragma unroll
    for (int s = 0; s < SLOTS; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) sum.x = fmaf(h[s][i], h[s][i], sum.x);
    sum = row_sum(sum, p.tpr_log, red);
    const float rstd = 1.f / sqrtf(sum.x * p.inv_c + p.eps);
    if (p.rstd && row_ok && t == 0) p.rstd[row] = rstd;
    if (!p.n && !p.ck.codes) return;
#pragma unroll
    for (int s = 0; s < SLOTS; s++) {
        const int ch = (s * tpr + t) * kGroup, n = row_ok ? p.channels - ch : 0;
        float g[16];
#pragma unroll
        for (int i = 0; i < 16; i++) h[s][i] *= rstd;
        if (p.n || p.ck_scaled) {
            load_gamma(p, ch, g);
#pragma unroll
            for (int i = 0; i < 16; i++) g[i] *= h[s][i];
        }
        if (p.n) store16((TB *)p.n + row * p.ld_b + ch, n, p.lv_n, g);
        if (p.ck.codes) {
            if (p.ck_scaled) {
#pragma unroll
                for (int i = 0; i < 16; i++) h[s][i] = g[i];
            }
            keep16<CODE>(p.ck, row, ch, row_ok && ch < p.groups * kGroup, h[s]);
        }
    }
}

// SRC 0: from h; 1: from a checkpoint of xh with CODE.  A thread keeps its channels for all rows it works on, and their dgamma in registers.
template <class TS, class TB, int SRC, int CODE, int SLOTS, int THREADS>
__global__ void __launch_bounds__(THREADS) rmsnorm_bwd_kernel(const NormArgs p) {
    __shared__ float2 red[THREADS / 32];
    __shared__ float sums[THREADS == 256 ? THREADS * 16 : 1];      // rows share a CTA only in the small one
    pdl_enter();
    const int tpr = 1 << p.tpr_log, t = threadIdx.x & (tpr - 1), rows_at_once = THREADS >> p.tpr_log, mine = threadIdx.x >> p.tpr_log;
    float dg[SLOTS][16];
#pragma unroll
    for (int s = 0; s < SLOTS; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) dg[s][i] = 0.f;
    for (size_t row0 = (size_t)blockIdx.x * rows_at_once; row0 < (size_t)p.rows; row0 += (size_t)gridDim.x * rows_at_once) {
        const size_t row = row0 + mine;
        const bool row_ok = row < (size_t)p.rows;
        float xh[SLOTS][16], dn[SLOTS][16];
        Raw16<TS> dh[SLOTS];
        float2 sum = make_float2(0.f, 0.f);
        float rstd = 0.f;
        if (SRC == 1 && row_ok) rstd = p.rstd_in[row];
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = (s * tpr + t) * kGroup, n = row_ok ? p.channels - ch : 0;
            load16((const TB *)p.dn + row * p.ld_b + ch, n, p.lv_dn, dn[s]);
            if (SRC == 0) load16((const TS *)p.x + row * p.ld_s + ch, n, p.lv_x, xh[s]);
            else if (n > 0) read16<CODE>(p.ck, row, ch, xh[s]);
            else {
#pragma unroll
                for (int i = 0; i < 16; i++) xh[s][i] = 0.f;
            }
            if (p.dh) load_raw((const TS *)p.dh + row * p.ld_s + ch, n, p.lv_dh, dh[s]);
        }
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = (s * tpr + t) * kGroup;
            float g[16];
            load_gamma(p, ch, g);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                if (SRC == 0) sum.y = fmaf(xh[s][i], xh[s][i], sum.y);
                sum.x = fmaf(dn[s][i] * g[i], xh[s][i], sum.x);
            }
        }
        sum = row_sum(sum, p.tpr_log, red);
        float m;
        if (SRC == 0) {
            rstd = 1.f / sqrtf(sum.y * p.inv_c + p.eps);
            m = sum.x * rstd * p.inv_c;              // of gamma dn h so far
        } else m = sum.x * p.inv_c;
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = (s * tpr + t) * kGroup, n = row_ok ? p.channels - ch : 0;
            float g[16], d[16];
            load_gamma(p, ch, g);
            if (p.dh) unpack(dh[s], d);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float x = SRC == 0 ? xh[s][i] * rstd : xh[s][i];
                if (row_ok) dg[s][i] = fmaf(dn[s][i], x, dg[s][i]);
                const float v = rstd * (dn[s][i] * g[i] - x * m);
                d[i] = p.dh ? d[i] + v : v;
            }
            store16((TS *)p.dx + row * p.ld_s + ch, n, p.lv_dx, d);
            if (p.dr) store16((TB *)p.dr + row * p.ld_b + ch, n, p.lv_dr, d);
        }
    }
    if (!p.dgamma) return;
    float *out = gridDim.x == 1 ? p.dgamma : p.partial + (size_t)blockIdx.x * p.channels;
    if (THREADS == 256 && rows_at_once > 1) {
        // the CTA's rows first, in a fixed order
#pragma unroll
        for (int i = 0; i < 16; i++) sums[threadIdx.x * 16 + i] = dg[0][i];
        __syncthreads();
        for (int c = threadIdx.x; c < p.channels; c += THREADS) {
            float v = 0.f;
            for (int k = 0; k < rows_at_once; k++) v += sums[(k << p.tpr_log) * 16 + c];
            out[c] = v;
        }
        return;
    }
#pragma unroll
    for (int s = 0; s < SLOTS; s++) {
        const int ch = (s * tpr + t) * kGroup;
#pragma unroll
        for (int i = 0; i < 16; i++) if (ch + i < p.channels) out[ch + i] = dg[s][i];
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

// groups of a row -> threads per row (log2), groups per thread and threads per CTA
struct Shape { int tpr_log, slots, threads; };
Shape shape_of(int groups) {
    Shape s{1, 1, groups > 256 ? 512 : 256};         // at least the two lanes of a block of 32
    while ((1 << s.tpr_log) < groups && (1 << s.tpr_log) < s.threads) s.tpr_log++;
    while ((s.slots << s.tpr_log) < groups) s.slots *= 2;
    return s;
}
int groups_of(int channels) { return ck_pitch(channels) / kGroup; }
// CTAs of the backward kernel: what can be resident, no more than there are rows for
int bwd_grid(const revnet_ctx *ctx, int64_t rows, const Shape &s) {
    const int64_t at_once = s.threads >> s.tpr_log, need = (rows + at_once - 1) / at_once;
    const int64_t most = (int64_t)ctx->sm_count * (s.threads == 512 ? 1 : 2);
    return (int)(need < most ? need : most);
}

template <class TS, class TB, int CODE> void fwd_t(Exec &ex, const NormArgs &p, const Shape &s, unsigned grid, double bytes) {
    if (s.slots == 2) launch_stream(ex, bytes, 0, rmsnorm_fwd_kernel<TS, TB, CODE, 2, 512>, grid, 512, 0, p);
    else if (s.threads == 512) launch_stream(ex, bytes, 0, rmsnorm_fwd_kernel<TS, TB, CODE, 1, 512>, grid, 512, 0, p);
    else launch_stream(ex, bytes, 0, rmsnorm_fwd_kernel<TS, TB, CODE, 1, 256>, grid, 256, 0, p);
}
template <class TS, class TB, int SRC, int CODE> void bwd_t(Exec &ex, const NormArgs &p, const Shape &s, unsigned grid, double bytes) {
    if (s.slots == 2) launch_stream(ex, bytes, 0, rmsnorm_bwd_kernel<TS, TB, SRC, CODE, 2, 512>, grid, 512, 0, p);
    else if (s.threads == 512) launch_stream(ex, bytes, 0, rmsnorm_bwd_kernel<TS, TB, SRC, CODE, 1, 512>, grid, 512, 0, p);
    else launch_stream(ex, bytes, 15, rmsnorm_bwd_kernel<TS, TB, SRC, CODE, 1, 256>, grid, 256, 0, p);
}
template <class F> void by_types(const revnet_norm_desc &d, F &&f) {
    if (d.stream_dtype == REVNET_BF16) f(bf16(), bf16());
    else if (d.branch_dtype == REVNET_BF16) f(float(), bf16());
    else f(float(), float());
}
NormArgs args_of(const revnet_norm_desc &d) {
    NormArgs p{};
    p.rows = d.rows; p.ld_s = d.ld_stream; p.ld_b = d.ld_branch;
    p.channels = d.channels; p.groups = groups_of(d.channels);
    p.eps = d.eps; p.inv_c = 1.f / (float)d.channels; p.ck_scaled = d.ck_scaled;
    return p;
}

}  // namespace

void rmsnorm_fwd(Exec &ex, const revnet_norm_desc &d, const void *x, const void *r, const float *gamma, void *h, void *n, void *ck, float *rstd) {
    if (d.rows == 0) return;
    const int ss = d.stream_dtype == REVNET_F32 ? 4 : 2, sb = d.branch_dtype == REVNET_F32 ? 4 : 2;
    NormArgs p = args_of(d);
    const Shape s = shape_of(p.groups);
    p.x = x; p.r = r; p.gamma = gamma; p.h = h; p.n = n; p.rstd = rstd; p.ck = ck_view(ck, d.rows, d.channels); p.tpr_log = s.tpr_log;
    p.lv_x = access_level(x, d.ld_stream, ss); p.lv_h = access_level(h, d.ld_stream, ss);
    p.lv_r = access_level(r, d.ld_branch, sb); p.lv_n = access_level(n, d.ld_branch, sb); p.lv_g = access_level(gamma, 0, 4);
    const double bytes = (double)d.rows * d.channels * (ss + (r ? sb : 0) + (h ? ss : 0) + (n ? sb : 0) + (ck ? 1 : 0));
    const unsigned grid = (unsigned)((d.rows + (s.threads >> s.tpr_log) - 1) / (s.threads >> s.tpr_log));
    by_types(d, [&](auto ts, auto tb) {
        if (d.code == REVNET_INT8) fwd_t<decltype(ts), decltype(tb), REVNET_INT8>(ex, p, s, grid, bytes);
        else fwd_t<decltype(ts), decltype(tb), REVNET_E4M3>(ex, p, s, grid, bytes);
    });
    ex.check("rmsnorm_fwd", bytes);
}

size_t rmsnorm_bwd_workspace(const revnet_ctx *ctx, const revnet_norm_desc &d) {
    return (size_t)bwd_grid(ctx, d.rows, shape_of(groups_of(d.channels))) * d.channels * sizeof(float) + 256;
}

void rmsnorm_bwd(Exec &ex, const revnet_norm_desc &d, const void *dn, const void *dh, const void *h, const void *ck, const float *rstd,
                 const float *gamma, void *dx, void *dr, float *dgamma, float *partial) {
    const int ss = d.stream_dtype == REVNET_F32 ? 4 : 2, sb = d.branch_dtype == REVNET_F32 ? 4 : 2;
    NormArgs p = args_of(d);
    const Shape s = shape_of(p.groups);
    const int grid = bwd_grid(ex.ctx, d.rows, s);
    if (grid > 0) {
        p.x = h; p.dn = dn; p.dh = dh; p.rstd_in = rstd; p.gamma = gamma; p.dx = dx; p.dr = dr; p.dgamma = dgamma; p.partial = partial;
        p.ck = ck_view(ck, d.rows, d.channels); p.tpr_log = s.tpr_log;
        p.lv_x = access_level(h, d.ld_stream, ss); p.lv_dh = access_level(dh, d.ld_stream, ss); p.lv_dx = access_level(dx, d.ld_stream, ss);
        p.lv_dn = access_level(dn, d.ld_branch, sb); p.lv_dr = access_level(dr, d.ld_branch, sb); p.lv_g = access_level(gamma, 0, 4);
        const double bytes = (double)d.rows * d.channels * (sb + (dh ? ss : 0) + (h ? ss : 1) + ss + (dr ? sb : 0));
        by_types(d, [&](auto ts, auto tb) {
            if (h) bwd_t<decltype(ts), decltype(tb), 0, 0>(ex, p, s, grid, bytes);
            else if (d.code == REVNET_INT8) bwd_t<decltype(ts), decltype(tb), 1, REVNET_INT8>(ex, p, s, grid, bytes);
            else bwd_t<decltype(ts), decltype(tb), 1, REVNET_E4M3>(ex, p, s, grid, bytes);
        });
        ex.check("rmsnorm_bwd", bytes);
    }
    if (dgamma && grid != 1) {
        launch(ex, rmsnorm_dgamma_kernel, (unsigned)((d.channels + 31) / 32), 1024, 0, (const float *)partial, grid, d.channels, dgamma);
        ex.check("rmsnorm_dgamma", (double)grid * d.channels * 4);
    }
}
