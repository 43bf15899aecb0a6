// Root-mean-square norm behind the residual's addition, with an output in 8 bits, and its backward pass.
//
//   forward   h = x + r,  rstd = 1 / sqrt(mean(h^2) + eps),  xh = h rstd,  n = xh gamma,  checkpoint of xh (or n)
//   backward  dx = dh + rstd (gamma dn - xh mean(gamma dn xh)),  dgamma = sum over rows of dn xh
//
// HBM bounds both.  A row stays in the registers of the threads that own it, so every tensor is read and written once: the sum of squares
// (backward: that and the sum of gamma dn h) is one reduction over the row, and everything else is local to a thread's 16 channels
// (token.cuh).  A row belongs to `tpr` threads, as few as its channels take: up to 32 of them reduce by shuffles, more through shared memory.
// Short rows share a CTA.  CTAs are resident and walk over the rows; while one row is reduced and written, the next ones are on their way into
// shared memory (rows in 16-byte pieces, as far as two fit; others are loaded when they are needed).  With idle threads up to the next power of
// two the warps' instructions bound rows in between: 8192 x 5120 bf16, forward 80 -> 63 us, backward 86 -> 69.
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
    int tpr;                         // threads per row
    int stages;                      // rows of a CTA in shared memory
    int ck_scaled;
    bool wide;                       // 32-byte accesses (token.cuh)
    float eps, inv_c;
};

// gamma of a thread's channels (ones where there is none, zeros behind the row's end)
template <int ROWS> __device__ __forceinline__ void load_gamma(const NormArgs &p, int ch, float (&g)[16]) {
    if (p.gamma) { load16<ROWS>(p.gamma + ch, ch, p.channels - ch, p.wide, g); return; }
#pragma unroll
    for (int i = 0; i < 16; i++) g[i] = ch + i < p.channels ? 1.f : 0.f;
}

// sums over the tpr threads of a row, given to all of them; red: N floats per warp, the other half of them at every call, so that one barrier
// is enough: who writes a half has passed the barrier behind its readers.  Every thread of the CTA calls it.
template <int N, int WARPS> __device__ __forceinline__ void row_sum(float (&v)[N], int tpr, int row, int &half, float (*red)[WARPS][N]) {
#pragma unroll
    for (int o = 16; o; o >>= 1)
        if (o < tpr) {
#pragma unroll
            for (int i = 0; i < N; i++) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        }
    if (tpr <= 32) return;
    const int lane = threadIdx.x & 31, warps = tpr >> 5, first = row * warps;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; i++) red[half][threadIdx.x >> 5][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = lane < warps ? red[half][first + lane][i] : 0.f;
#pragma unroll
    for (int o = WARPS / 2; o; o >>= 1) {
#pragma unroll
        for (int i = 0; i < N; i++) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = __shfl_sync(0xffffffffu, v[i], 0);
    half ^= 1;
}

// How many rows of a CTA lie in shared memory (the one that is worked on among them) and how many CTAs an SM holds.  Enough bytes have to be in
// flight, but the reads and writes that HBM sees at a time must not be scattered over too many rows.  Forward, us by CTAs x rows (KB of them per SM):
// 16384 x 4096 bf16 1 x 2 (32) 131, 1 x 3 (48) 112, 2 x 2 (64) 99, 2 x 3 (96) 114; 200704 x 512 float32 1 x 2 (64) 281, 1 x 3 (96) 306, 2 x 2 (128) 305;
// 8192 x 7168 float32 stream, bf16 branch 1 x 2 (84) 120, 1 x 3 (126) 137; 8192 x 6144 bf16, alone on its SM, 1 x 2 (48) 84, 1 x 3 (72) 73.
// Backward, with more reads per write, gains from more: 16384 x 4096 bf16 2 x 2 (80) 90, 2 x 3 (120) 83, 2 x 4 (160) 84; 4096 float32 2 x 2 (144)
// 138, 2 x 3 (216) 151; 200704 x 512 float32 from h 1 x 3 (144) 238, 2 x 2 (192) 239.  More than three rows never paid.  (With 80 registers, for three
// CTAs, a float32 stream with a bf16 branch spills: 16384 x 4096 150 against 136.)
// The forward's limit is less than 96 KB.  Two rows and three (2^26 values, us): at 96 KB, rows that fill all threads, bf16 4096 102 and 114, 8192 107 both,
// float32 512 281 and 306; just below it, bf16 4080 109 and 115, 4064 109 and 111, 4032 109 and 111, 1000 115 and 109, 8128 109 and 107, 8064 109 and
// 105, float32 4064 201 and 195, 2032 201 and 192, 2000 203 and 189; at 90 KB float32 3840 201 and 185.  A limit of 95 KB only moves the step.
constexpr int kMaxStages = 3, kFwdBytes = 96 * 1024 - 1, kBwdBytes = 160 * 1024;
__host__ __device__ constexpr int per_sm_of(int threads) { return threads == 512 ? 1 : 2; }        // of the most threads, with 128 registers each
__host__ __device__ constexpr int shared_of(int per_sm) { return (228 / per_sm - 2) * 1024; }        // bytes of a CTA for stages: an SM has 228 KB, the system takes 1 KB per CTA, the sums less than another
__host__ __device__ constexpr bool staged(int rows, int slots, int row, int threads) {        // do two stages fit
    return 2 * slots * (row * threads + (rows == kShifted ? 3 * threads / 32 : 0)) * 16 <= shared_of(1);
}
// the row that comes next has arrived: only the copies of the one behind it may be on their way
__device__ __forceinline__ void next_row_wait(int stages) {
    if (stages == 2) copies_wait<0>();
    else copies_wait<1>();
}

// SLOTS times 16 channels per thread
template <int ROWS, class TS, class TB, int CODE, int SLOTS, int THREADS>
__global__ void __launch_bounds__(THREADS, per_sm_of(THREADS)) rmsnorm_fwd_kernel(const __grid_constant__ NormArgs p) {
    extern __shared__ uint4 stages[];
    __shared__ float red[2][THREADS / 32][1];
    constexpr int kX = kChunks<TS>, kPer = kX + kChunks<TB>;      // chunks: of x; of 16 channels, r behind x
    constexpr bool kAsync = staged(ROWS, SLOTS, kPer, THREADS);
    const int threads = blockDim.x, tpr = p.tpr, at_once = threads / tpr, which = threadIdx.x / tpr, t = threadIdx.x - which * tpr;
    const int64_t step = (int64_t)gridDim.x * at_once;
    int64_t row = (int64_t)blockIdx.x * at_once + which;
    int half = 0;
    const int ch0 = t * kGroup;
    float gamma[16];
    pdl_enter();
    load_gamma<ROWS>(p, ch0, gamma);
    // the lanes of this warp that share the row, their first channel, and where their chunks lie in a part of a stage (one per thread)
    const int lanes = tpr < 32 ? tpr : 32, lane = t & (lanes - 1), chw = (t - lane) * kGroup, mine = (int)threadIdx.x - lane;
    // shifted rows have a chunk more per row and warp, in each part of a stage
    const int extra = ROWS == kShifted ? mine / lanes : 0, extras = ROWS == kShifted ? threads / lanes : 0;
    const int per_slot = kPer * threads + 3 * extras, per_stage = SLOTS * per_slot;
    auto fetch = [&](int stage, int64_t at) {
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            uint4 *to = stages + stage * per_stage + s * per_slot;
            const int ch = chw + s * tpr * kGroup, left = at < p.rows ? p.channels - ch : 0;
            fetch_row<ROWS>(to + mine * kX + extra, lanes, lane, (const TS *)p.x, at * p.ld_s + ch, left);
            if (p.r) fetch_row<ROWS>(to + kX * threads + extras + mine * kChunks<TB> + extra, lanes, lane, (const TB *)p.r, at * p.ld_b + ch, left);
        }
        copies_commit();
    };
    if constexpr (kAsync)
        for (int i = 0; i < p.stages - 1; i++) fetch(i, row + i * step);
    int stage = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * at_once; row0 < p.rows; row0 += step, row += step) {
        const bool row_ok = row < p.rows;
        const int64_t at_s = row * p.ld_s, at_b = row * p.ld_b;
        float h[SLOTS][16], sum[1] = {0.f};
        if constexpr (kAsync) { next_row_wait(p.stages); __syncwarp(); }
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = (s * tpr + t) * kGroup, left = row_ok ? p.channels - ch : 0;
            Raw16<TS> x;
            Raw16<TB> r;
            if constexpr (kAsync) {
                const uint4 *from = stages + stage * per_stage + s * per_slot;
                fetched<ROWS>(from + mine * kX + extra, lanes, lane, (const TS *)p.x + at_s, x);
                if (p.r) fetched<ROWS>(from + kX * threads + extras + mine * kChunks<TB> + extra, lanes, lane, (const TB *)p.r + at_b, r);
            } else {
                load_raw<ROWS>((const TS *)p.x + (at_s + ch), ch, left, p.wide, x);
                if (p.r) load_raw<ROWS>((const TB *)p.r + (at_b + ch), ch, left, p.wide, r);
            }
            unpack(x, h[s]);
            if (p.r) {
                float add[16];
                unpack(r, add);
#pragma unroll
                for (int i = 0; i < 16; i++) h[s][i] += add[i];
                pack(h[s], x);                       // the norm is of h as it is stored, so that the backward pass sees the same h
                unpack(x, h[s]);
                if (p.h) store_raw<ROWS>((TS *)p.h + (at_s + ch), ch, left, p.wide, x);
            }
#pragma unroll
            for (int i = 0; i < 16; i++) sum[0] = fmaf(h[s][i], h[s][i], sum[0]);
        }
        if constexpr (kAsync) {
            // into the stage that the row before this one has left
            fetch(stage == 0 ? p.stages - 1 : stage - 1, row + (p.stages - 1) * step);
            if (++stage == p.stages) stage = 0;
        }
        row_sum(sum, tpr, which, half, red);
        // (rsqrtf is off by two steps at most.  16384 x 4096: 415 of the bf16 outputs and 52 of the codes fall otherwise than exact ones would; with
        // divisions and roots in float32 throughout 474 and 65)
        const float rstd = rsqrtf(sum[0] * p.inv_c + p.eps);
        if (p.rstd && row_ok && t == 0) p.rstd[row] = rstd;
        if (!p.n && !p.ck.codes) continue;
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = (s * tpr + t) * kGroup, left = row_ok ? p.channels - ch : 0;
            float n[16];
            if (s > 0) load_gamma<ROWS>(p, ch, gamma);
#pragma unroll
            for (int i = 0; i < 16; i++) { h[s][i] *= rstd; n[i] = h[s][i] * gamma[i]; }
            if (p.n) store16<ROWS>((TB *)p.n + (at_b + ch), ch, left, p.wide, n);
            if (p.ck.codes) {
                if (p.ck_scaled) keep16<CODE>(p.ck, row, ch, row_ok, n);
                else keep16<CODE>(p.ck, row, ch, row_ok, h[s]);
            }
        }
        if (SLOTS > 1) load_gamma<ROWS>(p, ch0, gamma);
    }
    if constexpr (kAsync) copies_wait<0>();
}

// FROM_H: from h; else from a checkpoint of xh with CODE.  A thread keeps its channels for all rows it works on, and their dgamma in registers.
template <int ROWS, class TS, class TB, bool FROM_H, int CODE, int SLOTS, int THREADS>
__global__ void __launch_bounds__(THREADS, per_sm_of(THREADS)) rmsnorm_bwd_kernel(const __grid_constant__ NormArgs p) {
    extern __shared__ uint4 stages[];
    constexpr int kSums = FROM_H ? 2 : 1;                // gamma dn x, and the squares
    __shared__ float red[2][THREADS / 32][kSums];
    constexpr int kS = kChunks<TS>, kB = kChunks<TB>, kX = FROM_H ? kS : 1, kPer = kS + kB + kX;      // chunks of 16 channels: dh, dn, h or codes
    constexpr bool kAsync = staged(ROWS, SLOTS, kPer, THREADS);
    constexpr bool kAgain = kAsync && SLOTS > 1;         // longer rows are decoded a second time: their registers hold dgamma
    const int threads = blockDim.x, tpr = p.tpr, at_once = threads / tpr, which = threadIdx.x / tpr, t = threadIdx.x - which * tpr;
    const int64_t step = (int64_t)gridDim.x * at_once;
    int64_t row = (int64_t)blockIdx.x * at_once + which;
    int half = 0;
    const int ch0 = t * kGroup;
    float dg[SLOTS][16], gamma[16];
#pragma unroll
    for (int s = 0; s < SLOTS; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) dg[s][i] = 0.f;
    pdl_enter();
    load_gamma<ROWS>(p, ch0, gamma);
    // the lanes of this warp that share the row, their first channel, and where their chunks lie in a part of a stage (one per thread)
    const int lanes = tpr < 32 ? tpr : 32, lane = t & (lanes - 1), chw = (t - lane) * kGroup, mine = (int)threadIdx.x - lane;
    // shifted rows have a chunk more per row and warp, in each part of a stage
    const int extra = ROWS == kShifted ? mine / lanes : 0, extras = ROWS == kShifted ? threads / lanes : 0;
    const int per_slot = kPer * threads + 3 * extras, per_stage = SLOTS * per_slot;
    auto fetch = [&](int stage, int64_t at) {
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            uint4 *to = stages + stage * per_stage + s * per_slot;
            const int ch = chw + s * tpr * kGroup, left = at < p.rows ? p.channels - ch : 0;
            if (p.dh) fetch_row<ROWS>(to + mine * kS + extra, lanes, lane, (const TS *)p.dh, at * p.ld_s + ch, left);
            fetch_row<ROWS>(to + kS * threads + extras + mine * kB + extra, lanes, lane, (const TB *)p.dn, at * p.ld_b + ch, left);
            if constexpr (FROM_H) fetch_row<ROWS>(to + (kS + kB) * threads + 2 * extras + mine * kS + extra, lanes, lane, (const TS *)p.x, at * p.ld_s + ch, left);
            else copy16(to + (kS + kB) * threads + 2 * extras + threadIdx.x, p.ck.codes + (at * p.ck.pitch + ch + lane * kGroup), lane * kGroup < left ? 16 : 0);
        }
        copies_commit();
    };
    if constexpr (kAsync)
        for (int i = 0; i < p.stages - 1; i++) fetch(i, row + i * step);
    int stage = 0;
    // what a row has besides its channels is loaded a row ahead too
    float rstd_next = 0.f;
    uint32_t byte_next[SLOTS] = {}, bytes[SLOTS];
    auto ahead = [&](int64_t at) {
        if (FROM_H) return;
        rstd_next = at < p.rows ? p.rstd_in[at] : 0.f;
        if (kAsync) {
#pragma unroll
            for (int s = 0; s < SLOTS; s++) {
                const int ch = ch0 + s * tpr * kGroup;
                byte_next[s] = at < p.rows && ch < p.channels ? byte_of(p.ck.scales + scale_index(p.ck, at, ch)) : 0u;
            }
        }
    };
    // what the sums and dx need of slot s, out of a stage
    auto staged_row = [&](int stage, int s, int64_t at_s, int64_t at_b, float (&x)[16], float (&dn)[16]) {
        const uint4 *from = stages + stage * per_stage + s * per_slot;
        Raw16<TB> rn;
        fetched<ROWS>(from + kS * threads + extras + mine * kB + extra, lanes, lane, (const TB *)p.dn + at_b, rn);
        unpack(rn, dn);
        if constexpr (FROM_H) {
            Raw16<TS> rx;
            fetched<ROWS>(from + (kS + kB) * threads + 2 * extras + mine * kS + extra, lanes, lane, (const TS *)p.x + at_s, rx);
            unpack(rx, x);
        } else decode16<CODE>(from[(kS + kB) * threads + 2 * extras + threadIdx.x], bytes[s], x);
    };
    ahead(row);
    for (int64_t row0 = (int64_t)blockIdx.x * at_once; row0 < p.rows; row0 += step, row += step) {
        const bool row_ok = row < p.rows;
        const int64_t at_s = row * p.ld_s, at_b = row * p.ld_b;
        constexpr int kHeld = kAgain ? 1 : SLOTS;
        float x[kHeld][16], dn[kHeld][16], rstd = rstd_next, sum[kSums];
#pragma unroll
        for (int s = 0; s < SLOTS; s++) bytes[s] = byte_next[s];
#pragma unroll
        for (int i = 0; i < kSums; i++) sum[i] = 0.f;
        if constexpr (kAsync) { next_row_wait(p.stages); __syncwarp(); }
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = (s * tpr + t) * kGroup, left = row_ok ? p.channels - ch : 0;
            const int k = kAgain ? 0 : s;
            if constexpr (kAsync) staged_row(stage, s, at_s, at_b, x[k], dn[k]);
            else {
                load16<ROWS>((const TB *)p.dn + (at_b + ch), ch, left, p.wide, dn[k]);
                if constexpr (FROM_H) load16<ROWS>((const TS *)p.x + (at_s + ch), ch, left, p.wide, x[k]);
                else read16<CODE>(p.ck, row, ch, left, x[k]);
            }
            if (s > 0) load_gamma<ROWS>(p, ch, gamma);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                if constexpr (FROM_H) {
                    sum[0] = fmaf(dn[k][i] * gamma[i], x[k][i], sum[0]);
                    sum[1] = fmaf(x[k][i], x[k][i], sum[1]);
                } else {
                    dg[s][i] = fmaf(dn[k][i], x[k][i], dg[s][i]);         // (zeros where there is no row)
                    dn[k][i] *= gamma[i];
                    sum[0] = fmaf(dn[k][i], x[k][i], sum[0]);
                }
            }
        }
        ahead(row + step);
        if constexpr (kAsync) {
            // into the stage that the row before this one has left
            fetch(stage == 0 ? p.stages - 1 : stage - 1, row + (p.stages - 1) * step);
        }
        row_sum(sum, tpr, which, half, red);
        if constexpr (FROM_H) rstd = rsqrtf(sum[1] * p.inv_c + p.eps);
        // dx = dh + rstd gamma dn - xh (rstd mean(gamma dn xh)); from h: xh = h rstd, and the mean is rstd times that of gamma dn h
        const float back = -sum[0] * p.inv_c * rstd * (FROM_H ? rstd * rstd : 1.f);
#pragma unroll
        for (int s = 0; s < SLOTS; s++) {
            const int ch = (s * tpr + t) * kGroup, left = row_ok ? p.channels - ch : 0;
            float d[16];
            if (p.dh) {
                Raw16<TS> rh;
                if constexpr (kAsync) fetched<ROWS>(stages + stage * per_stage + s * per_slot + mine * kS + extra, lanes, lane, (const TS *)p.dh + at_s, rh);
                else load_raw<ROWS>((const TS *)p.dh + (at_s + ch), ch, left, p.wide, rh);
                unpack(rh, d);
            } else {
#pragma unroll
                for (int i = 0; i < 16; i++) d[i] = 0.f;
            }
            const int k = kAgain ? 0 : s;
            if (SLOTS > 1 && (FROM_H || kAgain)) load_gamma<ROWS>(p, ch, gamma);
            if constexpr (kAgain) staged_row(stage, s, at_s, at_b, x[0], dn[0]);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                float w = dn[k][i] * rstd;
                if constexpr (FROM_H) dg[s][i] = fmaf(w, x[k][i], dg[s][i]);
                if constexpr (FROM_H || kAgain) w *= gamma[i];
                d[i] = fmaf(x[k][i], back, d[i] + w);
            }
            store16<ROWS>((TS *)p.dx + (at_s + ch), ch, left, p.wide, d);
            if (p.dr) store16<ROWS>((TB *)p.dr + (at_b + ch), ch, left, p.wide, d);
        }
        if (SLOTS > 1) load_gamma<ROWS>(p, ch0, gamma);
        if constexpr (kAsync) { if (++stage == p.stages) stage = 0; }
    }
    if constexpr (kAsync) copies_wait<0>();
    if (!p.dgamma) return;
    float *out = gridDim.x == 1 ? p.dgamma : p.partial + (size_t)blockIdx.x * p.channels;
    if (SLOTS == 1 && at_once > 1) {
        // the CTA's rows first, in a fixed order, through the stages' memory
        float *sums = reinterpret_cast<float *>(stages);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; i++) sums[(threadIdx.x - t) * 16 + ch0 + i] = dg[0][i];
        __syncthreads();
        for (int c = threadIdx.x; c < p.channels; c += threads) {
            float v = 0.f;
            for (int k = 0; k < at_once; k++) v += sums[k * tpr * 16 + c];
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

// 16-channel groups of a row -> threads per row (a power of two, or whole warps), groups per thread, threads per CTA, and the most of them
struct Shape { int tpr, slots, threads, most; };
Shape shape_of(int channels) {
    const int groups = ck_pitch(channels) / kGroup;
    Shape s{2, groups > 512 ? 2 : 1, 0, groups > 256 ? 512 : 256};       // at least the two lanes of a block of 32
    const int need = (groups + s.slots - 1) / s.slots;
    while (s.tpr < need && s.tpr < 32) s.tpr *= 2;
    if (s.tpr < need) s.tpr = (need + 31) / 32 * 32;
    s.threads = s.most / s.tpr * s.tpr;
    return s;
}
// resident CTAs, no more than there are rows for
int grid_of(const revnet_ctx *ctx, int64_t rows, const Shape &s, int per_sm) {
    const int64_t at_once = s.threads / s.tpr, need = (rows + at_once - 1) / at_once, most = (int64_t)ctx->sm_count * per_sm;
    return (int)(need < most ? need : most);
}
// CTAs per SM and the stages of each, for rows that take `row` chunks per thread: as many CTAs as threads fit (`full` of the most threads), then
// up to kMaxStages stages, as long as the rows in them stay within `bytes` per SM.
struct Plan { int per_sm, stages; };
int stage_bytes(int rows, const Shape &s, int row) { return s.slots * (s.threads * row + (rows == kShifted ? 3 * s.threads / std::min(s.tpr, 32) : 0)) * 16; }
Plan plan_of(int rows, const Shape &s, int channels, int row, int full, int bytes) {
    const int used = s.threads / s.tpr * ((channels + kGroup - 1) / kGroup) * row * 16, stage = stage_bytes(rows, s, row);
    Plan p{full * s.most / s.threads, 2};
    while (p.per_sm > 1 && (p.per_sm * 2 * used > bytes || 2 * stage > shared_of(p.per_sm))) p.per_sm--;
    while (p.stages < kMaxStages && p.per_sm * (p.stages + 1) * used <= bytes && (p.stages + 1) * stage <= shared_of(p.per_sm)) p.stages++;
    return p;
}
// (shifted rows take more instructions than bytes: as many as fit)
Plan fwd_plan(int rows, const Shape &s, int channels, int row) { return plan_of(rows, s, channels, row, per_sm_of(s.most), rows == kShifted ? shared_of(1) : kFwdBytes); }
Plan bwd_plan(int rows, const Shape &s, int channels, int row) { return plan_of(rows, s, channels, row, per_sm_of(s.most), rows == kShifted ? shared_of(1) : kBwdBytes); }
// records of dgamma, of the largest grid that a call may have: its rows' alignment decides too
int parts_of(const revnet_ctx *ctx, const revnet_norm_desc &d) {
    const Shape s = shape_of(d.channels);
    return grid_of(ctx, d.rows, s, per_sm_of(s.most) * s.most / s.threads);
}

template <int ROWS, class TS, class TB, int CODE, int SLOTS, int THREADS> void fwd_k(Exec &ex, NormArgs p, const Shape &s, unsigned grid, double bytes) {
    static OncePerDevice once;
    constexpr int row = kChunks<TS> + kChunks<TB>;
    constexpr bool async = staged(ROWS, SLOTS, row, THREADS);
    p.stages = fwd_plan(ROWS, s, p.channels, row).stages;
    if (!shared_limit(once, ex.ctx->device, async ? shared_of(1) : 0, rmsnorm_fwd_kernel<ROWS, TS, TB, CODE, SLOTS, THREADS>)) return;
    launch_stream(ex, bytes, async ? 100 : 0, rmsnorm_fwd_kernel<ROWS, TS, TB, CODE, SLOTS, THREADS>, grid, s.threads, async ? (size_t)p.stages * stage_bytes(ROWS, s, row) : 0, p);
}
template <int ROWS, class TS, class TB, int CODE> void fwd_t(Exec &ex, const NormArgs &p, const Shape &s, unsigned grid, double bytes) {
    if (s.slots == 2) fwd_k<ROWS, TS, TB, CODE, 2, 512>(ex, p, s, grid, bytes);
    else if (s.most == 512) fwd_k<ROWS, TS, TB, CODE, 1, 512>(ex, p, s, grid, bytes);
    else fwd_k<ROWS, TS, TB, CODE, 1, 256>(ex, p, s, grid, bytes);
}
template <int ROWS, class TS, class TB, bool FROM_H, int CODE, int SLOTS, int THREADS> void bwd_k(Exec &ex, NormArgs p, const Shape &s, unsigned grid, double bytes) {
    static OncePerDevice once;
    constexpr int row = kChunks<TS> + kChunks<TB> + (FROM_H ? kChunks<TS> : 1);
    constexpr bool async = staged(ROWS, SLOTS, row, THREADS);
    p.stages = bwd_plan(ROWS, s, p.channels, row).stages;
    const size_t rows = async ? (size_t)p.stages * stage_bytes(ROWS, s, row) : 0, least = THREADS == 256 ? THREADS * 16 * sizeof(float) : 0, smem = rows > least ? rows : least;
    if (!shared_limit(once, ex.ctx->device, async ? shared_of(1) : least, rmsnorm_bwd_kernel<ROWS, TS, TB, FROM_H, CODE, SLOTS, THREADS>)) return;
    launch_stream(ex, bytes, async ? 100 : 15, rmsnorm_bwd_kernel<ROWS, TS, TB, FROM_H, CODE, SLOTS, THREADS>, grid, s.threads, smem, p);
}
template <int ROWS, class TS, class TB, bool FROM_H, int CODE> void bwd_t(Exec &ex, const NormArgs &p, const Shape &s, unsigned grid, double bytes) {
    if (s.slots == 2) bwd_k<ROWS, TS, TB, FROM_H, CODE, 2, 512>(ex, p, s, grid, bytes);
    else if (s.most == 512) bwd_k<ROWS, TS, TB, FROM_H, CODE, 1, 512>(ex, p, s, grid, bytes);
    else bwd_k<ROWS, TS, TB, FROM_H, CODE, 1, 256>(ex, p, s, grid, bytes);
}
template <class F> void by_types(const revnet_norm_desc &d, int rows, F &&f) {
    auto types = [&](auto s) {
        if (d.stream_dtype == REVNET_BF16) f(s, bf16(), bf16());
        else if (d.branch_dtype == REVNET_BF16) f(s, float(), bf16());
        else f(s, float(), float());
    };
    if (rows == kPieces) types(std::integral_constant<int, kPieces>()); else types(std::integral_constant<int, kShifted>());
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
    const int rows = access ? kPieces : kShifted;
    p.wide = access == 2;
    const Shape s = shape_of(d.channels);
    p.tpr = s.tpr;
    const double bytes = (double)d.rows * d.channels * (ss + (r ? sb : 0) + (h ? ss : 0) + (n ? sb : 0) + (ck ? 1 : 0));
    const unsigned grid = (unsigned)grid_of(ex.ctx, d.rows, s, fwd_plan(rows, s, d.channels, ss + sb).per_sm);
    by_types(d, rows, [&](auto sp, auto ts, auto tb) {
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
    const int rows = access ? kPieces : kShifted;
    p.wide = access == 2;
    const Shape s = shape_of(d.channels);
    p.tpr = s.tpr;
    const int grid = grid_of(ex.ctx, d.rows, s, bwd_plan(rows, s, d.channels, h ? ss + sb + ss : ss + sb + 1).per_sm);
    if (grid > 0) {
        const double bytes = (double)d.rows * d.channels * (sb + (dh ? ss : 0) + (h ? ss : 1) + ss + (dr ? sb : 0));
        by_types(d, rows, [&](auto sp, auto ts, auto tb) {
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
