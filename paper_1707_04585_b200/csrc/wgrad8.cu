// Weight gradient of a linear layer from an 8-bit checkpoint of its input: dW[o][c] = gamma[c] sum_t dy[t][o] x8[t][c].
//
// A matrix product over the rows t, both operands with t as the outer index, on the 5th-generation tensor cores as CTA pairs
// (tcgen05 cta_group::2).  The values of a checkpoint are bf16 numbers, so a tile of codes becomes an MMA operand without rounding:
//
//   dy     TMA -> shared memory, 64 rows x 64 channels per box, 128-byte swizzle, M-major: the A operand as it lies
//   codes  TMA -> shared memory (64 rows x 128 channels) -> twelve decoder warps -> bf16 in the same swizzled layout: the B operand
//   D      256 output channels x 256 input channels of fp32 in the pair's tensor memory, twice
//
// Long sums: the tensor cores round their running sum towards zero, an error that grows with the number of rows (operands of mean zero: 7.8e-6
// relative after about 10000) and is a bias where the operands have one sign.  So a run of MMAs covers 1024 rows; eight warps of their own then
// add its result to sums in registers (128 per thread), to nearest, while the MMAs of the next run fill the other half of tensor memory.  Relative
// error of 512 x 512 from 65536 rows, mean zero and one sign, by rows per run: 2048 4.3e-7 and 1.9e-6, 1024 2.2e-7 and 8e-7, 512 1.4e-7 and
// 3.2e-7, 256 1.2e-7 and 1.3e-7 (a sum in float32 throughout: 2e-7 and 1.7e-7); 16384 rows, 4096 x 4096: 346, 350, 364, 379 us.
//
// Decoding has to keep up with 512 clocks of MMAs per 64 x 128 codes, about 850 warp instructions.  What it took, 16384 rows, 4096 x 4096:
// 854 us with eight warps that reported every step at cluster scope, 740 at CTA scope, 557 with steps dealt out to groups of warps so that
// several are in flight, 415 with twelve warps of 40 registers beside the summing ones of 160, 390 in groups of two.  Without any decoding it
// takes 301, but twelve warps that decode also draw power: 382 us (1440 TFLOP/s) in a short burst, 465 (1180) back to back at the power limit,
// where the library's product of two bf16 matrices of this shape takes 419.  (With runs of 2048 rows; 1 % more with those of 1024.)
//
// Schedule: with P pairs resident, pair p takes the tiles p, p + P, ... as long as there is one for every pair, all of them at the same rows
// at the same time (so that L2 serves what they share); the steps of the tiles left over are dealt out evenly, tile after tile, pair p of P'
// getting [p n / P', (p + 1) n / P').  Parts of a tile go to the workspace, and a second kernel adds them in a fixed order.
#include "token.cuh"
#include "tc_ptx.cuh"
#include <algorithm>

namespace {
using namespace tc;

constexpr int kThreads = 768;        // warp 0: dy loads, 1: MMAs, 2: codes, 3: tensor memory; 4..11: sums and stores; 12..23: decoders
constexpr int kSummers = 8, kDecoders = 12;
constexpr int kGroups = 6, kGroupWarps = kDecoders / kGroups;    // every kGroups-th step is decoded by the same kGroupWarps warps
constexpr int kRegs = 80, kRegsFew = 40, kRegsSums = 160;        // registers per thread: at launch; then of the control and decoder warps, and of the summing ones
static_assert((4 + kDecoders) * kRegsFew + kSummers * kRegsSums == kThreads / 32 * kRegs, "the split is the launch's total");
constexpr int kStep = 64;            // rows per step
constexpr int kRun = 16;             // steps per run of the tensor cores' own sum
constexpr int kM = 256, kN = 256;    // output and input channels of a pair's tile, half of either in each CTA's shared memory
constexpr int kMaxPairs = 80;
constexpr int kStepsMin = 8;         // a pair's share of a tile is at least that long: shorter ones do not pay for their sums
constexpr int kSplitSteps = 32;      // tiles are cut only where that saves as many steps: parts have to be written, read and added (8192 rows, 4096 x 1024:
                                     // 78 us cut, 62 whole)
constexpr uint32_t kBlock = 64 * 128;        // bytes of 64 rows x 64 channels of bf16, the unit of both operands
constexpr int kA = 5, kB = 6, kC = 6;        // stages of the rings: dy, decoded x, codes
// A group meets every phase of the barriers that it waits on only if a stage is always the same group's: else it could take the phase before the
// one it wants, of the same parity as the one before that, for complete.
static_assert(kB % kGroups == 0 && kC % kGroups == 0, "a stage belongs to one group");
constexpr uint32_t kOperand = 2 * kBlock, kCodes = kStep * 128;
constexpr uint32_t kSmem = kA * kOperand + kB * kOperand + kC * (kCodes + kStep * 4) + 1024;
constexpr size_t kSlot = (size_t)kM * kN;    // floats of a part

struct Shared {
    uint64_t a_full[kA], a_empty[kA], b_full[kB], b_empty[kB], c_full[kC], c_empty[kC], d_full[2], d_empty[2];
    uint32_t tmem, failed;
};

struct alignas(64) Wgrad8Args {
    CUtensorMap dy, codes;
    const uint8_t *scales;
    const float *gamma;
    float *dW, *partial;
    int *status;
    int rows, cin, cout;
    int row_steps;                   // 64-row steps of one pass over the rows
    int steps;                       // of a tile: row_steps, or three times that (float32 dy as three bf16 parts)
    int tiles_c;                     // tiles along the input channels
    int pairs, waves;                // every pair takes `waves` whole tiles
    int rest, sharers;               // tiles left over, and how many pairs share their steps
    int begin[kMaxPairs + 1];        // first of the steps left over that pair q works on (below 2^31: at most 79 tiles of fewer than 3 * 2^23 steps)
    uint8_t first[kMaxPairs], last[kMaxPairs];       // of a tile left over: the pairs that work on it
    uint32_t rows_pad;
    int vec;                         // dW rows take stores of 16 bytes
};

// The pieces of work of a pair, in order; every role of both CTAs walks the same list.
struct Pieces {
    const Wgrad8Args &p;
    int pair, wave = 0;
    int from = 0, it = 0, to = 0;
    int tile, k0, k1, slot;          // steps [k0, k1) of a tile; slot: where a part of a tile goes, -1 for a whole one
    __device__ __forceinline__ Pieces(const Wgrad8Args &a, int q) : p(a), pair(q) {
        if (q < a.sharers) { from = it = a.begin[q]; to = a.begin[q + 1]; }
    }
    __device__ __forceinline__ bool next() {
        if (wave < p.waves) { tile = pair + wave++ * p.pairs; k0 = 0; k1 = p.steps; slot = -1; return true; }
        if (it >= to) return false;
        const int t = it / p.steps;
        tile = p.waves * p.pairs + t;
        k0 = it - t * p.steps;
        k1 = to - it < p.steps - k0 ? k0 + (to - it) : p.steps;
        // at most two parts per pair: the tile that its share starts in, and the one that it ends in
        slot = k0 == 0 && k1 == p.steps ? -1 : pair * 2 + (it == from ? 0 : 1);
        it += k1 - k0;
        return true;
    }
};

// bounded wait of a whole warp; false: gave up
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, uint32_t *failed) {
    const bool ok = mbar_wait(bar, parity);
    if (!ok) atomicExch(failed, 1u);
    return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// two codes (the bytes that SEL puts under a bf16 exponent of 128) -> two bf16, times a scale (twice the same bf16): exact
template <int CODE> __device__ __forceinline__ uint32_t decode2(uint32_t w, uint32_t sel, uint32_t scale2) {
    if constexpr (CODE == REVNET_INT8) {
        // 0x43 above the byte: a bf16 in [128, 256) whose last 7 bits are the code's; the sign bit alone makes it 256 = 128 + 128
        const uint32_t x = __byte_perm(w, 0x43434343u, sel);
        return mul_bf16x2(sub_bf16x2(x & 0xff7fff7fu, x & 0xff80ff80u), scale2);
    } else {
        // sign, exponent and mantissa bits moved to a bf16's places; its exponent bias is larger by 120
        const uint32_t big = (120u + 127u) << 7 | (120u + 127u) << 23;
        const uint32_t x = __byte_perm(w, 0u, sel) << 8;                 // the codes in the upper bytes
        return mul_bf16x2(mul_bf16x2((x & 0x80008000u) | ((x >> 4) & 0x07f007f0u), big), scale2);
    }
}

template <int CODE>
__global__ void __launch_bounds__(kThreads, 1) wgrad8_kernel(const __grid_constant__ Wgrad8Args p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ Shared sh;
    uint8_t *ring_a = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *ring_b = ring_a + kA * kOperand, *ring_c = ring_b + kB * kOperand;
    uint32_t *ring_s = (uint32_t *)(ring_c + kC * kCodes);
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    Pieces job(p, (int)(blockIdx.x >> 1));

    if (threadIdx.x == 0) {
        for (int i = 0; i < kA; i++) { mbar_init(&sh.a_full[i], 1); mbar_init(&sh.a_empty[i], 1); }
        for (int i = 0; i < kB; i++) { mbar_init(&sh.b_full[i], 2 * kGroupWarps); mbar_init(&sh.b_empty[i], 1); }
        for (int i = 0; i < kC; i++) { mbar_init(&sh.c_full[i], 1); mbar_init(&sh.c_empty[i], kGroupWarps); }
        for (int i = 0; i < 2; i++) { mbar_init(&sh.d_full[i], 1); mbar_init(&sh.d_empty[i], 2 * kSummers); }
        sh.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3) tmem2_alloc(&sh.tmem, 2 * kN);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    pdl_enter();
    const uint32_t tmem = sh.tmem;

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
    }
    if (warp == 0) {
        const uint32_t full0 = mapa_shared(smem_u32(&sh.a_full[0]), 0);
        int s = 0; uint32_t round = 0;
        bool ok = true;
        while (ok && job.next()) {
            const int o0 = (job.tile / p.tiles_c) * kM + (int)rank * 128;
            for (int k = job.k0; k < job.k1; k++) {
                if (round > 0 && !(ok = warp_wait(&sh.a_empty[s], (round - 1) & 1, &sh.failed))) break;
                if (elect_one()) {
                    if (rank == 0) mbar_expect_tx(&sh.a_full[s], 2 * kOperand);      // the leader's barrier counts the bytes of both CTAs
                    tma2_load_2d(ring_a + s * kOperand, &p.dy, full0 + 8u * s, o0, k * kStep);
                    tma2_load_2d(ring_a + s * kOperand + kBlock, &p.dy, full0 + 8u * s, o0 + 64, k * kStep);
                }
                __syncwarp();
                if (++s == kA) { s = 0; round++; }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = instr_desc_m256(kN) | (3u << 15);     // both operands M / N-major
            const uint64_t da0 = smem_desc_mn(smem_u32(ring_a), 128, kBlock), db0 = smem_desc_mn(smem_u32(ring_b), 128, kBlock);
            int sa = 0, sb = 0; uint32_t ra = 0, rb = 0, run = 0;
            bool ok = true;
            while (ok && job.next()) {
                for (int k = job.k0; k < job.k1 && ok; run++) {
                    const int end = k + kRun < job.k1 ? k + kRun : job.k1;
                    if (run > 1) ok = mbar_wait(&sh.d_empty[run & 1], ((run >> 1) - 1) & 1);
                    tc_fence_after();
                    const uint32_t acc = tmem + (run & 1) * kN;
                    for (bool first = true; k < end && ok; k++) {
                        ok = mbar_wait(&sh.a_full[sa], ra & 1) && mbar_wait(&sh.b_full[sb], rb & 1);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t da = da0 + (uint32_t)sa * (kOperand >> 4), db = db0 + (uint32_t)sb * (kOperand >> 4);
#pragma unroll
                        for (int ks = 0; ks < kStep / 16; ks++)          // 16 rows of 128 bytes per MMA
                            mma2_bf16(acc, da + (uint32_t)ks * 128u, db + (uint32_t)ks * 128u, idesc, first && ks == 0 ? 0u : 1u);
                        first = false;
                        mma2_commit_both(&sh.a_empty[sa]);
                        mma2_commit_both(&sh.b_empty[sb]);
                        if (++sa == kA) { sa = 0; ra++; }
                        if (++sb == kB) { sb = 0; rb++; }
                    }
                    mma2_commit_both(&sh.d_full[run & 1]);
                }
            }
            if (!ok) atomicExch(&sh.failed, 1u);
        }
    } else if (warp == 2) {
        int s = 0; uint32_t round = 0;
        bool ok = true;
        while (ok && job.next()) {
            const int c0 = (job.tile % p.tiles_c) * kN + (int)rank * 128;
            const bool in = c0 < p.cin;              // a CTA whose half of the tile lies behind the last channel has no scales to read
            int t = job.k0 % p.row_steps;
            for (int k = job.k0; k < job.k1; k++) {
                if (round > 0 && !(ok = warp_wait(&sh.c_empty[s], (round - 1) & 1, &sh.failed))) break;
                if (elect_one()) {
                    mbar_expect_tx(&sh.c_full[s], kCodes + (in ? kStep * 4 : 0));
                    tma_load_2d(ring_c + s * kCodes, &p.codes, &sh.c_full[s], c0, t * kStep);
                    if (in) bulk_load(ring_s + s * kStep, p.scales + ((size_t)(c0 >> 7) * p.rows_pad + (size_t)t * kStep) * 4, kStep * 4, &sh.c_full[s]);
                }
                __syncwarp();
                if (++t == p.row_steps) t = 0;
                if (++s == kC) { s = 0; round++; }
            }
        }
    } else if (warp >= 4 && warp < 4 + kSummers) {
        // sums: a warp holds 32 of the CTA's 128 output channels (its quarter of tensor memory) x 128 of the 256 input channels
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSums));
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t tmem_mine = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128);
        const uint32_t d_empty0 = mapa_shared(smem_u32(&sh.d_empty[0]), 0);
        uint32_t run = 0;
        bool ok = true;
        float sum[128];
        while (ok && job.next()) {
#pragma unroll
            for (int i = 0; i < 128; i++) sum[i] = 0.f;
            for (int k = job.k0; k < job.k1; k += kRun, run++) {
                const uint32_t buf = run & 1;
                if (!(ok = warp_wait(&sh.d_full[buf], (run >> 1) & 1, &sh.failed))) break;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < 128; c += 8) {
                    float v[8];
                    tmem_ld8(tmem_mine + buf * kN + c, v);
#pragma unroll
                    for (int i = 0; i < 8; i++) sum[c + i] += v[i];
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(d_empty0 + 8u * buf);
            }
            const int r = (int)rank * 128 + quarter * 32 + lane, o = (job.tile / p.tiles_c) * kM + r;
            const int c0 = (job.tile % p.tiles_c) * kN + half * 128;
            if (job.slot >= 0) {
                // a part: [column quad][row][4], so that a warp's 32 rows are one run of 512 bytes
                const int left = ok && o < p.cout ? p.cin - c0 : 0;
                float4 *part = reinterpret_cast<float4 *>(p.partial + (size_t)job.slot * kSlot) + (size_t)half * 32 * kM + r;
#pragma unroll
                for (int i = 0; i < 128; i += 4)
                    if (i < left) part[(size_t)(i / 4) * kM] = make_float4(sum[i], sum[i + 1], sum[i + 2], sum[i + 3]);
                continue;
            }
            // a tile: 32 x 32 squares transposed in registers, so that a store is 128 consecutive bytes of a row, whatever the row's alignment (24 rows,
            // 1682 x 3709: 180 us with every lane writing its own row)
            if (!ok) break;
            const int rows = p.cout - (o - lane);
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
                if (c0 + c >= p.cin || rows <= 0) break;                 // the same for the whole warp
#pragma unroll
                for (int s = 16; s; s >>= 1)
#pragma unroll
                    for (int j = 0; j < 32; j++)
                        if ((j & s) == 0) {
                            const bool up = (lane & s) != 0;
                            const float got = __shfl_xor_sync(0xffffffffu, up ? sum[c + j] : sum[c + j + s], s);
                            if (up) sum[c + j] = got; else sum[c + j + s] = got;
                        }
                if (c + lane < p.cin - c0) {
                    const float g = p.gamma ? p.gamma[c0 + c + lane] : 1.f;
                    float *out = p.dW + (size_t)(o - lane) * p.cin + c0 + c + lane;
#pragma unroll
                    for (int j = 0; j < 32; j++)
                        if (j < rows) out[(size_t)j * p.cin] = sum[c + j] * g;
                }
            }
        }
    } else if (warp >= 4 + kSummers) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
        const int d = warp - 4 - kSummers;
        // a step's 64 rows x 4 blocks of 32 channels: `sub` is half a column of them (32 rows, one per lane)
        const int group = d / kGroupWarps, sub0 = d % kGroupWarps;
        const uint32_t b_full0 = mapa_shared(smem_u32(&sh.b_full[0]), 0);
        const uint32_t x7 = (uint32_t)lane & 7;
        int sb = 0, sc = 0, turn = 0; uint32_t rb = 0, rc = 0;
        bool ok = true;
        while (ok && job.next()) {
            int row = (job.k0 % p.row_steps) * kStep;
            const int c0 = (job.tile % p.tiles_c) * kN + (int)rank * 128;
            for (int k = job.k0; k < job.k1; k++) {
                if (turn == group) {
                    if (!(ok = warp_wait(&sh.c_full[sc], rc & 1, &sh.failed))) break;
                    if (rb > 0 && !(ok = warp_wait(&sh.b_empty[sb], (rb - 1) & 1, &sh.failed))) break;
                    const uint8_t *src = ring_c + sc * kCodes;
                    uint8_t *dst = ring_b + sb * kOperand;
#pragma unroll
                    for (int i = 0; i < 8 / kGroupWarps; i++) {
                        const int sub = sub0 + i * kGroupWarps;
                        const uint32_t t = (uint32_t)((sub & 1) * 32 + lane), blk = (uint32_t)sub >> 1;
                        // eight neighbouring lanes have eight rows of different index mod 8, so both swizzles spread them over all banks
                        const uint4 q0 = *reinterpret_cast<const uint4 *>(src + t * 128 + (((2 * blk) ^ x7) << 4));
                        const uint4 q1 = *reinterpret_cast<const uint4 *>(src + t * 128 + (((2 * blk + 1) ^ x7) << 4));
                        // rows behind the last have codes 0 (the load fills them in) and no scale, channels behind the last likewise
                        uint32_t byte = (ring_s[sc * kStep + t] >> (8 * blk)) & 0xffu;
                        if (row + (int)t >= p.rows || c0 + (int)blk * 32 >= p.cin) byte = 127u;
                        const uint32_t scale2 = byte << 7 | byte << 23;
                        const uint32_t w[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
                        uint8_t *out = dst + (blk >> 1) * kBlock + t * 128;
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            *reinterpret_cast<uint4 *>(out + ((((blk & 1) * 4 + e) ^ x7) << 4)) =
                                make_uint4(decode2<CODE>(w[2 * e], 0x4140, scale2), decode2<CODE>(w[2 * e], 0x4342, scale2),
                                           decode2<CODE>(w[2 * e + 1], 0x4140, scale2), decode2<CODE>(w[2 * e + 1], 0x4342, scale2));
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(&sh.c_empty[sc]); mbar_arrive_remote(b_full0 + 8u * sb); }
                }
                if (++turn == kGroups) turn = 0;
                if (++sc == kC) { sc = 0; rc++; }
                if (++sb == kB) { sb = 0; rb++; }
                row += kStep;
                if (row >= p.row_steps * kStep) row = 0;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (sh.failed) {
        // a wait ran out: copies may still be on their way into this CTA's shared memory, which nothing waits for any more; 2 ms is ample
        if (threadIdx.x == 0) {
            atomicExch(p.status, (int)REVNET_E_TIMEOUT);
            for (int i = 0; i < 2000; i++) __nanosleep(1000);
        }
        __syncthreads();
    }
    cluster_sync_all();      // neither CTA leaves, or frees tensor memory, while the other may still read its operands
    if (warp == 3) {
        tc_fence_after();
        tmem2_dealloc(tmem, 2 * kN);
    }
}

// dW of the tiles that several pairs have worked on: the parts in a fixed order.  A CTA takes 8 rows x QUADS * 4 columns; LANES threads per quad
// add every LANES-th part (and one of them then their sums), which a tile cut into many parts needs: 16384 rows, 256 x 256, 74 parts: 57 us with one.
template <int LANES, int QUADS> __global__ void __launch_bounds__(8 * QUADS * LANES) wgrad8_sum_kernel(const __grid_constant__ Wgrad8Args p) {
    __shared__ float4 sm[LANES == 1 ? 1 : LANES][8 * QUADS];
    pdl_enter();
    constexpr int kPer = (kM / 8) * (kN / 4 / QUADS);                    // CTAs per tile
    const int t = (int)blockIdx.x / kPer, within = (int)blockIdx.x % kPer, tile = p.waves * p.pairs + t;
    const int first = p.first[t], last = p.last[t];
    if (first == last) return;                                           // one pair: the tile is there already
    const int item = (int)threadIdx.x % (8 * QUADS), lane = (int)threadIdx.x / (8 * QUADS);
    const int r = (within % (kM / 8)) * 8 + (item & 7), c = (within / (kM / 8)) * QUADS + (item >> 3);
    const int o = (tile / p.tiles_c) * kM + r, ch = (tile % p.tiles_c) * kN + 4 * c, left = o < p.cout ? p.cin - ch : 0;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (left > 0) {
#pragma unroll 4
        for (int q = first + lane; q <= last; q += LANES) {
            // the first pair's share may have begun before this tile: it is then the second part of that pair
            const size_t slot = (size_t)q * 2 + (q > first || p.begin[q] >= t * p.steps ? 0 : 1);
            const float4 v = reinterpret_cast<const float4 *>(p.partial + slot * kSlot)[(size_t)c * kM + r];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    if constexpr (LANES > 1) {
        sm[lane][item] = s;
        __syncthreads();
        if (lane) return;
#pragma unroll
        for (int l = 1; l < LANES; l++) { const float4 v = sm[l][item]; s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w; }
    }
    if (left <= 0) return;
    float *out = p.dW + (size_t)o * p.cin + ch;
    if (p.gamma) {
        const float *g = p.gamma + ch;
        s.x *= g[0];
        if (left > 1) s.y *= g[1];
        if (left > 2) s.z *= g[2];
        if (left > 3) s.w *= g[3];
    }
    if (left > 3 && p.vec) *reinterpret_cast<float4 *>(out) = s;
    else { out[0] = s.x; if (left > 1) out[1] = s.y; if (left > 2) out[2] = s.z; if (left > 3) out[3] = s.w; }
}
template <int LANES, int QUADS> void sum_t(Exec &ex, const Wgrad8Args &a) {
    launch(ex, wgrad8_sum_kernel<LANES, QUADS>, (unsigned)a.rest * (kM / 8) * (kN / 4 / QUADS), 8 * QUADS * LANES, 0, a);
}

// dy for the loads: rows of `pitch` bf16 on 16-byte boundaries.  float32 becomes three parts, the bits of a value 8 at a time: their sum is the
// value (infinities and NaN stay in the upper one).  The lowest part comes first: the tensor cores cut small products off at the last bits of
// the sum that they are added to, which should be small then (330 rows: error 1.7e-6 with the upper part first).  Rows of the last step behind the last one are zeros between the parts.
template <class T> __global__ void __launch_bounds__(256) wgrad8_prepare_kernel(const T *dy, int64_t ld, bool aligned, bf16 *out, int rows, int rows_step, int cout, int pitch, FastDiv groups) {
    pdl_enter();
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= (uint32_t)rows_step * groups.d) return;                     // (below 2^31, see the entry point)
    uint32_t row, g;
    groups.divmod(i, row, g);
    const int ch = (int)g * 8, n = row < (uint32_t)rows ? min(8, cout - ch) : 0;
    const T *src = dy + (size_t)row * ld + ch;
    float v[8];
    if constexpr (sizeof(T) == 4) {
        if (n == 8 && aligned) {
            const float4 a = reinterpret_cast<const float4 *>(src)[0], b = reinterpret_cast<const float4 *>(src)[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = j < n ? to_f(src[j]) : 0.f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = j < n ? to_f(src[j]) : 0.f;
    }
    for (int part = 0; part < (sizeof(T) == 4 ? 3 : 1); part++) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            uint32_t b = __float_as_uint(v[j]);
            const bool finite = (b & 0x7f800000u) != 0x7f800000u;
            if ((b & 0x7fffffffu) > 0x7f800000u) b |= 0x00400000u;       // a NaN whose payload lies in the low half stays one
            b &= 0xffff0000u;
            v[j] = finite ? v[j] - __uint_as_float(b) : 0.f;
            if (j & 1) w[j >> 1] |= b; else w[j >> 1] = b >> 16;
        }
        *reinterpret_cast<uint4 *>(out + ((size_t)(sizeof(T) == 4 ? 2 - part : 0) * rows_step + row) * pitch + ch) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

struct Plan {
    int row_steps, steps, tiles_c, tiles, pairs, waves, rest, sharers;
    int pitch;                       // elements per row of the prepared dy
    size_t prepared_bytes, partial_bytes;
};
// whether the loads can take dy from where it is (the entry point sees to its address)
bool direct(const revnet_wgrad_desc &d) { return d.dy_dtype == REVNET_BF16 && d.ld_dy % 8 == 0; }
Plan plan_of(const revnet_ctx *ctx, const revnet_wgrad_desc &d, bool prepared) {
    Plan w{};
    w.row_steps = (int)((d.rows + kStep - 1) / kStep);
    w.steps = w.row_steps * (d.dy_dtype == REVNET_F32 ? 3 : 1);
    w.tiles_c = (d.cin + kN - 1) / kN;
    w.tiles = w.tiles_c * ((d.cout + kM - 1) / kM);
    const int most = ctx->sm_count / 2 < kMaxPairs ? ctx->sm_count / 2 : kMaxPairs;
    // a pair for every kStepsMin steps, and for every tile however short
    auto sharers_of = [&](int64_t tiles) { const int64_t q = std::max(tiles, (tiles * w.steps + kStepsMin - 1) / kStepsMin); return (int)std::min<int64_t>(w.steps ? q : 0, most); };
    w.pairs = sharers_of(w.tiles);
    if (w.tiles < w.pairs && w.steps - (int64_t)w.tiles * w.steps / w.pairs < kSplitSteps) w.pairs = w.tiles;
    w.waves = w.pairs ? w.tiles / w.pairs : 0;
    w.rest = w.tiles - w.waves * w.pairs;
    w.sharers = sharers_of(w.rest);
    if (w.rest && w.steps - (int64_t)w.rest * w.steps / w.sharers < kSplitSteps) w.sharers = w.rest;         // one more round of whole tiles
    // the same number of pairs for every tile where that leaves few of them idle: no pair then has two parts to add and store
    else if (w.rest && w.sharers / w.rest * w.rest >= w.sharers * 85 / 100) w.sharers -= w.sharers % w.rest;
    w.pitch = (d.cout + 7) & ~7;
    w.prepared_bytes = prepared ? ((size_t)w.steps * kStep * w.pitch * 2 + 255) & ~size_t(255) : 0;
    w.partial_bytes = w.rest == 0 || w.rest % w.sharers == 0 ? 0 : (size_t)w.sharers * 2 * kSlot * 4;        // (a multiple: whole tiles for all of them)
    return w;
}

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                             const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
bool encode_2d(void *fn, CUtensorMap *map, CUtensorMapDataType type, const void *base, uint64_t inner, uint64_t outer, uint64_t stride, uint32_t box_inner) {
    cuuint64_t dims[2] = {inner, outer}, strides[1] = {stride};
    cuuint32_t box[2] = {box_inner, (cuuint32_t)kStep}, es[2] = {1, 1};
    return fn && ((EncodeFn)fn)(map, type, 2, (void *)base, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CODE> void run_t(Exec &ex, const Wgrad8Args &a, double bytes, double flops) {
    static OncePerDevice once;
    if (!shared_limit(once, ex.ctx->device, kSmem, wgrad8_kernel<CODE>)) { ex.check("wgrad8"); return; }
    // the split of the registers adds up to what a launch gets with kRegs per thread, no more: a kernel built with fewer would wait for ever
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, wgrad8_kernel<CODE>) != cudaSuccess || attr.numRegs != kRegs) {
        cudaGetLastError();
        ex.failed = true; ex.ctx->err = "revnet_linear_wgrad: the kernel was built with another number of registers";
        return;
    }
    launch_cluster(ex, wgrad8_kernel<CODE>, (unsigned)a.pairs * 2, kThreads, kSmem, 2, a);
    ex.check("wgrad8", bytes, flops);
}

}  // namespace

size_t wgrad8_workspace(const revnet_ctx *ctx, const revnet_wgrad_desc &d) {
    const Plan w = plan_of(ctx, d, !direct(d));
    return w.prepared_bytes + w.partial_bytes + 256;
}

void wgrad8(Exec &ex, const revnet_wgrad_desc &d, const void *dy, const void *ck, const float *gamma, float *dW, char *workspace) {
    if (d.rows == 0) { fill_zero(ex, dW, (size_t)d.cin * d.cout * 4); return; }
    const bool prepared = !direct(d);
    const Plan w = plan_of(ex.ctx, d, prepared);
    const Checkpoint c = ck_view(ck, d.rows, d.cin);
    Wgrad8Args a{};
    a.scales = c.scales; a.gamma = gamma; a.dW = dW; a.partial = (float *)(workspace + w.prepared_bytes); a.status = ex.ctx->dev_status;
    a.rows = (int)d.rows; a.cin = d.cin; a.cout = d.cout; a.row_steps = w.row_steps; a.steps = w.steps; a.tiles_c = w.tiles_c;
    a.pairs = w.pairs; a.waves = w.waves; a.rest = w.rest; a.sharers = w.sharers; a.rows_pad = c.rows_pad; a.vec = d.cin % 4 == 0;        // (dW itself is on 16 bytes)
    for (int q = 0; q <= w.sharers; q++) a.begin[q] = w.sharers ? (int)((int64_t)w.rest * w.steps * q / w.sharers) : 0;
    for (int t = 0, q = 0; t < w.rest; t++) {
        while (a.begin[q + 1] <= t * w.steps) q++;
        a.first[t] = (uint8_t)q;
        while (a.begin[q + 1] < (t + 1) * w.steps) q++;
        a.last[t] = (uint8_t)q;
    }
    const int rows_step = w.row_steps * kStep;
    if (prepared) {
        const uint32_t groups = (uint32_t)w.pitch / 8;
        const unsigned grid = (unsigned)(((uint64_t)rows_step * groups + 255) / 256);
        const double bytes = (double)d.rows * d.cout * (d.dy_dtype == REVNET_F32 ? 10 : 4);
        if (d.dy_dtype == REVNET_F32)
            launch_stream(ex, bytes, 0, wgrad8_prepare_kernel<float>, grid, 256, 0, (const float *)dy, d.ld_dy, row_access(dy, d.ld_dy, 4, 4) > 0, (bf16 *)workspace, a.rows, rows_step, d.cout, w.pitch, fast_div(groups));
        else
            launch_stream(ex, bytes, 0, wgrad8_prepare_kernel<bf16>, grid, 256, 0, (const bf16 *)dy, d.ld_dy, false, (bf16 *)workspace, a.rows, rows_step, d.cout, w.pitch, fast_div(groups));
        ex.check("wgrad8_prepare", bytes);
    }
    void *enc = tc_encoder(ex.ctx);
    const uint64_t dy_rows = prepared ? (uint64_t)w.steps * kStep : (uint64_t)d.rows;
    if (!encode_2d(enc, &a.dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, prepared ? workspace : dy, (uint64_t)d.cout, dy_rows, (prepared ? (uint64_t)w.pitch : (uint64_t)d.ld_dy) * 2, 64) ||
        !encode_2d(enc, &a.codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, c.codes, (uint64_t)c.pitch, (uint64_t)d.rows, (uint64_t)c.pitch, 128)) {
        ex.failed = true; ex.ctx->err = "revnet_linear_wgrad: tensor map rejected";
        return;
    }
    const double bytes = (double)d.rows * (2.0 * d.cout * (w.steps / w.row_steps) + d.cin) + 4.0 * d.cin * d.cout, flops = 2.0 * w.steps * kStep * d.cin * d.cout;
    if (d.code == REVNET_INT8) run_t<REVNET_INT8>(ex, a, bytes, flops);
    else run_t<REVNET_E4M3>(ex, a, bytes, flops);
    if (w.partial_bytes && !ex.failed) {
        if (w.sharers > 16 * w.rest) sum_t<16, 4>(ex, a);
        else if (w.sharers > 3 * w.rest) sum_t<4, 8>(ex, a);
        else sum_t<1, 32>(ex, a);
        ex.check("wgrad8_sum", (double)w.partial_bytes);
    }
}
