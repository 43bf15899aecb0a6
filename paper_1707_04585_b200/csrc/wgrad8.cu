// Weight gradient of a linear layer from an 8-bit checkpoint of its input: dW[o][c] = gamma[c] sum_t dy[t][o] x8[t][c].
//
// A matrix product over the rows t, both operands with t as the outer index, on the 5th-generation tensor cores as CTA pairs
// (tcgen05 cta_group::2).  The values of a checkpoint are bf16 numbers, so a tile of codes becomes an MMA operand without rounding:
//
//   dy     TMA -> shared memory, 64 rows x 64 channels per box, 128-byte swizzle, M-major: the A operand as it lies
//   codes  TMA -> shared memory (64 rows x 128 channels) -> eight decoder warps -> bf16 in the same swizzled layout: the B operand
//   D      512 (or 256) output channels x 256 input channels of fp32 in the pair's tensor memory
//
// What bounds it: shared memory and the tensor pipe about equally.  Decoding is on the side of N because an MMA of the pair reuses a
// decoded element for all its 512 rows: per 64 rows a CTA loads 32 KB of dy and 8 KB of codes and decodes 8192 values for 1024 clocks
// of MMAs.  (With x on the side of M it would decode twice as many, and shared memory would carry 144 bytes per clock, of 128.)
//
// The products of a tile (over all rows) are one after another and the tiles are cut where the pairs' shares end: pair p of P works on
// steps [p n / P, (p + 1) n / P) of the n = tiles x (64-row steps), so every SM is busy to the end for any shape.  A tile that one pair
// finishes goes straight to dW; parts of a tile go to the workspace, and a second kernel adds them in a fixed order.
#include "token.cuh"
#include "tc_ptx.cuh"

namespace {
using namespace tc;

constexpr int kThreads = 384;        // warp 0: dy loads, 1: MMAs, 2: codes, 3: tensor memory; 4..11: decoders, which also store the tiles
constexpr int kDecoders = 8;
constexpr int kStep = 64;            // rows per step
constexpr int kN = 256;              // input channels of a pair's tile, half of them per CTA
constexpr int kStepsMin = 8;         // a pair's share is at least that long where the work allows: shorter ones do not pay for their sums
constexpr uint32_t kBlock = 64 * 128;        // bytes of 64 rows x 64 channels of bf16, the unit of both operands

template <int GM> struct Tile {      // GM: groups of 128 output channels per CTA; a pair's tile has 256 GM of them
    static constexpr int kA = GM == 2 ? 4 : 5, kB = GM == 2 ? 3 : 4, kC = GM == 2 ? 3 : 4;      // stages of the rings
    static constexpr uint32_t kAStage = GM * 2 * kBlock, kBStage = 2 * kBlock, kCStage = kStep * 128;
    static constexpr uint32_t kSmem = kA * kAStage + kB * kBStage + kC * (kCStage + kStep * 4) + 1024;
};
struct Shared {
    uint64_t a_full[8], a_empty[8], b_full[8], b_empty[8], c_full[8], c_empty[8], d_full, d_empty;
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
    int tiles_c, tiles;              // tiles along the input channels; in all
    int pairs;
    uint32_t rows_pad;
    int vec;                         // dW rows take 16-byte stores
};
// first step of a pair's share
__host__ __device__ __forceinline__ int64_t share(int64_t n, int p, int pairs) { return n * p / pairs; }
// A part of a tile: where its partial sums go.  A pair has at most two parts that are not whole tiles: the one its share starts in and the one
// it ends in.
__device__ __forceinline__ size_t slot_floats(int gm) { return (size_t)gm * 256 * kN; }

// bounded wait by one lane for its warp; false: gave up, or somebody else in the CTA did
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, uint32_t *failed, bool cluster) {
    bool ok = true;
    if ((threadIdx.x & 31) == 0) {
        ok = cluster ? mbar_wait_cluster(bar, parity) : mbar_wait(bar, parity);
        if (!ok) atomicExch(failed, 1u);
    }
    return __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
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
// four codes -> four bf16, times a scale (twice the same bf16): exact
template <int CODE> __device__ __forceinline__ uint2 decode4(uint32_t w, uint32_t scale2) {
    if constexpr (CODE == REVNET_INT8) {
        const uint32_t u = w ^ 0x80808080u;
        float f[4];
#pragma unroll
        for (int j = 0; j < 4; j++) f[j] = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 + j)) - 8388736.f;
        return make_uint2(mul_bf16x2(bf16_pair(f[0], f[1]), scale2), mul_bf16x2(bf16_pair(f[2], f[3]), scale2));
    } else {
        // sign, exponent and mantissa bits in a bf16's places; its exponent bias is larger by 120
        const uint32_t big = (120u + 127u) << 7 | (120u + 127u) << 23;
        const uint32_t lo = __byte_perm(w, 0u, 0x1404), hi = __byte_perm(w, 0u, 0x3424);        // codes in the upper bytes
        const uint32_t l = (lo & 0x80008000u) | ((lo >> 4) & 0x07f007f0u), h = (hi & 0x80008000u) | ((hi >> 4) & 0x07f007f0u);
        return make_uint2(mul_bf16x2(mul_bf16x2(l, big), scale2), mul_bf16x2(mul_bf16x2(h, big), scale2));
    }
}

template <int GM, int CODE>
__global__ void __launch_bounds__(kThreads, 1) wgrad8_kernel(const __grid_constant__ Wgrad8Args p) {
    using T = Tile<GM>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Shared sh;
    uint8_t *ring_a = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *ring_b = ring_a + T::kA * T::kAStage, *ring_c = ring_b + T::kB * T::kBStage;
    uint32_t *ring_s = (uint32_t *)(ring_c + T::kC * T::kCStage);
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = (int)(blockIdx.x >> 1);
    constexpr uint32_t kCols = GM * kN;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 8; i++) {
            mbar_init(&sh.a_full[i], 1); mbar_init(&sh.a_empty[i], 1);
            mbar_init(&sh.b_full[i], 2 * kDecoders); mbar_init(&sh.b_empty[i], 1);
            mbar_init(&sh.c_full[i], 1); mbar_init(&sh.c_empty[i], kDecoders);
        }
        mbar_init(&sh.d_full, 1); mbar_init(&sh.d_empty, 2 * kDecoders);
        sh.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3) tmem2_alloc(&sh.tmem, kCols);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    pdl_enter();
    const uint32_t tmem = sh.tmem;
    const int64_t n = (int64_t)p.tiles * p.steps, from = share(n, pair, p.pairs), to = share(n, pair + 1, p.pairs);

    // every role walks the same list of (tile, steps k0 .. k1)
    if (warp == 0) {
        const uint32_t full0 = mapa_shared(smem_u32(&sh.a_full[0]), 0);
        int s = 0; uint32_t round = 0;
        bool ok = true;
        for (int64_t it = from; it < to && ok; it++) {
            const int tile = (int)(it / p.steps), k = (int)(it - (int64_t)tile * p.steps);
            const int o0 = (tile / p.tiles_c) * 256 * GM + (int)rank * 128;
            if (round > 0) ok = warp_wait(&sh.a_empty[s], (round - 1) & 1, &sh.failed, true);
            if (!ok) break;
            if (elect_one()) {
                if (rank == 0) mbar_expect_tx(&sh.a_full[s], 2 * T::kAStage);        // the leader's barrier counts the bytes of both CTAs
#pragma unroll
                for (int g = 0; g < GM; g++)
#pragma unroll
                    for (int b = 0; b < 2; b++)
                        tma2_load_2d(ring_a + s * T::kAStage + (g * 2 + b) * kBlock, &p.dy, full0 + 8u * s, o0 + g * 256 + b * 64, k * kStep);
            }
            __syncwarp();
            if (++s == T::kA) { s = 0; round++; }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = instr_desc_m256(kN) | (3u << 15);     // both operands M / N-major
            const uint64_t da0 = smem_desc_mn(smem_u32(ring_a), 128, kBlock), db0 = smem_desc_mn(smem_u32(ring_b), 128, kBlock);
            int sa = 0, sb = 0; uint32_t ra = 0, rb = 0, tiles_done = 0;
            bool ok = true;
            for (int64_t it = from; it < to && ok;) {
                const int tile = (int)(it / p.steps);
                const int64_t tile_end = (int64_t)(tile + 1) * p.steps, end = tile_end < to ? tile_end : to;
                if (tiles_done > 0) ok = mbar_wait_cluster(&sh.d_empty, (tiles_done - 1) & 1);
                tc_fence_after();
                for (bool first = true; it < end && ok; it++) {
                    ok = mbar_wait_cluster(&sh.a_full[sa], ra & 1) && mbar_wait_cluster(&sh.b_full[sb], rb & 1);
                    if (!ok) break;
                    tc_fence_after();
                    uint64_t db = db0 + (uint32_t)sb * (T::kBStage >> 4);
#pragma unroll
                    for (int g = 0; g < GM; g++) {
                        uint64_t da = da0 + (uint32_t)sa * (T::kAStage >> 4) + (uint32_t)g * (2 * kBlock >> 4);
#pragma unroll
                        for (int ks = 0; ks < kStep / 16; ks++)          // 16 rows of 128 bytes per MMA
                            mma2_bf16(tmem + (uint32_t)(g * kN), da + (uint32_t)ks * 128u, db + (uint32_t)ks * 128u, idesc, first && ks == 0 ? 0u : 1u);
                    }
                    first = false;
                    mma2_commit_both(&sh.a_empty[sa]);
                    mma2_commit_both(&sh.b_empty[sb]);
                    if (++sa == T::kA) { sa = 0; ra++; }
                    if (++sb == T::kB) { sb = 0; rb++; }
                }
                mma2_commit_both(&sh.d_full);
                tiles_done++;
            }
            if (!ok) atomicExch(&sh.failed, 1u);
        }
    } else if (warp == 2) {
        int s = 0; uint32_t round = 0;
        bool ok = true;
        for (int64_t it = from; it < to && ok; it++) {
            const int tile = (int)(it / p.steps), t0 = (int)((it - (int64_t)tile * p.steps) % p.row_steps) * kStep;
            const int c0 = (tile % p.tiles_c) * kN + (int)rank * 128;
            if (round > 0) ok = warp_wait(&sh.c_empty[s], (round - 1) & 1, &sh.failed, false);
            if (!ok) break;
            if (elect_one()) {
                const bool in = c0 < p.cin;          // a CTA whose half of the tile lies behind the last channel has no scales to read
                mbar_expect_tx(&sh.c_full[s], T::kCStage + (in ? kStep * 4 : 0));
                tma_load_2d(ring_c + s * T::kCStage, &p.codes, &sh.c_full[s], c0, t0);
                if (in) bulk_load(ring_s + s * kStep, p.scales + ((size_t)(c0 >> 7) * p.rows_pad + t0) * 4, kStep * 4, &sh.c_full[s]);
            }
            __syncwarp();
            if (++s == T::kC) { s = 0; round++; }
        }
    } else if (warp >= 4) {
        const int d = warp - 4;
        const uint32_t t = (uint32_t)((d & 1) * 32 + lane), blk = (uint32_t)d >> 1;       // this thread's row of a step, and its 32 channels
        // eight neighbouring lanes have eight rows of different index mod 8, so both swizzles spread them over all banks
        const uint32_t src0 = t * 128 + (((2 * blk) ^ (t & 7)) << 4), src1 = t * 128 + (((2 * blk + 1) ^ (t & 7)) << 4);
        const uint32_t dst_block = (blk >> 1) * kBlock + t * 128;
        const uint32_t b_full0 = mapa_shared(smem_u32(&sh.b_full[0]), 0), d_empty0 = mapa_shared(smem_u32(&sh.d_empty), 0);
        int sb = 0, sc = 0; uint32_t rb = 0, rc = 0, tiles_done = 0;
        bool ok = true;
        for (int64_t it = from; it < to && ok;) {
            const int tile = (int)(it / p.steps), k0 = (int)(it - (int64_t)tile * p.steps);
            const int64_t tile_end = (int64_t)(tile + 1) * p.steps, end = tile_end < to ? tile_end : to;
            const bool whole = k0 == 0 && end == tile_end;
            const size_t slot = (size_t)pair * 2 + (it == from ? 0 : 1);
            const int c0 = (tile % p.tiles_c) * kN, o0 = (tile / p.tiles_c) * 256 * GM;
            for (int k = k0; it < end; it++, k++) {
                const int row = (k % p.row_steps) * kStep + (int)t;
                ok = warp_wait(&sh.c_full[sc], rc & 1, &sh.failed, false);
                if (!ok) break;
                const uint4 q0 = *reinterpret_cast<const uint4 *>(ring_c + sc * T::kCStage + src0), q1 = *reinterpret_cast<const uint4 *>(ring_c + sc * T::kCStage + src1);
                // rows behind the last have codes 0 (the load fills them in) and no scale, channels behind the last likewise
                uint32_t byte = (ring_s[sc * kStep + t] >> (8 * blk)) & 0xffu;
                if (row >= p.rows || c0 + (int)rank * 128 + (int)blk * 32 >= p.cin) byte = 127u;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.c_empty[sc]);
                if (rb > 0) ok = warp_wait(&sh.b_empty[sb], (rb - 1) & 1, &sh.failed, true);
                if (!ok) break;
                const uint32_t scale2 = byte << 7 | byte << 23;
                uint8_t *dst = ring_b + sb * T::kBStage + dst_block;
                const uint32_t w[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const uint2 a = decode4<CODE>(w[2 * j], scale2), b = decode4<CODE>(w[2 * j + 1], scale2);
                    *reinterpret_cast<uint4 *>(dst + ((((blk & 1) * 4 + j) ^ (t & 7)) << 4)) = make_uint4(a.x, a.y, b.x, b.y);
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(b_full0 + 8u * sb);
                if (++sc == T::kC) { sc = 0; rc++; }
                if (++sb == T::kB) { sb = 0; rb++; }
            }
            if (!ok) break;
            // the tile, or this pair's part of it: warp = 32 rows of output channels, every other 32 columns
            ok = warp_wait(&sh.d_full, tiles_done & 1, &sh.failed, true);
            if (!ok) break;
            tc_fence_after();
            const int quarter = warp & 3;
#pragma unroll 1
            for (int g = 0; g < GM; g++) {
                const int r = g * 256 + (int)rank * 128 + quarter * 32 + lane, o = o0 + r;
                float *out = whole ? p.dW + (size_t)o * p.cin + c0 : p.partial + slot * slot_floats(GM) + (size_t)r * kN;
#pragma unroll 1
                for (int c = (d >> 2) * 16; c < kN; c += 32) {
                    if (c0 + c >= p.cin) break;                          // the same for the whole warp
                    float v[16];
                    tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(g * kN + c), v);
                    if (o >= p.cout) continue;
                    const int left = p.cin - c0 - c;
                    if (whole && p.gamma) {
#pragma unroll
                        for (int i = 0; i < 16; i++) if (i < left) v[i] *= p.gamma[c0 + c + i];
                    }
                    if (left >= 16 && (!whole || p.vec)) {
#pragma unroll
                        for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4 *>(out + c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; i++) if (i < left) out[c + i] = v[i];
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(d_empty0);
            tiles_done++;
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
        tmem2_dealloc(tmem, kCols);
    }
}

// dW of the tiles that several pairs have worked on: the parts in the order of their rows.  One CTA per 16 rows of a tile.
template <int GM> __global__ void __launch_bounds__(256) wgrad8_sum_kernel(const __grid_constant__ Wgrad8Args p) {
    pdl_enter();
    const int tile = (int)blockIdx.x / (16 * GM), r0 = ((int)blockIdx.x % (16 * GM)) * 16;
    const int64_t n = (int64_t)p.tiles * p.steps, begin = (int64_t)tile * p.steps, end = begin + p.steps;
    // the pair whose share holds step `begin`
    int first = (int)(begin * p.pairs / n);
    while (first > 0 && share(n, first, p.pairs) > begin) first--;
    while (share(n, first + 1, p.pairs) <= begin) first++;
    if (share(n, first + 1, p.pairs) >= end) return;                     // one pair: the tile is there already
    const int c0 = (tile % p.tiles_c) * kN, o0 = (tile / p.tiles_c) * 256 * GM;
    const int c = (int)threadIdx.x & 63, row4 = (int)threadIdx.x >> 6;   // 4 columns of every fourth row
    if (c0 + 4 * c >= p.cin) return;
    const int left = p.cin - c0 - 4 * c;
    for (int r = r0 + row4; r < r0 + 16; r += 4) {
        const int o = o0 + r;
        if (o >= p.cout) return;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int q = first; q < p.pairs; q++) {
            const int64_t start = share(n, q, p.pairs);
            if (start >= end) break;
            const size_t slot = (size_t)q * 2 + (start >= begin ? 0 : 1);
            const float *src = p.partial + slot * slot_floats(GM) + (size_t)r * kN + 4 * c;
            float4 v;
            if (left >= 4) v = *reinterpret_cast<const float4 *>(src);
            else v = make_float4(src[0], left > 1 ? src[1] : 0.f, left > 2 ? src[2] : 0.f, 0.f);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        float *out = p.dW + (size_t)o * p.cin + c0 + 4 * c;
        const float *g = p.gamma ? p.gamma + c0 + 4 * c : nullptr;
        if (left >= 4) {
            if (g) { s.x *= g[0]; s.y *= g[1]; s.z *= g[2]; s.w *= g[3]; }
            if (p.vec) *reinterpret_cast<float4 *>(out) = s;
            else { out[0] = s.x; out[1] = s.y; out[2] = s.z; out[3] = s.w; }
        } else {
            out[0] = g ? s.x * g[0] : s.x;
            if (left > 1) out[1] = g ? s.y * g[1] : s.y;
            if (left > 2) out[2] = g ? s.z * g[2] : s.z;
        }
    }
}

// dy for the loads: rows of `pitch` bf16 on 16-byte boundaries.  float32 becomes three parts, the bits of a value 8 at a time: their sum is the
// value (infinities and NaN stay in the first).  Rows of the last step behind the last one are zeros between the parts.
template <class T> __global__ void __launch_bounds__(256) wgrad8_prepare_kernel(const T *dy, int64_t ld, int level, bf16 *out, int rows, int rows_step, int cout, int pitch, FastDiv groups) {
    pdl_enter();
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    uint32_t row, g;
    groups.divmod(i, row, g);
    if (row >= (uint32_t)rows_step) return;
    const int ch = (int)g * 8, n = row < (uint32_t)rows ? min(8, cout - ch) : 0;
    const T *src = dy + (size_t)row * ld + ch;
    float v[8];
    if constexpr (sizeof(T) == 4) {
        if (n == 8 && level >= 1) {
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
        *reinterpret_cast<uint4 *>(out + ((size_t)part * rows_step + row) * pitch + ch) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

struct Plan {
    int gm, row_steps, steps, tiles_c, tiles, pairs;
    bool prepared;                   // dy goes through the workspace
    int pitch;
    size_t prepared_bytes, partial_bytes;
};
bool direct(const revnet_wgrad_desc &d) { return d.dy_dtype == REVNET_BF16 && d.ld_dy % 8 == 0; }
Plan plan_of(const revnet_ctx *ctx, const revnet_wgrad_desc &d, bool prepared) {
    Plan w{};
    w.gm = d.cout > 256 ? 2 : 1;
    w.row_steps = (int)((d.rows + kStep - 1) / kStep);
    w.steps = w.row_steps * (d.dy_dtype == REVNET_F32 ? 3 : 1);
    w.tiles_c = (d.cin + kN - 1) / kN;
    w.tiles = w.tiles_c * ((d.cout + 256 * w.gm - 1) / (256 * w.gm));
    const int64_t n = (int64_t)w.tiles * w.steps;
    int64_t pairs = (n + kStepsMin - 1) / kStepsMin;
    const int most = ctx->sm_count / 2;
    w.pairs = (int)(pairs > most ? most : pairs);
    w.prepared = prepared;
    w.pitch = (d.cout + 7) & ~7;
    w.prepared_bytes = prepared ? ((size_t)w.steps * kStep * w.pitch * 2 + 255) & ~size_t(255) : 0;
    w.partial_bytes = w.pairs == 0 || w.tiles % w.pairs == 0 ? 0 :          // whole tiles for every pair: no parts
                      (size_t)w.pairs * 2 * w.gm * 256 * kN * 4;
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

template <int GM, int CODE> void run_t(Exec &ex, const Wgrad8Args &a, double bytes, double flops) {
    static OncePerDevice once;
    if (once.first(ex.ctx->device))
        cudaFuncSetAttribute(wgrad8_kernel<GM, CODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Tile<GM>::kSmem);
    launch_cluster(ex, wgrad8_kernel<GM, CODE>, (unsigned)a.pairs * 2, kThreads, Tile<GM>::kSmem, 2, a);
    ex.check("wgrad8", bytes, flops);
}

}  // namespace

size_t wgrad8_workspace(const revnet_ctx *ctx, const revnet_wgrad_desc &d) {
    // whether dy can be loaded from where it is also depends on its address: the workspace serves either
    const Plan w = plan_of(ctx, d, true);
    return w.prepared_bytes + w.partial_bytes + 256;
}

void wgrad8(Exec &ex, const revnet_wgrad_desc &d, const void *dy, const void *ck, const float *gamma, float *dW, char *workspace) {
    if (d.rows == 0) { fill_zero(ex, dW, (size_t)d.cin * d.cout * 4); return; }
    const bool prepared = !direct(d) || ((uintptr_t)dy & 15);
    const Plan w = plan_of(ex.ctx, d, prepared);
    const Checkpoint c = ck_view(ck, d.rows, d.cin);
    Wgrad8Args a{};
    a.scales = c.scales; a.gamma = gamma; a.dW = dW; a.partial = (float *)(workspace + w.prepared_bytes); a.status = ex.ctx->dev_status;
    a.rows = (int)d.rows; a.cin = d.cin; a.cout = d.cout; a.row_steps = w.row_steps; a.steps = w.steps; a.tiles_c = w.tiles_c; a.tiles = w.tiles;
    a.pairs = w.pairs; a.rows_pad = c.rows_pad; a.vec = d.cin % 4 == 0;
    const int rows_step = w.row_steps * kStep;
    if (prepared) {
        const uint32_t groups = (uint32_t)w.pitch / 8;
        const unsigned grid = (unsigned)(((uint64_t)rows_step * groups + 255) / 256);
        const double bytes = (double)d.rows * d.cout * (d.dy_dtype == REVNET_F32 ? 10 : 4);
        if (d.dy_dtype == REVNET_F32)
            launch_stream(ex, bytes, 0, wgrad8_prepare_kernel<float>, grid, 256, 0, (const float *)dy, d.ld_dy, access_level(dy, d.ld_dy, 4), (bf16 *)workspace, a.rows, rows_step, d.cout, w.pitch, fast_div(groups));
        else
            launch_stream(ex, bytes, 0, wgrad8_prepare_kernel<bf16>, grid, 256, 0, (const bf16 *)dy, d.ld_dy, 0, (bf16 *)workspace, a.rows, rows_step, d.cout, w.pitch, fast_div(groups));
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
    if (w.gm == 2) { if (d.code == REVNET_INT8) run_t<2, REVNET_INT8>(ex, a, bytes, flops); else run_t<2, REVNET_E4M3>(ex, a, bytes, flops); }
    else { if (d.code == REVNET_INT8) run_t<1, REVNET_INT8>(ex, a, bytes, flops); else run_t<1, REVNET_E4M3>(ex, a, bytes, flops); }
    if (w.partial_bytes) {
        if (w.gm == 2) launch(ex, wgrad8_sum_kernel<2>, (unsigned)w.tiles * 32, 256, 0, a);
        else launch(ex, wgrad8_sum_kernel<1>, (unsigned)w.tiles * 16, 256, 0, a);
        ex.check("wgrad8_sum", (double)w.partial_bytes);
    }
}
