// Shared by the operators on rows of tokens: loads and stores of sixteen channels, and the 8-bit checkpoint format
// (include/revnet.h, "An 8-bit checkpoint").
#pragma once
#include "common.cuh"
#include <cuda_fp8.h>

// ---------------------------------------------------------------- host side
struct Checkpoint {            // a checkpoint buffer taken apart
    uint8_t *codes, *scales;
    int pitch;                 // bytes per row of codes: channels rounded up to 32
    uint32_t rows_pad;         // rows rounded up to 64
};
static inline int ck_pitch(int channels) { return (channels + 31) & ~31; }
static inline size_t ck_scales_at(int64_t rows, int channels) { return ((size_t)rows * ck_pitch(channels) + 255) & ~size_t(255); }
static inline size_t ck_bytes(int64_t rows, int channels) {
    return ck_scales_at(rows, channels) + (size_t)((channels + 127) / 128) * (((size_t)rows + 63) & ~size_t(63)) * 4;
}
static inline Checkpoint ck_view(const void *buf, int64_t rows, int channels) {
    uint8_t *b = (uint8_t *)buf;
    return Checkpoint{b, b ? b + ck_scales_at(rows, channels) : nullptr, ck_pitch(channels), (uint32_t)((rows + 63) & ~int64_t(63))};
}
// How wide the accesses to the rows of a tensor at p can be, `ld` elements of `size` bytes apart, `channels` of them in use: 2: 32 bytes at multiples
// of 16 channels; 1: 16 bytes; 0: rows that do not consist of 16-byte pieces on 16-byte boundaries (null: 2).
static inline int row_access(const void *p, int64_t ld, int size, int channels) {
    if (!p) return 2;
    const uint64_t a = (uint64_t)(uintptr_t)p | (uint64_t)ld * size;
    return a % 16 || channels * size % 16 ? 0 : (a % 32 ? 1 : 2);
}

// ---------------------------------------------------------------- act8.cu, norm.cu, wgrad8.cu, logprobs.cu
// q not 0: x is int32 fixed point with that step (float32 descriptor, a null)
void act8_store(Exec &ex, const revnet_act_desc &d, const void *x, void *ck, void *a, float q = 0.f);
void act8_load(Exec &ex, const revnet_act_desc &d, const void *ck, void *a);
void act8_bwd(Exec &ex, const revnet_act_desc &d, const void *ck, const void *da, void *dx, void *a_ck);
void rmsnorm_fwd(Exec &ex, const revnet_norm_desc &d, const void *x, const void *r, const float *gamma, void *h, void *n, void *ck, float *rstd);
size_t rmsnorm_bwd_workspace(const revnet_ctx *ctx, const revnet_norm_desc &d);
void rmsnorm_bwd(Exec &ex, const revnet_norm_desc &d, const void *dn, const void *dh, const void *h, const void *ck, const float *rstd,
                 const float *gamma, void *dx, void *dr, float *dgamma, float *partial);
size_t wgrad8_workspace(const revnet_ctx *ctx, const revnet_wgrad_desc &d);
void wgrad8(Exec &ex, const revnet_wgrad_desc &d, const void *dy, const void *ck, const float *gamma, float *dW, char *workspace);
void logprobs_fwd(Exec &ex, const revnet_logprob_desc &d, const void *logits, const int32_t *targets, float *logp, float *entropy, float *lse,
                  float *top_logp, int32_t *top_index);
void logprobs_bwd(Exec &ex, const revnet_logprob_desc &d, const void *logits, const int32_t *targets, const float *lse, const float *entropy,
                  const float *dlogp, const float *dentropy, void *dlogits);

#ifdef __CUDACC__
// 2^v to two steps of 2^-23, results below 2^-126 become 0 (keeping those takes four more instructions); 1 / v likewise
__device__ __forceinline__ float exp2_ftz(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float rcp_ftz(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

// ---------------------------------------------------------------- sixteen channels of a row
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float &d, float v) { d = v; }
__device__ __forceinline__ void put(bf16 &d, float v) { d = __float2bfloat16_rn(v); }
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ uint32_t byte_of(const uint8_t *p) { return *p; }

// A thread's 16 channels.  Rows of 16-byte pieces on 16-byte boundaries: 16 consecutive ones, moved by accesses of 32 (`wide`) or 16 bytes.  Any
// other rows (SPREAD): every 32nd of 512, the lanes of a warp side by side, so that a warp's accesses are whole lines where a thread's
// would be an element each.  `left` is the row's length minus the thread's first channel.
constexpr int kGroup = 16;
template <bool SPREAD> __device__ __forceinline__ int first_channel(int t) { return SPREAD ? (t & ~31) * kGroup + (t & 31) : t * kGroup; }
template <bool SPREAD> __device__ __forceinline__ int step_of(int i) { return SPREAD ? 32 * i : i; }

// raw words of 16 elements, so that a load can be in flight while earlier values are worked on
template <class T> struct Raw16 { uint32_t w[16 * sizeof(T) / 4]; };
__device__ __forceinline__ uint32_t bits_of(const float *p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t bits_of(const bf16 *p) { return *reinterpret_cast<const uint16_t *>(p); }

// elements of p (the thread's first channel), zeros where there is none
template <bool SPREAD, class T> __device__ __forceinline__ void load_raw(const T *p, int left, bool wide, Raw16<T> &r) {
    constexpr int W = 16 * sizeof(T) / 4;
    if constexpr (!SPREAD) {
        if (left >= 16 && wide) {
#pragma unroll
            for (int i = 0; i < W; i += 8) {
                uint32_t t[8];
                ld8(reinterpret_cast<const char *>(p) + 4 * i, t, true);
#pragma unroll
                for (int j = 0; j < 8; j++) r.w[i + j] = t[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 4) {
                uint4 q = make_uint4(0u, 0u, 0u, 0u);
                if (i * 4 / (int)sizeof(T) < left) q = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) + 4 * i);
                r.w[i] = q.x; r.w[i + 1] = q.y; r.w[i + 2] = q.z; r.w[i + 3] = q.w;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; i++) {
            if constexpr (sizeof(T) == 4) r.w[i] = 32 * i < left ? bits_of(p + 32 * i) : 0u;
            else r.w[i] = (64 * i < left ? bits_of(p + 64 * i) : 0u) | (64 * i + 32 < left ? bits_of(p + 64 * i + 32) : 0u) << 16;
        }
    }
}
__device__ __forceinline__ void unpack(const Raw16<float> &r, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; i++) v[i] = __uint_as_float(r.w[i]);
}
__device__ __forceinline__ void unpack(const Raw16<bf16> &r, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 8; i++) { v[2 * i] = bf16_lo(r.w[i]); v[2 * i + 1] = bf16_hi(r.w[i]); }
}
__device__ __forceinline__ void pack(const float (&v)[16], Raw16<float> &r) {
#pragma unroll
    for (int i = 0; i < 16; i++) r.w[i] = __float_as_uint(v[i]);
}
// bf16 outputs: the one rounding of a value, to nearest even
__device__ __forceinline__ void pack(const float (&v)[16], Raw16<bf16> &r) {
#pragma unroll
    for (int i = 0; i < 8; i++) r.w[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void put_bits(float *p, uint32_t w) { *p = __uint_as_float(w); }
__device__ __forceinline__ void put_bits(bf16 *p, uint32_t w) { *reinterpret_cast<uint16_t *>(p) = (uint16_t)w; }
template <bool SPREAD, class T> __device__ __forceinline__ void store_raw(T *p, int left, bool wide, const Raw16<T> &r) {
    constexpr int W = 16 * sizeof(T) / 4;
    if constexpr (!SPREAD) {
        if (left >= 16 && wide) {
#pragma unroll
            for (int i = 0; i < W; i += 8) {
                uint32_t t[8];
#pragma unroll
                for (int j = 0; j < 8; j++) t[j] = r.w[i + j];
                st8(reinterpret_cast<char *>(p) + 4 * i, t, true);
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 4)
                if (i * 4 / (int)sizeof(T) < left)
                    *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(p) + 4 * i) = make_uint4(r.w[i], r.w[i + 1], r.w[i + 2], r.w[i + 3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; i++)
            if (32 * i < left) put_bits(p + 32 * i, sizeof(T) == 4 ? r.w[i * sizeof(T) / 4] : r.w[i / 2] >> (16 * (i & 1)));
    }
}
template <bool SPREAD, class T> __device__ __forceinline__ void load16(const T *p, int left, bool wide, float (&v)[16]) {
    Raw16<T> r;
    load_raw<SPREAD>(p, left, wide, r);
    unpack(r, v);
}
template <bool SPREAD, class T> __device__ __forceinline__ void store16(T *p, int left, bool wide, const float (&v)[16]) {
    Raw16<T> r;
    pack(v, r);
    store_raw<SPREAD>(p, left, wide, r);
}

// ---------------------------------------------------------------- rows on their way
// Channels of the rows to come, fetched into shared memory by asynchronous copies of 16 bytes: unlike loads into registers they cost none
// while they are in flight.  The lanes of a warp that share a row (`lanes` of them, 16 channels each) copy side by side, whole lines per
// instruction, and wait for each other (__syncwarp behind the wait) before a thread reads its own 16 channels.  A thread's chunks are
// neighbours, so eight lanes that read their k-th chunk would meet in half or a quarter of the banks: chunk c lies at c ^ (bits 3.. of c).
// Not for SPREAD.
__device__ __forceinline__ void copy16(void *dst, const void *src, bool in) {        // in = false: zeros, nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }
template <class T> constexpr int kChunks = 16 * (int)sizeof(T) / 16;
template <class T> __device__ __forceinline__ int chunk_place(int c) { return c ^ ((c >> 3) & (kChunks<T> - 1)); }
// p: the first of the lanes' channels, `left` of them in the row; to: the lanes' part of a stage
template <class T> __device__ __forceinline__ void fetch_row(uint4 *to, int lanes, int lane, const T *p, int left) {
#pragma unroll
    for (int k = 0; k < kChunks<T>; k++) {
        const int c = k * lanes + lane;
        copy16(to + chunk_place<T>(c), reinterpret_cast<const char *>(p) + 16 * c, c * (16 / (int)sizeof(T)) < left);
    }
}
template <class T> __device__ __forceinline__ void fetched(const uint4 *from, int lane, Raw16<T> &r) {
#pragma unroll
    for (int k = 0; k < kChunks<T>; k++) {
        const uint4 q = from[chunk_place<T>(lane * kChunks<T> + k)];
        r.w[4 * k] = q.x; r.w[4 * k + 1] = q.y; r.w[4 * k + 2] = q.z; r.w[4 * k + 3] = q.w;
    }
}

// ---------------------------------------------------------------- codes
// Scale byte of a block whose largest magnitude has the bits `top` (sign cleared): the exponent field of the smallest power of two s with
// top <= 127 s (448 s), read off the bits: 127 = 1.984375 * 2^6, 448 = 1.75 * 2^8, so it is top's exponent - 6 (- 8), one more where top's
// mantissa exceeds that of 127 (448).  Not below 10 (2^-117), so that the least value, 2^-9 * 2^-117 in e4m3, is a normal bf16 number;
// 255 for an infinity or a NaN, whose bits are the largest.
template <int CODE> __device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return 255u;
    const uint32_t m = top & 0x7fffffu;
    const int e = (int)(top >> 23) - (CODE == REVNET_INT8 ? 6 : 8) + (m > (CODE == REVNET_INT8 ? 0x7e0000u : 0x600000u) ? 1 : 0);
    return (uint32_t)(e < 10 ? 10 : e);
}
// the largest magnitude of 16 values, a NaN if one of them is
__device__ __forceinline__ float abs_max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
    return r;
}
__device__ __forceinline__ uint32_t abs_max16(const float (&v)[16]) {
    float t = abs_max3(v[0], v[1], v[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) t = abs_max3(t, v[i], v[i + 1]);
    return __float_as_uint(abs_max3(t, v[15], v[15])) & 0x7fffffffu;
}
// codes of 16 values: the multiplication by a power of two is exact, the one rounding is to nearest even
template <int CODE> __device__ __forceinline__ uint4 encode16(const float (&v)[16], uint32_t byte) {
    uint32_t w[4];
    if (byte == 255u) return make_uint4(0u, 0u, 0u, 0u);
    const float inv = __uint_as_float((254u - byte) << 23);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (CODE == REVNET_INT8) {
            // 1.5 * 2^23 added: the sum's last mantissa bits are the integer nearest to v * inv, in two's complement
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; j++) b[j] = __float_as_uint(__fmaf_rn(v[4 * i + j], inv, 12582912.f));
            w[i] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        } else {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i] * inv, v[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2] * inv, v[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
            w[i] = lo | hi << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// sign, 4 exponent and 3 mantissa bits of an e4m3 byte moved to a float's places: the exponent's bias is 7 and not 127, which the factor 2^120
// makes up for (subnormal codes included)
__device__ __forceinline__ float e4m3_to_f(uint32_t b) {
    return __uint_as_float((b & 0x80u) << 24 | (b & 0x7fu) << 20) * __uint_as_float((120u + 127u) << 23);
}
template <int CODE> __device__ __forceinline__ void decode16(uint4 q, uint32_t byte, float (&v)[16]) {
    const float s = __uint_as_float(byte << 23);             // byte 255: infinity, and 0 * infinity = NaN
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (CODE == REVNET_INT8) {
            const uint32_t u = w[i] ^ 0x80808080u;           // code + 128 in each byte: 2^23 + that is a float whose last byte it is
#pragma unroll
            for (int j = 0; j < 4; j++) v[4 * i + j] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 + j)) - 8388736.f) * s;
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) v[4 * i + j] = e4m3_to_f(w[i] >> (8 * j)) * s;
        }
    }
}
__device__ __forceinline__ size_t scale_index(const Checkpoint &ck, size_t row, int ch) {
    return ((size_t)(ch >> 7) * ck.rows_pad + row) * 4 + ((ch >> 5) & 3);
}
// 16 channels into a checkpoint (all lanes of the warp call it, SPREAD: all of one row).  live: the row exists.  v holds zeros behind the row's
// last channel.  end: first channel that is not to be written (a multiple of 32; 0: the padded row's end).
template <bool SPREAD, int CODE> __device__ __forceinline__ void keep16(const Checkpoint &ck, size_t row, int ch, bool live, const float (&v)[16], int end = 0) {
    if (end == 0) end = ck.pitch;
    if constexpr (SPREAD) {
        // the lanes of a warp hold the 32 channels of a block; lane i writes the scale of block i
        const int ch0 = ch & ~31, lane = ch & 31;
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 16; i++) {
            if (ch0 + 32 * i >= end) break;
            const uint32_t byte = scale_byte<CODE>(__reduce_max_sync(0xffffffffu, __float_as_uint(v[i]) & 0x7fffffffu));
            if (lane == i) mine = byte;
            const float inv = __uint_as_float((254u - byte) << 23);
            uint32_t c;
            if constexpr (CODE == REVNET_INT8) c = __float_as_uint(__fmaf_rn(v[i], inv, 12582912.f));
            else c = __nv_cvt_float_to_fp8(v[i] * inv, __NV_SATFINITE, __NV_E4M3);
            if (live) ck.codes[row * ck.pitch + ch + 32 * i] = byte == 255u ? (uint8_t)0 : (uint8_t)c;
        }
        if (live && lane < 16 && ch0 + 32 * lane < end) ck.scales[scale_index(ck, row, ch0 + 32 * lane)] = (uint8_t)mine;
    } else {
        uint32_t top = abs_max16(v);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        const uint32_t byte = scale_byte<CODE>(top);
        if (!live || ch >= end) return;
        *reinterpret_cast<uint4 *>(ck.codes + row * ck.pitch + ch) = encode16<CODE>(v, byte);
        if ((ch & 16) == 0) ck.scales[scale_index(ck, row, ch)] = (uint8_t)byte;
    }
}
// 16 channels' codes, not yet decoded: 16 bytes and a scale byte, or (SPREAD) 16 bytes of 16 blocks and their scales
template <bool SPREAD> struct RawCodes;
template <> struct RawCodes<false> { uint4 q; uint32_t byte; };
template <> struct RawCodes<true> { uint4 q, bytes; };
// left as for load_raw; ch a multiple of 16 unless SPREAD
template <bool SPREAD> __device__ __forceinline__ void load_codes(const Checkpoint &ck, size_t row, int ch, int left, RawCodes<SPREAD> &r) {
    if constexpr (SPREAD) {
        uint32_t c[4] = {0u, 0u, 0u, 0u}, b[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 16; i++)
            if (32 * i < left) {
                c[i / 4] |= byte_of(ck.codes + row * ck.pitch + ch + 32 * i) << (8 * (i & 3));
                // the scales of four blocks are one word where the first is a multiple of four (always but in a gated row's second half); bytes behind the
                // last block are not used
                if (i % 4 == 0 && (ch & 96) == 0) b[i / 4] = *reinterpret_cast<const uint32_t *>(ck.scales + scale_index(ck, row, ch + 32 * i));
                if ((ch & 96) != 0) b[i / 4] |= byte_of(ck.scales + scale_index(ck, row, ch + 32 * i)) << (8 * (i & 3));
            }
        r.q = make_uint4(c[0], c[1], c[2], c[3]);
        r.bytes = make_uint4(b[0], b[1], b[2], b[3]);
    } else if (left > 0) {
        r.q = *reinterpret_cast<const uint4 *>(ck.codes + row * ck.pitch + ch);
        r.byte = byte_of(ck.scales + scale_index(ck, row, ch));
    } else {
        r.q = make_uint4(0u, 0u, 0u, 0u);
        r.byte = 0u;
    }
}
template <bool SPREAD, int CODE> __device__ __forceinline__ void decode(const RawCodes<SPREAD> &r, float (&v)[16]) {
    if constexpr (SPREAD) {
        decode16<CODE>(r.q, 127u, v);
        const uint32_t b[4] = {r.bytes.x, r.bytes.y, r.bytes.z, r.bytes.w};
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] *= __uint_as_float(((b[i / 4] >> (8 * (i & 3))) & 0xffu) << 23);
    } else decode16<CODE>(r.q, r.byte, v);
}
template <bool SPREAD, int CODE> __device__ __forceinline__ void read16(const Checkpoint &ck, size_t row, int ch, int left, float (&v)[16]) {
    RawCodes<SPREAD> r;
    load_codes<SPREAD>(ck, row, ch, left, r);
    decode<SPREAD, CODE>(r, v);
}
#endif
