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

// The context's device has to be current: its kernels and their parameters belong to it.
static inline bool device_is_current(const revnet_ctx *ctx) {
    int dev = -1;
    if (ctx->device >= 0 && cudaGetDevice(&dev) == cudaSuccess && dev == ctx->device) return true;
    cudaGetLastError();
    return false;
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

// A thread's 16 channels.
//   kPieces   rows of 16-byte pieces on 16-byte boundaries: 16 consecutive ones, moved by accesses of 32 (`wide`) or 16 bytes
//   kShifted  any other rows: 16 consecutive ones too, loaded as the aligned 16 bytes that hold them and shifted into place; stored the same way, with
//             the end of the lane before.  Elements one by one only at the ends of a row (stores: of a warp's part of it)
//   kCut      the same, of gated rows whose second half's codes start inside 16
// `left` is the row's length minus the thread's first channel.
constexpr int kGroup = 16;
enum { kPieces, kShifted, kCut };

// raw words of 16 elements, so that a load can be in flight while earlier values are worked on
template <class T> struct Raw16 { uint32_t w[16 * sizeof(T) / 4]; };
__device__ __forceinline__ uint32_t bits_of(const float *p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t bits_of(const bf16 *p) { return *reinterpret_cast<const uint16_t *>(p); }

// r = w from `bytes` (0 to 16, a multiple of SIZE) on; w holds four words more than r.  (A branch for each whole word instead of the selections
// saves nothing: 8192 x 2500 norms in bf16 54.6 and 55.4 us forward, float32 with rows of 100 channels 10 % slower.)
template <int SIZE, int N, int W> __device__ __forceinline__ void shift_words(uint32_t (&w)[N], uint32_t bytes, uint32_t (&r)[W]) {
    static_assert(N == W + 4, "");
    if (bytes & 16u) {
#pragma unroll
        for (int i = 0; i < N - 4; i++) w[i] = w[i + 4];
    }
    if (bytes & 8u) {
#pragma unroll
        for (int i = 0; i < N - 2; i++) w[i] = w[i + 2];
    }
    if (bytes & 4u) {
#pragma unroll
        for (int i = 0; i < N - 1; i++) w[i] = w[i + 1];
    }
#pragma unroll
    for (int i = 0; i < W; i++) r[i] = SIZE < 4 ? __funnelshift_r(w[i], w[i + 1], 8u * (bytes & (SIZE == 2 ? 2u : 3u))) : w[i];
}
// kShifted, reads nothing outside the row; ch: p's channel (0: the row's start)
template <class T> __device__ __forceinline__ void load_shifted(const T *p, int ch, int left, Raw16<T> &r) {
    constexpr int kSize = sizeof(T), kN = kSize + 1, kBytes = 16 * kSize;       // aligned pieces
    const uint32_t o = (uint32_t)(uintptr_t)p & 15u;
    const char *from = reinterpret_cast<const char *>(p) - o;
    const int first = ch == 0 ? 0 : -16, end = left * kSize;
    uint32_t w[4 * kN];
#pragma unroll
    for (int k = 0; k < kN; k++) {
        const int at = 16 * k - (int)o;
        uint4 q = make_uint4(0u, 0u, 0u, 0u);
        if (at >= first && at + 16 <= end) { if (at < kBytes) q = *reinterpret_cast<const uint4 *>(from + 16 * k); }
        else if (at < end && at < kBytes) {
            uint32_t e[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < 16 / kSize; j++)
                if (at + j * kSize >= 0 && at + j * kSize < end)
                    e[j * kSize / 4] |= bits_of(reinterpret_cast<const T *>(from + 16 * k) + j) << (8 * (j * kSize & 3));
            q = make_uint4(e[0], e[1], e[2], e[3]);
        }
        w[4 * k] = q.x; w[4 * k + 1] = q.y; w[4 * k + 2] = q.z; w[4 * k + 3] = q.w;
    }
    shift_words<kSize>(w, o, r.w);
}

// elements of p (the thread's first channel), zeros where there is none
template <int ROWS, class T> __device__ __forceinline__ void load_raw(const T *p, int ch, int left, bool wide, Raw16<T> &r) {
    constexpr int W = 16 * sizeof(T) / 4;
    if constexpr (ROWS != kPieces) load_shifted(p, ch, left, r);
    else {
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
// kShifted: all lanes of the warp call it, neighbours that share a row with neighbouring groups of it
template <class T> __device__ __forceinline__ void store_shifted(T *p, int ch, int left, const Raw16<T> &r) {
    constexpr int kSize = sizeof(T), W = 4 * kSize, kBytes = 16 * kSize;
    const int o = (int)((uint32_t)(uintptr_t)p & 15u), lane = threadIdx.x & 31, n = left >= 16 ? kBytes : (left > 0 ? left * kSize : 0);
    char *to = reinterpret_cast<char *>(p) - o;
    uint32_t w[W + 4];
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = __shfl_up_sync(0xffffffffu, r.w[W - 4 + i], 1);
#pragma unroll
    for (int i = 0; i < W; i++) w[4 + i] = r.w[i];
    uint32_t v[W];
    shift_words<kSize>(w, 16u - o, v);
    // the first piece holds the end of the lane before, if that has one; the last elements go with the next lane's first piece, if that is whole
    const bool head = o == 0 || (lane > 0 && ch > 0), tail = o == 0 || (lane < 31 && left * kSize - kBytes >= 16 - o);
#pragma unroll
    for (int k = 0; k < kSize; k++)
        if ((k > 0 || head) && 16 * k + 16 - o <= n) *reinterpret_cast<uint4 *>(to + 16 * k) = make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    auto put = [&](int i) { put_bits(p + i, r.w[i * kSize / 4] >> (8 * (i * kSize & 3))); };
    if (n < kBytes) {                // the row's end
        if (n > 0) {
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int piece = (i * kSize + o) >> 4;
                if (i * kSize < n && (16 * piece + 16 - o > n || (piece == 0 && !head))) put(i);
            }
        }
        return;
    }
    if (!head) {
#pragma unroll
        for (int i = 0; i < 16 / kSize; i++) if (i * kSize < 16 - o) put(i);
    }
    if (!tail) {
#pragma unroll
        for (int i = 16 - 16 / kSize; i < 16; i++) if (i * kSize >= kBytes - o) put(i);
    }
}
template <int ROWS, class T> __device__ __forceinline__ void store_raw(T *p, int ch, int left, bool wide, const Raw16<T> &r) {
    constexpr int W = 16 * sizeof(T) / 4;
    if constexpr (ROWS != kPieces) store_shifted(p, ch, left, r);
    else {
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
    }
}
template <int ROWS, class T> __device__ __forceinline__ void load16(const T *p, int ch, int left, bool wide, float (&v)[16]) {
    Raw16<T> r;
    load_raw<ROWS>(p, ch, left, wide, r);
    unpack(r, v);
}
template <int ROWS, class T> __device__ __forceinline__ void store16(T *p, int ch, int left, bool wide, const float (&v)[16]) {
    Raw16<T> r;
    pack(v, r);
    store_raw<ROWS>(p, ch, left, wide, r);
}

// ---------------------------------------------------------------- rows on their way
// Channels of the rows to come, fetched into shared memory by asynchronous copies of 16 bytes: unlike loads into registers they cost none
// while they are in flight.  The lanes of a warp that share a row (`lanes` of them, 16 channels each) copy side by side, whole lines per
// instruction, and wait for each other (__syncwarp behind the wait) before a thread reads its own 16 channels.  A thread's chunks are
// neighbours, so eight lanes that read their k-th chunk would meet in half or a quarter of the banks: chunk c lies at c ^ (bits 3.. of c).
// kShifted: the aligned chunks that hold the channels, one more than their number (which lies behind them as it is); the first may start with
// up to 15 bytes of the row before, or of what lies between the rows (shifted away), but with nothing in front of the tensor.
__device__ __forceinline__ void copy16(void *dst, const void *src, int bytes) {       // bytes of src, zeros behind them (0: nothing is read)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }
template <class T> constexpr int kChunks = 16 * (int)sizeof(T) / 16;
template <class T> __device__ __forceinline__ int chunk_place(int c) { return c ^ ((c >> 3) & (kChunks<T> - 1)); }
// at: the first of the lanes' channels in the tensor, `left` of them in the row; to: the lanes' part of a stage
template <int ROWS, class T> __device__ __forceinline__ void fetch_row(uint4 *to, int lanes, int lane, const T *tensor, int64_t at, int left) {
    const char *p = reinterpret_cast<const char *>(tensor + at);
    if constexpr (ROWS == kPieces) {
#pragma unroll
        for (int k = 0; k < kChunks<T>; k++) {
            const int c = k * lanes + lane;
            copy16(to + chunk_place<T>(c), p + 16 * c, c * (16 / (int)sizeof(T)) < left ? 16 : 0);
        }
    } else {
        const int o = (int)((uint32_t)(uintptr_t)p & 15u), bytes = left > 0 ? left * (int)sizeof(T) + o : 0;
        p -= o;
        auto in = [&](int c) { const int n = bytes - 16 * c; return n < 0 ? 0 : (n < 16 ? n : 16); };
        const bool front = lane == 0 && bytes > 0 && p < reinterpret_cast<const char *>(tensor);
#pragma unroll
        for (int k = 0; k < kChunks<T>; k++) {
            const int c = k * lanes + lane;
            if (k > 0 || !front) copy16(to + chunk_place<T>(c), p + 16 * c, in(c));
        }
        if (lane == 0) copy16(to + kChunks<T> * lanes, p + 16 * kChunks<T> * lanes, o ? in(kChunks<T> * lanes) : 0);
        if (front) {
            uint32_t e[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < 16 / (int)sizeof(T); j++)
                if (j * (int)sizeof(T) >= o && j * (int)sizeof(T) < bytes)
                    e[j * sizeof(T) / 4] |= bits_of(reinterpret_cast<const T *>(p) + j) << (8 * (j * sizeof(T) & 3));
            to[0] = make_uint4(e[0], e[1], e[2], e[3]);
        }
    }
}
// row: any address that is a multiple of 16 channels away from the row's start
template <int ROWS, class T> __device__ __forceinline__ void fetched(const uint4 *from, int lanes, int lane, const T *row, Raw16<T> &r) {
    constexpr int W = 4 * kChunks<T>;
    uint32_t w[W + 4];
#pragma unroll
    for (int k = 0; k < kChunks<T> + (ROWS == kShifted); k++) {
        const int c = lane * kChunks<T> + k;
        const uint4 q = from[k == kChunks<T> && lane == lanes - 1 ? c : chunk_place<T>(c)];
        w[4 * k] = q.x; w[4 * k + 1] = q.y; w[4 * k + 2] = q.z; w[4 * k + 3] = q.w;
    }
    if constexpr (ROWS == kShifted) shift_words<sizeof(T)>(w, (uint32_t)(uintptr_t)row & 15u, r.w);
    else {
#pragma unroll
        for (int i = 0; i < W; i++) r.w[i] = w[i];
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
// 16 channels into a checkpoint (all lanes of the warp call it).  live: the row exists.  v holds zeros behind the row's last channel.  end: first
// channel that is not to be written (a multiple of 32; 0: the padded row's end).
template <int CODE> __device__ __forceinline__ void keep16(const Checkpoint &ck, size_t row, int ch, bool live, const float (&v)[16], int end = 0) {
    if (end == 0) end = ck.pitch;
    uint32_t top = abs_max16(v);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t byte = scale_byte<CODE>(top);
    if (!live || ch >= end) return;
    *reinterpret_cast<uint4 *>(ck.codes + row * ck.pitch + ch) = encode16<CODE>(v, byte);
    if ((ch & 16) == 0) ck.scales[scale_index(ck, row, ch)] = (uint8_t)byte;
}
// 16 channels' codes, not yet decoded
struct RawCodes { uint4 q; uint32_t byte; };
// left as for load_raw; ch a multiple of 16
__device__ __forceinline__ void load_codes(const Checkpoint &ck, size_t row, int ch, int left, RawCodes &r) {
    if (left > 0) {
        r.q = *reinterpret_cast<const uint4 *>(ck.codes + row * ck.pitch + ch);
        r.byte = byte_of(ck.scales + scale_index(ck, row, ch));
    } else {
        r.q = make_uint4(0u, 0u, 0u, 0u);
        r.byte = 0u;
    }
}
template <int CODE> __device__ __forceinline__ void decode(const RawCodes &r, float (&v)[16]) { decode16<CODE>(r.q, r.byte, v); }
template <int CODE> __device__ __forceinline__ void read16(const Checkpoint &ck, size_t row, int ch, int left, float (&v)[16]) {
    RawCodes r;
    load_codes(ck, row, ch, left, r);
    decode<CODE>(r, v);
}
// the same from any channel on: out of the two aligned pieces that hold them, under the scales of up to two blocks
struct RawCodesAt { uint4 q; uint32_t byte, next; int cut; };            // next: the scale byte from the cut-th on
__device__ __forceinline__ void load_codes_at(const Checkpoint &ck, size_t row, int ch, int left, RawCodesAt &r) {
    r.q = make_uint4(0u, 0u, 0u, 0u);
    r.byte = r.next = 0u;
    r.cut = 32 - (ch & 31);
    if (left <= 0) return;
    const int at = ch & ~15;
    const uint4 *from = reinterpret_cast<const uint4 *>(ck.codes + row * ck.pitch + at);
    const uint4 a = from[0], b = at + 16 < (int)ck.pitch ? from[1] : make_uint4(0u, 0u, 0u, 0u);
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, c[4];
    shift_words<1>(w, ch & 15u, c);
    r.q = make_uint4(c[0], c[1], c[2], c[3]);
    r.byte = byte_of(ck.scales + scale_index(ck, row, ch));
    r.next = r.cut < left && r.cut < 16 ? byte_of(ck.scales + scale_index(ck, row, ch + r.cut)) : 0u;
}
template <int CODE> __device__ __forceinline__ void decode(const RawCodesAt &r, float (&v)[16]) {
    decode16<CODE>(r.q, 127u, v);
    const float s = __uint_as_float(r.byte << 23), t = __uint_as_float(r.next << 23);
#pragma unroll
    for (int i = 0; i < 16; i++) v[i] *= i < r.cut ? s : t;
}
#endif
