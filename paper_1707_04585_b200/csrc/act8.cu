// Activations kept in 8 bits: store (with the activation function beside it), load, and the activation's backward pass from what was kept.
//
//   store  ck = checkpoint of x, a = act(x)          load  a = act(x8)          bwd  dx = da act'(x8), checkpoint of act(x8)
//
// Every value is read and written once, so HBM bounds all of them.  A thread owns 16 channels (token.cuh): consecutive ones in rows
// of any alignment (kShifted), the amax of a block of 32 being one shuffle between two lanes.  No shared memory and no second pass.  Flat indexing over (row, group), since rows of any length then leave no thread idle but in the last CTA.
#include "token.cuh"
#include <algorithm>
#include <type_traits>

namespace {

constexpr int kThreads = 256;

// act(x) and d act / dx.  1 / (1 + e^-x): e^-x = inf gives 0, which is right to float32's least normal number.
__device__ __forceinline__ float sigmoid(float x) { return rcp_ftz(1.f + exp2_ftz(-1.4426950408889634f * x)); }
__device__ __forceinline__ float gelu_arg(float x) { return 1.5957691216057308f * (x + 0.044715f * x * x * x); }   // 2 sqrt(2 / pi) (...)
template <int ACT> __device__ __forceinline__ float act(float x) {
    if (ACT == REVNET_ACT_RELU) return x > 0.f ? x : (x != x ? x : 0.f);
    if (ACT == REVNET_ACT_GELU) return x * sigmoid(gelu_arg(x));
    if (ACT == REVNET_ACT_SILU) return x * sigmoid(x);
    return x;
}
template <int ACT> __device__ __forceinline__ void act_grad(float x, float &a, float &d) {
    if (ACT == REVNET_ACT_RELU) { a = x > 0.f ? x : (x != x ? x : 0.f); d = x > 0.f ? 1.f : (x != x ? x : 0.f); }
    else if (ACT == REVNET_ACT_GELU) {
        const float s = sigmoid(gelu_arg(x));
        a = x * s;
        // (x^2 would be infinite from 1.8e19 on; the factor before it is 0 long before 1e30)
        d = s + a * (1.f - s) * (1.5957691216057308f * (1.f + 0.134145f * fminf(x * x, 1e30f)));
    } else if (ACT == REVNET_ACT_SILU) {
        const float s = sigmoid(x);
        a = x * s;
        d = s * (1.f + x * (1.f - s));
    } else { a = x; d = 1.f; }
}

struct Act8Args {
    const void *x; void *a;          // store: x -> a; load: a; bwd: x = da, a = dx
    Checkpoint ck, out;              // of x; bwd: of act(x8)
    int channels, half;              // of x; of a when gated
    int64_t ld_x, ld_a;              // of x, a above
    uint32_t total;                  // groups in all
    FastDiv per_row;                 // of a row
    bool wide;                       // 32-byte accesses (token.cuh)
    float q;                         // not 0: x is int32 fixed point, value = i * q (a coupling state)
};

// this thread's row and first channel; false behind the last row
__device__ __forceinline__ bool place(const Act8Args &p, size_t &row, int &ch) {
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    uint32_t r, g;
    p.per_row.divmod(i < p.total ? i : p.total - 1, r, g);
    row = r;
    ch = (int)g * kGroup;
    return i < p.total;
}
// the gated form's operands; kCut: a half ends inside the 16 codes, and the second starts there
template <int ROWS, int CODE> struct GatedCodes {
    RawCodes g, u;
    __device__ __forceinline__ void load(const Act8Args &p, size_t row, int ch, int left) { load_codes(p.ck, row, ch, left, g); load_codes(p.ck, row, p.half + ch, left, u); }
    __device__ __forceinline__ void values(int, float (&a)[16], float (&b)[16]) const { decode<CODE>(g, a); decode<CODE>(u, b); }
};
template <int CODE> struct GatedCodes<kCut, CODE> {
    RawCodes g; RawCodesAt u;
    __device__ __forceinline__ void load(const Act8Args &p, size_t row, int ch, int left) { load_codes(p.ck, row, ch, left, g); load_codes_at(p.ck, row, p.half + ch, left, u); }
    __device__ __forceinline__ void values(int left, float (&a)[16], float (&b)[16]) const {
        decode<CODE>(g, a); decode<CODE>(u, b);
#pragma unroll
        for (int i = 0; i < 16; i++) if (i >= left) a[i] = b[i] = 0.f;
    }
};

template <int ROWS, class T, int CODE, int ACT, bool WITH_A>
__global__ void __launch_bounds__(kThreads) act8_store_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    const bool live = place(p, row, ch);
    const int left = live ? p.channels - ch : 0;
    float v[16];
    load16<ROWS>((const T *)p.x + row * p.ld_x + ch, ch, left, p.wide, v);
    if (sizeof(T) == 4 && !WITH_A && p.q != 0.f) {
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] = __int2float_rn(__float_as_int(v[i])) * p.q;
    }
    keep16<CODE>(p.ck, row, ch, live, v);
    if constexpr (WITH_A) {
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] = act<ACT>(v[i]);
        store16<ROWS>((T *)p.a + row * p.ld_a + ch, ch, left, p.wide, v);
    }
}
// gated, halves in whole blocks of 32 (CODE -1: without the checkpoint, halves of any length): the thread that needs g and u for a encodes both
template <int ROWS, class T, int CODE>
__global__ void __launch_bounds__(kThreads) act8_store_gated_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    const bool live = place(p, row, ch);
    const int left = live ? p.half - ch : 0;
    float g[16], u[16];
    Raw16<T> rg, ru;
    const T *x = (const T *)p.x + row * p.ld_x + ch;
    load_raw<ROWS>(x, ch, left, p.wide, rg);
    load_raw<ROWS>(x + p.half, ch, left, p.wide, ru);
    unpack(rg, g); unpack(ru, u);
    if constexpr (CODE >= 0) {
        keep16<CODE>(p.ck, row, ch, live, g, p.half);            // the first half ends where the second begins
        keep16<CODE>(p.ck, row, ch + p.half, live, u);
    }
#pragma unroll
    for (int i = 0; i < 16; i++) g[i] = act<REVNET_ACT_SILU>(g[i]) * u[i];
    store16<ROWS>((T *)p.a + row * p.ld_a + ch, ch, left, p.wide, g);
}

template <int ROWS, class T, int CODE, int ACT>
__global__ void __launch_bounds__(kThreads) act8_load_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    const bool live = place(p, row, ch);
    const int left = live ? p.half - ch : 0;         // (not above 0: the second group of a padded block)
    if (ROWS == kPieces && left <= 0) return;
    float v[16];
    if constexpr (ACT == REVNET_ACT_SWIGLU) {
        float u[16];
        GatedCodes<ROWS, CODE> r;
        r.load(p, row, ch, left);
        r.values(left, v, u);
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] = act<REVNET_ACT_SILU>(v[i]) * u[i];
    } else {
        read16<CODE>(p.ck, row, ch, left, v);
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] = act<ACT>(v[i]);
    }
    store16<ROWS>((T *)p.a + row * p.ld_a + ch, ch, left, p.wide, v);
}

template <int ROWS, class T, int CODE, int ACT>
__global__ void __launch_bounds__(kThreads) act8_bwd_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    const bool live = place(p, row, ch);
    const int left = live ? p.half - ch : 0;
    float x[16], da[16];
    Raw16<T> rd;
    RawCodes rx;
    GatedCodes<ROWS, CODE> rg;
    load_raw<ROWS>((const T *)p.x + row * p.ld_x + ch, ch, left, p.wide, rd);
    if constexpr (ACT == REVNET_ACT_SWIGLU) rg.load(p, row, ch, left);
    else load_codes(p.ck, row, ch, left, rx);
    unpack(rd, da);
    T *dx = (T *)p.a + row * p.ld_a + ch;
    if constexpr (ACT == REVNET_ACT_SWIGLU) {
        float u[16];
        rg.values(left, x, u);
#pragma unroll
        for (int i = 0; i < 16; i++) {
            float s, d;
            act_grad<REVNET_ACT_SILU>(x[i], s, d);
            x[i] = da[i] * u[i] * d;
            u[i] *= s;                               // (codes that were not loaded are zeros, as the padding of the checkpoint has to be)
            da[i] *= s;
        }
        store16<ROWS>(dx, ch, left, p.wide, x);
        store16<ROWS>(dx + p.half, ch, left, p.wide, da);
        if (p.out.codes) keep16<CODE>(p.out, row, ch, live, u);
    } else {
        decode<CODE>(rx, x);
#pragma unroll
        for (int i = 0; i < 16; i++) {
            float a, d;
            act_grad<ACT>(x[i], a, d);
            da[i] = ACT == REVNET_ACT_RELU && !(x[i] > 0.f) && x[i] == x[i] ? 0.f : da[i] * d;      // an infinite gradient stops at a closed ReLU too
            x[i] = a;
        }
        store16<ROWS>(dx, ch, left, p.wide, da);
        if (p.out.codes) keep16<CODE>(p.out, row, ch, live, x);
    }
}

// channels_per_row: of the tensor that the threads walk along, padded to whole blocks
bool fill(Act8Args &p, const revnet_act_desc &d, int channels_per_row) {
    p.channels = d.channels;
    p.half = d.act == REVNET_ACT_SWIGLU ? d.channels / 2 : d.channels;
    const uint32_t per_row = (uint32_t)ck_pitch(channels_per_row) / kGroup;
    p.per_row = fast_div(per_row);
    p.total = (uint32_t)d.rows * per_row;            // the entry points keep it below 2^31
    return p.total > 0;
}
unsigned blocks(const Act8Args &p) { return (p.total + kThreads - 1) / kThreads; }
template <int ROWS, class T, int CODE> void store_t(Exec &ex, const Act8Args &p, const revnet_act_desc &d, double bytes) {
    const unsigned g = blocks(p);
    if (!p.a) launch_stream(ex, bytes, 0, act8_store_kernel<ROWS, T, CODE, REVNET_ACT_NONE, false>, g, kThreads, 0, p);
    else switch (d.act) {
        case REVNET_ACT_NONE: launch_stream(ex, bytes, 0, act8_store_kernel<ROWS, T, CODE, REVNET_ACT_NONE, true>, g, kThreads, 0, p); break;
        case REVNET_ACT_RELU: launch_stream(ex, bytes, 0, act8_store_kernel<ROWS, T, CODE, REVNET_ACT_RELU, true>, g, kThreads, 0, p); break;
        case REVNET_ACT_GELU: launch_stream(ex, bytes, 0, act8_store_kernel<ROWS, T, CODE, REVNET_ACT_GELU, true>, g, kThreads, 0, p); break;
        case REVNET_ACT_SILU: launch_stream(ex, bytes, 0, act8_store_kernel<ROWS, T, CODE, REVNET_ACT_SILU, true>, g, kThreads, 0, p); break;
        default: launch_stream(ex, bytes, 0, act8_store_gated_kernel<ROWS, T, CODE>, g, kThreads, 0, p); break;
    }
    ex.check("act8_store", bytes);
}
template <int ROWS, class T, int CODE> void load_t(Exec &ex, const Act8Args &p, const revnet_act_desc &d, double bytes) {
    const unsigned g = blocks(p);
    if constexpr (ROWS == kCut) launch_stream(ex, bytes, 0, act8_load_kernel<ROWS, T, CODE, REVNET_ACT_SWIGLU>, g, kThreads, 0, p);
    else switch (d.act) {
        case REVNET_ACT_NONE: launch_stream(ex, bytes, 0, act8_load_kernel<ROWS, T, CODE, REVNET_ACT_NONE>, g, kThreads, 0, p); break;
        case REVNET_ACT_RELU: launch_stream(ex, bytes, 0, act8_load_kernel<ROWS, T, CODE, REVNET_ACT_RELU>, g, kThreads, 0, p); break;
        case REVNET_ACT_GELU: launch_stream(ex, bytes, 0, act8_load_kernel<ROWS, T, CODE, REVNET_ACT_GELU>, g, kThreads, 0, p); break;
        case REVNET_ACT_SILU: launch_stream(ex, bytes, 0, act8_load_kernel<ROWS, T, CODE, REVNET_ACT_SILU>, g, kThreads, 0, p); break;
        default: launch_stream(ex, bytes, 0, act8_load_kernel<ROWS, T, CODE, REVNET_ACT_SWIGLU>, g, kThreads, 0, p); break;
    }
    ex.check("act8_load", bytes);
}
template <int ROWS, class T, int CODE> void bwd_t(Exec &ex, const Act8Args &p, const revnet_act_desc &d, double bytes) {
    const unsigned g = blocks(p);
    if constexpr (ROWS == kCut) launch_stream(ex, bytes, 0, act8_bwd_kernel<ROWS, T, CODE, REVNET_ACT_SWIGLU>, g, kThreads, 0, p);
    else switch (d.act) {
        case REVNET_ACT_NONE: launch_stream(ex, bytes, 0, act8_bwd_kernel<ROWS, T, CODE, REVNET_ACT_NONE>, g, kThreads, 0, p); break;
        case REVNET_ACT_RELU: launch_stream(ex, bytes, 0, act8_bwd_kernel<ROWS, T, CODE, REVNET_ACT_RELU>, g, kThreads, 0, p); break;
        case REVNET_ACT_GELU: launch_stream(ex, bytes, 0, act8_bwd_kernel<ROWS, T, CODE, REVNET_ACT_GELU>, g, kThreads, 0, p); break;
        case REVNET_ACT_SILU: launch_stream(ex, bytes, 0, act8_bwd_kernel<ROWS, T, CODE, REVNET_ACT_SILU>, g, kThreads, 0, p); break;
        default: launch_stream(ex, bytes, 0, act8_bwd_kernel<ROWS, T, CODE, REVNET_ACT_SWIGLU>, g, kThreads, 0, p); break;
    }
    ex.check("act8_bwd", bytes);
}
template <bool CUT, class F> void by_type(const revnet_act_desc &d, int rows, F &&f) {
    auto code = [&](auto s, auto t) {
        if (d.code == REVNET_INT8) f(s, t, std::integral_constant<int, REVNET_INT8>());
        else f(s, t, std::integral_constant<int, REVNET_E4M3>());
    };
    auto type = [&](auto s) { if (d.dtype == REVNET_F32) code(s, float()); else code(s, bf16()); };
    if (rows == kPieces) type(std::integral_constant<int, kPieces>());
    else if (rows == kShifted) type(std::integral_constant<int, kShifted>());
    else if constexpr (CUT) type(std::integral_constant<int, kCut>());
}

}  // namespace

void act8_store(Exec &ex, const revnet_act_desc &d, const void *x, void *ck, void *a, float q) {
    const int size = d.dtype == REVNET_F32 ? 4 : 2, half = d.channels / 2;
    const bool gated = d.act == REVNET_ACT_SWIGLU && a;
    Act8Args p{};
    p.x = x; p.a = a; p.ck = ck_view(ck, d.rows, d.channels); p.q = q;
    p.ld_x = d.ld_x; p.ld_a = d.ld_a;
    const double n = (double)d.rows * d.channels, out = a ? (gated ? n / 2 : n) * size : 0;
    // (a gated row's second half starts on a block's boundary here, so on 32 bytes too)
    const int access = std::min(row_access(x, d.ld_x, size, d.channels), row_access(a, d.ld_a, size, gated ? half : d.channels));
    p.wide = access == 2;
    if (!gated || half % 32 == 0) {
        const int rows = access ? kPieces : kShifted;
        if (!fill(p, d, gated ? half : d.channels)) return;
        by_type<false>(d, rows, [&](auto s, auto t, auto c) { store_t<decltype(s)::value, decltype(t), decltype(c)::value>(ex, p, d, n * (size + 1) + out); });
        return;
    }
    // halves that end inside a block: the checkpoint first, then the activation alone
    Act8Args only = p;
    only.a = nullptr;
    const int first = row_access(x, d.ld_x, size, d.channels);
    only.wide = first == 2;
    const int rows = first ? kPieces : kShifted;
    if (!fill(only, d, d.channels)) return;
    by_type<false>(d, rows, [&](auto s, auto t, auto c) { store_t<decltype(s)::value, decltype(t), decltype(c)::value>(ex, only, d, n * (size + 1)); });
    fill(p, d, half);
    if (d.dtype == REVNET_F32) launch_stream(ex, n * size + out, 0, act8_store_gated_kernel<kShifted, float, -1>, blocks(p), kThreads, 0, p);
    else launch_stream(ex, n * size + out, 0, act8_store_gated_kernel<kShifted, bf16, -1>, blocks(p), kThreads, 0, p);
    ex.check("act8_gate", n * size + out);
}

void act8_load(Exec &ex, const revnet_act_desc &d, const void *ck, void *a) {
    const int size = d.dtype == REVNET_F32 ? 4 : 2, out = d.act == REVNET_ACT_SWIGLU ? d.channels / 2 : d.channels;
    Act8Args p{};
    p.a = a; p.ck = ck_view(ck, d.rows, d.channels);
    p.ld_a = d.ld_a;
    // (the codes of a gated row's second half: 16 bytes on 16-byte boundaries under one scale, or not)
    const int access = row_access(a, d.ld_a, size, out), rows = d.act == REVNET_ACT_SWIGLU && out % 16 ? kCut : (access ? kPieces : kShifted);
    p.wide = access == 2;
    if (!fill(p, d, out)) return;
    const double bytes = (double)d.rows * (d.channels + (double)p.half * size);
    by_type<true>(d, rows, [&](auto s, auto t, auto c) { load_t<decltype(s)::value, decltype(t), decltype(c)::value>(ex, p, d, bytes); });
}

void act8_bwd(Exec &ex, const revnet_act_desc &d, const void *ck, const void *da, void *dx, void *a_ck) {
    const int size = d.dtype == REVNET_F32 ? 4 : 2, out = d.act == REVNET_ACT_SWIGLU ? d.channels / 2 : d.channels;
    Act8Args p{};
    p.x = da; p.a = dx; p.ck = ck_view(ck, d.rows, d.channels); p.out = ck_view(a_ck, d.rows, out);
    p.ld_x = d.ld_a; p.ld_a = d.ld_x;
    const int access = std::min(row_access(da, d.ld_a, size, out), row_access(dx, d.ld_x, size, d.channels));
    const int rows = d.act == REVNET_ACT_SWIGLU && out % 16 ? kCut : (access ? kPieces : kShifted);
    p.wide = access == 2;
    if (!fill(p, d, out)) return;
    const double bytes = (double)d.rows * (d.channels * (1.0 + size) + out * (size + (a_ck ? 1.0 : 0.0)));
    by_type<true>(d, rows, [&](auto s, auto t, auto c) { bwd_t<decltype(s)::value, decltype(t), decltype(c)::value>(ex, p, d, bytes); });
}
