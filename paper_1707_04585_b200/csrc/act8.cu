// Activations kept in 8 bits: store (with the activation function beside it), load, and the activation's backward pass from what was kept.
//
//   store  ck = checkpoint of x, a = act(x)          load  a = act(x8)          bwd  dx = da act'(x8), checkpoint of act(x8)
//
// Every value is read and written once, so HBM bounds all of them.  A thread owns groups of 16 channels (see token.cuh): the amax of a block
// of 32 is one shuffle between two lanes, no shared memory and no second pass.  Flat indexing over (row, group), since rows of any length
// then leave no thread idle but in the last CTA.
#include "token.cuh"
#include <type_traits>

namespace {

constexpr int kThreads = 256;

// act(x) and d act / dx.  1 / (1 + e^-x): e^-x = inf gives 0, which is right to float32's least normal number.
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }
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
        d = s + a * (1.f - s) * (1.5957691216057308f * (1.f + 0.134145f * x * x));
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
    int lv_x, lv_a, lv_u;            // access levels (token.cuh); lv_u: of the second half of a gated row
    uint32_t total;                  // groups in all
    FastDiv per_row;                 // groups per row
};
__device__ __forceinline__ int left(int channels, int ch) { return channels - ch; }

// the group that thread i of the flat index works on; false behind the last one
__device__ __forceinline__ bool place(const Act8Args &p, uint32_t i, size_t &row, int &ch) {
    uint32_t r, g;
    p.per_row.divmod(i < p.total ? i : p.total - 1, r, g);
    row = r;
    ch = (int)g * kGroup;
    return i < p.total;
}

template <class T, int CODE, int ACT, bool WITH_A>
__global__ void __launch_bounds__(kThreads) act8_store_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    const bool live = place(p, blockIdx.x * kThreads + threadIdx.x, row, ch);
    const int n = live ? left(p.channels, ch) : 0;
    float v[16];
    load16((const T *)p.x + row * p.ld_x + ch, n, p.lv_x, v);
    keep16<CODE>(p.ck, row, ch, live, v);
    if constexpr (WITH_A) {
        float a[16];
#pragma unroll
        for (int i = 0; i < 16; i++) a[i] = act<ACT>(v[i]);
        store16((T *)p.a + row * p.ld_a + ch, n, p.lv_a, a);
    }
}
// gated, halves in whole blocks of 32: the thread that needs g and u for a encodes both
template <class T, int CODE>
__global__ void __launch_bounds__(kThreads) act8_store_gated_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    const bool live = place(p, blockIdx.x * kThreads + threadIdx.x, row, ch);
    const int n = live ? left(p.half, ch) : 0;
    float g[16], u[16];
    Raw16<T> rg, ru;
    const T *x = (const T *)p.x + row * p.ld_x + ch;
    load_raw(x, n, p.lv_x, rg);
    load_raw(x + p.half, n, p.lv_u, ru);
    unpack(rg, g); unpack(ru, u);
    keep16<CODE>(p.ck, row, ch, live, g);
    keep16<CODE>(p.ck, row, ch + p.half, live, u);
#pragma unroll
    for (int i = 0; i < 16; i++) g[i] = act<REVNET_ACT_SILU>(g[i]) * u[i];
    store16((T *)p.a + row * p.ld_a + ch, n, p.lv_a, g);
}
// the gated activation alone, for halves that end inside a block
template <class T>
__global__ void __launch_bounds__(kThreads) act8_gate_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    const bool live = place(p, blockIdx.x * kThreads + threadIdx.x, row, ch);
    const int n = live ? left(p.half, ch) : 0;
    float g[16], u[16];
    const T *x = (const T *)p.x + row * p.ld_x + ch;
    load16(x, n, p.lv_x, g);
    load16(x + p.half, n, p.lv_u, u);
#pragma unroll
    for (int i = 0; i < 16; i++) g[i] = act<REVNET_ACT_SILU>(g[i]) * u[i];
    store16((T *)p.a + row * p.ld_a + ch, n, p.lv_a, g);
}

// 16 channels of the second half: where the half is no multiple of 16 their codes are not aligned and may have two scales
template <int CODE> __device__ __forceinline__ void read_up(const Act8Args &p, size_t row, int ch, int n, float (&u)[16]) {
    const int c0 = p.half + ch;
    if ((p.half & 15) == 0 && n > 0) {
        read16<CODE>(p.ck, row, c0, u);
        return;
    }
    const uint8_t *codes = p.ck.codes + row * p.ck.pitch + c0;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        u[i] = 0.f;
        if (i < n) {
            float t[16];
            decode16<CODE>(make_uint4(codes[i], 0u, 0u, 0u), byte_of(p.ck.scales + scale_index(p.ck, row, c0 + i)), t);
            u[i] = t[0];
        }
    }
}

template <class T, int CODE, int ACT>
__global__ void __launch_bounds__(kThreads) act8_load_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    if (!place(p, blockIdx.x * kThreads + threadIdx.x, row, ch)) return;
    const int n = left(p.half, ch);
    if (n <= 0) return;                              // the second group of a padded block
    float v[16];
    read16<CODE>(p.ck, row, ch, v);
    if constexpr (ACT == REVNET_ACT_SWIGLU) {
        float u[16];
        read_up<CODE>(p, row, ch, n, u);
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] = act<REVNET_ACT_SILU>(v[i]) * u[i];
    } else {
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] = act<ACT>(v[i]);
    }
    store16((T *)p.a + row * p.ld_a + ch, n, p.lv_a, v);
}

template <class T, int CODE, int ACT>
__global__ void __launch_bounds__(kThreads) act8_bwd_kernel(const Act8Args p) {
    pdl_enter();
    size_t row; int ch;
    const bool live = place(p, blockIdx.x * kThreads + threadIdx.x, row, ch);
    const int n = live ? left(p.half, ch) : 0;
    float x[16], da[16], a[16];
    load16((const T *)p.x + row * p.ld_x + ch, n, p.lv_x, da);
    read16<CODE>(p.ck, row, ch, x);                  // codes of a padded row end are zeros
    T *dx = (T *)p.a + row * p.ld_a + ch;
    if constexpr (ACT == REVNET_ACT_SWIGLU) {
        float u[16], du[16];
        read_up<CODE>(p, row, ch, n, u);
#pragma unroll
        for (int i = 0; i < 16; i++) {
            float s, d;
            act_grad<REVNET_ACT_SILU>(x[i], s, d);
            a[i] = i < n ? s * u[i] : 0.f;           // behind the half's end x and u are the neighbours' values
            du[i] = da[i] * s;
            x[i] = da[i] * u[i] * d;
        }
        store16(dx, n, p.lv_a, x);
        store16(dx + p.half, n, p.lv_u, du);
    } else {
#pragma unroll
        for (int i = 0; i < 16; i++) {
            float d;
            act_grad<ACT>(x[i], a[i], d);
            x[i] = ACT == REVNET_ACT_RELU && d == 0.f ? 0.f : da[i] * d;      // an infinite gradient stops at a closed ReLU too
        }
        store16(dx, n, p.lv_a, x);
    }
    if (p.out.codes) keep16<CODE>(p.out, row, ch, live, a);
}

bool fill(Act8Args &p, const revnet_act_desc &d, int channels_per_row) {
    const bool gated = d.act == REVNET_ACT_SWIGLU;
    p.channels = d.channels;
    p.half = gated ? d.channels / 2 : d.channels;
    const uint32_t per_row = (uint32_t)ck_pitch(channels_per_row) / kGroup;
    p.per_row = fast_div(per_row);
    p.total = (uint32_t)d.rows * per_row;            // the entry points keep it below 2^31
    return p.total > 0;
}
unsigned blocks(const Act8Args &p) { return (p.total + kThreads - 1) / kThreads; }
int upper_level(const void *x, int64_t ld, int half, int size) { return access_level((const char *)x + (size_t)half * size, ld, size); }

template <class T, int CODE> void store_t(Exec &ex, Act8Args p, const revnet_act_desc &d, double bytes) {
    const unsigned g = blocks(p);
    if (!p.a) launch_stream(ex, bytes, 0, act8_store_kernel<T, CODE, REVNET_ACT_NONE, false>, g, kThreads, 0, p);
    else if (d.act == REVNET_ACT_NONE) launch_stream(ex, bytes, 0, act8_store_kernel<T, CODE, REVNET_ACT_NONE, true>, g, kThreads, 0, p);
    else if (d.act == REVNET_ACT_RELU) launch_stream(ex, bytes, 0, act8_store_kernel<T, CODE, REVNET_ACT_RELU, true>, g, kThreads, 0, p);
    else if (d.act == REVNET_ACT_GELU) launch_stream(ex, bytes, 0, act8_store_kernel<T, CODE, REVNET_ACT_GELU, true>, g, kThreads, 0, p);
    else launch_stream(ex, bytes, 0, act8_store_kernel<T, CODE, REVNET_ACT_SILU, true>, g, kThreads, 0, p);
    ex.check("act8_store", bytes);
}
template <class T, int CODE> void load_t(Exec &ex, const Act8Args &p, const revnet_act_desc &d, double bytes) {
    const unsigned g = blocks(p);
    switch (d.act) {
        case REVNET_ACT_NONE: launch_stream(ex, bytes, 0, act8_load_kernel<T, CODE, REVNET_ACT_NONE>, g, kThreads, 0, p); break;
        case REVNET_ACT_RELU: launch_stream(ex, bytes, 0, act8_load_kernel<T, CODE, REVNET_ACT_RELU>, g, kThreads, 0, p); break;
        case REVNET_ACT_GELU: launch_stream(ex, bytes, 0, act8_load_kernel<T, CODE, REVNET_ACT_GELU>, g, kThreads, 0, p); break;
        case REVNET_ACT_SILU: launch_stream(ex, bytes, 0, act8_load_kernel<T, CODE, REVNET_ACT_SILU>, g, kThreads, 0, p); break;
        default: launch_stream(ex, bytes, 0, act8_load_kernel<T, CODE, REVNET_ACT_SWIGLU>, g, kThreads, 0, p); break;
    }
    ex.check("act8_load", bytes);
}
template <class T, int CODE> void bwd_t(Exec &ex, const Act8Args &p, const revnet_act_desc &d, double bytes) {
    const unsigned g = blocks(p);
    switch (d.act) {
        case REVNET_ACT_NONE: launch_stream(ex, bytes, 0, act8_bwd_kernel<T, CODE, REVNET_ACT_NONE>, g, kThreads, 0, p); break;
        case REVNET_ACT_RELU: launch_stream(ex, bytes, 0, act8_bwd_kernel<T, CODE, REVNET_ACT_RELU>, g, kThreads, 0, p); break;
        case REVNET_ACT_GELU: launch_stream(ex, bytes, 0, act8_bwd_kernel<T, CODE, REVNET_ACT_GELU>, g, kThreads, 0, p); break;
        case REVNET_ACT_SILU: launch_stream(ex, bytes, 0, act8_bwd_kernel<T, CODE, REVNET_ACT_SILU>, g, kThreads, 0, p); break;
        default: launch_stream(ex, bytes, 0, act8_bwd_kernel<T, CODE, REVNET_ACT_SWIGLU>, g, kThreads, 0, p); break;
    }
    ex.check("act8_bwd", bytes);
}
template <class F> void by_type(const revnet_act_desc &d, F &&f) {
    if (d.dtype == REVNET_F32) { if (d.code == REVNET_INT8) f(float(), std::integral_constant<int, REVNET_INT8>()); else f(float(), std::integral_constant<int, REVNET_E4M3>()); }
    else { if (d.code == REVNET_INT8) f(bf16(), std::integral_constant<int, REVNET_INT8>()); else f(bf16(), std::integral_constant<int, REVNET_E4M3>()); }
}

}  // namespace

void act8_store(Exec &ex, const revnet_act_desc &d, const void *x, void *ck, void *a) {
    const int size = d.dtype == REVNET_F32 ? 4 : 2;
    const bool gated = d.act == REVNET_ACT_SWIGLU;
    Act8Args p{};
    p.x = x; p.a = a; p.ck = ck_view(ck, d.rows, d.channels);
    p.ld_x = d.ld_x; p.ld_a = d.ld_a;
    p.lv_x = access_level(x, d.ld_x, size); p.lv_a = access_level(a, d.ld_a, size);
    p.lv_u = upper_level(x, d.ld_x, d.channels / 2, size);
    const double n = (double)d.rows * d.channels, out = a ? (gated ? n / 2 : n) * size : 0;
    if (!(gated && a)) {
        if (fill(p, d, d.channels)) by_type(d, [&](auto t, auto c) { store_t<decltype(t), decltype(c)::value>(ex, p, d, n * (size + 1) + out); });
        return;
    }
    if (d.channels / 2 % 32 == 0) {
        if (!fill(p, d, d.channels / 2)) return;
        by_type(d, [&](auto t, auto c) {
            launch_stream(ex, n * (size + 1) + out, 0, act8_store_gated_kernel<decltype(t), decltype(c)::value>, blocks(p), kThreads, 0, p);
        });
        ex.check("act8_store", n * (size + 1) + out);
        return;
    }
    Act8Args only = p;
    only.a = nullptr;
    if (!fill(only, d, d.channels)) return;
    by_type(d, [&](auto t, auto c) { store_t<decltype(t), decltype(c)::value>(ex, only, d, n * (size + 1)); });
    fill(p, d, d.channels / 2);
    if (d.dtype == REVNET_F32) launch_stream(ex, n * size + out, 0, act8_gate_kernel<float>, blocks(p), kThreads, 0, p);
    else launch_stream(ex, n * size + out, 0, act8_gate_kernel<bf16>, blocks(p), kThreads, 0, p);
    ex.check("act8_gate", n * size + out);
}

void act8_load(Exec &ex, const revnet_act_desc &d, const void *ck, void *a) {
    const int size = d.dtype == REVNET_F32 ? 4 : 2;
    Act8Args p{};
    p.a = a; p.ck = ck_view(ck, d.rows, d.channels);
    p.ld_a = d.ld_a; p.lv_a = access_level(a, d.ld_a, size);
    if (!fill(p, d, d.act == REVNET_ACT_SWIGLU ? d.channels / 2 : d.channels)) return;
    const double bytes = (double)d.rows * (d.channels + (double)p.half * size);
    by_type(d, [&](auto t, auto c) { load_t<decltype(t), decltype(c)::value>(ex, p, d, bytes); });
}

void act8_bwd(Exec &ex, const revnet_act_desc &d, const void *ck, const void *da, void *dx, void *a_ck) {
    const int size = d.dtype == REVNET_F32 ? 4 : 2;
    const int out = d.act == REVNET_ACT_SWIGLU ? d.channels / 2 : d.channels;
    Act8Args p{};
    p.x = da; p.a = dx; p.ck = ck_view(ck, d.rows, d.channels); p.out = ck_view(a_ck, d.rows, out);
    p.ld_x = d.ld_a; p.ld_a = d.ld_x;
    p.lv_x = access_level(da, d.ld_a, size); p.lv_a = access_level(dx, d.ld_x, size);
    p.lv_u = upper_level(dx, d.ld_x, d.channels / 2, size);
    if (!fill(p, d, out)) return;
    const double bytes = (double)d.rows * (d.channels * (1.0 + size) + out * (size + (a_ck ? 1.0 : 0.0)));
    by_type(d, [&](auto t, auto c) { bwd_t<decltype(t), decltype(c)::value>(ex, p, d, bytes); });
}
