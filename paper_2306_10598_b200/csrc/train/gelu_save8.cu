// dc_gelu_save8 and its backward pass: gelu with x kept as 8-bit integers and one scale per 128 neighbours of a row.
//
// Both kernels touch every element once (16-bit types: forward 2 bytes in, 2 + 1 out; backward 2 + 1 in, 2 + 2 out) and do
// about 30 operations on it, so memory bounds them.  A group of 128 is held by 128/V lanes with V adjacent elements each
// (V = 16 bytes' worth), which makes its maximum a few shuffles and leaves nothing to pass through shared memory.
#include "train_common.cuh"

namespace dct {

constexpr int kGroup = DC_SAVE8_GROUP;
constexpr float kTwoA = 1.5957691216057308f;   // 2 sqrt(2/pi)
constexpr float kB = 0.044715f;
constexpr int kThreads = 256;

// sigma(2u), u = sqrt(2/pi)(v + B v^3), so that gelu(v) = v gate(v).  exp overflows to +inf for very negative v, which
// gives the gate 0.
__device__ __forceinline__ float gate(float v)
{
    return __fdividef(1.0f, 1.0f + __expf(-kTwoA * (v + kB * v * v * v)));
}

// How the lanes of a warp hold a group: packs of V elements, LPG lanes to a group, K packs to a lane.
template <class T, int V> struct Hold {
    static constexpr int LPG = kGroup / V < 32 ? kGroup / V : 32;
    static constexpr int K = kGroup / (V * LPG);
};

// The groups a thread works on: first, then every `step`-th, as (row, group of the row) without a division per group.
struct GroupWalk {
    int64_t row, drow, left;
    int32_t g, dg, per_row;
    __device__ GroupWalk(int64_t first, int64_t step, int64_t total, int32_t per_row_) : per_row(per_row_)
    {
        row = first / per_row;
        g = (int32_t)(first - row * per_row);
        drow = step / per_row;
        dg = (int32_t)(step - drow * per_row);
        left = first < total ? (total - first + step - 1) / step : 0;
    }
    __device__ __forceinline__ void next()
    {
        --left;
        row += drow;
        g += dg;
        if (g >= per_row) { g -= per_row; ++row; }
    }
};

template <class T, int V>
__global__ void __launch_bounds__(kThreads) gelu_save8_kernel(const T *__restrict__ x, int64_t xs, int64_t N, int32_t D, T *__restrict__ y, int64_t ys,
                                                              int8_t *__restrict__ q, float *__restrict__ scales)
{
    using H = Hold<T, V>;
    const int lane = threadIdx.x % H::LPG;
    const int32_t per_row = (D + kGroup - 1) / kGroup;
    const int64_t total = N * per_row, step = (int64_t)gridDim.x * (kThreads / H::LPG);
    GroupWalk w((int64_t)blockIdx.x * (kThreads / H::LPG) + threadIdx.x / H::LPG, step, total, per_row);
    // the lanes of a warp stay together: all go on while one of them has a group left
    while (__any_sync(~0u, w.left > 0)) {
        float v[H::K][V];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < H::K; ++k) {
            const int32_t c = w.g * kGroup + (k * H::LPG + lane) * V;
            Pack<T, V> p = {};
            if (w.left > 0 && c < D) p = *reinterpret_cast<const Pack<T, V> *>(x + w.row * xs + c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i] = to_f(p.v[i]);
                top = max(top, __float_as_uint(fabsf(v[k][i])));   // the bits of non-negative floats keep their order; NaN is on top
            }
        }
#pragma unroll
        for (int m = H::LPG / 2; m; m >>= 1) top = max(top, __shfl_xor_sync(~0u, top, m));
        const float a = __uint_as_float(top);
        const bool finite = top < 0x7f800000u;
        const bool live = a > 0x1p-100f && finite;
        const float inv = live ? __fdiv_rn(127.0f, a) : 0.0f;
        const float scale = live ? __fmul_rn(a, 1.0f / 127.0f) : finite ? 0.0f : __uint_as_float(0x7fffffffu);
        if (w.left > 0) {
            if (lane == 0) scales[w.row * per_row + w.g] = scale;
#pragma unroll
            for (int k = 0; k < H::K; ++k) {
                const int32_t c = w.g * kGroup + (k * H::LPG + lane) * V;
                if (c >= D) continue;
                Pack<T, V> o;
                Pack<int8_t, V> b;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    o.v[i] = from_f<T>(v[k][i] * gate(v[k][i]));
                    b.v[i] = live ? (int8_t)__float2int_rn(__fmul_rn(v[k][i], inv)) : (int8_t)0;
                }
                *reinterpret_cast<Pack<T, V> *>(y + w.row * ys + c) = o;
                *reinterpret_cast<Pack<int8_t, V> *>(q + w.row * D + c) = b;
            }
        }
        if (w.left > 0) w.next();
    }
}

template <class T, int V>
__global__ void __launch_bounds__(kThreads) gelu_save8_backward_kernel(const T *__restrict__ dy, int64_t dys, const int8_t *__restrict__ q,
                                                                       const float *__restrict__ scales, int64_t N, int32_t D, T *__restrict__ dx,
                                                                       int64_t dxs, T *__restrict__ y, int64_t ys)
{
    using H = Hold<T, V>;
    const int lane = threadIdx.x % H::LPG;
    const int32_t per_row = (D + kGroup - 1) / kGroup;
    const int64_t total = N * per_row, step = (int64_t)gridDim.x * (kThreads / H::LPG);
    for (GroupWalk w((int64_t)blockIdx.x * (kThreads / H::LPG) + threadIdx.x / H::LPG, step, total, per_row); w.left > 0; w.next()) {
        const float scale = scales[w.row * per_row + w.g];
#pragma unroll
        for (int k = 0; k < H::K; ++k) {
            const int32_t c = w.g * kGroup + (k * H::LPG + lane) * V;
            if (c >= D) continue;
            const Pack<T, V> d = *reinterpret_cast<const Pack<T, V> *>(dy + w.row * dys + c);
            const Pack<int8_t, V> b = *reinterpret_cast<const Pack<int8_t, V> *>(q + w.row * D + c);
            Pack<T, V> o, r;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float v = (float)b.v[i] * scale, s = gate(v);
                const float near = fminf(fmaxf(v, -64.0f), 64.0f);   // beyond, s (1 - s) is 0 and v^2 must not make it NaN
                const float slope = s + near * s * (1.0f - s) * (kTwoA + 3.0f * kB * kTwoA * near * near);
                o.v[i] = from_f<T>(to_f(d.v[i]) * (isnan(v) ? v : slope));
                r.v[i] = from_f<T>(v * s);
            }
            *reinterpret_cast<Pack<T, V> *>(dx + w.row * dxs + c) = o;
            if (y) *reinterpret_cast<Pack<T, V> *>(y + w.row * ys + c) = r;
        }
    }
}

// As many blocks as the device holds at once, or as there is work for.
inline int64_t grid_for(int64_t N, int64_t D, int lanes_per_group)
{
    const int64_t groups = N * ceil_div(D, kGroup), blocks = ceil_div(groups, kThreads / lanes_per_group);
    const int64_t most = (int64_t)sm_count() * (2048 / kThreads);
    return blocks < most ? blocks : most;
}

inline int check(int64_t N, int64_t D, int32_t dtype)
{
    if (N < 0 || D <= 0) return DC_ERR_SHAPE;
    if (N > kMaxDim || D > kMaxDim) return DC_ERR_RANGE;
    if (dtype != DC_BF16 && dtype != DC_F16 && dtype != DC_F32) return DC_ERR_UNSUPPORTED;
    return DC_OK;
}

template <class T, int V>
int forward(const void *x, int64_t xs, int64_t N, int64_t D, void *y, int64_t ys, int8_t *q, float *scales, cudaStream_t st)
{
    gelu_save8_kernel<T, V><<<(unsigned)grid_for(N, D, Hold<T, V>::LPG), kThreads, 0, st>>>((const T *)x, xs, N, (int32_t)D, (T *)y, ys, q, scales);
    return launched();
}
template <class T, int V>
int backward(const void *dy, int64_t dys, const int8_t *q, const float *scales, int64_t N, int64_t D, void *dx, int64_t dxs, void *y, int64_t ys,
             cudaStream_t st)
{
    gelu_save8_backward_kernel<T, V><<<(unsigned)grid_for(N, D, Hold<T, V>::LPG), kThreads, 0, st>>>((const T *)dy, dys, q, scales, N, (int32_t)D,
                                                                                                     (T *)dx, dxs, (T *)y, ys);
    return launched();
}

}  // namespace dct

using namespace dct;

extern "C" int dc_gelu_save8(const void *x, int64_t x_stride, int32_t dtype, int64_t N, int64_t D, void *y, int64_t y_stride, int8_t *q,
                             float *scales, void *stream)
{
    if (int e = check(N, D, dtype)) return e;
    if (N == 0) return DC_OK;
    if (!x || !y || !q || !scales) return DC_ERR_NULL;
    const int eb = elem_bytes(dtype), V = 16 / eb;
    if (x_stride < D || y_stride < D) return DC_ERR_SHAPE;
    if (!on(x, eb) || !on(y, eb) || !on(scales, 4)) return DC_ERR_ALIGN;
    if (sm_count() == 0) return DC_ERR_CUDA;
    const bool wide = D % V == 0 && rows_on(x, x_stride, eb, 16) && rows_on(y, y_stride, eb, 16) && on(q, V);
    const cudaStream_t st = (cudaStream_t)stream;
    if (dtype == DC_BF16) return wide ? forward<__nv_bfloat16, 8>(x, x_stride, N, D, y, y_stride, q, scales, st)
                                      : forward<__nv_bfloat16, 1>(x, x_stride, N, D, y, y_stride, q, scales, st);
    if (dtype == DC_F16) return wide ? forward<__half, 8>(x, x_stride, N, D, y, y_stride, q, scales, st)
                                     : forward<__half, 1>(x, x_stride, N, D, y, y_stride, q, scales, st);
    return wide ? forward<float, 4>(x, x_stride, N, D, y, y_stride, q, scales, st) : forward<float, 1>(x, x_stride, N, D, y, y_stride, q, scales, st);
}

extern "C" int dc_gelu_save8_backward(const void *dy, int64_t dy_stride, int32_t dtype, const int8_t *q, const float *scales, int64_t N, int64_t D,
                                      void *dx, int64_t dx_stride, void *y_again, int64_t y_again_stride, void *stream)
{
    if (int e = check(N, D, dtype)) return e;
    if (N == 0) return DC_OK;
    if (!dy || !q || !scales || !dx) return DC_ERR_NULL;
    const int eb = elem_bytes(dtype), V = 16 / eb;
    if (dy_stride < D || dx_stride < D || (y_again && y_again_stride < D)) return DC_ERR_SHAPE;
    if (!on(dy, eb) || !on(dx, eb) || !on(y_again, eb) || !on(scales, 4)) return DC_ERR_ALIGN;
    if (sm_count() == 0) return DC_ERR_CUDA;
    const bool wide = D % V == 0 && rows_on(dy, dy_stride, eb, 16) && rows_on(dx, dx_stride, eb, 16) &&
                      (!y_again || rows_on(y_again, y_again_stride, eb, 16)) && on(q, V);
    const cudaStream_t st = (cudaStream_t)stream;
#define DCT_BACK(T, V) backward<T, V>(dy, dy_stride, q, scales, N, D, dx, dx_stride, y_again, y_again_stride, st)
    if (dtype == DC_BF16) return wide ? DCT_BACK(__nv_bfloat16, 8) : DCT_BACK(__nv_bfloat16, 1);
    if (dtype == DC_F16) return wide ? DCT_BACK(__half, 8) : DCT_BACK(__half, 1);
    return wide ? DCT_BACK(float, 4) : DCT_BACK(float, 1);
#undef DCT_BACK
}
