// The three products of the vocabulary loss, with what is done to a tile of them before it leaves the chip.
#pragma once

#include "train_common.cuh"

namespace dct {

__device__ unsigned int g_train_wait_expired = 0;

constexpr int kTileM = 256, kTileN = 256;   // rows and columns of a tile of the result
constexpr int kRowBlock = 64;               // what a product over rows or tokens takes at a time
constexpr int64_t kPieceBytes = int64_t(256) << 20;   // g of one piece of the vocabulary

// What vocab_gather finds out on the device.
struct Head {
    int32_t rows;                           // labelled rows
    float grad_scale, grad_unscale;         // power of two that g carries, and its inverse
};

// Partial products of dh: one.
__host__ __device__ inline int32_t split_of(int32_t rows, int32_t tiles_d, int32_t vocab_blocks) { return 1; }
inline int64_t acc_rows(int64_t N, int32_t tiles_d) { return ceil_div(N, kTileM) * kTileM; }

// ---- a plain tile product: 64 x 64 results, 256 threads with 4 x 4 each --------------------------------------------------

constexpr int kS = 64, kK = 16;

// C[i][j] = sum_k A(i,k) B(j,k); A(i,k) = a[i*ai + k*ak], zero outside [0,I) x [0,K); B alike.
template <class T>
__device__ __forceinline__ void tile_product(float (&c)[4][4], const T *a, int64_t ai, int64_t ak, int64_t i0, int64_t I, const T *b, int64_t bj, int64_t bk,
                                             int64_t j0, int64_t J, int64_t K, float (*sa)[kS + 1], float (*sb)[kS + 1])
{
    const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = 0.0f;
    for (int64_t k0 = 0; k0 < K; k0 += kK) {
        __syncthreads();
        for (int e = tid; e < kS * kK; e += 256) {
            const int ia = ak == 1 ? e / kK : e % kS, ka = ak == 1 ? e % kK : e / kS;
            sa[ka][ia] = i0 + ia < I && k0 + ka < K ? to_f(a[(i0 + ia) * ai + (k0 + ka) * ak]) : 0.0f;
            const int ib = bk == 1 ? e / kK : e % kS, kb = bk == 1 ? e % kK : e / kS;
            sb[kb][ib] = j0 + ib < J && k0 + kb < K ? to_f(b[(j0 + ib) * bj + (k0 + kb) * bk]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            float x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = sa[k][ty * 4 + i]; y[i] = sb[k][tx * 4 + i]; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) c[i][j] = fmaf(x[i], y[j], c[i][j]);
        }
    }
}

#define DCT_SHARED __shared__ float sa[kK][kS + 1], sb[kK][kS + 1]; float c[4][4]; const int ty = threadIdx.x / 16, tx = threadIdx.x % 16

template <class T>
__global__ void __launch_bounds__(256) loss_kernel(const Head *head, const T *h, int64_t hs, const T *w, int64_t ws, const int32_t *label, int64_t V, int64_t D,
                                                   float scale, float2 *part, float *hit, int32_t tiles_v)
{
    DCT_SHARED;
    const int64_t L = head->rows, i0 = (int64_t)blockIdx.y * kS, t = blockIdx.x;
    if (i0 >= L) return;
    float m[4], s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { m[i] = -INFINITY; s[i] = 0.0f; }
    for (int64_t j0 = t * kTileN; j0 < (t + 1) * kTileN && j0 < V; j0 += kS) {
        tile_product(c, h, hs, 1, i0, L, w, ws, 1, j0, V, D, sa, sb);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = i0 + ty * 4 + i;
            float top = m[i];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j0 + tx * 4 + j < V) {
                    top = fmaxf(top, c[i][j] * scale);
                    if (r < L && label[r] == j0 + tx * 4 + j) hit[r] = c[i][j] * scale;
                }
            float sum = m[i] == -INFINITY ? s[i] : s[i] * __expf(m[i] - top);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j0 + tx * 4 + j < V) sum += top == -INFINITY && c[i][j] * scale == -INFINITY ? 0.0f : __expf(c[i][j] * scale - top);
            m[i] = top;
            s[i] = sum;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int d = 8; d; d >>= 1) {
            const float om = __shfl_xor_sync(~0u, m[i], d), os = __shfl_xor_sync(~0u, s[i], d), n = fmaxf(m[i], om);
            s[i] = (m[i] == -INFINITY ? s[i] : s[i] * __expf(m[i] - n)) + (om == -INFINITY ? os : os * __expf(om - n));
            m[i] = n;
        }
        if (tx == 0 && i0 + ty * 4 + i < L) part[(i0 + ty * 4 + i) * tiles_v + t] = make_float2(m[i], s[i]);
    }
}

template <class T>
__global__ void __launch_bounds__(256) grad_kernel(const Head *head, const T *h, int64_t hs, const T *w, int64_t ws, const int32_t *label, const float *lse,
                                                   const float *dloss, int64_t v0, int64_t nv, int64_t D, float scale, T *g, int64_t gs)
{
    DCT_SHARED;
    const int64_t L = head->rows, i0 = (int64_t)blockIdx.y * kS, j0 = (int64_t)blockIdx.x * kS;
    if (i0 >= L) return;
    tile_product(c, h, hs, 1, i0, L, w, ws, 1, j0, nv, D, sa, sb);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t r = i0 + ty * 4 + i, v = j0 + tx * 4 + j;
            float x = 0.0f;
            if (r < L && v < nv) x = (__expf(c[i][j] * scale - lse[r]) - (label[r] == v0 + v ? 1.0f : 0.0f)) * (dloss[r] * head->grad_scale);
            g[r * gs + v] = from_f<T>(x);
        }
}

template <class T, class O>
__global__ void __launch_bounds__(256) weight_grad_kernel(const Head *head, const T *g, int64_t gs, const T *h, int64_t hs, int64_t nv, int64_t D, O *dw,
                                                          int64_t dws, bool accumulate)
{
    DCT_SHARED;
    const int64_t L = head->rows, i0 = (int64_t)blockIdx.y * kS, j0 = (int64_t)blockIdx.x * kS;
    tile_product(c, g, 1, gs, i0, nv, h, 1, hs, j0, D, L, sa, sb);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t v = i0 + ty * 4 + i, d = j0 + tx * 4 + j;
            if (v >= nv || d >= D) continue;
            O *o = dw + v * dws + d;
            *o = from_f<O>((accumulate ? to_f(*o) : 0.0f) + c[i][j] * head->grad_unscale);
        }
}

template <class T>
__global__ void __launch_bounds__(256) hidden_grad_kernel(const Head *head, const T *g, int64_t gs, const T *w, int64_t ws, int64_t nv, int64_t D, float *acc,
                                                          int64_t as, bool first)
{
    DCT_SHARED;
    const int64_t L = head->rows, i0 = (int64_t)blockIdx.y * kS, j0 = (int64_t)blockIdx.x * kS;
    if (i0 >= L) return;
    tile_product(c, g, gs, 1, i0, L, w, 1, ws, j0, D, nv, sa, sb);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t r = i0 + ty * 4 + i, d = j0 + tx * 4 + j;
            if (r >= L || d >= D) continue;
            float *o = acc + r * as + d;
            *o = (first ? 0.0f : *o) + c[i][j];
        }
}
#undef DCT_SHARED

// ---- launches -------------------------------------------------------------------------------------------------------------

inline dim3 tiles(int64_t x, int64_t y, int s) { return dim3((unsigned)ceil_div(x, s), (unsigned)ceil_div(y, kS)); }

template <class T>
int loss_product(const Head *head, const void *rows, int64_t rs, const void *w, int64_t ws, const int32_t *label, int64_t N, int64_t V, int64_t D, float scale,
                 float2 *part, float *hit, int32_t tiles_v, cudaStream_t st)
{
    loss_kernel<T><<<tiles(V, N, kTileN), 256, 0, st>>>(head, (const T *)rows, rs, (const T *)w, ws, label, V, D, scale, part, hit, tiles_v);
    return launched();
}

template <class T>
int grad_product(const Head *head, const void *rows, int64_t rs, const void *w, int64_t ws, const int32_t *label, const float *lse, const float *dloss, int64_t N,
                 int64_t v0, int64_t nv, int64_t D, float scale, void *g, int64_t gs, cudaStream_t st)
{
    grad_kernel<T><<<tiles(nv, N, kS), 256, 0, st>>>(head, (const T *)rows, rs, (const T *)w, ws, label, lse, dloss, v0, nv, D, scale, (T *)g, gs);
    return launched();
}

template <class T>
int back_products(const Head *head, const void *g, int64_t gs, const void *rows, int64_t rs, const void *w, int64_t ws, int64_t N, int64_t nv, int64_t D,
                  void *dw, int64_t dws, bool dw_f32, bool accumulate, float *acc, int64_t as, int32_t, int32_t, bool first, cudaStream_t st)
{
    if (dw && dw_f32) weight_grad_kernel<T, float><<<tiles(D, nv, kS), 256, 0, st>>>(head, (const T *)g, gs, (const T *)rows, rs, nv, D, (float *)dw, dws, accumulate);
    if (dw && !dw_f32) weight_grad_kernel<T, T><<<tiles(D, nv, kS), 256, 0, st>>>(head, (const T *)g, gs, (const T *)rows, rs, nv, D, (T *)dw, dws, accumulate);
    if (acc) hidden_grad_kernel<T><<<tiles(D, N, kS), 256, 0, st>>>(head, (const T *)g, gs, (const T *)w, ws, nv, D, acc, as, first);
    return launched();
}

}  // namespace dct
