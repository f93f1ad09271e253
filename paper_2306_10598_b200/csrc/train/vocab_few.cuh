// The loss of a few tokens: one pass over the weight, which is all that such a call costs.
//
// With up to 16 tokens the tiles of the general path are nearly empty, and its gathering of rows and setting up of tensor
// memory cost as much as the weight's bytes.  Here a warp multiplies 16 rows of the weight with all tokens by small matrix
// instructions (16 x 8 x 16); it reads the rows straight into their operands, 16 bytes to a thread.  The order of the summed
// elements is free as long as both operands have the same one: thread t of a row's four takes elements 8t ... 8t + 7 of each
// 32, which feed two instructions.  Maximum and sum of exp stay in registers over all rows of the vocabulary that a warp meets.
// Bound by the weight's bytes: 8 tokens x 32000 x 1024 bf16 are 65.5 MB, 10 us at the copy rate.  Measured, this path / the
// general one: 1 token 17.9 / 25.8 us, 8 tokens 17.7 / 26.2, 16 tokens 20.0 / 26.4, and 32 tokens, which it was built for too,
// 28.9 / 27.2 (every block brings in all tokens), hence the limit; 8 tokens x 128000 49 us (5.3 TB/s).
#pragma once

#include "tensor_core.cuh"

namespace dct {

constexpr int kFewTokens = 16, kFewThreads = 256, kFewSmem = 96 * 1024, kMostFewBlocks = 512;
// rows of h in shared memory are 64 bytes further apart than their length, so that 8 threads reading 16 bytes meet no bank twice
inline int few_pitch(int64_t D) { return (int)(ceil_div(D, 32) * 64 + 64); }
inline int few_tiles(int64_t N) { return N <= 8 ? 1 : 2; }
// tokens, and rows that can be read 16 bytes at a time
inline bool few(int64_t N, int64_t D, const void *hidden, int64_t hs, const void *weight, int64_t ws)
{
    return N <= kFewTokens && D % 8 == 0 && rows_on(hidden, hs, 2, 16) && rows_on(weight, ws, 2, 16) && D <= 65536 &&
           8 * few_tiles(N) * few_pitch(D) <= kFewSmem;
}

__device__ __forceinline__ void few_product(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void few_product(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes that are read once: the memory's whole 256 bytes come into L2, where the warp's next reads find them
__device__ __forceinline__ uint4 read_once(const void *p)
{
    uint4 r;
    asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

struct Few {
    const void *hidden; int64_t hs;
    const void *weight; int64_t ws;
    const int64_t *targets; int64_t ignore, V;
    int32_t N, D, pitch;
    float scale;                 // logit_scale * log2(e)
    float2 *part; float *hit;    // [tokens][blocks], [tokens]
};

template <class T, int NT>
__global__ void __launch_bounds__(kFewThreads, 2) vocab_few(const __grid_constant__ Few a)
{
    constexpr int U = 8, W = kFewThreads / 32;                   // U times 32 elements of 16 rows on their way
    extern __shared__ __align__(16) uint8_t room[];
    __shared__ float2 of_warp[W][NT * 8];
    __shared__ int32_t label[NT * 8];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const T *weight = (const T *)a.weight;
    const int32_t groups = (int32_t)((a.V + 15) / 16), step = gridDim.x * W;
    uint4 x[U], y[U];
    auto fetch = [&](int64_t v, int32_t k0) {
        const T *r0 = weight + v * a.ws, *r1 = r0 + 8 * a.ws;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t k = k0 + u * 32 + t * 8;
            x[u] = y[u] = make_uint4(0, 0, 0, 0);
            if (k < a.D) {
                if (v < a.V) x[u] = read_once(r0 + k);
                if (v + 8 < a.V) y[u] = read_once(r1 + k);
            }
        }
    };
    follow();
    int32_t group = blockIdx.x * W + warp;
    if (group < groups) fetch((int64_t)group * 16 + g, 0);       // on its way while the tokens come in
    if (tid < NT * 8) {
        int64_t l = -1;
        if (tid < a.N) {
            l = a.targets[tid];
            if (l == a.ignore || l < 0 || l >= a.V) l = -1;
        }
        label[tid] = (int32_t)l;
    }
    __syncthreads();
    for (int32_t i = tid; i < NT * 8 * (a.pitch / 16); i += kFewThreads) {
        const int32_t n = i / (a.pitch / 16), k = (i - n * (a.pitch / 16)) * 8;
        uint4 h = make_uint4(0, 0, 0, 0);                        // rows without a label too: what they hold is not used
        if (label[n] >= 0 && k < a.D) h = *reinterpret_cast<const uint4 *>((const T *)a.hidden + n * a.hs + k);
        *reinterpret_cast<uint4 *>(room + n * a.pitch + k * 2) = h;
    }
    __syncthreads();

    float m[NT][2], s[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) { m[j][e] = -INFINITY; s[j][e] = 0.0f; }
    const uint8_t *mine = room + g * a.pitch + t * 16;
    bool first = true;
    for (; group < groups; group += step) {
        const int64_t v = (int64_t)group * 16 + g;
        float c[NT][4] = {};
        for (int32_t k0 = 0; k0 < a.D; k0 += 32 * U) {
            if (!first) fetch(v, k0);
            first = false;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int32_t k = k0 + u * 32;
                if (k >= a.D) break;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const uint4 h = *reinterpret_cast<const uint4 *>(mine + j * 8 * a.pitch + k * 2);
                    few_product(c[j], x[u].x, y[u].x, x[u].y, y[u].y, h.x, h.y, T());
                    few_product(c[j], x[u].z, y[u].z, x[u].w, y[u].w, h.z, h.w, T());
                }
            }
        }
        // c[j][0], c[j][1]: row v with tokens 8j + 2t and the next; c[j][2], c[j][3]: row v + 8
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int32_t l = label[j * 8 + 2 * t + e];
                const float z0 = v < a.V ? c[j][e] * a.scale : -INFINITY, z1 = v + 8 < a.V ? c[j][2 + e] * a.scale : -INFINITY;
                if (l == v) a.hit[j * 8 + 2 * t + e] = z0 * 0.6931471805599453f;
                if (l == v + 8) a.hit[j * 8 + 2 * t + e] = z1 * 0.6931471805599453f;
                const float top = fmaxf(fmaxf(z0, z1), m[j][e]), ref = top == -INFINITY ? 0.0f : top;
                s[j][e] = s[j][e] * exp2_fast(m[j][e] - ref) + exp2_fast(z0 - ref) + exp2_fast(z1 - ref);
                m[j][e] = top;
            }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) join_parts(m[j][e], s[j][e], __shfl_xor_sync(~0u, m[j][e], d), __shfl_xor_sync(~0u, s[j][e], d));
            if (g == 0) of_warp[warp][j * 8 + 2 * t + e] = make_float2(m[j][e], s[j][e]);
        }
    __syncthreads();
    if (tid < a.N) {
        float2 r = of_warp[0][tid];
        for (int w = 1; w < W; ++w) join_parts(r.x, r.y, of_warp[w][tid].x, of_warp[w][tid].y);
        a.part[(int64_t)tid * gridDim.x + blockIdx.x] = r;
    }
}

// A warp per token: the blocks' parts joined, and the label's logit in fp32; tokens without a label are written here.
template <class T>
__global__ void __launch_bounds__(128) vocab_few_join(const __grid_constant__ Few a, int32_t blocks, float *__restrict__ loss, float *__restrict__ lse)
{
    const int lane = threadIdx.x & 31;
    const int32_t n = blockIdx.x * 4 + (threadIdx.x >> 5);
    follow();
    if (n >= a.N) return;
    const int64_t l = a.targets[n];
    if (l == a.ignore || l < 0 || l >= a.V) {
        if (lane == 0) loss[n] = lse[n] = l == a.ignore ? 0.0f : __uint_as_float(0x7fffffffu);
        return;
    }
    float exact = 0.0f;
    for (int32_t d = lane * 8; d < a.D; d += 256) {
        const Pack<T, 8> h = *reinterpret_cast<const Pack<T, 8> *>((const T *)a.hidden + n * a.hs + d);
        const Pack<T, 8> w = *reinterpret_cast<const Pack<T, 8> *>((const T *)a.weight + l * a.ws + d);
#pragma unroll
        for (int i = 0; i < 8; ++i) exact = fmaf(to_f(h.v[i]), to_f(w.v[i]), exact);
    }
    float m = -INFINITY, s = 0.0f;
    for (int32_t b = lane; b < blocks; b += 32) join_parts(m, s, a.part[(int64_t)n * blocks + b].x, a.part[(int64_t)n * blocks + b].y);
    for (int d = 16; d; d >>= 1) {
        exact += __shfl_xor_sync(~0u, exact, d);
        join_parts(m, s, __shfl_xor_sync(~0u, m, d), __shfl_xor_sync(~0u, s, d));
    }
    if (lane == 0) {
        exact *= a.scale * 0.6931471805599453f;
        const float z = with_label((m + log2f(s)) * 0.6931471805599453f, a.hit[n], exact);
        lse[n] = z;
        loss[n] = z - exact;
    }
}

// Two blocks to a multiprocessor, fewer where the vocabulary has not as many rows.
inline int32_t few_blocks(int64_t V)
{
    const int64_t held = 2 * (int64_t)sm_count(), most = held < kMostFewBlocks ? held : kMostFewBlocks, need = ceil_div(ceil_div(V, 16), kFewThreads / 32);
    return (int32_t)(need < most ? need : most);
}

template <class T, int NT> int few_launch(const Few &a, int32_t blocks, cudaStream_t st)
{
    static int ready[64] = {};                                   // the kernel may use its shared memory on this device
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return DC_ERR_CUDA;
    if (!__atomic_load_n(&ready[dev], __ATOMIC_ACQUIRE)) {
        if (cudaFuncSetAttribute(vocab_few<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem) != cudaSuccess) return DC_ERR_CUDA;
        __atomic_store_n(&ready[dev], 1, __ATOMIC_RELEASE);
    }
    return launch(vocab_few<T, NT>, dim3((unsigned)blocks), kFewThreads, (size_t)(8 * NT * a.pitch), st, a);
}

}  // namespace dct
