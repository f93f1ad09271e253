// dc_vocab_loss and dc_vocab_loss_backward: softmax cross entropy over a vocabulary from the hidden states and the output
// weight, without keeping the logits.
//
// With h the labelled rows and W the weight, the logits l = c h W^T of a tile live in registers only:
//   forward   per (row, tile of the vocabulary) the maximum and the sum of exp(l - maximum) leave the kernel; lse joins them
//   backward  per piece of the vocabulary l is formed again, g = (exp(l - lse) - [label]) dloss c is kept in 16 bits,
//             then dW = g^T h and dh += g W
// Rows without a label are taken out first (vocab_gather), so the products run over labelled rows alone and whatever the
// others hold never meets a product.
#include "train_common.cuh"
#include "vocab_gemm.cuh"

namespace dct {

constexpr int kGatherRows = 32;

// ---- taking out the labelled rows ------------------------------------------------------------------------------------------

struct Gather {
    const void *hidden; int64_t hs;
    const int64_t *targets; int64_t ignore;
    const float *lse, *dloss;              // backward only
    int64_t N, V; int32_t D, Dp;
    float logit_scale;
    Head *head; int32_t *row_of, *pos_of, *label; float *row_lse, *row_dloss;
    void *rows;                            // [Lp][Dp]
    float *loss_out, *lse_out;             // forward only: rows without a label are written here
    int32_t scale_grad;                    // whether g needs a power of two (fp16)
};

template <class T, int V>
__global__ void __launch_bounds__(256) vocab_gather(Gather a)
{
    __shared__ int32_t count[8];
    __shared__ float top[8];
    __shared__ int32_t where[kGatherRows];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t first = (int64_t)blockIdx.x * kGatherRows;
    const bool last_block = blockIdx.x == gridDim.x - 1;
    // labelled rows before this block's, and for the last block the largest |dloss|: every block reads what it needs itself
    int32_t c = 0;
    float m = 0.0f;
    for (int64_t i = tid; i < first; i += 256) {
        const int64_t t = a.targets[i];
        const bool ok = t != a.ignore && t >= 0 && t < a.V;
        c += ok;
        if (last_block && a.dloss && ok) m = fmaxf(m, fabsf(a.dloss[i]));
    }
    c = __reduce_add_sync(~0u, c);
    if (lane == 0) count[warp] = c;
    __syncthreads();
    int32_t base = 0;
    for (int w = 0; w < 8; ++w) base += count[w];
    int32_t labelled = 0;
    if (warp == 0) {
        const int64_t i = first + lane;
        const int64_t t = i < a.N ? a.targets[i] : a.ignore;
        const bool ok = i < a.N && t != a.ignore && t >= 0 && t < a.V;
        const uint32_t all = __ballot_sync(~0u, ok);
        const int32_t p = base + __popc(all & ((1u << lane) - 1));
        where[lane] = ok ? p : -1;
        if (i < a.N) {
            a.pos_of[i] = ok ? p : -1;
            if (!ok && a.loss_out) a.loss_out[i] = a.lse_out[i] = t == a.ignore ? 0.0f : __uint_as_float(0x7fffffffu);
        }
        if (ok) {
            a.row_of[p] = (int32_t)i;
            a.label[p] = (int32_t)t;
            if (a.dloss) {
                a.row_lse[p] = a.lse[i];
                a.row_dloss[p] = a.dloss[i] * a.logit_scale;
                m = fmaxf(m, fabsf(a.dloss[i]));
            }
        }
        labelled = __popc(all);
    }
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    if (lane == 0) top[warp] = m;
    __syncthreads();
    if (last_block && tid == 0) {
        for (int w = 0; w < 8; ++w) m = fmaxf(m, top[w]);
        m *= fabsf(a.logit_scale);
        // |g| <= 2^14 in fp16, whatever dloss is: probabilities down to 2^-28 of it stay normal numbers
        int e = 0;
        if (a.scale_grad && m > 0.0f && m < INFINITY) e = min(max(13 - ilogbf(m), -100), 100);
        a.head->rows = base + labelled;
        a.head->grad_scale = ldexpf(1.0f, e);
        a.head->grad_unscale = ldexpf(1.0f, -e);
    }
    const T *hidden = (const T *)a.hidden;
    T *rows = (T *)a.rows;
    for (int j = warp; j < kGatherRows; j += 8) {
        const int32_t p = where[j];
        if (p < 0) continue;
        const T *from = hidden + (first + j) * a.hs;
        T *to = rows + (int64_t)p * a.Dp;
        for (int32_t d = lane * V; d < a.Dp; d += 32 * V) {
            Pack<T, V> x = {};
            if (d < a.D) x = *reinterpret_cast<const Pack<T, V> *>(from + d);
            *reinterpret_cast<Pack<T, V> *>(to + d) = x;
        }
    }
    if (last_block) {
        // the product over rows takes whole blocks of kRowBlock: what follows the last row there is zero
        __shared__ int32_t total;
        if (tid == 0) total = base + labelled;
        __syncthreads();
        const int64_t from = (int64_t)total * a.Dp, to = ceil_div(total, kRowBlock) * kRowBlock * (int64_t)a.Dp;
        for (int64_t d = from + tid * 8; d < to; d += 256 * 8) *reinterpret_cast<uint4 *>(rows + d) = make_uint4(0, 0, 0, 0);
    }
}

// A copy of the weight with rows that start on 16-byte boundaries, where its own do not.
template <class T>
__global__ void __launch_bounds__(256) vocab_copy_weight(const T *__restrict__ w, int64_t ws, int64_t V, int32_t D, int32_t Dp, T *__restrict__ to)
{
    for (int64_t v = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); v < V; v += (int64_t)gridDim.x * 8)
        for (int32_t d = threadIdx.x & 31; d < Dp; d += 32) to[v * Dp + d] = d < D ? w[v * ws + d] : from_f<T>(0.0f);
}

// ---- joining the tiles of the vocabulary: a warp per row --------------------------------------------------------------------

__global__ void __launch_bounds__(256) vocab_join(const Head *__restrict__ head, const int32_t *__restrict__ row_of, const float2 *__restrict__ part,
                                                  const float *__restrict__ hit, int32_t tiles, float *__restrict__ loss, float *__restrict__ lse)
{
    const int lane = threadIdx.x & 31;
    const int64_t j = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (j >= head->rows) return;
    const float2 *p = part + j * tiles;
    float m = -INFINITY, s = 0.0f;
    for (int32_t t = lane; t < tiles; t += 32) {
        const float2 x = p[t];
        const float n = fmaxf(m, x.x);
        // a maximum of -inf stands for a part without a finite logit; its sum is 0, or NaN if it holds one
        s = (m == -INFINITY ? s : s * __expf(m - n)) + (x.x == -INFINITY ? x.y : x.y * __expf(x.x - n));
        m = n;
    }
    for (int d = 16; d; d >>= 1) {
        const float om = __shfl_xor_sync(~0u, m, d), os = __shfl_xor_sync(~0u, s, d), n = fmaxf(m, om);
        s = (m == -INFINITY ? s : s * __expf(m - n)) + (om == -INFINITY ? os : os * __expf(om - n));
        m = n;
    }
    if (lane == 0) {
        const float z = m + logf(s);
        lse[row_of[j]] = z;
        loss[row_of[j]] = z - hit[j];
    }
}

// ---- the gradient of the hidden states: partial products joined in order and put back to their rows ------------------------

template <class T>
__global__ void __launch_bounds__(256) vocab_put_back(const Head *__restrict__ head, const int32_t *__restrict__ pos_of, const float *__restrict__ acc,
                                                      int64_t N, int32_t D, int32_t Dp, int32_t tiles_d, int32_t vocab_blocks, T *__restrict__ out, int64_t os)
{
    const int64_t n = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (n >= N) return;
    const int32_t p = pos_of[n], rows = head->rows, parts = split_of(rows, tiles_d, vocab_blocks);
    const float unscale = head->grad_unscale;
    for (int32_t d = threadIdx.x & 31; d < D; d += 32) {
        float s = 0.0f;
        if (p >= 0) {
            for (int32_t k = 0; k < parts; ++k) s += acc[((int64_t)k * rows + p) * Dp + d];
            s *= unscale;
        }
        out[n * os + d] = from_f<T>(s);
    }
}

// ---- host --------------------------------------------------------------------------------------------------------------------

struct Plan {
    int32_t Dp, tiles_v, tiles_d, piece, pieces;   // piece: columns of the vocabulary that g holds at a time
    bool copy_weight;
    Head *head; int32_t *row_of, *pos_of, *label; float *row_lse, *row_dloss, *hit; float2 *part; char *rows, *weight, *grad; float *acc;
    size_t bytes;
};

inline Plan make_plan(void *base, int64_t N, int64_t V, int64_t D, const void *weight, int64_t ws, bool backward)
{
    Plan p{};
    char *b = (char *)base;
    size_t at = 0;
    auto take = [&](size_t bytes) { char *r = b + at; at += align_up(bytes, 1024); return r; };
    const int64_t Lp = ceil_div(N > 0 ? N : 1, kTileM) * kTileM;
    p.Dp = (int32_t)(ceil_div(D, 64) * 64);
    p.tiles_v = (int32_t)ceil_div(V, kTileN);
    p.tiles_d = (int32_t)ceil_div(D, kTileN);
    p.copy_weight = !rows_on(weight, ws, 2, 16);
    p.head = (Head *)take(sizeof(Head));
    p.row_of = (int32_t *)take(Lp * 4);
    p.pos_of = (int32_t *)take(Lp * 4);
    p.label = (int32_t *)take(Lp * 4);
    p.rows = take((size_t)Lp * p.Dp * 2);
    if (p.copy_weight) p.weight = take((size_t)V * p.Dp * 2);
    if (!backward) {
        p.hit = (float *)take(Lp * 4);
        p.part = (float2 *)take((size_t)Lp * p.tiles_v * 8);
    } else {
        p.row_lse = (float *)take(Lp * 4);
        p.row_dloss = (float *)take(Lp * 4);
        const int64_t most = kPieceBytes / (2 * Lp) / kTileM * kTileM, whole = ceil_div(V, kTileM) * kTileM;
        p.piece = (int32_t)(most < kTileM ? kTileM : most < whole ? most : whole);
        p.pieces = (int32_t)ceil_div(V, p.piece);
        p.grad = take((size_t)Lp * p.piece * 2);
        p.acc = (float *)take((size_t)acc_rows(N, p.tiles_d) * p.Dp * 4);
    }
    p.bytes = at;
    return p;
}

inline int check(const void *hidden, int64_t hs, const void *weight, int64_t ws, int32_t dtype, const int64_t *targets, int64_t N, int64_t V, int64_t D)
{
    if (N < 0 || V <= 0 || D <= 0) return DC_ERR_SHAPE;
    if (N > kMaxDim || V > kMaxDim || D > kMaxDim) return DC_ERR_RANGE;
    if (dtype != DC_BF16 && dtype != DC_F16) return DC_ERR_UNSUPPORTED;
    if (N == 0) return DC_OK;
    if (!hidden || !weight || !targets) return DC_ERR_NULL;
    if (hs < D || ws < D) return DC_ERR_SHAPE;
    if (!on(hidden, 2) || !on(weight, 2) || !on(targets, 8)) return DC_ERR_ALIGN;
    return DC_OK;
}

template <class T>
int gather(const Gather &g, cudaStream_t st)
{
    const unsigned blocks = (unsigned)ceil_div(g.N, kGatherRows);
    if (g.D % 8 == 0 && rows_on(g.hidden, g.hs, 2, 16)) vocab_gather<T, 8><<<blocks, 256, 0, st>>>(g);
    else vocab_gather<T, 1><<<blocks, 256, 0, st>>>(g);
    return launched();
}

template <class T>
int forward(Gather g, const Plan &p, const void *weight, int64_t ws, float *loss, float *lse, cudaStream_t st)
{
    if (int e = gather<T>(g, st)) return e;
    if (p.copy_weight) {
        vocab_copy_weight<T><<<(unsigned)(sm_count() * 8), 256, 0, st>>>((const T *)weight, ws, g.V, g.D, p.Dp, (T *)p.weight);
        weight = p.weight;
        ws = p.Dp;
    }
    if (int e = loss_product<T>(p.head, p.rows, p.Dp, weight, ws, p.label, g.N, g.V, g.D, g.logit_scale, p.part, p.hit, p.tiles_v, st)) return e;
    vocab_join<<<(unsigned)ceil_div(g.N, 8), 256, 0, st>>>(p.head, p.row_of, p.part, p.hit, p.tiles_v, loss, lse);
    return launched();
}

template <class T>
int backward(Gather g, const Plan &p, const void *weight, int64_t ws, void *dh, int64_t dhs, void *dw, int64_t dws, bool dw_f32, bool accumulate, cudaStream_t st)
{
    if (int e = gather<T>(g, st)) return e;
    if (p.copy_weight) {
        vocab_copy_weight<T><<<(unsigned)(sm_count() * 8), 256, 0, st>>>((const T *)weight, ws, g.V, g.D, p.Dp, (T *)p.weight);
        weight = p.weight;
        ws = p.Dp;
    }
    for (int32_t k = 0; k < p.pieces; ++k) {
        const int64_t v0 = (int64_t)k * p.piece, nv = g.V - v0 < p.piece ? g.V - v0 : p.piece;
        const T *w = (const T *)weight + v0 * ws;
        if (int e = grad_product<T>(p.head, p.rows, p.Dp, w, ws, p.label, p.row_lse, p.row_dloss, g.N, v0, nv, g.D, g.logit_scale, p.grad, p.piece, st)) return e;
        char *dwk = dw ? (char *)dw + v0 * dws * (dw_f32 ? 4 : 2) : nullptr;
        if (int e = back_products<T>(p.head, p.grad, p.piece, p.rows, p.Dp, w, ws, g.N, nv, g.D, dwk, dws, dw_f32, accumulate, dh ? p.acc : nullptr,
                                     p.Dp, p.tiles_d, p.piece / kRowBlock, k == 0, st)) return e;
    }
    if (dh) vocab_put_back<T><<<(unsigned)ceil_div(g.N, 8), 256, 0, st>>>(p.head, p.pos_of, p.acc, g.N, g.D, p.Dp, p.tiles_d, p.piece / kRowBlock, (T *)dh, dhs);
    return launched();
}

}  // namespace dct

using namespace dct;

extern "C" size_t dc_vocab_loss_workspace_bytes(int64_t N, int64_t V, int64_t D, const void *weight, int64_t weight_stride, int32_t backward)
{
    if (N < 0 || V <= 0 || D <= 0 || N > kMaxDim || V > kMaxDim || D > kMaxDim) return 0;
    return make_plan(nullptr, N, V, D, weight, weight_stride, backward != 0).bytes;
}

extern "C" int dc_vocab_loss(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride, int32_t dtype, const int64_t *targets,
                             int64_t N, int64_t V, int64_t D, int64_t ignore_index, float logit_scale, float *loss, float *lse, void *workspace,
                             size_t workspace_bytes, void *stream)
{
    if (int e = check(hidden, hidden_stride, weight, weight_stride, dtype, targets, N, V, D)) return e;
    if (N == 0) return DC_OK;
    if (!loss || !lse) return DC_ERR_NULL;
    if (!on(loss, 4) || !on(lse, 4)) return DC_ERR_ALIGN;
    const Plan p = make_plan(workspace, N, V, D, weight, weight_stride, false);
    if (!workspace || !on(workspace, 256) || workspace_bytes < p.bytes) return DC_ERR_WORKSPACE;
    if (sm_count() == 0) return DC_ERR_CUDA;
    Gather g{};
    g.hidden = hidden; g.hs = hidden_stride; g.targets = targets; g.ignore = ignore_index; g.N = N; g.V = V; g.D = (int32_t)D; g.Dp = p.Dp;
    g.logit_scale = logit_scale; g.head = p.head; g.row_of = p.row_of; g.pos_of = p.pos_of; g.label = p.label; g.rows = p.rows;
    g.loss_out = loss; g.lse_out = lse;
    const cudaStream_t st = (cudaStream_t)stream;
    return dtype == DC_BF16 ? forward<__nv_bfloat16>(g, p, weight, weight_stride, loss, lse, st) : forward<__half>(g, p, weight, weight_stride, loss, lse, st);
}

extern "C" int dc_vocab_loss_backward(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride, int32_t dtype,
                                      const int64_t *targets, int64_t N, int64_t V, int64_t D, int64_t ignore_index, float logit_scale, const float *lse,
                                      const float *dloss, void *dhidden, int64_t dhidden_stride, void *dweight, int64_t dweight_stride, int32_t dweight_dtype,
                                      int32_t accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int e = check(hidden, hidden_stride, weight, weight_stride, dtype, targets, N, V, D)) return e;
    if (!dhidden && !dweight) return DC_ERR_NULL;
    if (dweight && dweight_dtype != dtype && dweight_dtype != DC_F32) return DC_ERR_UNSUPPORTED;
    if ((dhidden && N > 0 && dhidden_stride < D) || (dweight && dweight_stride < D)) return DC_ERR_SHAPE;
    const int ob = dweight_dtype == DC_F32 ? 4 : 2;
    if (!on(dhidden, 2) || !on(dweight, ob)) return DC_ERR_ALIGN;
    const cudaStream_t st = (cudaStream_t)stream;
    if (N == 0) {
        if (!dweight || accumulate) return DC_OK;
        return cudaMemset2DAsync(dweight, (size_t)dweight_stride * ob, 0, (size_t)D * ob, (size_t)V, st) == cudaSuccess ? DC_OK : DC_ERR_CUDA;
    }
    if (!lse || !dloss) return DC_ERR_NULL;
    if (!on(lse, 4) || !on(dloss, 4)) return DC_ERR_ALIGN;
    const Plan p = make_plan(workspace, N, V, D, weight, weight_stride, true);
    if (!workspace || !on(workspace, 256) || workspace_bytes < p.bytes) return DC_ERR_WORKSPACE;
    if (sm_count() == 0) return DC_ERR_CUDA;
    Gather g{};
    g.hidden = hidden; g.hs = hidden_stride; g.targets = targets; g.ignore = ignore_index; g.lse = lse; g.dloss = dloss; g.N = N; g.V = V;
    g.D = (int32_t)D; g.Dp = p.Dp; g.logit_scale = logit_scale; g.head = p.head; g.row_of = p.row_of; g.pos_of = p.pos_of; g.label = p.label;
    g.row_lse = p.row_lse; g.row_dloss = p.row_dloss; g.rows = p.rows; g.scale_grad = dtype == DC_F16;
    return dtype == DC_BF16
               ? backward<__nv_bfloat16>(g, p, weight, weight_stride, dhidden, dhidden_stride, dweight, dweight_stride, dweight_dtype == DC_F32, accumulate != 0, st)
               : backward<__half>(g, p, weight, weight_stride, dhidden, dhidden_stride, dweight, dweight_stride, dweight_dtype == DC_F32, accumulate != 0, st);
}

extern "C" int dc_train_status(uint32_t *flags)
{
    unsigned int f = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&f, g_train_wait_expired, sizeof(f)) != cudaSuccess) return DC_ERR_CUDA;
    if (f != 0 && cudaMemcpyToSymbol(g_train_wait_expired, &zero, sizeof(zero)) != cudaSuccess) return DC_ERR_CUDA;
    if (flags) *flags = f;
    return f == 0 ? DC_OK : DC_ERR_DEVICE;
}
