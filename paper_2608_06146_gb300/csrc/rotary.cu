// rotary.cu -- what stands between a model's projections and the attention kernels: the RMS norm of every
// query and key head (or none) and rotary positions with up to four axes (time, height, width of images
// and video), for packed rows (the training forward) with their gradients, and for a step's or a
// prefix's rows on their way into the paged pool (C5, Algorithm 1's append).
#include <cfloat>
#include <cmath>

#include "common.cuh"
#include "rotary.cuh"

namespace padoc_rotary_dev {

namespace {

constexpr int kWarps = 8;   // warps per CTA

struct Args {
    Spec sp;
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;   // elements
    const int32_t *pos;
    int64_t rows;                           // source rows
    int32_t hq, hkv;
    void *q_out, *k_out;
    int64_t q_out_stride, k_out_stride;
    int32_t group, splits;                  // lanes per head; warps per row
    // append
    void *v_out;                            // with k_out: the pool's arrays
    const int32_t *src_rows, *slots;
    int64_t count, pool_slots;
    int32_t block_size;
    int *err;
};

// A warp per row (or `splits` warps), 32 / group heads at a time. Bound by HBM in large calls: every
// element is read once and written once. kAppend: row i of the call is source row src_rows[i]; its K and V
// heads go to pool slot slots[i], its query heads to row i of q_out.
template <typename T, int V, bool kAdjacent, bool kNorm, bool kAppend>
__global__ void __launch_bounds__(32 * kWarps) rotary_kernel(const Args p)
{
    pdl_wait_prerequisite();
    pdl_launch_dependents();
    const int64_t wid = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int64_t i = wid / p.splits;
    const int split = (int)(wid - i * p.splits);
    if (i >= p.count) return;
    const int lane = threadIdx.x & 31;
    int64_t row = i, slot = 0;
    if constexpr (kAppend) {
        if (p.src_rows) row = p.src_rows[i];
        slot = p.slots[i];
        if (slot < 0 || slot >= p.pool_slots || row < 0 || row >= p.rows) {
            if (lane == 0 && split == 0)
                padoc_record_error(p.err, PADOC_DEVERR_BLOCK_ID,
                                   (slot < 0 || slot >= p.pool_slots) ? (int)slot : (int)row);
            return;
        }
    }
    const int group = p.group, heads = 32 / group;
    const int sub = lane / group, chunk = lane & (group - 1);
    const Place pl = lane_place<V, kAdjacent>(chunk, p.sp.d, p.sp.rot);
    float c[V], s[V];
    if (pl.turned) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            cos_sin(p.sp.freq[chunk * V + j], p.pos + row * p.sp.axes, p.sp.amplitude, c[j], s[j]);
    }
    const T *q = static_cast<const T *>(p.q) + row * p.q_stride, *k = static_cast<const T *>(p.k) + row * p.k_stride;
    const int nq = p.q ? p.hq : 0, turned = nq + p.hkv, total = kAppend ? turned + p.hkv : turned;
    for (int h0 = split * heads; h0 < total; h0 += p.splits * heads) {
        const int h = h0 + sub;
        const bool here = h < total && pl.active;
        const bool is_q = h < nq, is_v = kAppend && h >= turned;
        const int hk = is_v ? h - turned : h - nq;
        const T *src;
        T *dst;
        if (is_q) {
            src = q + (int64_t)h * p.sp.d;
            dst = static_cast<T *>(p.q_out) + i * p.q_out_stride + (int64_t)h * p.sp.d;
        } else if constexpr (kAppend) {
            src = is_v ? static_cast<const T *>(p.v) + row * p.v_stride + (int64_t)hk * p.sp.d : k + (int64_t)hk * p.sp.d;
            dst = static_cast<T *>(is_v ? p.v_out : p.k_out) +
                  ((slot / p.block_size * p.hkv + hk) * p.block_size + slot % p.block_size) * p.sp.d;
        } else {
            src = k + (int64_t)hk * p.sp.d;
            dst = static_cast<T *>(p.k_out) + i * p.k_out_stride + (int64_t)hk * p.sp.d;
        }
        float a[V], b[V];
        if (here) {
            load_vec<V>(src + pl.a, a);
            load_vec<V>(src + pl.b, b);
        }
        if constexpr (kNorm) {
            float na[V], nb[V];
#pragma unroll
            for (int j = 0; j < V; ++j) na[j] = a[j], nb[j] = b[j];
            Place pn = pl;
            pn.active = here;
            norm_head<T, V>(na, nb, static_cast<const T *>(is_q ? p.sp.q_weight : p.sp.k_weight), pn, p.sp, group);
            if (!is_v) {
#pragma unroll
                for (int j = 0; j < V; ++j) a[j] = na[j], b[j] = nb[j];
            }
        }
        if (here) {
            if (pl.turned && !is_v) turn_pairs<V, kAdjacent, false>(a, b, c, s);
            store_vec<V>(dst + pl.a, a);
            store_vec<V>(dst + pl.b, b);
        }
    }
}

struct BwdArgs {
    Spec sp;
    const void *q, *k;                      // the forward's inputs (with the norm)
    int64_t q_stride, k_stride;
    const int32_t *pos;
    int64_t rows;
    int32_t hq, hkv, group;
    const void *dq_out, *dk_out;
    int64_t dq_out_stride, dk_out_stride;
    void *dq, *dk;
    int64_t dq_stride, dk_stride;
    float *part;                            // [CTAs][2][d]
};

// The gradient of one kind's heads (the queries or the keys) of a row; acc: the lane's sums of g x r.
template <typename T, int V, bool kAdjacent, bool kNorm>
__device__ __forceinline__ void bwd_heads(const BwdArgs &p, const T *x, const T *dy, T *dx, int n, const T *w, const Place &pl,
                                          int sub, const float (&c)[V], const float (&s)[V], float (&acc)[2 * V])
{
    const int group = p.group, heads = 32 / group;
    for (int h0 = 0; h0 < n; h0 += heads) {
        const int h = h0 + sub;
        const bool here = h < n && pl.active;
        const int64_t at = (int64_t)h * p.sp.d;
        float a[V], b[V];
        if (here) {
            load_vec<V>(dy + at + pl.a, a);
            load_vec<V>(dy + at + pl.b, b);
            if (pl.turned) turn_pairs<V, kAdjacent, true>(a, b, c, s);
        }
        if constexpr (kNorm) {
            float xa[V], xb[V], wa[V], wb[V];
            float ss = 0.f, dot = 0.f;
            if (here) {
                load_vec<V>(x + at + pl.a, xa);
                load_vec<V>(x + at + pl.b, xb);
                load_vec<V>(w + pl.a, wa);
                load_vec<V>(w + pl.b, wb);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    ss = fmaf(xa[j], xa[j], fmaf(xb[j], xb[j], ss));
                    dot = fmaf(a[j] * wa[j], xa[j], fmaf(b[j] * wb[j], xb[j], dot));
                }
            }
            const float r = rsqrtf(group_sum(ss, group) / (float)p.sp.d + p.sp.eps);
            const float m = group_sum(dot, group) * r / (float)p.sp.d;   // mean of w g x r
            if (here) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float ha = xa[j] * r, hb = xb[j] * r;
                    acc[j] = fmaf(a[j], ha, acc[j]);
                    acc[V + j] = fmaf(b[j], hb, acc[V + j]);
                    a[j] = r * fmaf(-ha, m, wa[j] * a[j]);
                    b[j] = r * fmaf(-hb, m, wb[j] * b[j]);
                }
            }
        }
        if (here) {
            store_vec<V>(dx + at + pl.a, a);
            store_vec<V>(dx + at + pl.b, b);
        }
    }
}

// A warp per row, rows in a grid-wide stride. With the norm every lane keeps fp32 sums of the weights'
// gradient for its dims; a CTA joins them in a fixed order and writes one partial row, which
// rotary_weight_grad_kernel adds up (no atomics: the same call gives the same bits).
template <typename T, int V, bool kAdjacent, bool kNorm>
__global__ void __launch_bounds__(32 * kWarps) rotary_bwd_kernel(const BwdArgs p)
{
    extern __shared__ float sums[];   // [kWarps][2][d]
    pdl_wait_prerequisite();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane / p.group, chunk = lane & (p.group - 1);
    const Place pl = lane_place<V, kAdjacent>(chunk, p.sp.d, p.sp.rot);
    float acc_q[2 * V], acc_k[2 * V];
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) acc_q[j] = acc_k[j] = 0.f;
    for (int64_t row = (int64_t)blockIdx.x * kWarps + warp; row < p.rows; row += (int64_t)gridDim.x * kWarps) {
        float c[V], s[V];
        if (pl.turned) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                cos_sin(p.sp.freq[chunk * V + j], p.pos + row * p.sp.axes, p.sp.amplitude, c[j], s[j]);
        }
        const T *xq = nullptr, *xk = nullptr;
        if constexpr (kNorm) {
            xq = static_cast<const T *>(p.q) + row * p.q_stride;
            xk = static_cast<const T *>(p.k) + row * p.k_stride;
        }
        bwd_heads<T, V, kAdjacent, kNorm>(p, xq, static_cast<const T *>(p.dq_out) + row * p.dq_out_stride,
                                          static_cast<T *>(p.dq) + row * p.dq_stride, p.hq,
                                          static_cast<const T *>(p.sp.q_weight), pl, sub, c, s, acc_q);
        bwd_heads<T, V, kAdjacent, kNorm>(p, xk, static_cast<const T *>(p.dk_out) + row * p.dk_out_stride,
                                          static_cast<T *>(p.dk) + row * p.dk_stride, p.hkv,
                                          static_cast<const T *>(p.sp.k_weight), pl, sub, c, s, acc_k);
    }
    if constexpr (kNorm) {
        const int d = p.sp.d;
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            float(&acc)[2 * V] = kind ? acc_k : acc_q;
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) {
                float v = acc[j];
                for (int m = p.group; m < 32; m <<= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
                if (sub == 0 && pl.active) sums[(warp * 2 + kind) * d + (j < V ? pl.a + j : pl.b + j - V)] = v;
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 2 * d; e += 32 * kWarps) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) v += sums[w * 2 * d + e];
            p.part[(int64_t)blockIdx.x * 2 * d + e] = v;
        }
    }
}

// Column sums of the CTAs' partial rows: 32 columns a CTA, eight warps that take the rows in turn.
__global__ void __launch_bounds__(256) rotary_weight_grad_kernel(const float *__restrict__ part, int n, int d, float *dqw, float *dkw)
{
    __shared__ float sums[8][32];
    pdl_wait_prerequisite();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (col < 2 * d)
        for (int r = warp; r < n; r += 8) v += part[(int64_t)r * 2 * d + col];
    sums[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && col < 2 * d) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += sums[w][lane];
        (col < d ? dqw[col] : dkw[col - d]) = t;
    }
}

size_t elt_size(padoc_dtype t) { return t == PADOC_DTYPE_BF16 ? 2 : 4; }

// Elements of a lane's vectors: 16 bytes where the rotated and the other dims come in whole chunks of
// them, else 8 bytes (bf16 heads whose dims are an odd multiple of 8).
int vec_of(const padoc_rotary *r, padoc_dtype t)
{
    return t == PADOC_DTYPE_BF16 && r->head_dim % 16 == 0 && r->rotary_dim % 16 == 0 ? 8 : 4;
}
int group_of(const padoc_rotary *r, int vec)
{
    int g = 1;
    while (g * 2 * vec < r->head_dim) g *= 2;
    return g;
}

padoc_status check_ptr(const void *p, int64_t stride, int64_t rows, int64_t least, size_t esz)
{
    if (!p) return PADOC_ERR_INVALID_ARGUMENT;
    if (((uintptr_t)p) & 15) return PADOC_ERR_INVALID_ARGUMENT;
    if (stride < least || (stride * (int64_t)esz) % 16 != 0) return PADOC_ERR_INVALID_ARGUMENT;
    if (rows > 0 && stride > INT64_MAX / 8 / rows) return PADOC_ERR_INVALID_ARGUMENT;
    return PADOC_OK;
}

template <typename K>
padoc_status launch(K kernel, unsigned grid, int block, size_t smem, padoc_stream_t stream, const void *args)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(grid);
    lc.blockDim = dim3(block);
    lc.dynamicSmemBytes = smem;
    lc.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // every kernel here waits for its predecessor
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    void *argv[1] = {const_cast<void *>(args)};
    PADOC_CUDA_TRY(cudaLaunchKernelExC(&lc, (const void *)kernel, argv));
    return padoc_launch_status();
}

template <typename T, int V, bool kAppend>
padoc_status launch_rows(const Args &p, bool adjacent, bool norm, unsigned grid, padoc_stream_t stream)
{
    auto *k = adjacent ? (norm ? rotary_kernel<T, V, true, true, kAppend> : rotary_kernel<T, V, true, false, kAppend>)
                       : (norm ? rotary_kernel<T, V, false, true, kAppend> : rotary_kernel<T, V, false, false, kAppend>);
    return launch(k, grid, 32 * kWarps, 0, stream, &p);
}

// Warps per row: one when the rows fill the GPU by themselves, else as many as the heads can use.
int splits_of(int64_t rows, int heads_total, int group)
{
    const int steps = (heads_total + 32 / group - 1) / (32 / group);
    const int64_t want = (int64_t)padoc_num_sms() * 32 / (rows > 0 ? rows : 1);
    return (int)(want < 1 ? 1 : want > steps ? steps : want);
}

template <bool kAppend>
padoc_status launch_any(Args &p, const padoc_rotary *rot, padoc_dtype dtype, padoc_stream_t stream)
{
    const int vec = vec_of(rot, dtype);
    p.group = group_of(rot, vec);
    p.splits = splits_of(p.count, (p.q ? p.hq : 0) + (kAppend ? 2 : 1) * p.hkv, p.group);
    const int64_t ctas = (p.count * p.splits + kWarps - 1) / kWarps;
    if (ctas > INT32_MAX) return PADOC_ERR_UNSUPPORTED;
    const bool adj = rot->adjacent != 0, norm = rot->q_weight != nullptr;
    if (dtype == PADOC_DTYPE_F32) return launch_rows<float, 4, kAppend>(p, adj, norm, (unsigned)ctas, stream);
    return vec == 8 ? launch_rows<__nv_bfloat16, 8, kAppend>(p, adj, norm, (unsigned)ctas, stream)
                    : launch_rows<__nv_bfloat16, 4, kAppend>(p, adj, norm, (unsigned)ctas, stream);
}

// CTAs of the backward: with the norm each leaves a partial row of weight gradients.
int bwd_ctas(int64_t rows)
{
    const int64_t need = (rows + kWarps - 1) / kWarps, most = 4 * (int64_t)padoc_default_ctas();
    return (int)(need < most ? need : most);
}

template <typename T, int V>
padoc_status launch_bwd(const BwdArgs &p, bool adjacent, bool norm, int ctas, padoc_stream_t stream)
{
    auto *k = adjacent ? (norm ? rotary_bwd_kernel<T, V, true, true> : rotary_bwd_kernel<T, V, true, false>)
                       : (norm ? rotary_bwd_kernel<T, V, false, true> : rotary_bwd_kernel<T, V, false, false>);
    return launch(k, (unsigned)ctas, 32 * kWarps, norm ? (size_t)kWarps * 2 * p.sp.d * sizeof(float) : 0, stream, &p);
}

}  // namespace

padoc_status check_spec(const padoc_rotary *r)
{
    if (!r || !r->freq || (((uintptr_t)r->freq) & 7)) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->head_dim < 1 || r->rotary_dim < 1 || r->rotary_dim > r->head_dim) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->num_axes < 1 || r->num_axes > 4 || (r->adjacent != 0 && r->adjacent != 1)) return PADOC_ERR_INVALID_ARGUMENT;
    if (!std::isfinite(r->amplitude)) return PADOC_ERR_INVALID_ARGUMENT;
    if ((r->q_weight == nullptr) != (r->k_weight == nullptr)) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->q_weight && (!(r->eps >= 0.f) || !std::isfinite(r->eps))) return PADOC_ERR_INVALID_ARGUMENT;
    if ((((uintptr_t)r->q_weight) | ((uintptr_t)r->k_weight)) & 15) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->head_dim > 256 || r->head_dim % 8 != 0 || r->rotary_dim % 8 != 0) return PADOC_ERR_UNSUPPORTED;
    return PADOC_OK;
}

padoc_status check_rows(const padoc_qkv_rows *in, const padoc_rotary *rot, bool with_v)
{
    if (!in || in->rows < 0 || in->num_kv_heads < 1 || in->num_q_heads < 0 || (in->q && in->num_q_heads < 1))
        return PADOC_ERR_INVALID_ARGUMENT;
    if (in->dtype != PADOC_DTYPE_BF16 && in->dtype != PADOC_DTYPE_F32) return PADOC_ERR_INVALID_ARGUMENT;
    if (in->rows > INT32_MAX || in->num_q_heads > 4096 || in->num_kv_heads > 4096) return PADOC_ERR_UNSUPPORTED;
    if (in->rows == 0) return PADOC_OK;
    const size_t e = elt_size(in->dtype);
    if (!in->pos || (((uintptr_t)in->pos) & 3)) return PADOC_ERR_INVALID_ARGUMENT;
    padoc_status st = check_ptr(in->k, in->k_stride, in->rows, (int64_t)in->num_kv_heads * rot->head_dim, e);
    if (st == PADOC_OK && in->q) st = check_ptr(in->q, in->q_stride, in->rows, (int64_t)in->num_q_heads * rot->head_dim, e);
    if (st == PADOC_OK && with_v) st = check_ptr(in->v, in->v_stride, in->rows, (int64_t)in->num_kv_heads * rot->head_dim, e);
    return st;
}

}  // namespace padoc_rotary_dev

using namespace padoc_rotary_dev;

extern "C" padoc_status padoc_build_rotary_table(const double *inv_freq, const int32_t *axis_of, int32_t num_freqs,
                                                 int32_t num_axes, uint64_t *table)
{
    if (!inv_freq || !table || num_freqs < 1 || num_axes < 1 || num_axes > 4 || (num_axes > 1 && !axis_of))
        return PADOC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < num_freqs; ++i) {
        if (!std::isfinite(inv_freq[i])) return PADOC_ERR_INVALID_ARGUMENT;
        if (axis_of && (axis_of[i] < 0 || axis_of[i] >= num_axes)) return PADOC_ERR_INVALID_ARGUMENT;
    }
    for (int32_t i = 0; i < num_freqs; ++i) {
        const double turns = inv_freq[i] / 6.283185307179586476925;
        const double frac = turns - std::floor(turns);                     // [0, 1]
        const double units = std::nearbyint(std::ldexp(frac, 62));         // the axis takes the two lowest bits
        const uint64_t u = units >= 0x1p62 ? 0 : (uint64_t)units;          // (a whole turn is none)
        table[i] = u << 2 | (uint64_t)(axis_of ? axis_of[i] : 0);
    }
    return PADOC_OK;
}

extern "C" padoc_status padoc_qk_rotary(const padoc_rotary *rot, const padoc_qkv_rows *in, void *q_out, int64_t q_out_stride,
                                        void *k_out, int64_t k_out_stride, padoc_stream_t stream)
{
    padoc_status st = check_spec(rot);
    if (st != PADOC_OK) return st;
    st = check_rows(in, rot, false);
    if (st != PADOC_OK) return st;
    if (in->num_q_heads < 1) return PADOC_ERR_INVALID_ARGUMENT;
    if (in->rows == 0) return PADOC_OK;
    if (!in->q) return PADOC_ERR_INVALID_ARGUMENT;
    const size_t e = elt_size(in->dtype);
    st = check_ptr(q_out, q_out_stride, in->rows, (int64_t)in->num_q_heads * rot->head_dim, e);
    if (st == PADOC_OK) st = check_ptr(k_out, k_out_stride, in->rows, (int64_t)in->num_kv_heads * rot->head_dim, e);
    if (st != PADOC_OK) return st;
    Args p = {};
    p.sp = make_spec(rot);
    p.q = in->q, p.k = in->k;
    p.q_stride = in->q_stride, p.k_stride = in->k_stride;
    p.pos = in->pos;
    p.rows = p.count = in->rows;
    p.hq = in->num_q_heads, p.hkv = in->num_kv_heads;
    p.q_out = q_out, p.k_out = k_out;
    p.q_out_stride = q_out_stride, p.k_out_stride = k_out_stride;
    return launch_any<false>(p, rot, in->dtype, stream);
}

extern "C" padoc_status padoc_append_rotary_inputs(const padoc_kv_pool *pool, const padoc_rotary *rot, const padoc_qkv_rows *in,
                                                   void *q_dst, const int32_t *src_rows, const int32_t *slots, int32_t count,
                                                   padoc_stream_t stream)
{
    if (!pool || count < 0) return PADOC_ERR_INVALID_ARGUMENT;
    padoc_status st = check_spec(rot);
    if (st != PADOC_OK) return st;
    st = check_rows(in, rot, true);
    if (st != PADOC_OK) return st;
    if (pool->dtype != in->dtype || pool->head_dim != rot->head_dim || pool->num_kv_heads != in->num_kv_heads ||
        pool->num_blocks < 1 || pool->block_size < 1)
        return PADOC_ERR_INVALID_ARGUMENT;
    if (count == 0) return PADOC_OK;
    if (in->rows == 0 || !slots || !pool->k_pool || !pool->v_pool || (in->q && !q_dst)) return PADOC_ERR_INVALID_ARGUMENT;
    if ((((uintptr_t)pool->k_pool) | ((uintptr_t)pool->v_pool) | ((uintptr_t)q_dst)) & 15) return PADOC_ERR_INVALID_ARGUMENT;
    int *err = padoc_device_error_word();
    if (!err) return PADOC_ERR_CUDA;
    Args p = {};
    p.sp = make_spec(rot);
    p.q = in->q, p.k = in->k, p.v = in->v;
    p.q_stride = in->q_stride, p.k_stride = in->k_stride, p.v_stride = in->v_stride;
    p.pos = in->pos;
    p.rows = in->rows;
    p.hq = in->num_q_heads, p.hkv = in->num_kv_heads;
    p.q_out = q_dst, p.q_out_stride = (int64_t)in->num_q_heads * rot->head_dim;
    p.k_out = const_cast<void *>(pool->k_pool), p.v_out = const_cast<void *>(pool->v_pool);
    p.src_rows = src_rows, p.slots = slots;
    p.count = count;
    p.pool_slots = (int64_t)pool->num_blocks * pool->block_size;
    p.block_size = pool->block_size;
    p.err = err;
    return launch_any<true>(p, rot, in->dtype, stream);
}

extern "C" padoc_status padoc_qk_rotary_bwd_workspace_size(const padoc_rotary *rot, int64_t rows, size_t *bytes)
{
    const padoc_status st = check_spec(rot);
    if (st != PADOC_OK) return st;
    if (rows < 0 || !bytes) return PADOC_ERR_INVALID_ARGUMENT;
    if (rows > INT32_MAX) return PADOC_ERR_UNSUPPORTED;
    *bytes = rot->q_weight ? (size_t)bwd_ctas(rows) * 2 * rot->head_dim * sizeof(float) : 0;
    return PADOC_OK;
}

extern "C" padoc_status padoc_qk_rotary_bwd(const padoc_rotary *rot, const padoc_qkv_rows *in, const void *dq_out,
                                            int64_t dq_out_stride, const void *dk_out, int64_t dk_out_stride, void *dq,
                                            int64_t dq_stride, void *dk, int64_t dk_stride, float *dq_weight, float *dk_weight,
                                            void *workspace, size_t workspace_bytes, padoc_stream_t stream)
{
    padoc_status st = check_spec(rot);
    if (st != PADOC_OK) return st;
    if (!in || in->num_q_heads < 1) return PADOC_ERR_INVALID_ARGUMENT;
    const bool norm = rot->q_weight != nullptr;
    padoc_qkv_rows rows = *in;
    if (!norm) {   // the rotation's gradient does not depend on the rows: dk_out stands in for their checks
        rows.q = nullptr;
        rows.k = dk_out;
        rows.k_stride = dk_out_stride;
    }
    st = check_rows(&rows, rot, false);
    if (st != PADOC_OK) return st;
    if (norm) {
        if (!dq_weight || !dk_weight || ((((uintptr_t)dq_weight) | ((uintptr_t)dk_weight)) & 3)) return PADOC_ERR_INVALID_ARGUMENT;
        if (in->rows > 0 && !in->q) return PADOC_ERR_INVALID_ARGUMENT;
    }
    if (in->rows > 0) {
        const size_t e = elt_size(in->dtype);
        const int64_t nq = (int64_t)in->num_q_heads * rot->head_dim, nk = (int64_t)in->num_kv_heads * rot->head_dim;
        st = check_ptr(dq_out, dq_out_stride, in->rows, nq, e);
        if (st == PADOC_OK) st = check_ptr(dk_out, dk_out_stride, in->rows, nk, e);
        if (st == PADOC_OK) st = check_ptr(dq, dq_stride, in->rows, nq, e);
        if (st == PADOC_OK) st = check_ptr(dk, dk_stride, in->rows, nk, e);
        if (st != PADOC_OK) return st;
    }
    const int ctas = bwd_ctas(in->rows);
    if (norm && ctas > 0) {
        if (!workspace || (((uintptr_t)workspace) & 255)) return PADOC_ERR_INVALID_ARGUMENT;
        if (workspace_bytes < (size_t)ctas * 2 * rot->head_dim * sizeof(float)) return PADOC_ERR_WORKSPACE_TOO_SMALL;
    }
    if (ctas > 0) {
        BwdArgs p = {};
        p.sp = make_spec(rot);
        p.q = in->q, p.k = in->k;
        p.q_stride = in->q_stride, p.k_stride = in->k_stride;
        p.pos = in->pos;
        p.rows = in->rows;
        p.hq = in->num_q_heads, p.hkv = in->num_kv_heads;
        p.dq_out = dq_out, p.dk_out = dk_out;
        p.dq_out_stride = dq_out_stride, p.dk_out_stride = dk_out_stride;
        p.dq = dq, p.dk = dk;
        p.dq_stride = dq_stride, p.dk_stride = dk_stride;
        p.part = (float *)workspace;
        const int vec = vec_of(rot, in->dtype);
        p.group = group_of(rot, vec);
        const bool adj = rot->adjacent != 0;
        st = in->dtype == PADOC_DTYPE_F32 ? launch_bwd<float, 4>(p, adj, norm, ctas, stream)
             : vec == 8                   ? launch_bwd<__nv_bfloat16, 8>(p, adj, norm, ctas, stream)
                                          : launch_bwd<__nv_bfloat16, 4>(p, adj, norm, ctas, stream);
        if (st != PADOC_OK) return st;
    }
    if (!norm) return PADOC_OK;
    // no rows: the weights' gradients are zero
    const int d = rot->head_dim;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)((2 * d + 31) / 32));
    lc.blockDim = dim3(256);
    lc.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    PADOC_CUDA_TRY(cudaLaunchKernelEx(&lc, rotary_weight_grad_kernel, (const float *)workspace, ctas, d, dq_weight, dk_weight));
    return padoc_launch_status();
}
