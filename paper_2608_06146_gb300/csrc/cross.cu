// cross.cu -- cross attention (query rows over an encoder's states of another length): the host entry points, their
// validation, the kernels that join split rows, and the fp32 kernels. The bf16 kernels run on the tensor cores
// (cross_tc.cu, cross_bwd_tc.cu).
//
// Per segment, query head h of KV head g:  S = scale Q K^T,  lse = ln sum_j exp S_j,  O = sum_j exp(S_j - lse) V_j;
//   P = exp(S - lse),  D = rowsum(dO * O),  dS = P (dO V^T - D),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
#include <math.h>

#include <algorithm>

#include "cross.cuh"

namespace {

// ------------------------------------------------------------------------------------------------
// Joining split rows
// ------------------------------------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ void store4(T *p, float4 x)
{
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p) = x;
    } else {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w));
    }
}

// A packed row by one warp, or by the eight of a CTA (W 8: a warp each eighth part) where there are many parts. Parts
// hold O / l and lse * log2(e), so O = sum_i w_i O_i with w_i = 2^(lse2_i - lse2); dq's are plain sums. The order is
// fixed. Rows without parts (segments without keys) get O = 0, lse = -inf.
template <typename T, int D, bool kDq, int W>
__global__ void __launch_bounds__(256) cross_merge_kernel(const padoc_cross_args a)
{
    constexpr int E = D / 32;
    const int unit_rows = a.unit_rows, per = unit_rows * W / 8;   // (multiples of 8)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w0 = W == 8 ? warp : 0;
    const int row = W == 8 ? (int)blockIdx.x % per : (int)blockIdx.x % per * 8 + warp;
    pdl_launch_dependents();
    // The plan too is read behind the wait: the forward lets this kernel start before it has itself waited for the one
    // before it, which may have written the plan.
    pdl_wait_prerequisite();
    const padoc_cross_merge m = a.merges[(int)blockIdx.x / per];
    int token, head;
    if (!cross_row(a, m.tok, m.ntok, row, token, head)) return;
    const int n = (m.parts - w0 + W - 1) / W;   // this warp's parts: w0, w0 + W, ..
    auto at = [&](int i) { return (size_t)(m.slot + w0 + i * W) * unit_rows + row; };
    float acc[E], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    if (!kDq) {
        for (int i = lane; i < n; i += 32) top = fmaxf(top, a.part_lse[at(i)]);
#pragma unroll
        for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    }
    for (int i0 = 0; i0 < n; i0 += 32) {
        float w = 1.f;
        if (!kDq) {
            const float l = i0 + lane < n ? a.part_lse[at(i0 + lane)] : -INFINITY;
            w = l == -INFINITY ? 0.f : exp2f(l - top);
        }
        const int k = min(32, n - i0);
#pragma unroll 4
        for (int j = 0; j < k; ++j) {
            const float *p = a.part + at(i0 + j) * D + lane * E;
            const float wj = kDq ? 1.f : __shfl_sync(0xffffffffu, w, j);
            float x[E];
            if constexpr (E == 4) *reinterpret_cast<float4 *>(x) = *reinterpret_cast<const float4 *>(p);
            else *reinterpret_cast<float2 *>(x) = *reinterpret_cast<const float2 *>(p);
            sum += wj;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(wj, x[e], acc[e]);
        }
    }
    if constexpr (W == 8) {
        __shared__ float parts[8][D + 2];
#pragma unroll
        for (int e = 0; e < E; ++e) parts[warp][lane * E + e] = acc[e];
        if (lane == 0) {
            parts[warp][D] = top;
            parts[warp][D + 1] = sum;
        }
        __syncthreads();
        if (warp) return;
        float most = -INFINITY;
        if (!kDq)
            for (int i = 0; i < 8; ++i) most = fmaxf(most, parts[i][D]);
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = parts[i][D], w = kDq ? 1.f : t == -INFINITY ? 0.f : exp2f(t - most);
            sum = fmaf(w, parts[i][D + 1], sum);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(w, parts[i][lane * E + e], acc[e]);
        }
        top = most;
    }
    const float mul = kDq ? a.scale : sum == 0.f ? 0.f : 1.f / sum;
    const size_t h = (size_t)token * a.hq + m.g * a.group + head;
    T *dst = kDq ? (T *)a.dq + (size_t)token * a.dq_stride + (size_t)(m.g * a.group + head) * D + lane * E
                 : (T *)a.o + h * D + lane * E;
    if constexpr (E == 4) {
        store4(dst, make_float4(acc[0] * mul, acc[1] * mul, acc[2] * mul, acc[3] * mul));
    } else {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float2 *>(dst) = make_float2(acc[0] * mul, acc[1] * mul);
        else *reinterpret_cast<uint32_t *>(dst) = pack_bf16x2(acc[0] * mul, acc[1] * mul);
    }
    if (!kDq && lane == 0) a.lse[h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * PADOC_LN2;
}

template <typename T, int D, bool kDq, int W>
padoc_status launch_merge(const padoc_cross_args &a, bool pdl, cudaStream_t stream)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(a.num_merges * (a.unit_rows * W / 8)));
    lc.blockDim = dim3(256);
    lc.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = pdl ? 1 : 0;
    PADOC_CUDA_TRY(cudaLaunchKernelEx(&lc, cross_merge_kernel<T, D, kDq, W>, a));
    return padoc_launch_status();
}

template <typename T, bool kDq>
padoc_status merge_rows(const padoc_cross_args &a, int head_dim, bool pdl, cudaStream_t stream)
{
    if (head_dim == 64) return a.max_parts > 16 ? launch_merge<T, 64, kDq, 8>(a, pdl, stream) : launch_merge<T, 64, kDq, 1>(a, pdl, stream);
    return a.max_parts > 16 ? launch_merge<T, 128, kDq, 8>(a, pdl, stream) : launch_merge<T, 128, kDq, 1>(a, pdl, stream);
}

// ------------------------------------------------------------------------------------------------
// fp32: 64 packed rows a CTA of 256 threads, in steps of 64 keys. Tiles lie in shared memory, rows four
// floats further apart than their length (a quarter warp's 16-byte reads of eight rows then meet no bank twice); a
// thread keeps four rows by four columns of a 64 x 64 product, or four rows by D / 16 columns of a 64 x D one.
// Meant for small pages: bound by the chain of a step (5 us with 64 dims: two products, three barriers), so keys are cut
// until every four SMs have an item of four such CTAs, in the dQ pass every two one of two (368 rows of 4 heads over 260
// states 33 -> 14 us, parts joined by a second kernel). Where a segment has few rows, an item's other CTAs end at once and
// their SMs stay idle: a token over 150001 states is 38 items with one CTA at work each.
// ------------------------------------------------------------------------------------------------

constexpr int kB = PADOC_CROSS_BLOCK;

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }

template <int D>
struct Simt {
    static constexpr int P = D + 4;          // pitch of a tile's rows
    static constexpr int PS = kB + 4;        // ... of a 64 x 64 product's
    static constexpr int kTile = kB * P;

    // 64 rows of D values; row r at base(r), or zeros where that is null
    template <typename F>
    static __device__ __forceinline__ void load(float *dst, F base)
    {
        for (int i = threadIdx.x; i < kB * (D / 4); i += 256) {
            const int r = i / (D / 4), c = i % (D / 4) * 4;
            const float *p = base(r);
            *reinterpret_cast<float4 *>(dst + r * P + c) = p ? load4(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    // acc[i][j] = x[4 ty + i] . y[tx + 16 j]
    static __device__ __forceinline__ void dots(const float *x, const float *y, float (&acc)[4][4])
    {
        const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
            float4 a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = *reinterpret_cast<const float4 *>(x + (4 * ty + i) * P + d);
                b[i] = *reinterpret_cast<const float4 *>(y + (tx + 16 * i) * P + d);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    acc[i][j] = fmaf(a[i].x, b[j].x, acc[i][j]);
                    acc[i][j] = fmaf(a[i].y, b[j].y, acc[i][j]);
                    acc[i][j] = fmaf(a[i].z, b[j].z, acc[i][j]);
                    acc[i][j] = fmaf(a[i].w, b[j].w, acc[i][j]);
                }
        }
    }
    // acc[i][4 j + e] += sum_k s[4 ty + i][k] y[k][64 j + 4 tx + e]
    static __device__ __forceinline__ void add_product(const float *s, const float *y, float (&acc)[4][D / 16])
    {
        const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 2
        for (int k = 0; k < kB; k += 4) {
            float w[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(w[i]) = *reinterpret_cast<const float4 *>(s + (4 * ty + i) * PS + k);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const float4 b = *reinterpret_cast<const float4 *>(y + (k + e) * P + 64 * j + 4 * tx);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        acc[i][4 * j] = fmaf(w[i][e], b.x, acc[i][4 * j]);
                        acc[i][4 * j + 1] = fmaf(w[i][e], b.y, acc[i][4 * j + 1]);
                        acc[i][4 * j + 2] = fmaf(w[i][e], b.z, acc[i][4 * j + 2]);
                        acc[i][4 * j + 3] = fmaf(w[i][e], b.w, acc[i][4 * j + 3]);
                    }
                }
        }
    }
    static __device__ __forceinline__ void zero(float (&acc)[4][D / 16])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < D / 16; ++c) acc[i][c] = 0.f;
    }
};

// over the 16 threads that share rows 4 ty .. 4 ty + 3
__device__ __forceinline__ float max16(float x)
{
#pragma unroll
    for (int s = 8; s; s >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, s));
    return x;
}
__device__ __forceinline__ float sum16(float x)
{
#pragma unroll
    for (int s = 8; s; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    return x;
}

template <int D>
__global__ void __launch_bounds__(256) cross_fwd_simt_kernel(const padoc_cross_args a)
{
    using S = Simt<D>;
    extern __shared__ __align__(16) float sm[];
    float *sq = sm, *sk = sq + S::kTile, *sv = sk + S::kTile, *sp = sv + S::kTile;
    const int unit = blockIdx.x / PADOC_CROSS_UNIT_BLOCKS, blk = blockIdx.x % PADOC_CROSS_UNIT_BLOCKS;
    const padoc_cross_unit u = a.units[unit];
    const int g = u.g, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    pdl_launch_dependents();
    if (blk * a.block_tokens >= u.ntok) return;
    auto heads_row = [&](const void *base, int64_t stride, int r) -> const float * {
        int token, head;
        if (!cross_row(a, u.tok, u.ntok, blk * kB + r, token, head)) return nullptr;
        return (const float *)base + (size_t)token * stride + (size_t)(g * a.group + head) * D;
    };
    S::load(sq, [&](int r) { return heads_row(a.q, a.q_stride, r); });
    float acc[4][D / 16], m[4], l[4];
    S::zero(acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) { m[i] = -INFINITY; l[i] = 0.f; }
    for (int j0 = 0; j0 < u.nk; j0 += kB) {
        __syncthreads();
        auto key_row = [&](const void *base, int64_t stride, int r) -> const float * {
            return j0 + r < u.nk ? (const float *)base + (size_t)(u.k0 + j0 + r) * stride + (size_t)g * D : nullptr;
        };
        S::load(sk, [&](int r) { return key_row(a.k, a.k_stride, r); });
        S::load(sv, [&](int r) { return key_row(a.v, a.v_stride, r); });
        __syncthreads();
        float s[4][4];
        S::dots(sq, sk, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mx = m[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = j0 + tx + 16 * j < u.nk ? s[i][j] * a.scale_log2 : -INFINITY;
                mx = fmaxf(mx, s[i][j]);
            }
            mx = max16(mx);
            const float ref = mx == -INFINITY ? 0.f : mx, alpha = exp2f(m[i] - ref);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = exp2f(s[i][j] - ref);
                sum += p;
                sp[(4 * ty + i) * S::PS + tx + 16 * j] = p;
            }
            l[i] = l[i] * alpha + sum16(sum);
            m[i] = mx;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) acc[i][c] *= alpha;
        }
        __syncwarp();   // (a product's rows are written and read by the same half warp)
        S::add_product(sp, sv, acc);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = blk * kB + 4 * ty + i;
        int token, head;
        if (!cross_row(a, u.tok, u.ntok, r, token, head)) continue;
        const float inv = l[i] == 0.f ? 0.f : 1.f / l[i], lse2 = l[i] == 0.f ? -INFINITY : m[i] + log2f(l[i]);
        const size_t h = (size_t)token * a.hq + g * a.group + head;
        const size_t pr = (size_t)max(u.slot, 0) * (PADOC_CROSS_UNIT_BLOCKS * kB) + r;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const float4 x = make_float4(acc[i][4 * j] * inv, acc[i][4 * j + 1] * inv, acc[i][4 * j + 2] * inv, acc[i][4 * j + 3] * inv);
            if (u.slot < 0) store4((float *)a.o + h * D + 64 * j + 4 * tx, x);
            else store4(a.part + pr * D + 64 * j + 4 * tx, x);
        }
        if (tx == 0) {
            if (u.slot < 0) a.lse[h] = lse2 * PADOC_LN2;
            else a.part_lse[pr] = lse2;
        }
    }
}

// dQ, and the rows' statistics for the dK/dV pass.
template <int D>
__global__ void __launch_bounds__(256) cross_dq_simt_kernel(const padoc_cross_args a)
{
    using S = Simt<D>;
    extern __shared__ __align__(16) float sm[];
    float *sq = sm, *sg = sq + S::kTile, *sk = sg + S::kTile, *sv = sk + S::kTile, *sp = sv + S::kTile;
    float *st = sp + kB * S::PS;   // -lse2 and D
    const int unit = blockIdx.x / PADOC_CROSS_DQ_BLOCKS, blk = blockIdx.x % PADOC_CROSS_DQ_BLOCKS;
    const padoc_cross_unit u = a.units[unit];
    const int g = u.g, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    if (blk * a.block_tokens >= u.ntok) return;
    auto heads_row = [&](const void *base, int64_t stride, int r) -> const float * {
        int token, head;
        if (!cross_row(a, u.tok, u.ntok, blk * kB + r, token, head)) return nullptr;
        return (const float *)base + (size_t)token * stride + (size_t)(g * a.group + head) * D;
    };
    S::load(sq, [&](int r) { return heads_row(a.q, a.q_stride, r); });
    S::load(sg, [&](int r) { return heads_row(a.dout, (int64_t)a.hq * D, r); });
    for (int r = threadIdx.x >> 5; r < kB; r += 8) {   // a warp per row
        const float *o = heads_row(a.out, (int64_t)a.hq * D, r), *d = heads_row(a.dout, (int64_t)a.hq * D, r);
        const int c = threadIdx.x & 31;
        float x = 0.f;
        if (o && c < D / 4) {
            const float4 u4 = load4(o + 4 * c), v4 = load4(d + 4 * c);
            x = fmaf(u4.x, v4.x, fmaf(u4.y, v4.y, fmaf(u4.z, v4.z, u4.w * v4.w)));
        }
#pragma unroll
        for (int s = 16; s; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
        if (c == 0) {
            int token, head;
            const bool in = cross_row(a, u.tok, u.ntok, blk * kB + r, token, head);
            const float l = in ? a.lse_in[(size_t)token * a.hq + g * a.group + head] : -INFINITY;
            st[r] = l == -INFINITY ? -INFINITY : -l * PADOC_LOG2E;
            st[kB + r] = in ? x : 0.f;
            if (u.sub >= 0) {
                const size_t at = ((size_t)g * a.num_subs + u.sub + blk) * kB + r;
                a.neg_lse2[at] = st[r];
                a.dsum[at] = st[kB + r];
            }
        }
    }
    float acc[4][D / 16];
    S::zero(acc);
    for (int j0 = 0; j0 < u.nk; j0 += kB) {
        __syncthreads();
        auto key_row = [&](const void *base, int64_t stride, int r) -> const float * {
            return j0 + r < u.nk ? (const float *)base + (size_t)(u.k0 + j0 + r) * stride + (size_t)g * D : nullptr;
        };
        S::load(sk, [&](int r) { return key_row(a.k, a.k_stride, r); });
        S::load(sv, [&](int r) { return key_row(a.v, a.v_stride, r); });
        __syncthreads();
        float s[4][4], dp[4][4];
        S::dots(sq, sk, s);
        S::dots(sg, sv, dp);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = exp2f(fmaf(s[i][j], a.scale_log2, st[4 * ty + i]));
                sp[(4 * ty + i) * S::PS + tx + 16 * j] = j0 + tx + 16 * j < u.nk ? p * (dp[i][j] - st[kB + 4 * ty + i]) : 0.f;
            }
        __syncwarp();
        S::add_product(sp, sk, acc);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = blk * kB + 4 * ty + i;
        int token, head;
        if (!cross_row(a, u.tok, u.ntok, r, token, head)) continue;
        const float mul = u.slot < 0 ? a.scale : 1.f;
        const size_t pr = (size_t)max(u.slot, 0) * (PADOC_CROSS_DQ_BLOCKS * kB) + r;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const float4 x = make_float4(acc[i][4 * j] * mul, acc[i][4 * j + 1] * mul, acc[i][4 * j + 2] * mul, acc[i][4 * j + 3] * mul);
            if (u.slot < 0) store4((float *)a.dq + (size_t)token * a.dq_stride + (size_t)(g * a.group + head) * D + 64 * j + 4 * tx, x);
            else store4(a.part + pr * D + 64 * j + 4 * tx, x);
        }
    }
}

// dK and dV of 64 keys: the sums over every block of rows that sees them, in the covers' order. A cluster of NC CTAs
// shares out the blocks; the CTAs' sums are added through distributed shared memory in rank order.
template <int D, int NC>
__global__ void __launch_bounds__(256) cross_dkv_simt_kernel(const padoc_cross_args a)
{
    using S = Simt<D>;
    extern __shared__ __align__(16) float sm[];
    float *sq = sm, *sg = sq + S::kTile, *sk = sg + S::kTile, *sv = sk + S::kTile, *sp = sv + S::kTile, *sd = sp + kB * S::PS;
    const int rank = blockIdx.x % NC, part = blockIdx.x / NC, half = part & 1, unit = part >> 1, g = unit % a.hkv, i0 = unit / a.hkv;
    padoc_cross_key_tile t;
    if (i0 < a.num_tiles) t = a.tiles[i0];
    else {
        t.k0 = a.tail_begin + (i0 - a.num_tiles) * PADOC_CROSS_KEY_TILE;
        t.nk = (int)min((int64_t)PADOC_CROSS_KEY_TILE, a.key_rows - t.k0);
        t.cover = t.ncover = t.steps = 0;
    }
    const int k0 = t.k0 + half * kB, nk = min(kB, t.nk - half * kB), ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    if (nk <= 0) return;   // (the whole cluster)
    float ak[4][D / 16], av[4][D / 16];
    S::zero(ak);
    S::zero(av);
    if (t.steps > 0) {
        auto key_row = [&](const void *base, int64_t stride, int r) -> const float * {
            return r < nk ? (const float *)base + (size_t)(k0 + r) * stride + (size_t)g * D : nullptr;
        };
        S::load(sk, [&](int r) { return key_row(a.k, a.k_stride, r); });
        S::load(sv, [&](int r) { return key_row(a.v, a.v_stride, r); });
    }
    // this CTA's blocks of the tile's: from .. to
    const int from = (int)((int64_t)t.steps * rank / NC), to = (int)((int64_t)t.steps * (rank + 1) / NC);
    int first = 0;   // of the cover
    for (int ci = 0; ci < t.ncover && first < to; ++ci) {
        const padoc_cross_cover c = a.covers[t.cover + ci];
        const int b0 = max(from - first, 0), b1 = min(c.nsub, to - first);
        first += c.nsub;
        if (c.k0 >= k0 + nk || c.k0 + c.nk <= k0) continue;
        for (int b = b0; b < b1; ++b) {
            auto heads_row = [&](const void *base, int64_t stride, int r) -> const float * {
                int token, head;
                if (!cross_row(a, c.tok, c.ntok, b * kB + r, token, head)) return nullptr;
                return (const float *)base + (size_t)token * stride + (size_t)(g * a.group + head) * D;
            };
            __syncthreads();
            S::load(sq, [&](int r) { return heads_row(a.q, a.q_stride, r); });
            S::load(sg, [&](int r) { return heads_row(a.dout, (int64_t)a.hq * D, r); });
            __syncthreads();
            float s[4][4], dp[4][4];
            S::dots(sk, sq, s);
            S::dots(sv, sg, dp);
            const size_t at = ((size_t)g * a.num_subs + c.sub + b) * kB;
            // Rows whose q or dO is not finite, where a key does not see them: as 0 x NaN would reach the key's sums all the
            // same, the rows become zeros and the weights of the keys that see them NaN. Such a row's lse or D is not
            // finite; where nothing is left of its scores (lse = -inf, finite D) its weights stay zeros.
            const bool some_blind = c.k0 > k0 || c.k0 + c.nk < k0 + nk;
            if (some_blind) {
                __syncthreads();   // (both products have read the rows)
                const int r = threadIdx.x >> 2;
                if (!isfinite(a.neg_lse2[at + r]) || !isfinite(a.dsum[at + r]))
                    for (int e = threadIdx.x & 3; e < D / 4; e += 4)
                        *reinterpret_cast<float4 *>(sq + r * S::P + 4 * e) = *reinterpret_cast<float4 *>(sg + r * S::P + 4 * e) =
                            make_float4(0.f, 0.f, 0.f, 0.f);
                __syncthreads();
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = tx + 16 * j;
                const float l = a.neg_lse2[at + r], d = a.dsum[at + r];
                const bool odd_nan = some_blind && (isnan(l) || !isfinite(d));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool sees = k0 + 4 * ty + i >= c.k0 && k0 + 4 * ty + i < c.k0 + c.nk;
                    // (rows past the segment's: l = -inf)
                    const float p = !sees ? 0.f : odd_nan ? NAN : exp2f(fmaf(s[i][j], a.scale_log2, l));
                    sp[(4 * ty + i) * S::PS + r] = p;
                    sd[(4 * ty + i) * S::PS + r] = sees ? p * (dp[i][j] - d) : 0.f;
                }
            }
            __syncwarp();
            S::add_product(sp, sg, av);
            S::add_product(sd, sq, ak);
        }
    }
    auto write = [&](int r, int c, float4 xk, float4 xv) {
        store4((float *)a.dk + (size_t)(k0 + r) * a.dk_stride + (size_t)g * D + c,
               make_float4(xk.x * a.scale, xk.y * a.scale, xk.z * a.scale, xk.w * a.scale));
        store4((float *)a.dv + (size_t)(k0 + r) * a.dv_stride + (size_t)g * D + c, xv);
    };
    auto cols = [](const float (&x)[D / 16], int j) { return make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]); };
    if constexpr (NC == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 64; ++j)
                if (4 * ty + i < nk) write(4 * ty + i, 64 * j + 4 * tx, cols(ak[i], j), cols(av[i], j));
    } else {
        __syncthreads();
        float *xk = sm, *xv = sm + S::kTile;   // [64][P] each, over the tiles
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                *reinterpret_cast<float4 *>(xk + (4 * ty + i) * S::P + 64 * j + 4 * tx) = cols(ak[i], j);
                *reinterpret_cast<float4 *>(xv + (4 * ty + i) * S::P + 64 * j + 4 * tx) = cols(av[i], j);
            }
        cluster_sync();
        const int mine = (nk - rank + NC - 1) / NC;   // rows rank, rank + NC, ..
        for (int i = threadIdx.x; i < mine * (D / 4); i += 256) {
            const int r = rank + i / (D / 4) * NC, c = i % (D / 4) * 4;
            float4 yk = make_float4(0.f, 0.f, 0.f, 0.f), yv = yk;
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const float4 u = ld_cluster_v4(cluster_map(smem_u32(xk + r * S::P + c), n));
                const float4 v = ld_cluster_v4(cluster_map(smem_u32(xv + r * S::P + c), n));
                yk = make_float4(yk.x + u.x, yk.y + u.y, yk.z + u.z, yk.w + u.w);
                yv = make_float4(yv.x + v.x, yv.y + v.y, yv.z + v.z, yv.w + v.w);
            }
            write(r, c, yk, yv);
        }
        cluster_sync();   // no CTA leaves while another reads its shared memory
    }
}

template <int D>
padoc_status run_fwd_simt(const padoc_cross_args &a, cudaStream_t cs)
{
    constexpr int bytes = (3 * Simt<D>::kTile + kB * Simt<D>::PS) * 4;
    auto kernel = cross_fwd_simt_kernel<D>;
    if (const padoc_status st = padoc_set_max_smem((const void *)kernel, bytes)) return st;
    kernel<<<(unsigned)(a.num_units * PADOC_CROSS_UNIT_BLOCKS), 256, bytes, cs>>>(a);
    return padoc_launch_status();
}

template <int D, int NC>
padoc_status run_dkv_simt(const padoc_cross_args &a, cudaStream_t cs)
{
    constexpr int bytes = (4 * Simt<D>::kTile + 2 * kB * Simt<D>::PS) * 4;
    auto kernel = cross_dkv_simt_kernel<D, NC>;
    if (const padoc_status st = padoc_set_max_smem((const void *)kernel, bytes)) return st;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)((a.num_tiles + a.tail_tiles) * a.hkv * 2 * NC));
    lc.blockDim = dim3(256);
    lc.dynamicSmemBytes = bytes;
    lc.stream = cs;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = NC;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = NC > 1 ? 1 : 0;
    PADOC_CUDA_TRY(cudaLaunchKernelEx(&lc, kernel, a));
    return padoc_launch_status();
}

template <int D>
padoc_status run_bwd_simt(const padoc_cross_args &a, int cluster, cudaStream_t cs)
{
    constexpr int bytes = (4 * Simt<D>::kTile + kB * Simt<D>::PS + 2 * kB) * 4;
    auto dq = cross_dq_simt_kernel<D>;
    if (a.num_units) {
        if (const padoc_status st = padoc_set_max_smem((const void *)dq, bytes)) return st;
        dq<<<(unsigned)(a.num_units * PADOC_CROSS_DQ_BLOCKS), 256, bytes, cs>>>(a);
        if (const padoc_status st = padoc_launch_status()) return st;
    }
    if (!(a.num_tiles + a.tail_tiles)) return PADOC_OK;
    switch (cluster) {
        case 8: return run_dkv_simt<D, 8>(a, cs);
        case 4: return run_dkv_simt<D, 4>(a, cs);
        case 2: return run_dkv_simt<D, 2>(a, cs);
        default: return run_dkv_simt<D, 1>(a, cs);
    }
}

// ------------------------------------------------------------------------------------------------
// Validation
// ------------------------------------------------------------------------------------------------

// Bytes that rows of `width` bytes every `stride` bytes take.
struct Span {
    uintptr_t base;
    int64_t stride, width, rows;
};

// Whether two arrays of rows share a byte. Rows that lie side by side (slices of one buffer, equal strides) do not.
bool overlap(const Span &x, const Span &y)
{
    if (x.rows == 0 || y.rows == 0) return false;
    const uintptr_t xe = x.base + (uintptr_t)((x.rows - 1) * x.stride + x.width), ye = y.base + (uintptr_t)((y.rows - 1) * y.stride + y.width);
    if (xe <= y.base || ye <= x.base) return false;
    if (x.stride != y.stride) return true;
    const int64_t d = (int64_t)((y.base >= x.base ? y.base - x.base : x.base - y.base) % (uintptr_t)x.stride);
    const int64_t first = y.base >= x.base ? x.width : y.width, second = y.base >= x.base ? y.width : x.width;
    return d < first || d + second > x.stride;
}

padoc_status check_rows(const padoc_cross_plan *info, const int32_t *plan, const padoc_cross_rows *r, float scale)
{
    if (!info || !r) return PADOC_ERR_INVALID_ARGUMENT;
    const padoc_cross_config &c = info->cfg;
    if (c.num_q_heads < 1 || c.num_kv_heads < 1 || c.num_q_heads % c.num_kv_heads) return PADOC_ERR_INVALID_ARGUMENT;
    if (c.dtype != PADOC_DTYPE_F32 && c.dtype != PADOC_DTYPE_BF16) return PADOC_ERR_UNSUPPORTED;
    if ((c.head_dim != 64 && c.head_dim != 128) || c.num_q_heads / c.num_kv_heads > kB) return PADOC_ERR_UNSUPPORTED;
    if (!(scale > 0.f) || !isfinite(scale)) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->query_rows < info->query_rows || r->key_rows < info->key_rows || r->query_rows < 0 || r->key_rows < 0 ||
        r->query_rows > INT32_MAX - 1024 || r->key_rows > INT32_MAX - 1024)
        return PADOC_ERR_INVALID_ARGUMENT;
    const int64_t e = c.dtype == PADOC_DTYPE_F32 ? 4 : 2;
    const int64_t most = (int64_t)1 << 39;   // (a tensor map's strides have 40 bits)
    for (const int64_t s : {r->q_stride, r->k_stride, r->v_stride})
        if (s < 0 || s > most / e || s * e % 16) return PADOC_ERR_INVALID_ARGUMENT;
    // (what the overlap checks add up stays in 64 bits)
    if (r->q_stride * e > INT64_MAX / 4 / (r->query_rows + 1) || std::max(r->k_stride, r->v_stride) * e > INT64_MAX / 4 / (r->key_rows + 1))
        return PADOC_ERR_INVALID_ARGUMENT;
    if (r->q_stride < (int64_t)c.num_q_heads * c.head_dim || r->k_stride < (int64_t)c.num_kv_heads * c.head_dim ||
        r->v_stride < (int64_t)c.num_kv_heads * c.head_dim)
        return PADOC_ERR_INVALID_ARGUMENT;
    if ((((uintptr_t)r->q) | ((uintptr_t)r->k) | ((uintptr_t)r->v) | ((uintptr_t)plan)) & 15) return PADOC_ERR_INVALID_ARGUMENT;
    if (info->query_rows > 0 && (!r->q || !plan)) return PADOC_ERR_INVALID_ARGUMENT;
    if (info->key_rows > 0 && (!r->k || !r->v)) return PADOC_ERR_INVALID_ARGUMENT;
    return PADOC_OK;
}

void fill_args(padoc_cross_args &a, const padoc_cross_plan *info, const padoc_cross_rows *r, float scale)
{
    a = padoc_cross_args{};
    a.q = r->q;
    a.k = r->k;
    a.v = r->v;
    a.q_stride = r->q_stride;
    a.k_stride = r->k_stride;
    a.v_stride = r->v_stride;
    a.query_rows = r->query_rows;
    a.key_rows = r->key_rows;
    a.hq = info->cfg.num_q_heads;
    a.hkv = info->cfg.num_kv_heads;
    a.group = a.hq / a.hkv;
    a.block_tokens = kB / a.group;
    a.scale = scale;
    a.scale_log2 = scale * PADOC_LOG2E;
}

}  // namespace

extern "C" padoc_status padoc_cross_attn(const padoc_cross_plan *info, const int32_t *plan_dev, const padoc_cross_rows *rows,
                                         float scale, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                         padoc_stream_t stream)
{
    padoc_status st = check_rows(info, plan_dev, rows, scale);
    if (st != PADOC_OK) return st;
    if (info->query_rows == 0) return PADOC_OK;
    if (!out || !lse || (((uintptr_t)out) & 15) || (((uintptr_t)lse) & 3)) return PADOC_ERR_INVALID_ARGUMENT;
    size_t need = 0;
    if ((st = padoc_cross_workspace_size(info, &need)) != PADOC_OK) return st;
    if (need && (!workspace || (((uintptr_t)workspace) & 255))) return PADOC_ERR_INVALID_ARGUMENT;
    if (workspace_bytes < need) return PADOC_ERR_WORKSPACE_TOO_SMALL;
    const padoc_cross_config &c = info->cfg;
    const int64_t e = c.dtype == PADOC_DTYPE_F32 ? 4 : 2, qw = (int64_t)c.num_q_heads * c.head_dim * e, kw = (int64_t)c.num_kv_heads * c.head_dim * e;
    const Span in[] = {{(uintptr_t)rows->q, rows->q_stride * e, qw, info->query_rows},
                       {(uintptr_t)rows->k, rows->k_stride * e, kw, info->key_rows},
                       {(uintptr_t)rows->v, rows->v_stride * e, kw, info->key_rows}};
    const Span to[] = {{(uintptr_t)out, qw, qw, info->query_rows},
                       {(uintptr_t)lse, (int64_t)c.num_q_heads * 4, (int64_t)c.num_q_heads * 4, info->query_rows}};
    if (overlap(to[0], to[1])) return PADOC_ERR_INVALID_ARGUMENT;
    for (const Span &x : to)
        for (const Span &y : in)
            if (overlap(x, y)) return PADOC_ERR_INVALID_ARGUMENT;

    padoc_cross_args a;
    fill_args(a, info, rows, scale);
    a.units = (const padoc_cross_unit *)(plan_dev + info->off_units);
    a.merges = (const padoc_cross_merge *)(plan_dev + info->off_merges);
    a.num_units = info->num_units;
    a.num_merges = info->num_merges;
    a.o = out;
    a.lse = lse;
    a.part = (float *)workspace;
    a.ctas = info->num_ctas ? plan_dev + info->off_ctas : nullptr;
    a.num_ctas = info->num_ctas;
    a.max_parts = info->max_parts;
    a.unit_rows = info->unit_rows;
    a.part_lse = a.part + (size_t)info->num_slots * a.unit_rows * c.head_dim;
    cudaStream_t cs = (cudaStream_t)stream;
    if (a.num_units) {
        if (c.dtype == PADOC_DTYPE_F32) st = c.head_dim == 64 ? run_fwd_simt<64>(a, cs) : run_fwd_simt<128>(a, cs);
        else if (info->few) st = padoc_cross_launch_few(a, c.head_dim, info->few, cs);
        else st = padoc_cross_launch_tc(a, c.head_dim, cs);
        if (st != PADOC_OK) return st;
    }
    if (!a.num_merges) return PADOC_OK;
    return c.dtype == PADOC_DTYPE_F32 ? merge_rows<float, false>(a, c.head_dim, a.num_units > 0, cs)
                                      : merge_rows<__nv_bfloat16, false>(a, c.head_dim, a.num_units > 0, cs);
}

extern "C" padoc_status padoc_cross_attn_bwd(const padoc_cross_plan *info, const int32_t *plan_dev, const padoc_cross_rows *rows,
                                             const void *out, const void *dout, const float *lse, float scale,
                                             const padoc_cross_grads *grads, void *workspace, size_t workspace_bytes,
                                             padoc_stream_t stream)
{
    padoc_status st = check_rows(info, plan_dev, rows, scale);
    if (st != PADOC_OK) return st;
    if (!grads || !info->cfg.backward) return PADOC_ERR_INVALID_ARGUMENT;
    const padoc_cross_config &c = info->cfg;
    const int64_t e = c.dtype == PADOC_DTYPE_F32 ? 4 : 2;
    for (const int64_t s : {grads->dq_stride, grads->dk_stride, grads->dv_stride})
        if (s < 0 || s > ((int64_t)1 << 39) / e || s * e % 16) return PADOC_ERR_INVALID_ARGUMENT;
    if (grads->dq_stride * e > INT64_MAX / 4 / (rows->query_rows + 1) ||
        std::max(grads->dk_stride, grads->dv_stride) * e > INT64_MAX / 4 / (rows->key_rows + 1))
        return PADOC_ERR_INVALID_ARGUMENT;
    if (grads->dq_stride < (int64_t)c.num_q_heads * c.head_dim || grads->dk_stride < (int64_t)c.num_kv_heads * c.head_dim ||
        grads->dv_stride < (int64_t)c.num_kv_heads * c.head_dim)
        return PADOC_ERR_INVALID_ARGUMENT;
    if (info->query_rows > 0 && (!out || !dout || !lse || !grads->dq)) return PADOC_ERR_INVALID_ARGUMENT;
    if (rows->key_rows > 0 && (!grads->dk || !grads->dv)) return PADOC_ERR_INVALID_ARGUMENT;
    if (((((uintptr_t)out) | ((uintptr_t)dout) | ((uintptr_t)grads->dq) | ((uintptr_t)grads->dk) | ((uintptr_t)grads->dv)) & 15) ||
        (((uintptr_t)lse) & 3))
        return PADOC_ERR_INVALID_ARGUMENT;
    size_t need = 0;
    if ((st = padoc_cross_bwd_workspace_size(info, &need)) != PADOC_OK) return st;
    if (need && (!workspace || (((uintptr_t)workspace) & 255))) return PADOC_ERR_INVALID_ARGUMENT;
    if (workspace_bytes < need) return PADOC_ERR_WORKSPACE_TOO_SMALL;
    const int64_t qw = (int64_t)c.num_q_heads * c.head_dim * e, kw = (int64_t)c.num_kv_heads * c.head_dim * e, lw = (int64_t)c.num_q_heads * 4;
    const Span in[] = {{(uintptr_t)rows->q, rows->q_stride * e, qw, info->query_rows},
                       {(uintptr_t)rows->k, rows->k_stride * e, kw, info->key_rows},
                       {(uintptr_t)rows->v, rows->v_stride * e, kw, info->key_rows},
                       {(uintptr_t)out, qw, qw, info->query_rows},
                       {(uintptr_t)dout, qw, qw, info->query_rows},
                       {(uintptr_t)lse, lw, lw, info->query_rows}};
    const Span to[] = {{(uintptr_t)grads->dq, grads->dq_stride * e, qw, info->query_rows},
                       {(uintptr_t)grads->dk, grads->dk_stride * e, kw, rows->key_rows},
                       {(uintptr_t)grads->dv, grads->dv_stride * e, kw, rows->key_rows}};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(to[i], to[j])) return PADOC_ERR_INVALID_ARGUMENT;
        for (const Span &y : in)
            if (overlap(to[i], y)) return PADOC_ERR_INVALID_ARGUMENT;
    }

    padoc_cross_args a;
    fill_args(a, info, rows, scale);
    a.units = (const padoc_cross_unit *)(plan_dev + info->off_dq_units);
    a.merges = (const padoc_cross_merge *)(plan_dev + info->off_dq_merges);
    a.tiles = (const padoc_cross_key_tile *)(plan_dev + info->off_key_tiles);
    a.covers = (const padoc_cross_cover *)(plan_dev + info->off_covers);
    a.ctas = info->num_dq_ctas ? plan_dev + info->off_dq_ctas : nullptr;
    a.num_units = info->num_dq_units;
    a.num_ctas = info->num_dq_ctas;
    a.max_parts = info->max_dq_parts;
    a.unit_rows = PADOC_CROSS_DQ_BLOCKS * kB;
    a.num_merges = info->num_dq_merges;
    a.num_tiles = info->num_key_tiles;
    a.num_subs = info->num_subs;
    // the key tiles reach to the last key that a row sees; behind it the gradients are zero
    a.tail_begin = info->key_rows;
    a.tail_tiles = (int32_t)((rows->key_rows - info->key_rows + PADOC_CROSS_KEY_TILE - 1) / PADOC_CROSS_KEY_TILE);
    if ((int64_t)(a.num_tiles + (int64_t)a.tail_tiles) * a.hkv * 16 > INT32_MAX) return PADOC_ERR_UNSUPPORTED;
    if (a.num_units + a.num_merges + a.num_tiles + a.tail_tiles == 0) return PADOC_OK;
    a.out = out;
    a.dout = dout;
    a.lse_in = lse;
    a.dq = grads->dq;
    a.dk = grads->dk;
    a.dv = grads->dv;
    a.dq_stride = grads->dq_stride;
    a.dk_stride = grads->dk_stride;
    a.dv_stride = grads->dv_stride;
    const size_t stats = (size_t)info->num_subs * a.hkv * kB;
    a.neg_lse2 = (float *)workspace;
    a.dsum = a.neg_lse2 + stats;
    a.part = a.dsum + (c.dtype == PADOC_DTYPE_F32 ? 1 : 4) * stats;   // (bf16: 16 bytes a row)
    a.dkv = (const padoc_cross_dkv *)(plan_dev + info->off_dkv);
    a.dkv_ctas = plan_dev + info->off_dkv_ctas;
    a.dkv_sums = (const padoc_cross_dkv_sum *)(plan_dev + info->off_dkv_sums);
    a.num_dkv_ctas = info->num_dkv_ctas;
    a.num_dkv_sums = info->num_dkv_sums;
    a.num_dkv_slots = info->num_dkv_slots;
    a.gap_tile = info->num_key_tiles - info->num_gap_tiles;
    a.part_dkv = a.part + (size_t)info->num_dq_slots * a.unit_rows * c.head_dim;
    cudaStream_t cs = (cudaStream_t)stream;
    if (c.dtype == PADOC_DTYPE_F32) st = c.head_dim == 64 ? run_bwd_simt<64>(a, info->cluster, cs) : run_bwd_simt<128>(a, info->cluster, cs);
    else st = padoc_cross_launch_bwd_tc(a, c.head_dim, cs);
    if (st != PADOC_OK) return st;
    if (!a.num_merges) return PADOC_OK;
    return c.dtype == PADOC_DTYPE_F32 ? merge_rows<float, true>(a, c.head_dim, false, cs)
                                      : merge_rows<__nv_bfloat16, true>(a, c.head_dim, false, cs);
}
