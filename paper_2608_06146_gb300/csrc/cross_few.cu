// cross_few.cu -- cross attention forward for few rows: at most 32 packed (token, head) rows of a KV head over a
// segment's keys (single tokens, the streams of one page under as many KV heads as query heads).
//
// K and V are read once and used for few rows, so the call is bound by their bytes and, when those are few, by the
// latency of its launches. Four warps with warp-level MMAs (m16n8k16) take 16 keys each of every 64-key tile and keep
// their own maximum, sum and O in registers; their results are joined in shared memory. Tiles come by TMA through a ring
// deep enough that two or three CTAs of an SM keep some 190 KB on the way. With kTiles = 1 a row tile of 16 is computed,
// with 2 two. A unit is run by a cluster of NC CTAs that share its tiles and join their results through distributed
// shared memory, or its keys are cut into parts that a later kernel joins.
//
// Measured: 670 streams over 32 pages of up to 1201 states, 16 heads of 64 dims: 23.3 us, 92 MB at 58% of the copy rate
// (the items' starts and ends, as the pages' lengths differ); one stream over 961 states 5.3 us in a graph, most of it the
// launch (on tcgen05 items, cut and joined, the two took 39 and 16 us).
//
// As in the other kernels, what lies behind a segment's keys may be anything: scores past the end become -inf and V's
// rows zeros.
#include <math.h>

#include "cross.cuh"

namespace {

constexpr int kWarps = 4;
constexpr int kKeys = PADOC_CROSS_FEW_STEP;      // keys of a tile, 16 a warp
constexpr int kPanel = kKeys * 128;              // [64 keys][64 bf16]
static_assert(kKeys == 16 * kWarps, "");

template <int D, int kTiles>
struct Few {
    static constexpr int kRows = 16 * kTiles;
    static constexpr int kStages = D == 64 ? 4 : 3;
    static constexpr int kStage = 2 * (D / 64) * kPanel;     // K and V
    static constexpr int kPitch = D + 4;                     // floats of a row of the joined results
    static constexpr int kCtas = D == 64 ? 3 : 2;            // an SM
    static constexpr size_t kRing = (size_t)kStages * kStage;
    static constexpr size_t kSmemBytes = 1024 + kRing + (size_t)kRows * D * 2 + 2 * kStages * 8 + 64;
    static_assert((size_t)(kWarps + 1) * kRows * (kPitch + 2) * 4 <= kRing, "");
};

template <int D, int kTiles, int NC>
__global__ void __launch_bounds__(32 * kWarps, Few<D, kTiles>::kCtas)
cross_few_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const padoc_cross_args a)
{
    using F = Few<D, kTiles>;
    constexpr int kStages = F::kStages, kRows = F::kRows, kPanels = D / 64, kPitch = F::kPitch;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sq = smem + F::kRing;                            // [panel][kRows][64], swizzled
    uint64_t *bars = (uint64_t *)(sq + kRows * D * 2);        // [stage] full, [stage] empty
    volatile int *abort_flag = (volatile int *)(bars + 2 * kStages);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int rank = NC > 1 ? (int)cluster_rank() : 0;
    auto full = [&](int s) { return smem_u32(bars + s); };
    auto empty = [&](int s) { return smem_u32(bars + kStages + s); };
    if (tid == 0) {
        tma_prefetch_desc(&kmap);
        tma_prefetch_desc(&vmap);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), kWarps);
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    pdl_launch_dependents();
    pdl_wait_prerequisite();
    const padoc_cross_unit u = a.units[blockIdx.x / NC];
    // this CTA's tiles of the unit
    const int tiles = (u.nk + kKeys - 1) / kKeys, t0 = (int)((int64_t)tiles * rank / NC), n = (int)((int64_t)tiles * (rank + 1) / NC) - t0;
    const int rows = u.ntok * a.group;
    __syncthreads();
    auto issue = [&](int t) {
        const int s = t % kStages, row = u.k0 + (t0 + t) * kKeys;
        mbar_arrive_expect_tx(full(s), F::kStage);
#pragma unroll
        for (int p = 0; p < kPanels; ++p) {
            tma_load_2d(smem_u32(smem + s * F::kStage + p * kPanel), &kmap, u.g * D + 64 * p, row, full(s));
            tma_load_2d(smem_u32(smem + s * F::kStage + (kPanels + p) * kPanel), &vmap, u.g * D + 64 * p, row, full(s));
        }
    };
    int issued = 0;
    if (tid == 0)
        for (; issued < min(n, kStages - 1); ++issued) issue(issued);
    // Q's rows (zeros past the unit's), then as A fragments
    for (int i = tid; i < kRows * (D / 8); i += 32 * kWarps) {
        const int r = i / (D / 8), c = i % (D / 8) * 8;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (r < rows) {
            const int t = r / a.group;
            x = *reinterpret_cast<const uint4 *>((const __nv_bfloat16 *)a.q + (size_t)(u.tok + t) * a.q_stride +
                                                 (size_t)(u.g * a.group + r - t * a.group) * D + c);
        }
        *reinterpret_cast<uint4 *>(sq + (c >> 6) * kRows * 128 + sw128_offset(r, c & 63)) = x;
    }
    __syncthreads();
    uint32_t qf[kTiles][D / 16][4];
#pragma unroll
    for (int m = 0; m < kTiles; ++m)
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const int r = 16 * m + (lane & 15), c = 16 * k + (lane >> 4) * 8;
            ldmatrix_x4(qf[m][k], smem_u32(sq + (c >> 6) * kRows * 128 + sw128_offset(r, c & 63)));
        }
    float o[kTiles][D / 8][4], mref[kTiles][2], l[kTiles][2];
#pragma unroll
    for (int m = 0; m < kTiles; ++m) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[m][i][0] = o[m][i][1] = o[m][i][2] = o[m][i][3] = 0.f;
        mref[m][0] = mref[m][1] = -INFINITY;
        l[m][0] = l[m][1] = 0.f;
    }
    bool ok = true;
    for (int t = 0; t < n; ++t) {
        if (warp == 0 && t + kStages - 1 < n) {   // the tile before this one has been read by every warp
            const int s = (t + kStages - 1) % kStages;
            if (t > 0 && !mbar_wait_warp(empty(s), ((t - 1) / kStages) & 1, a.err, 220, abort_flag)) { ok = false; break; }
            if (lane == 0) {
                issue(t + kStages - 1);
                ++issued;
            }
        }
        const int s = t % kStages;
        if (!mbar_wait_warp(full(s), (t / kStages) & 1, a.err, 221, abort_flag)) { ok = false; break; }
        const uint8_t *kt = smem + s * F::kStage;
        uint8_t *vt = smem + s * F::kStage + kPanels * kPanel;
        const int left = u.nk - (t0 + t) * kKeys - 16 * warp;   // keys from this warp's first one on
        if (left > 0) {
            float sc[kTiles][2][4];
#pragma unroll
            for (int m = 0; m < kTiles; ++m)
#pragma unroll
                for (int j = 0; j < 2; ++j) sc[m][j][0] = sc[m][j][1] = sc[m][j][2] = sc[m][j][3] = 0.f;
            {
                const int r = 16 * warp + (lane & 7) + (lane >> 4) * 8;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const int c = 16 * k + ((lane >> 3) & 1) * 8;
                    uint32_t b[4];
                    ldmatrix_x4(b, smem_u32(kt + (c >> 6) * kPanel + sw128_offset(r, c & 63)));
#pragma unroll
                    for (int m = 0; m < kTiles; ++m) {
                        mma_bf16_16816(sc[m][0], qf[m][k], b[0], b[1]);
                        mma_bf16_16816(sc[m][1], qf[m][k], b[2], b[3]);
                    }
                }
            }
            if (left < 16) {
#pragma unroll
                for (int m = 0; m < kTiles; ++m)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (8 * j + 2 * (lane & 3) + (e & 1) >= left) sc[m][j][e] = -INFINITY;
                // V's rows past the end (this warp's own 16)
                for (int i = lane; i < (16 - left) * 8 * kPanels; i += 32)
                    *reinterpret_cast<uint4 *>(vt + i / 8 / (16 - left) * kPanel + (16 * warp + left + i / 8 % (16 - left)) * 128 + i % 8 * 16) =
                        make_uint4(0, 0, 0, 0);
                __syncwarp();
            }
            uint32_t pf[kTiles][4];
            bool grow = false;
            float mx[kTiles][2];
#pragma unroll
            for (int m = 0; m < kTiles; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x = fmaxf(fmaxf(sc[m][0][2 * h], sc[m][0][2 * h + 1]), fmaxf(sc[m][1][2 * h], sc[m][1][2 * h + 1]));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                    mx[m][h] = fmaxf(mref[m][h], x);
                    // the reference moves only when the maximum has grown by more than 2^8: P <= 256
                    if (mref[m][h] == -INFINITY) mref[m][h] = mx[m][h];
                    grow |= (mx[m][h] - mref[m][h]) * a.scale_log2 > 8.f;
                }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int m = 0; m < kTiles; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bool g = (mx[m][h] - mref[m][h]) * a.scale_log2 > 8.f;
                        const float alpha = g ? fast_exp2((mref[m][h] - mx[m][h]) * a.scale_log2) : 1.f;
                        if (g) mref[m][h] = mx[m][h];
                        l[m][h] *= alpha;
#pragma unroll
                        for (int i = 0; i < D / 8; ++i) {
                            o[m][i][2 * h] *= alpha;
                            o[m][i][2 * h + 1] *= alpha;
                        }
                    }
            }
#pragma unroll
            for (int m = 0; m < kTiles; ++m) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float off = mref[m][h] == -INFINITY ? 0.f : -mref[m][h] * a.scale_log2;
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = fast_exp2(fmaf(sc[m][e >> 1][2 * h + (e & 1)], a.scale_log2, off));
                    l[m][h] += (p[0] + p[1]) + (p[2] + p[3]);
                    // (bf16, the MMA's operand type; l adds the unrounded weights)
                    pf[m][h] = pack_bf16x2(p[0], p[1]);
                    pf[m][2 + h] = pack_bf16x2(p[2], p[3]);
                }
            }
            const int r = 16 * warp + (lane & 15);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int c = 16 * i + (lane >> 4) * 8;
                uint32_t b[4];
                ldmatrix_x4_trans(b, smem_u32(vt + (c >> 6) * kPanel + sw128_offset(r, c & 63)));
#pragma unroll
                for (int m = 0; m < kTiles; ++m) {
                    mma_bf16_16816(o[m][2 * i], pf[m], b[0], b[1]);
                    mma_bf16_16816(o[m][2 * i + 1], pf[m], b[2], b[3]);
                }
            }
        }
        __syncwarp();
        mbar_arrive_warp(empty(s));
    }
    // copies still in flight must land before the ring is used for something else
    if (tid == 0)
        for (int t = max(issued - kStages, 0); t < issued; ++t) mbar_wait_bounded(full(t % kStages), (t / kStages) & 1, a.err, 222);
#pragma unroll
    for (int m = 0; m < kTiles; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[m][h] += __shfl_xor_sync(0xffffffffu, l[m][h], 1);
            l[m][h] += __shfl_xor_sync(0xffffffffu, l[m][h], 2);
        }
    __syncthreads();
    // The warps' results: [warp][row][kPitch] O, then [warp][row] maxima and sums (log2 units), then the joined ones.
    float *so = (float *)smem, *sm = so + kWarps * kRows * kPitch, *sl = sm + kWarps * kRows;
    float *jo = sl + kWarps * kRows, *jl = jo + kRows * kPitch;
#pragma unroll
    for (int m = 0; m < kTiles; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 16 * m + 8 * h + (lane >> 2);
            float *row = so + (warp * kRows + r) * kPitch;
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
                *reinterpret_cast<float2 *>(row + 8 * i + 2 * (lane & 3)) = make_float2(o[m][i][2 * h], o[m][i][2 * h + 1]);
            if ((lane & 3) == 0) {
                sm[warp * kRows + r] = mref[m][h] == -INFINITY ? -INFINITY : mref[m][h] * a.scale_log2;
                sl[warp * kRows + r] = l[m][h];
            }
        }
    __syncthreads();
    // Joined row by row, four dims a thread. What the row holds then is O / l and lse * log2(e), which the cluster's
    // CTAs join once more (rows rank, rank + NC, ..).
    auto write = [&](int r, int c, float4 x, float lse2) {
        const int t = r / a.group;
        const size_t h = (size_t)(u.tok + t) * a.hq + u.g * a.group + (r - t * a.group);
        if (u.slot < 0) {
            *reinterpret_cast<uint2 *>((__nv_bfloat16 *)a.o + h * D + c) = make_uint2(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w));
            if (c == 0) a.lse[h] = lse2 * PADOC_LN2;
        } else {
            const size_t pr = (size_t)u.slot * a.unit_rows + r;
            *reinterpret_cast<float4 *>(a.part + pr * D + c) = x;
            if (c == 0) a.part_lse[pr] = lse2;
        }
    };
    for (int i = tid; ok && i < rows * (D / 4); i += 32 * kWarps) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm[w * kRows + r]);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float mw = sm[w * kRows + r], f = mw == -INFINITY ? (sl[w * kRows + r] == 0.f ? 0.f : 1.f) : fast_exp2(mw - top);
            const float4 y = *reinterpret_cast<const float4 *>(so + (w * kRows + r) * kPitch + c);
            sum = fmaf(f, sl[w * kRows + r], sum);
            x.x = fmaf(f, y.x, x.x);
            x.y = fmaf(f, y.y, x.y);
            x.z = fmaf(f, y.z, x.z);
            x.w = fmaf(f, y.w, x.w);
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum, lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
        x = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
        if (NC == 1) {
            write(r, c, x, lse2);
        } else {
            *reinterpret_cast<float4 *>(jo + r * kPitch + c) = x;
            if (c == 0) jl[r] = lse2;
        }
    }
    if (NC > 1) {
        cluster_sync();
        const int mine = (rows - rank + NC - 1) / NC;
        for (int i = tid; ok && i < mine * (D / 4); i += 32 * kWarps) {
            const int r = rank + i / (D / 4) * NC, c = i % (D / 4) * 4;
            float lse2[NC], top = -INFINITY, sum = 0.f;
            float4 y[NC], x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                lse2[k] = ld_cluster(cluster_map(smem_u32(jl + r), k));
                y[k] = ld_cluster_v4(cluster_map(smem_u32(jo + r * kPitch + c), k));
            }
#pragma unroll
            for (int k = 0; k < NC; ++k) top = fmaxf(top, lse2[k]);
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const float f = lse2[k] == -INFINITY ? 0.f : fast_exp2(lse2[k] - top);
                sum += f;
                x.x = fmaf(f, y[k].x, x.x);
                x.y = fmaf(f, y[k].y, x.y);
                x.z = fmaf(f, y[k].z, x.z);
                x.w = fmaf(f, y[k].w, x.w);
            }
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            write(r, c, make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv), sum == 0.f ? -INFINITY : top + log2f(sum));
        }
        cluster_sync();   // no CTA leaves while another reads its shared memory
    }
}

template <int D, int kTiles, int NC>
padoc_status launch(const padoc_cross_args &a, cudaStream_t stream)
{
    auto kernel = cross_few_kernel<D, kTiles, NC>;
    constexpr size_t bytes = Few<D, kTiles>::kSmemBytes;
    if (const padoc_status st = padoc_set_max_smem((const void *)kernel, (int)bytes)) return st;
    CUtensorMap kmap, vmap;
    if (!padoc_make_tmap_bf16(&kmap, a.k, (uint64_t)a.hkv * D, a.key_rows, a.k_stride * 2, 64, kKeys) ||
        !padoc_make_tmap_bf16(&vmap, a.v, (uint64_t)a.hkv * D, a.key_rows, a.v_stride * 2, 64, kKeys))
        return PADOC_ERR_CUDA;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(a.num_units * NC));
    lc.blockDim = dim3(32 * kWarps);
    lc.dynamicSmemBytes = bytes;
    lc.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // set up behind the last kernel's end
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = NC;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = NC > 1 ? 2 : 1;
    PADOC_CUDA_TRY(cudaLaunchKernelEx(&lc, kernel, kmap, vmap, a));
    return padoc_launch_status();
}

template <int D, int kTiles>
padoc_status run(const padoc_cross_args &a, int cluster, cudaStream_t stream)
{
    switch (cluster) {
        case 8: return launch<D, kTiles, 8>(a, stream);
        case 4: return launch<D, kTiles, 4>(a, stream);
        case 2: return launch<D, kTiles, 2>(a, stream);
        default: return launch<D, kTiles, 1>(a, stream);
    }
}

}  // namespace

padoc_status padoc_cross_launch_few(const padoc_cross_args &args, int head_dim, int cluster, cudaStream_t stream)
{
    padoc_cross_args a = args;
    a.err = padoc_device_error_word();
    if (!a.err) return PADOC_ERR_CUDA;
    if (head_dim == 64) return a.unit_rows == 16 ? run<64, 1>(a, cluster, stream) : run<64, 2>(a, cluster, stream);
    return a.unit_rows == 16 ? run<128, 1>(a, cluster, stream) : run<128, 2>(a, cluster, stream);
}
