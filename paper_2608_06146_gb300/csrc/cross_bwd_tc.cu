// cross_bwd_tc.cu -- gradients of cross attention on the 5th-generation tensor cores, in two passes without atomics.
//
// With c = scale * log2(e), lse2 = lse * log2(e), D = rowsum(dO * O):
//   P = exp2(S c - lse2),  dS = P (dP - D),  S = Q K^T,  dP = dO V^T.
//
// dQ pass: a unit is a 128-row tile of packed (token, head) rows of one KV head over a segment's keys, or a part of
//   them (parts are joined by a later kernel). It walks 64-key steps: S = Q K^T (Q in tensor memory), dP = dO V^T (dO in
//   shared memory), dS as bf16 over S, dQ += dS K. It also writes -lse2 and D of its rows for the other pass. A
//   running CTA takes over units not yet launched (cluster launch control).
// dK/dV pass: a unit is a tile of at most 128 keys and a KV head, or a part of the rows that see it (whose sums a later
//   kernel adds in order). Each CTA has a list of units of about equal time. A step is a block of 64 packed rows:
//   S^T = K Q^T, dP^T = V dO^T, P^T and dS^T as bf16 over S^T, dV += P^T dO, dK += dS^T Q. Query heads of the group and the
//   segments that share keys are thus summed in a fixed order. The next unit's K, V and first rows come while this one's
//   steps run, its first scores while this one's sums are written.
//
// Masks are needed at ends only: where a segment's keys (dQ) or rows (dK/dV) end inside a step, the weights past the end
// become 0 and the operand rows there zeros, because what lies behind may be anything; and keys of a tile that the
// step's segment does not see (key ranges that overlap) get weights 0. Rows of such a segment that are not finite get zeros
// as operands and NaN as the weights of the keys that see them.
//
// A step is bound by its chain S -> softmax -> accumulation -> S more than by its MMAs, so S, dP and the accumulating
// MMAs are issued by a warp each; P and dS share S's columns, so dP's buffer is free as soon as it is read; waits and
// roles are uniform per warp. A softmax warp owns 32 TMEM lanes (rows) and one 32-column half of a step; its bf16
// results go to the first 16 columns of its own half of S (dS of the dK/dV pass to the other 16).
// Warp roles: eight softmax and epilogue warps (or two groups of eight), then the TMA producer, S (and TMEM allocation),
// the accumulating MMAs, dP (converged warps, one elected lane issues). Every wait is bounded; a wait that runs out records
// an error and all roles leave their loops, the MMA warps wait for their MMAs, the producer for its copies, and tensor
// memory is released.
//
// Measured: 32768 rows over 8 x 2560 states of 16 query and 2 KV heads of 128 dims 1357 to 1387 us, by themselves dQ 586 and
// dK/dV 781 (1735 to 1770 TFLOP/s over the seven products made, as much as a library product sustains). A step of 64 rows
// of the dK/dV pass lasts 1290 cycles, of which the tensor cores' pipe is busy 93% (MMAs 1056 cycles, or their operands' way
// from shared memory); one of 64 keys of the dQ pass 1005, 87%. 8 pages of 25 segments over 1601 states 131 us (63 and 65,
// sums 8); 9 pages of 16 heads of 64 dims 147 (64 and 84). The short calls lose an item's start and end (3 to 4 us) and the launches.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "cross.cuh"
#include "tc.cuh"

namespace {

constexpr int kBlk = PADOC_CROSS_BLOCK;

__device__ __forceinline__ bool wait_or_abort(uint32_t bar, uint32_t parity, int *err, int site, volatile int *abort_flag)
{
    if (*abort_flag) return false;
    if (mbar_wait_bounded(bar, parity, err, site)) return true;
    *abort_flag = 1;
    return false;
}

// TMEM column of k-slice k (16 values) of a 64-wide bf16 operand written by the softmax warps: column half c packs its
// 32 values into the first 16 columns of its own half.
__host__ __device__ constexpr uint32_t slice_col(int k) { return (uint32_t)((k / 2) * 32 + (k % 2) * 8); }

__device__ __forceinline__ void store_row_bf16(__nv_bfloat16 *dst, const float (&o)[16], float mul)
{
#pragma unroll
    for (int i = 0; i < 16; i += 8) {
        uint4 w;
        w.x = pack_bf16x2(o[i] * mul, o[i + 1] * mul);
        w.y = pack_bf16x2(o[i + 2] * mul, o[i + 3] * mul);
        w.z = pack_bf16x2(o[i + 4] * mul, o[i + 5] * mul);
        w.w = pack_bf16x2(o[i + 6] * mul, o[i + 7] * mul);
        *reinterpret_cast<uint4 *>(dst + i) = w;
    }
}

__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[32]) { tmem_ld32(taddr, r); }
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[16]) { tmem_ld16(taddr, r); }

// A thread's 16-byte pieces of a row of D / 2 dims, its column half of the row (panels of 64 dims, 128-byte swizzle),
// and the same as the A operand in tensor memory.
template <int D>
struct HalfRow {
    static constexpr int kPieces = D / 16;
    static __device__ __forceinline__ int offset(int ch, int row, int i, int panel_bytes)
    {
        if constexpr (D == 128) return ch * panel_bytes + row * 128 + ((i ^ (row & 7)) * 16);
        return row * 128 + (((4 * ch + i) ^ (row & 7)) * 16);
    }
    static __device__ __forceinline__ void to_tmem(uint32_t taddr, const uint8_t *tile, int ch, int row, int panel_bytes)
    {
        uint32_t w[4 * kPieces];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint4 x = *reinterpret_cast<const uint4 *>(tile + offset(ch, row, i, panel_bytes));
            w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
        }
        if constexpr (D == 128) tmem_st32(taddr + 32 * ch, w);
        else tmem_st16(taddr + 16 * ch, w);
    }
};

// ================================================================================================
// dK/dV pass
// ================================================================================================
namespace dkv {
constexpr int kKT = PADOC_CROSS_KEY_TILE;   // 128 keys: the M of every MMA
constexpr int kMaxStages = 8;
constexpr int kKPanel = kKT * 128;           // [128 rows][64 bf16]
constexpr int kQPanel = kBlk * 128;          // [64 rows][64 bf16]
// -lse2[64], then -D of each row as eight bf16, the first three of which add up to it. They are a B operand: a last product
// of 16 (with ones for these three, zeros for the rest) subtracts D from dP. Read as fp32 like -lse2, each value by a whole
// warp, D kept shared memory busy for 256 cycles a step more (1439 us against 1349 for 32768 rows over 8 x 2560 states).
constexpr int kAuxBytes = kBlk * 4 + kBlk * 16;
constexpr int kSelBytes = 2 * kKT * 16;      // ... that product's A: 128 rows of three ones, 128 of zeros
// With 64 dims two groups of eight softmax warps take the steps in turn: one group's work on a step lasts longer than its
// 16 MMAs (98 us against 110 for 9 pages of 16 heads, both before items came in lists). With 128 dims, 24 MMAs, one group
// with all registers is faster (937 us against 983 for 32768 rows over 8 x 2560 states, before the lists too).
// Tensor memory: S buffers, dP buffers, V as an A operand (128 dims; with 64 it is read from shared memory), dV and dK.
template <int D>
struct Cols {
    static constexpr int kGroups = D == 64 ? 2 : 1, kSoft = 8 * kGroups, kThreads = 32 * (kSoft + 4);
    static constexpr int kBuffers = 2 * kGroups, kDPs = kGroups;
    static constexpr uint32_t kDP = 64 * kBuffers, kV = 192, kAcc = D == 64 ? 384 : 256;
    static_assert(kAcc + 2 * D <= 512 && kDP + 64 * kDPs <= (D == 64 ? kAcc : kV), "");
    // Steps on their way: a step of 64 dims copies 16 KB in the time of 16 MMAs, and with four stages it waited for them
    // (128 us against 98 with ten, before items came in lists; now eight, and K and V of the next item beside them: 82).
    static constexpr int kStages = D == 64 ? 8 : 4, kKBufs = D == 64 ? 2 : 1;   // K and V of the unit, and of the next
    static_assert(kStages <= kMaxStages && kStages % kGroups == 0, "a stage belongs to one group");
    static constexpr int kShare = 2 * D / (kSoft / 4);                          // columns of dV | dK a softmax thread writes
};
struct Unit {   // steps < 0: no more units
    int32_t k0, nk, cover, g;
    int32_t first, steps, slot, pad;
};
enum {
    B_UFULL = 0,                      // [unit parity]
    B_UEMPTY = 2,                     // [unit parity], an arrival per reading warp
    B_KFULL = 4,                      // [K buffer]
    B_KFREE = 6,                      // [K buffer]: the unit's last S is done
    B_VFULL = 8,                      // [V buffer]
    B_VFREE = 10,                     // [V buffer]: V is in tensor memory (an arrival per softmax warp) or its last dP is done
    B_VT = 12,                        // V is in tensor memory (an arrival per softmax warp)
    B_DPLAST = 13,                    // the unit's last dP is done
    B_ACCFULL = 14,                   // the unit's dV and dK are complete
    B_ACCFREE = 15,                   // ... and read (an arrival per softmax warp)
    B_FINAL = 16,                     // [issuing warp]
    B_SFULL = 19,                     // [S buffer]
    B_PFULL = 23,                     // [S buffer], an arrival per softmax warp of a group
    B_ACC = 27,                       // [S buffer]: the step's accumulating MMAs are done
    B_DPFREE = 31,                    // [dP buffer]: dP is read (an arrival per softmax warp of a group)
    B_QFULL = 33,                     // [stage]
    B_QEMPTY = 33 + kMaxStages,       // [stage]
    B_COUNT = 33 + 2 * kMaxStages
};
template <int D>
constexpr size_t smem_bytes()
{
    return 1024 + 2 * (size_t)Cols<D>::kKBufs * (D / 64) * kKPanel + 2 * (size_t)Cols<D>::kStages * (D / 64) * kQPanel +
           (size_t)Cols<D>::kStages * kAuxBytes + kSelBytes + 2 * sizeof(Unit) + B_COUNT * 8 + 16;
}
static_assert(smem_bytes<64>() <= 232448 && smem_bytes<128>() <= 232448, "shared memory per CTA");
}  // namespace dkv

// The blocks of rows that a key tile's steps are, one after the other.
struct Steps {
    const padoc_cross_cover *covers;
    padoc_cross_cover c;
    int i, b;
    __device__ __forceinline__ Steps(const padoc_cross_args &a, int cover, int first) : covers(a.covers + cover), i(0), b(first)
    {
        c = covers[0];
        while (b >= c.nsub) {
            b -= c.nsub;
            c = covers[++i];
        }
    }
    __device__ __forceinline__ void next(bool more)
    {
        if (++b == c.nsub && more) {
            b = 0;
            c = covers[++i];
        }
    }
    __device__ __forceinline__ int tokens(const padoc_cross_args &a) const { return min(a.block_tokens, c.ntok - b * a.block_tokens); }
};

// Key rows that no row sees: gap tiles of the plan, then those it does not reach.
template <int D>
__device__ __forceinline__ void zero_gaps(const padoc_cross_args &a, int first, int stride, int thread, int threads)
{
    const int gaps = a.num_tiles - a.gap_tile;
    for (int n = first; n < (gaps + a.tail_tiles) * a.hkv; n += stride) {
        const int i = n / a.hkv, g = n % a.hkv;
        int k0 = a.tail_begin + (i - gaps) * PADOC_CROSS_KEY_TILE, nk = (int)min((int64_t)PADOC_CROSS_KEY_TILE, a.key_rows - k0);
        if (i < gaps) {
            k0 = a.tiles[a.gap_tile + i].k0;
            nk = a.tiles[a.gap_tile + i].nk;
        }
        for (int t = thread; t < nk * (D / 8); t += threads) {
            const size_t r = (size_t)(k0 + t / (D / 8));
            const int c = g * D + t % (D / 8) * 8;
            *reinterpret_cast<uint4 *>((__nv_bfloat16 *)a.dk + r * a.dk_stride + c) = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4 *>((__nv_bfloat16 *)a.dv + r * a.dv_stride + c) = make_uint4(0, 0, 0, 0);
        }
    }
}
template <int D>
__global__ void __launch_bounds__(256) cross_zero_kernel(const padoc_cross_args a)
{
    zero_gaps<D>(a, blockIdx.x, gridDim.x, threadIdx.x, 256);
}

template <int D>
__global__ void __launch_bounds__(dkv::Cols<D>::kThreads, 1)
cross_dkv_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap gmap,
                 const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const padoc_cross_args a)
{
    using namespace dkv;
    using T = Cols<D>;
    constexpr int kPanels = D / 64, kKTile = kPanels * kKPanel, kQTile = kPanels * kQPanel, kBuf = T::kBuffers, kDPs = T::kDPs,
                  kStages = T::kStages, kKBufs = T::kKBufs, kGroups = T::kGroups, kSoft = T::kSoft;
    constexpr uint32_t kColS = 0, kColDP = T::kDP, kColV = T::kV, kColAcc = T::kAcc;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sk = smem;                        // [buffer]
    uint8_t *sv = sk + kKBufs * kKTile;        // [buffer]
    uint8_t *sq = sv + kKBufs * kKTile;        // [stage] Q step tiles
    uint8_t *sg = sq + kStages * kQTile;       // [stage] dO step tiles
    uint8_t *aux = sg + kStages * kQTile;      // [stage] -lse2, -D
    uint8_t *sel = aux + kStages * kAuxBytes;
    Unit *units = (Unit *)(sel + kSelBytes);   // [2]
    uint64_t *bars = (uint64_t *)(units + 2);
    uint32_t *tmem_slot = (uint32_t *)(bars + B_COUNT);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // (a value the compiler knows to be warp-uniform)
    const int used = a.block_tokens * a.group;   // rows of a block that its copies write
    auto bar = [&](int i) { return smem_u32(&bars[i]); };

    if (tid < B_COUNT) {
        const int i = tid;
        int n = 1;
        if (i == B_UEMPTY || i == B_UEMPTY + 1) n = kSoft + 3;
        if (i == B_VFREE || i == B_VFREE + 1) n = D == 128 ? 8 : 1;
        if (i == B_VT || (i >= B_PFULL && i < B_ACC) || i == B_DPFREE || i == B_DPFREE + 1) n = 8;
        if (i == B_ACCFREE) n = kSoft;
        if (i >= B_SFULL && i < B_PFULL) n = 2;
        mbar_init(bar(i), n);
        if (i == 0) *abort_flag = 0;
        fence_barrier_init();
    }
    if (used < kBlk) {   // the others are zeros throughout: they are summed over
        for (int i = tid; i < 2 * kStages * kPanels * (kBlk - used) * 8; i += T::kThreads) {
            const int r = i / 8 % (kBlk - used) + used, b = i / 8 / (kBlk - used);
            *reinterpret_cast<uint4 *>(sq + b * kQPanel + r * 128 + i % 8 * 16) = make_uint4(0, 0, 0, 0);
        }
    }
    if (tid < 2 * kKT) reinterpret_cast<uint4 *>(sel)[tid] = tid < kKT ? make_uint4(0x3f803f80u, 0x3f80u, 0, 0) : make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    if (warp == kSoft + 1) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    auto wait_w = [&](int b, uint32_t parity, int site) {
        return mbar_wait_warp(bar(b), parity, a.err, site, abort_flag);
    };
    // the n-th unit, as every lane of a reading warp sees it
    auto read_unit = [&](int n, Unit &u, int site) {
        if (!wait_w(B_UFULL + (n & 1), (n >> 1) & 1, site)) return false;
        const Unit v = units[n & 1];
        u.k0 = __shfl_sync(0xffffffffu, v.k0, 0);
        u.nk = __shfl_sync(0xffffffffu, v.nk, 0);
        u.cover = __shfl_sync(0xffffffffu, v.cover, 0);
        u.g = __shfl_sync(0xffffffffu, v.g, 0);
        u.first = __shfl_sync(0xffffffffu, v.first, 0);
        u.steps = __shfl_sync(0xffffffffu, v.steps, 0);
        u.slot = __shfl_sync(0xffffffffu, v.slot, 0);
        __syncwarp();   // (every lane's read has returned before the slot may be written again)
        mbar_arrive_warp(bar(B_UEMPTY + (n & 1)));
        return true;
    };

    if (warp == kSoft) {
        // ---------------------------------------------------------------- TMA producer
        if (lane == 0) {
            tma_prefetch_desc(&qmap);
            tma_prefetch_desc(&gmap);
            tma_prefetch_desc(&kmap);
            tma_prefetch_desc(&vmap);
            auto wait = [&](int b, uint32_t parity, int site) {
                return wait_or_abort(bar(b), parity, a.err, site, abort_flag);
            };
            pdl_wait_prerequisite();   // -lse2 and D are the dQ pass's
            int x = a.dkv_ctas[blockIdx.x];
            const int xe = a.dkv_ctas[blockIdx.x + 1];
            int issued = 0, nk = 0;    // steps, K and V tiles issued so far
            bool ok = true;
            for (int n = 0; ok; ++n, ++x) {
                if (n >= 2 && !(ok = wait(B_UEMPTY + (n & 1), ((n >> 1) - 1) & 1, 149))) break;
                Unit un = {0, 0, 0, 0, 0, -1, 0, 0};
                if (x < xe) {
                    const padoc_cross_dkv w = a.dkv[x];
                    un = {w.k0, w.nk, w.cover, w.g, w.first, w.steps, w.slot, 0};
                }
                units[n & 1] = un;
                mbar_arrive(bar(B_UFULL + (n & 1)));
                if (un.steps < 0) break;
                Steps st(a, un.cover, un.first);
                for (int j = 0; j < un.steps; ++j) {
                    const int s = issued % kStages;
                    if (issued >= kStages && !(ok = wait(B_QEMPTY + s, (issued / kStages - 1) & 1, 150))) break;
                    const int tok = st.c.tok + st.b * a.block_tokens;
                    const size_t at = ((size_t)un.g * a.num_subs + st.c.sub + st.b) * kBlk;
                    const uint32_t fb = bar(B_QFULL + s);
                    const uint32_t qb = smem_u32(sq + s * kQTile), gb = smem_u32(sg + s * kQTile);
                    const uint32_t ab = smem_u32(aux + s * kAuxBytes);
                    mbar_arrive_expect_tx(fb, 2 * kPanels * used * 128 + kAuxBytes);
#pragma unroll
                    for (int p = 0; p < kPanels; ++p) {
                        tma_load_3d(qb + p * kQPanel, &qmap, 64 * p, un.g * a.group, tok, fb);
                        tma_load_3d(gb + p * kQPanel, &gmap, 64 * p, un.g * a.group, tok, fb);
                    }
                    bulk_load(ab, a.neg_lse2 + at, kBlk * 4, fb);
                    bulk_load(ab + kBlk * 4, a.dsum + 4 * at, kBlk * 16, fb);
                    ++issued;
                    st.next(j + 1 < un.steps);
                    if (j == 0) {   // (K's and V's places may be free later than the first step's)
                        const int kb = n % kKBufs;
                        if (n >= kKBufs && !(ok = wait(B_KFREE + kb, (n / kKBufs - 1) & 1, 147) && wait(B_VFREE + kb, (n / kKBufs - 1) & 1, 148)))
                            break;
                        mbar_arrive_expect_tx(bar(B_KFULL + kb), kKTile);
                        mbar_arrive_expect_tx(bar(B_VFULL + kb), kKTile);
#pragma unroll
                        for (int p = 0; p < kPanels; ++p) {
                            tma_load_2d(smem_u32(sk + kb * kKTile) + p * kKPanel, &kmap, un.g * D + 64 * p, un.k0, bar(B_KFULL + kb));
                            tma_load_2d(smem_u32(sv + kb * kKTile) + p * kKPanel, &vmap, un.g * D + 64 * p, un.k0, bar(B_VFULL + kb));
                        }
                        ++nk;
                    }
                }
            }
            // copies still in flight must land before the CTA's shared memory is released
            for (int i = max(nk - kKBufs, 0); i < nk; ++i) {
                mbar_wait_bounded(bar(B_KFULL + i % kKBufs), (i / kKBufs) & 1, a.err, 151);
                mbar_wait_bounded(bar(B_VFULL + i % kKBufs), (i / kKBufs) & 1, a.err, 151);
            }
            for (int u = max(issued - kStages, 0); u < issued; ++u)
                mbar_wait_bounded(bar(B_QFULL + u % kStages), (u / kStages) & 1, a.err, 152);
        }
    } else if (warp > kSoft) {
        // ---------------------------------------------------------------- MMA issuers (whole warps)
        // the first S, the third dP, the second the accumulating MMAs; u counts the steps of all units
        constexpr uint32_t idS = umma_idesc_bf16(128, kBlk, false), idAcc = umma_idesc_bf16(128, D, true);
        int u = 0;
        bool ok = true;
        Unit un;
        for (int n = 0; ok && (ok = read_unit(n, un, 159)) && un.steps >= 0; ++n) {
            const int kb = n % kKBufs;
            const uint32_t kph = n / kKBufs & 1;
            if (warp == kSoft + 1) {
                const uint64_t dK = umma_desc_sw128(smem_u32(sk + kb * kKTile), 16, 1024);
                ok = wait_w(B_KFULL + kb, kph, 160);
                for (int j = 0; ok && j < un.steps; ++j, ++u) {
                    const int s = u % kStages, b = u % kBuf;
                    ok = wait_w(B_QFULL + s, (u / kStages) & 1, 161) && (u < kBuf || wait_w(B_ACC + b, (u / kBuf - 1) & 1, 163));
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t dq = umma_desc_sw128(smem_u32(sq + s * kQTile), 16, 1024);
                    if constexpr (D == 128) umma_bf16_ss_k128_warp<1, kKPanel, kQPanel>(tmem + kColS + 64 * b, dK, dq, idS);
                    else umma_bf16_ss_k64_warp(tmem + kColS + 64 * b, dK, dq, idS);
                    umma_commit_warp(bar(B_SFULL + b));
                }
                umma_commit_warp(bar(B_KFREE + kb));
            } else if (warp == kSoft + 3) {
                const uint64_t dV = umma_desc_sw128(smem_u32(sv + kb * kKTile), 16, 1024), ds = umma_desc_plain(smem_u32(sel), kKT * 16, 128);
                ok = D == 64 ? wait_w(B_VFULL + kb, kph, 166) : wait_w(B_VT, n & 1, 166);
                for (int j = 0; ok && j < un.steps; ++j, ++u) {
                    const int s = u % kStages;
                    ok = wait_w(B_QFULL + s, (u / kStages) & 1, 167) && (u < kDPs || wait_w(B_DPFREE + u % kDPs, (u / kDPs - 1) & 1, 165));
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t dg = umma_desc_sw128(smem_u32(sg + s * kQTile), 16, 1024);
                    if constexpr (D == 128) umma_bf16_ts_k128_warp<kQPanel>(tmem + kColDP + 64 * (u % kDPs), tmem + kColV, dg, idS);
                    else umma_bf16_ss_k64_warp(tmem + kColDP + 64 * (u % kDPs), dV, dg, idS);
                    // (the eight further values that the zeros meet are the first again)
                    const uint64_t db = umma_desc_plain(smem_u32(aux + s * kAuxBytes + kBlk * 4), 0, 128);
                    umma_bf16_ss_k16_add_warp(tmem + kColDP + 64 * (u % kDPs), ds, db, idS);
                    umma_commit_warp(bar(B_SFULL + u % kBuf));
                }
                if (D == 64) umma_commit_warp(bar(B_VFREE + kb));
                else umma_commit_warp(bar(B_DPLAST));
            } else {
                for (int j = 0; ok && j < un.steps; ++j, ++u) {
                    const int s = u % kStages, b = u % kBuf;
                    // (the sums of the unit before are read before this one's first products overwrite them)
                    ok = wait_w(B_PFULL + b, (u / kBuf) & 1, 162) && (j > 0 || n == 0 || wait_w(B_ACCFREE, (n - 1) & 1, 158));
                    if (!ok) break;
                    tc_fence_after();
                    // the step's Q and dO as MN-major B operands (N = head dim, K = the 64 rows)
                    const uint64_t gmn = umma_desc_sw128(smem_u32(sg + s * kQTile), kQPanel, 1024);
                    const uint64_t qmn = umma_desc_sw128(smem_u32(sq + s * kQTile), kQPanel, 1024);
                    umma_bf16_ts_k64_mn_warp<1, slice_col(1), slice_col(2), slice_col(3)>(tmem + kColAcc, tmem + kColS + 64 * b, gmn, idAcc, j > 0);
                    umma_bf16_ts_k64_mn_warp<1, slice_col(1), slice_col(2), slice_col(3)>(tmem + kColAcc + D, tmem + kColS + 64 * b + 16, qmn, idAcc, j > 0);
                    umma_commit_warp(bar(B_ACC + b));
                    umma_commit_warp(bar(B_QEMPTY + s));
                }
                umma_commit_warp(bar(B_ACCFULL));
            }
        }
        // every MMA issued above must complete before tensor memory is released
        umma_commit_warp(bar(B_FINAL + warp - kSoft - 1));
        mbar_wait_bounded(bar(B_FINAL + warp - kSoft - 1), 0, a.err, 164);
    } else {
        // ---------------------------------------------------------------- softmax + epilogue
        const int lq = warp & 3, ch = warp >> 2 & 1, grp = warp >> 3;   // TMEM lane quarter, column half, group
        const int row = lq * 32 + lane;
        const uint32_t lanes = (uint32_t)(lq * 32) << 16;
        const uint64_t c2 = f2_pack(a.scale_log2, a.scale_log2);
        zero_gaps<D>(a, blockIdx.x, gridDim.x, tid, 32 * kSoft);   // (while the first unit is on its way)
        int u0 = 0;             // steps of the units before
        Unit un, last = {};
        bool ok = true;
        for (int n = 0; ok && (ok = read_unit(n, un, 157)); ++n) {
            if (D == 128 && un.steps >= 0) {   // V's rows into tensor memory, half of the dims a thread
                if (!(ok = wait_w(B_VFULL, n & 1, 173) && (n == 0 || wait_w(B_DPLAST, (n - 1) & 1, 174)))) break;
                tc_fence_after();
                HalfRow<D>::to_tmem(tmem + lanes + kColV, sv, ch, row, kKPanel);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                mbar_arrive_warp(bar(B_VT));
                mbar_arrive_warp(bar(B_VFREE));
            }
            // The unit before's sums, kShare columns of dV | dK a thread: dV, and dK times scale, or both in fp32 as parts.
            if (n > 0) {
                if (!(ok = wait_w(B_ACCFULL, (n - 1) & 1, 172))) break;
                tc_fence_after();
                const int c0 = T::kShare * (warp >> 2);
#pragma unroll 1
                for (int c = 0; c < T::kShare; c += 16) {
                    uint32_t o[16];
                    tmem_ld16(tmem + lanes + kColAcc + c0 + c, o);
                    tmem_ld_wait();
                    if (c + 16 == T::kShare) {
                        tc_fence_before();
                        __syncwarp();
                        mbar_arrive_warp(bar(B_ACCFREE));
                    }
                    float x[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(o[i]);
                    const int col = c0 + c;
                    if (row < last.nk) {
                        if (last.slot >= 0) {
                            float *dst = a.part_dkv + ((size_t)last.slot * kKT + row) * (2 * D) + col;
                            st_global_v8(dst, x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]);
                            st_global_v8(dst + 8, x[8], x[9], x[10], x[11], x[12], x[13], x[14], x[15]);
                        } else {
                            const bool isk = col >= D;                       // dV first, then dK (times scale)
                            store_row_bf16(isk ? (__nv_bfloat16 *)a.dk + (size_t)(last.k0 + row) * a.dk_stride + last.g * D + (col - D)
                                               : (__nv_bfloat16 *)a.dv + (size_t)(last.k0 + row) * a.dv_stride + last.g * D + col,
                                           x, isk ? a.scale : 1.f);
                        }
                    }
                }
            }
            if (un.steps < 0) break;
            last = un;
            // this group's steps
            const int j0 = kGroups == 2 ? (u0 & 1) ^ grp : 0;
            Steps st(a, un.cover, un.first + (j0 < un.steps ? j0 : 0));
            for (int j = j0; ok && j < un.steps; j += kGroups) {
                const int u = u0 + j, s = u % kStages, sb = u % kBuf;
                const uint32_t b = (uint32_t)sb * 64 + 32 * ch;
                const int rows = __shfl_sync(0xffffffffu, st.tokens(a), 0) * a.group;
                const bool partial = rows < used;
                // keys of the tile that the segment does not see
                const int key = un.k0 + row;
                const bool blind = key < st.c.k0 || key >= st.c.k0 + st.c.nk;
                const bool some_blind = __any_sync(0xffffffffu, st.c.k0 > un.k0 || st.c.k0 + st.c.nk < un.k0 + un.nk);
                if (!(ok = wait_w(B_QFULL + s, (u / kStages) & 1, 171) && wait_w(B_SFULL + sb, (u / kBuf) & 1, 170))) break;
                tc_fence_after();
                for (int i = 1; i <= kGroups; ++i) st.next(j + i < un.steps);
                uint32_t vis = 0xffffffffu;
                if (partial) {
                    // the block's rows past the segment's, which the products below sum over: zeros (S and dP, which
                    // have read them, are done)
                    vis = interval_bits(0, rows, 32 * ch);
                    for (int i = tid & 255; i < (kBlk - rows) * 8 * kPanels; i += 256) {
                        const int r = rows + i / 8 % (kBlk - rows), p = i / 8 / (kBlk - rows), o = p * kQPanel + r * 128 + i % 8 * 16;
                        *reinterpret_cast<uint4 *>(sq + s * kQTile + o) = make_uint4(0, 0, 0, 0);
                        *reinterpret_cast<uint4 *>(sg + s * kQTile + o) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                }
                const float4 *la = reinterpret_cast<const float4 *>(aux + s * kAuxBytes) + 8 * ch;
                constexpr int kCols = kGroups == 2 ? 16 : 32;   // row columns at a time (96 registers a thread with two groups)
                uint32_t pk[16], dk[16];
#pragma unroll
                for (int h = 0; h < 32; h += kCols) {
                    uint32_t sr[kCols], dr[kCols];
                    tmem_ld_cols(tmem + lanes + kColS + b + h, sr);
                    tmem_ld_cols(tmem + lanes + kColDP + 64 * (u % kDPs) + 32 * ch + h, dr);
                    tmem_ld_wait();
                    if (h + kCols == 32) {
                        tc_fence_before();
                        __syncwarp();
                        mbar_arrive_warp(bar(B_DPFREE + u % kDPs));
                    }
                    // two row columns per packed instruction: P = exp2(S c - lse2), dS = P (dP - D), where dP has lost D
                    // already, both rounded to the MMAs' operand type (half a step, 2^-9 of a value on average)
                    auto column_pairs = [&](auto masked) {
#pragma unroll
                        for (int i4 = 0; i4 < kCols / 4; ++i4) {
                            const float4 l4 = la[h / 4 + i4];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const int i = 4 * i4 + 2 * k;
                                float x0, x1;
                                f2_unpack(f2_fma(f2_pack(__uint_as_float(sr[i]), __uint_as_float(sr[i + 1])), c2,
                                                 k ? f2_pack(l4.z, l4.w) : f2_pack(l4.x, l4.y)), x0, x1);
                                float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
                                float d0, d1;
                                f2_unpack(f2_mul(f2_pack(p0, p1), f2_pack(__uint_as_float(dr[i]), __uint_as_float(dr[i + 1]))), d0, d1);
                                if (decltype(masked)::value) {
                                    p0 = (vis >> (h + i)) & 1u ? p0 : 0.f;
                                    p1 = (vis >> (h + i + 1)) & 1u ? p1 : 0.f;
                                    d0 = (vis >> (h + i)) & 1u ? d0 : 0.f;
                                    d1 = (vis >> (h + i + 1)) & 1u ? d1 : 0.f;
                                }
                                pk[(h + i) >> 1] = pack_bf16x2(p0, p1);
                                dk[(h + i) >> 1] = pack_bf16x2(d0, d1);
                            }
                        }
                    };
                    if (partial) column_pairs(std::true_type{}); else column_pairs(std::false_type{});
                }
                if (some_blind) {
                    // Rows whose q or dO is not finite: 0 x NaN would reach the sums of the keys that do not see them, so their
                    // operand rows become zeros and the weights of the keys that see them NaN. Such a row's lse or D is
                    // not finite; where nothing is left of its scores (lse = -inf, finite D) its weights stay zeros.
                    const int r = 32 * ch + lane;
                    const uint8_t *stats = aux + s * kAuxBytes;
                    const float l = reinterpret_cast<const float *>(stats)[r];
                    const float d = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(stats + kBlk * 4 + r * 16) << 16);
                    const uint32_t odd = __ballot_sync(0xffffffffu, r < rows && !(isfinite(l) && isfinite(d)));
                    if (odd) {
                        const uint32_t nan = __ballot_sync(0xffffffffu, r < rows && (isnan(l) || !isfinite(d)));
                        for (int i = 0; i < 32; ++i)   // (the four warps of a column half write the same zeros)
                            if (((odd >> i) & 1u) && lane < 16 * kPanels)
                                *reinterpret_cast<uint4 *>((lane < 8 * kPanels ? sq : sg) + s * kQTile + (lane >> 3) % kPanels * kQPanel +
                                                           (32 * ch + i) * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t w = (((nan >> (2 * i)) & 1u) ? 0x7fffu : 0u) | (((nan >> (2 * i)) & 2u) ? 0x7fff0000u : 0u);
                            pk[i] |= w;
                            dk[i] |= w;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        pk[i] = blind ? 0u : pk[i];
                        dk[i] = blind ? 0u : dk[i];
                    }
                }
                tmem_st16(tmem + lanes + kColS + b, pk);
                tmem_st16(tmem + lanes + kColS + b + 16, dk);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                mbar_arrive_warp(bar(B_PFULL + sb));
            }
            u0 += un.steps;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kSoft + 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Parts' sums: four columns of a key row's dV | dK a thread, in the order of the parts. With W = 8 a warp adds an eighth of
// the parts and the warps' sums follow in their order: a tile in 76 parts 26 -> 4 us, while tiles in two or three (104 of
// them, 128 dims) took 26 us that way and take 8 with one thread for all parts.
template <int D, int W>
__global__ void __launch_bounds__(256) cross_dkv_sum_kernel(const padoc_cross_args a)
{
    constexpr int kThreadsOut = 256 / W, kRow = 2 * D / 4;   // sums of a CTA, of a row
    __shared__ float4 sums[W][kThreadsOut];
    const int w = threadIdx.x / kThreadsOut, at = blockIdx.x * kThreadsOut + threadIdx.x % kThreadsOut;
    const padoc_cross_dkv_sum t = a.dkv_sums[at / (dkv::kKT * kRow)];
    const int r = at / kRow % dkv::kKT, col = at % kRow * 4;
    pdl_wait_prerequisite();
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < t.nk) {
        const float *src = a.part_dkv + ((size_t)t.slot * dkv::kKT + r) * (2 * D) + col;
#pragma unroll 4
        for (int p = w; p < t.parts; p += W) {
            const float4 y = *reinterpret_cast<const float4 *>(src + (size_t)p * dkv::kKT * (2 * D));
            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
        }
    }
    if constexpr (W > 1) {
        sums[w][threadIdx.x % kThreadsOut] = x;
        __syncthreads();
        if (w) return;
#pragma unroll
        for (int i = 1; i < W; ++i) {
            const float4 y = sums[i][threadIdx.x];
            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
        }
    }
    if (r >= t.nk) return;
    const bool isk = col >= D;
    const float mul = isk ? a.scale : 1.f;
    __nv_bfloat16 *dst = isk ? (__nv_bfloat16 *)a.dk + (size_t)(t.k0 + r) * a.dk_stride + t.g * D + (col - D)
                             : (__nv_bfloat16 *)a.dv + (size_t)(t.k0 + r) * a.dv_stride + t.g * D + col;
    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16x2(x.x * mul, x.y * mul), pack_bf16x2(x.z * mul, x.w * mul));
}

// ================================================================================================
// dQ pass
// ================================================================================================
namespace dqp {
constexpr int kQT = PADOC_CROSS_DQ_BLOCKS * kBlk;   // 128 rows: the M of every MMA
constexpr int kW = PADOC_CROSS_DQ_STEP;             // 64 keys per step
constexpr int kThreads = 384;
constexpr int kMaxStages = 10;
constexpr int kQPanel = kQT * 128;           // [128 rows][64 bf16]
constexpr int kKPanel = kW * 128;            // [64 rows][64 bf16]
// Tensor memory columns: Q as an A operand, three S buffers (a step's dS takes its S's place), two dP, dQ.
constexpr int kSlots = 3;
constexpr uint32_t kColQ = 0, kColS = 64, kColDP = 256, kColDQ = 384;
template <int D>
constexpr int stages() { return D == 64 ? 10 : 4; }   // (with 64 dims 81 -> 65 us, as in the dK/dV pass)
enum {
    B_QROWS = 0,                   // the unit's Q has landed
    B_GROWS = 1,                   // its dO and O have landed
    B_QT = 2,                      // its Q is in tensor memory (an arrival per softmax warp)
    B_D = 3,                       // its rows' halves of D are in shared memory (an arrival per softmax warp)
    B_DREAD = 4,                   // ... and have been read, as dO and O (an arrival per softmax warp)
    B_QFREE = 5,                   // Q's place is free for the next unit's (an arrival per softmax warp)
    B_GFREE = 6,                   // the unit's last dP is done
    B_DQFULL = 7,                  // the unit's dQ is complete
    B_DQFREE = 8,                  // ... and read (an arrival per softmax warp)
    B_NEXT = 9,                    // the launch control's answer
    B_UFULL = 10,                  // [unit parity]
    B_UEMPTY = 12,                 // [unit parity], an arrival per reading warp
    B_KFULL = 14,                  // [stage]
    B_KEMPTY = 14 + kMaxStages,       // [stage]
    B_SFULL = 14 + 2 * kMaxStages,    // [slot]: S and dP (an arrival each)
    B_PFULL = 17 + 2 * kMaxStages,    // [slot]: dS (an arrival per softmax warp)
    B_ACC = 20 + 2 * kMaxStages,      // [slot]: the accumulating MMAs that read it are done
    B_DPFREE = 23 + 2 * kMaxStages,   // [step parity]: dP is read (an arrival per softmax warp)
    B_FINAL = 25 + 2 * kMaxStages,    // [issuing warp]
    B_COUNT = 28 + 2 * kMaxStages
};
struct Unit {   // steps < 0: no more units
    int32_t tok, ntok, k0, nk;
    int32_t g, slot, sub, steps;
};
constexpr int kReaders = 11;       // softmax and issuing warps
template <int D>
constexpr size_t smem_bytes()
{
    return 1024 + 3 * (size_t)(D / 64) * kQPanel + 2 * (size_t)stages<D>() * (D / 64) * kKPanel + 2 * sizeof(Unit) + 16 +
           B_COUNT * 8 + 32 + 2 * kQT * 4;
}
static_assert(smem_bytes<128>() <= 232448 && smem_bytes<64>() <= 232448, "shared memory per CTA");
}  // namespace dqp

template <int D>
__global__ void __launch_bounds__(dqp::kThreads, 1)
cross_dq_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap gmap,
                const __grid_constant__ CUtensorMap omap, const __grid_constant__ CUtensorMap kmap,
                const __grid_constant__ CUtensorMap vmap, const padoc_cross_args a)
{
    using namespace dqp;
    constexpr int kPanels = D / 64, kQTile = kPanels * kQPanel, kKTile = kPanels * kKPanel, kStages = stages<D>();
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sq = smem;                        // Q, dO and O rows; dQ leaves by way of Q's place
    uint8_t *sg = sq + kQTile;
    uint8_t *so = sg + kQTile;
    uint8_t *sk = so + kQTile;                 // [stage] K step tiles
    uint8_t *sv = sk + kStages * kKTile;       // [stage] V step tiles
    Unit *units = (Unit *)(sv + kStages * kKTile);   // [2]
    uint8_t *answer = (uint8_t *)(units + 2);  // 16 bytes
    uint64_t *bars = (uint64_t *)(answer + 16);
    uint32_t *tmem_slot = (uint32_t *)(bars + B_COUNT);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    float *dsum = (float *)(tmem_slot + 8);    // [2][128]: the two column halves' parts of D

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // (a value the compiler knows to be warp-uniform)
    const int used = a.block_tokens * a.group;
    pdl_launch_dependents();   // the dK/dV pass may take the SMs that run out of work here
    auto bar = [&](int i) { return smem_u32(&bars[i]); };

    if (tid < B_COUNT) {
        const int i = tid;
        const bool soft = i == B_QT || i == B_D || i == B_DREAD || i == B_QFREE || i == B_DQFREE ||
                          (i >= B_PFULL && i < B_PFULL + kSlots) || i == B_DPFREE || i == B_DPFREE + 1;
        mbar_init(bar(i), soft ? 8 : i == B_UEMPTY || i == B_UEMPTY + 1 ? kReaders : i >= B_SFULL && i < B_SFULL + kSlots ? 2 : 1);
        if (i == 0) *abort_flag = 0;
        fence_barrier_init();
    }
    if (used < kBlk) {   // rows that no copy writes (dQ's way out puts what it likes there)
        for (int i = tid; i < 6 * kPanels * (kBlk - used) * 8; i += kThreads) {
            const int r = i / 8 % (kBlk - used) + used, b = i / 8 / (kBlk - used);
            *reinterpret_cast<uint4 *>(sq + b * kBlk * 128 + r * 128 + i % 8 * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
    }
    if (warp == 9) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    auto wait_w = [&](int b, uint32_t parity, int site) {
        return mbar_wait_warp(bar(b), parity, a.err, site, abort_flag);
    };
    // the n-th unit, as every lane of a reading warp sees it
    auto read_unit = [&](int n, Unit &u, int site) {
        if (!wait_w(B_UFULL + (n & 1), (n >> 1) & 1, site)) return false;
        const Unit v = units[n & 1];
        u.tok = __shfl_sync(0xffffffffu, v.tok, 0);
        u.ntok = __shfl_sync(0xffffffffu, v.ntok, 0);
        u.nk = __shfl_sync(0xffffffffu, v.nk, 0);
        u.g = __shfl_sync(0xffffffffu, v.g, 0);
        u.slot = __shfl_sync(0xffffffffu, v.slot, 0);
        u.sub = __shfl_sync(0xffffffffu, v.sub, 0);
        u.steps = __shfl_sync(0xffffffffu, v.steps, 0);
        __syncwarp();   // (every lane's read has returned before the slot may be written again)
        mbar_arrive_warp(bar(B_UEMPTY + (n & 1)));
        return true;
    };

    if (warp == 8) {
        // ---------------------------------------------------------------- TMA producer
        if (lane == 0) {
            auto wait = [&](int b, uint32_t parity, int site) {
                return wait_or_abort(bar(b), parity, a.err, site, abort_flag);
            };
            int x = blockIdx.x, y = 0, xe = 0;   // items: x and, of a list, those up to xe
            if (a.ctas) {
                xe = a.ctas[x + 1];
                x = a.ctas[x];
            }
            int tk = 0, nq = 0, ng = 0;   // K/V tiles, Q tiles, dO and O tiles issued so far
            bool ok = true, more = true, asked = false;
            // asked eight steps before the unit's last copies: early enough for the answer and the next unit's rows, and
            // late enough that no CTA holds a second unit for long while others run out of work
            constexpr int kAsk = 8;
            auto ask = [&]() {
                if (a.ctas) return;
                mbar_arrive_expect_tx(bar(B_NEXT), 16);
                launch_control_ask(smem_u32(answer), bar(B_NEXT));
                asked = true;
            };
            int n = 0;
            for (;; ++n) {
                if (n >= 2 && !wait(B_UEMPTY + (n & 1), ((n >> 1) - 1) & 1, 183)) break;
                Unit u = {0, 0, 0, 0, 0, 0, 0, -1};
                if (more) {
                    const padoc_cross_unit w = a.units[x];
                    u = {w.tok, w.ntok, w.k0, w.nk, w.g, w.slot, w.sub, (w.nk + kW - 1) / kW};
                }
                units[n & 1] = u;
                mbar_arrive(bar(B_UFULL + (n & 1)));
                if (u.steps < 0) break;
                auto rows = [&](uint8_t *dst, const CUtensorMap *map, int b) {
#pragma unroll
                    for (int i = 0; i < 2 * kPanels; ++i)   // [panel][block]
                        tma_load_3d(smem_u32(dst) + (i >> 1) * kQPanel + (i & 1) * kBlk * 128, map, 64 * (i >> 1), u.g * a.group,
                                    u.tok + (i & 1) * a.block_tokens, bar(b));
                };
                // (dO and O cannot be copied before the unit before has used its own: their way from memory starts now)
                if (n > 0)
#pragma unroll
                    for (int i = 0; i < 2 * kPanels; ++i) {
                        tma_prefetch_l2_3d(&gmap, 64 * (i >> 1), u.g * a.group, u.tok + (i & 1) * a.block_tokens);
                        tma_prefetch_l2_3d(&omap, 64 * (i >> 1), u.g * a.group, u.tok + (i & 1) * a.block_tokens);
                    }
                if (n > 0 && !wait(B_QFREE, (n - 1) & 1, 184)) break;
                mbar_arrive_expect_tx(bar(B_QROWS), 2 * kPanels * used * 128);
                rows(sq, &qmap, B_QROWS);
                ++nq;
                for (int j = 0; j < u.steps; ++j, ++tk) {
                    if (j == max(u.steps - kAsk, 0)) ask();
                    const int s = tk % kStages;
                    if (tk >= kStages && !(ok = wait(B_KEMPTY + s, (tk / kStages - 1) & 1, 180))) break;
                    const int row = u.k0 + j * kW;
                    const uint32_t fb = bar(B_KFULL + s);
                    mbar_arrive_expect_tx(fb, 2 * kKTile);
#pragma unroll
                    for (int p = 0; p < kPanels; ++p) {
                        tma_load_2d(smem_u32(sk + s * kKTile) + p * kKPanel, &kmap, u.g * D + 64 * p, row, fb);
                        tma_load_2d(smem_u32(sv + s * kKTile) + p * kKPanel, &vmap, u.g * D + 64 * p, row, fb);
                    }
                    if (j == 0) {   // the first K and V tiles go before dO, whose place is free later
                        if (n > 0 && !(ok = wait(B_DREAD, (n - 1) & 1, 185) && wait(B_GFREE, (n - 1) & 1, 186))) { ++tk; break; }
                        mbar_arrive_expect_tx(bar(B_GROWS), 4 * kPanels * used * 128);
                        rows(sg, &gmap, B_GROWS);
                        rows(so, &omap, B_GROWS);
                        ++ng;
                    }
                }
                if (!ok) break;
                if (a.ctas) {
                    more = ++x < xe;
                    continue;
                }
                if (!wait(B_NEXT, n & 1, 187)) break;
                asked = false;
                more = launch_control_answer(smem_u32(answer), x, y);
                fence_proxy_async_smem();   // the answer is read before the next one may be written
            }
            // copies still in flight must land before the CTA's shared memory is released
            if (asked) mbar_wait_bounded(bar(B_NEXT), n & 1, a.err, 188);
            if (nq) mbar_wait_bounded(bar(B_QROWS), (nq - 1) & 1, a.err, 181);
            if (ng) mbar_wait_bounded(bar(B_GROWS), (ng - 1) & 1, a.err, 181);
            for (int i = max(tk - kStages, 0); i < tk; ++i)
                mbar_wait_bounded(bar(B_KFULL + i % kStages), (i / kStages) & 1, a.err, 182);
        }
    } else if (warp >= 9) {
        // ---------------------------------------------------------------- MMA issuers (whole warps)
        // warp 9 S, warp 11 dP, warp 10 dQ; c counts the steps of all units
        int c = 0, slot = 0;
        uint32_t ph = 0;   // parity of the slot's use
        bool ok = true;
        auto next_step = [&]() {
            ++c;
            if (++slot == kSlots) { slot = 0; ph ^= 1; }
        };
        constexpr uint32_t idS = umma_idesc_bf16(128, kW, false), idAcc = umma_idesc_bf16(128, D, true);
        Unit un;
        for (int n = 0; ok && (ok = read_unit(n, un, 201)) && un.steps >= 0; ++n) {
            if (warp == 9) {
                // S = Q K^T, A from tensor memory
                ok = wait_w(B_QT, n & 1, 190);
                for (int u = 0; ok && u < un.steps; ++u, next_step()) {
                    const int s = c % kStages;
                    ok = wait_w(B_KFULL + s, (c / kStages) & 1, 191) && (c < kSlots || wait_w(B_ACC + slot, ph ^ 1, 193));
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t dk = umma_desc_sw128(smem_u32(sk + s * kKTile), 16, 1024);
                    if constexpr (D == 128) umma_bf16_ts_k128_warp<kKPanel>(tmem + kColS + 64 * slot, tmem + kColQ, dk, idS);
                    else umma_bf16_ts_k64_warp(tmem + kColS + 64 * slot, tmem + kColQ, dk, idS);
                    umma_commit_warp(bar(B_SFULL + slot));
                }
            } else if (warp == 11) {
                // dP = dO V^T, both from shared memory (dO in tensor memory as Q is: 32768 rows over 8 x 2560 states 1548 ->
                // 1521 us, as the product's 48 KB a step take longer than its MMAs, but an item then begins later and there
                // is one dP buffer: 8 pages of 25 segments 137 -> 140 us, 9 pages of 16 heads 156 -> 157.5)
                const uint64_t dg = umma_desc_sw128(smem_u32(sg), 16, 1024);
                ok = wait_w(B_GROWS, n & 1, 197);
                for (int u = 0; ok && u < un.steps; ++u, next_step()) {
                    const int s = c % kStages;
                    ok = wait_w(B_KFULL + s, (c / kStages) & 1, 198) &&
                         (c < 2 || wait_w(B_DPFREE + (c & 1), ((c >> 1) - 1) & 1, 199));
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t dv = umma_desc_sw128(smem_u32(sv + s * kKTile), 16, 1024);
                    if constexpr (D == 128) umma_bf16_ss_k128_warp<1, kQPanel, kKPanel>(tmem + kColDP + 64 * (c & 1), dg, dv, idS);
                    else umma_bf16_ss_k64_warp(tmem + kColDP + 64 * (c & 1), dg, dv, idS);
                    umma_commit_warp(bar(B_SFULL + slot));
                }
                umma_commit_warp(bar(B_GFREE));
            } else {
                for (int u = 0; ok && u < un.steps; ++u, next_step()) {
                    const int s = c % kStages;
                    // (the dQ of the unit before is read before this one's first product overwrites it)
                    ok = wait_w(B_PFULL + slot, ph, 192) && (u > 0 || n == 0 || wait_w(B_DQFREE, (n - 1) & 1, 202));
                    if (!ok) break;
                    tc_fence_after();
                    // the step's K as an MN-major B operand (N = head dim, K = the 64 keys)
                    const uint64_t kmn = umma_desc_sw128(smem_u32(sk + s * kKTile), kKPanel, 1024);
                    umma_bf16_ts_k64_mn_warp<1, slice_col(1), slice_col(2), slice_col(3)>(tmem + kColDQ, tmem + kColS + 64 * slot, kmn,
                                                                                         idAcc, u > 0);
                    umma_commit_warp(bar(B_ACC + slot));
                    umma_commit_warp(bar(B_KEMPTY + s));
                }
                umma_commit_warp(bar(B_DQFULL));
            }
        }
        umma_commit_warp(bar(B_FINAL + warp - 9));
        mbar_wait_bounded(bar(B_FINAL + warp - 9), 0, a.err, 194);
    } else {
        // ---------------------------------------------------------------- softmax + epilogue
        const int lq = warp & 3, ch = warp >> 2;
        const int row = lq * 32 + lane;
        const uint32_t lanes = (uint32_t)(lq * 32) << 16;
        const uint64_t c2 = f2_pack(a.scale_log2, a.scale_log2);
        int c = 0, slot = 0;   // steps of all units
        uint32_t ph = 0;
        Unit un, last = {};
        int64_t last_at = -1;  // where the last unit's row of dQ goes
        bool ok = true;
        for (int n = 0; ok && (ok = read_unit(n, un, 203)); ++n) {
            int token = 0, head = 0;
            const bool in = un.steps >= 0 && cross_row(a, un.tok, un.ntok, row, token, head);
            float nlrow = -INFINITY;
            if (un.steps >= 0) {
                if (in) {
                    const float l = a.lse_in[(size_t)token * a.hq + un.g * a.group + head];
                    nlrow = l == -INFINITY ? -INFINITY : -l * PADOC_LOG2E;
                }
                // Q's row into tensor memory (half of its dims); the S of the unit before that read the last
                // one are done, as their steps are
                if (!(ok = wait_w(B_QROWS, n & 1, 200))) break;
                HalfRow<D>::to_tmem(tmem + lanes + kColQ, sq, ch, row, kQPanel);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                mbar_arrive_warp(bar(B_QT));
            }
            // the unit before's dQ, half of its columns: times scale as bf16 by way of this warp's part of Q's place,
            // so that neighbouring lanes write a row's bytes, or in fp32 as a part
            if (n > 0) {
                if (!(ok = wait_w(B_DQFULL, (n - 1) & 1, 196))) break;
                tc_fence_after();
                constexpr int kCols = D / 2;
                uint32_t o[kCols / 32][32];
#pragma unroll
                for (int i = 0; i < kCols / 32; ++i) tmem_ld32(tmem + lanes + kColDQ + kCols * ch + 32 * i, o[i]);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                mbar_arrive_warp(bar(B_DQFREE));
                if (last.slot >= 0) {
                    const size_t pr = (size_t)last.slot * kQT + row;
                    auto v = [&](int i) { return __uint_as_float(o[i >> 5][i & 31]); };
                    if (last_at >= 0)
#pragma unroll
                        for (int i = 0; i < kCols; i += 8)
                            st_global_v8(a.part + pr * D + kCols * ch + i, v(i), v(i + 1), v(i + 2), v(i + 3), v(i + 4), v(i + 5),
                                         v(i + 6), v(i + 7));
                } else {
#pragma unroll
                    for (int i = 0; i < kCols; i += 8) {
                        auto v = [&](int k) { return __uint_as_float(o[i >> 5][(i & 31) + k]) * a.scale; };
                        *reinterpret_cast<uint4 *>(sq + HalfRow<D>::offset(ch, row, i / 8, kQPanel)) =
                            make_uint4(pack_bf16x2(v(0), v(1)), pack_bf16x2(v(2), v(3)), pack_bf16x2(v(4), v(5)), pack_bf16x2(v(6), v(7)));
                    }
                    __syncwarp();
                    constexpr int kPer = D / 16;   // lanes a row
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        const int r = i * (32 / kPer) + lane / kPer, k = lane % kPer;
                        const int64_t to = __shfl_sync(0xffffffffu, last_at, r);
                        const uint4 w = *reinterpret_cast<const uint4 *>(sq + HalfRow<D>::offset(ch, lq * 32 + r, k, kQPanel));
                        if (to >= 0) *reinterpret_cast<uint4 *>((__nv_bfloat16 *)a.dq + to + kCols * ch + 8 * k) = w;
                    }
                    fence_proxy_async_smem();   // (the next unit's Q is copied over what was read)
                }
                __syncwarp();
            }
            if (un.steps < 0) break;
            mbar_arrive_warp(bar(B_QFREE));
            last = un;
            last_at = in ? (int64_t)token * a.dq_stride + (un.g * a.group + head) * D : -1;
            // the row's statistics: D = dO . O (fp32, the two column halves added through shared memory) and -lse2;
            // rows past the segment's get -lse2 = -inf and D = 0, so that the dK/dV pass adds nothing for them
            if (!(ok = wait_w(B_GROWS, n & 1, 204) && (n == 0 || wait_w(B_DREAD, (n - 1) & 1, 205)))) break;
            uint64_t acc2 = f2_pack(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < HalfRow<D>::kPieces; ++i) {
                const uint4 x = *reinterpret_cast<const uint4 *>(sg + HalfRow<D>::offset(ch, row, i, kQPanel));
                const uint4 w = *reinterpret_cast<const uint4 *>(so + HalfRow<D>::offset(ch, row, i, kQPanel));
                const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc2 = f2_fma(f2_pack(__uint_as_float(xs[j] << 16), __uint_as_float(xs[j] & 0xffff0000u)),
                                  f2_pack(__uint_as_float(ws[j] << 16), __uint_as_float(ws[j] & 0xffff0000u)), acc2);
            }
            float lo, hi;
            f2_unpack(acc2, lo, hi);
            dsum[ch * kQT + row] = lo + hi;
            __syncwarp();
            mbar_arrive_warp(bar(B_D));
            if (!(ok = wait_w(B_D, n & 1, 206))) break;
            const float drow = in ? dsum[row] + dsum[kQT + row] : 0.f;
            __syncwarp();
            mbar_arrive_warp(bar(B_DREAD));
            if (ch == 0 && un.sub >= 0 && row / kBlk * a.block_tokens < un.ntok) {
                const size_t at = ((size_t)un.g * a.num_subs + un.sub) * kBlk + row;
                a.neg_lse2[at] = nlrow;
                // -D as three bf16, which hold its 24 bits
                const float x = -drow, x1 = x - __bfloat162float(__float2bfloat16_rn(x)), x2 = x1 - __bfloat162float(__float2bfloat16_rn(x1));
                reinterpret_cast<uint4 *>(a.dsum)[at] = make_uint4(pack_bf16x2(x, x1), pack_bf16x2(x2, 0.f), 0, 0);
            }
            const uint64_t nl2 = f2_pack(nlrow, nlrow), d2 = f2_pack(drow, drow);
            for (int u = 0; ok && u < un.steps; ++u, ++c) {
                const uint32_t b = tmem + lanes + kColS + 64 * slot + 32 * ch;
                const int left = un.nk - u * kW;   // keys from this step on
                const bool partial = left < kW;
                if (!(ok = wait_w(B_SFULL + slot, ph, 195))) break;
                tc_fence_after();
                uint32_t vis = 0xffffffffu;
                if (partial) {
                    // K's rows past the end, which dQ's product sums over: zeros (S, which has read them, is done)
                    vis = interval_bits(0, left, 32 * ch);
                    uint8_t *kb = sk + c % kStages * kKTile;
                    for (int i = tid; i < (kW - left) * 8 * kPanels; i += 256)
                        *reinterpret_cast<uint4 *>(kb + i / 8 / (kW - left) * kKPanel + (left + i / 8 % (kW - left)) * 128 + i % 8 * 16) =
                            make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                }
                uint32_t sr[32], dr[32], dk[16];
                tmem_ld32(b, sr);
                tmem_ld32(tmem + lanes + kColDP + 64 * (c & 1) + 32 * ch, dr);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                mbar_arrive_warp(bar(B_DPFREE + (c & 1)));
                // two key columns per packed instruction: P = exp2(S c - lse2), dS = P (dP - D)
                auto column_pairs = [&](auto masked) {
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float x0, x1;
                        f2_unpack(f2_fma(f2_pack(__uint_as_float(sr[i]), __uint_as_float(sr[i + 1])), c2, nl2), x0, x1);
                        const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
                        const uint64_t t2 = f2_sub(f2_pack(__uint_as_float(dr[i]), __uint_as_float(dr[i + 1])), d2);
                        float d0, d1;
                        f2_unpack(f2_mul(f2_pack(p0, p1), t2), d0, d1);
                        if (decltype(masked)::value) {
                            d0 = (vis >> i) & 1u ? d0 : 0.f;
                            d1 = (vis >> (i + 1)) & 1u ? d1 : 0.f;
                        }
                        dk[i >> 1] = pack_bf16x2(d0, d1);
                    }
                };
                if (partial) column_pairs(std::true_type{}); else column_pairs(std::false_type{});
                tmem_st16(b, dk);   // over the first half of this thread's own S columns
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                mbar_arrive_warp(bar(B_PFULL + slot));
                if (++slot == kSlots) { slot = 0; ph ^= 1; }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int D>
padoc_status run(const padoc_cross_args &a, cudaStream_t stream)
{
    if (!a.num_units) {   // no row sees a key: the key rows' zeros alone
        const int64_t n = (int64_t)(a.num_tiles - a.gap_tile + a.tail_tiles) * a.hkv;
        if (n) cross_zero_kernel<D><<<(unsigned)(n < 4096 ? n : 4096), 256, 0, stream>>>(a);
        return padoc_launch_status();
    }
    const uint64_t row = (uint64_t)a.hq * D * 2, cols = (uint64_t)a.hkv * D;
    CUtensorMap qmap, gmap, omap, kmap, vmap, kmap2, vmap2;
    if (!padoc_make_tmap_bf16_heads(&qmap, a.q, D, a.hq, a.query_rows, a.q_stride * 2, a.group, a.block_tokens) ||
        !padoc_make_tmap_bf16_heads(&gmap, a.dout, D, a.hq, a.query_rows, row, a.group, a.block_tokens) ||
        !padoc_make_tmap_bf16_heads(&omap, a.out, D, a.hq, a.query_rows, row, a.group, a.block_tokens) ||
        !padoc_make_tmap_bf16(&kmap, a.k, cols, a.key_rows, a.k_stride * 2, 64, dqp::kW) ||
        !padoc_make_tmap_bf16(&vmap, a.v, cols, a.key_rows, a.v_stride * 2, 64, dqp::kW) ||
        !padoc_make_tmap_bf16(&kmap2, a.k, cols, a.key_rows, a.k_stride * 2, 64, dkv::kKT) ||
        !padoc_make_tmap_bf16(&vmap2, a.v, cols, a.key_rows, a.v_stride * 2, 64, dkv::kKT))
        return PADOC_ERR_CUDA;
    auto dq = cross_dq_kernel<D>;
    auto dkv = cross_dkv_kernel<D>;
    padoc_status st = padoc_set_max_smem((const void *)dq, (int)dqp::smem_bytes<D>());
    if (st == PADOC_OK) st = padoc_set_max_smem((const void *)dkv, (int)dkv::smem_bytes<D>());
    if (st != PADOC_OK) return st;
    dq<<<(unsigned)(a.ctas ? a.num_ctas : a.num_units), dqp::kThreads, dqp::smem_bytes<D>(), stream>>>(qmap, gmap, omap, kmap, vmap, a);
    if ((st = padoc_launch_status()) != PADOC_OK) return st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see the producer's wait
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)a.num_dkv_ctas);
    lc.blockDim = dim3(dkv::Cols<D>::kThreads);
    lc.dynamicSmemBytes = dkv::smem_bytes<D>();
    lc.stream = stream;
    lc.attrs = attr;
    lc.numAttrs = 1;
    PADOC_CUDA_TRY(cudaLaunchKernelEx(&lc, dkv, qmap, gmap, kmap2, vmap2, a));
    if ((st = padoc_launch_status()) != PADOC_OK || !a.num_dkv_sums) return st;
    const bool many = a.num_dkv_slots > 8 * a.num_dkv_sums;
    auto sum = many ? cross_dkv_sum_kernel<D, 8> : cross_dkv_sum_kernel<D, 1>;
    lc.gridDim = dim3((unsigned)(a.num_dkv_sums * (dkv::kKT * 2 * D / 4 / 256) * (many ? 8 : 1)));
    lc.blockDim = dim3(256);
    lc.dynamicSmemBytes = 0;
    PADOC_CUDA_TRY(cudaLaunchKernelEx(&lc, sum, a));
    return padoc_launch_status();
}

}  // namespace

padoc_status padoc_cross_launch_bwd_tc(const padoc_cross_args &args, int head_dim, cudaStream_t stream)
{
    padoc_cross_args a = args;
    a.err = padoc_device_error_word();
    if (!a.err) return PADOC_ERR_CUDA;
    return head_dim == 64 ? run<64>(a, stream) : run<128>(a, stream);
}
