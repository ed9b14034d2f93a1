// cross_tc.cu -- cross attention forward on the 5th-generation tensor cores: S = Q K^T, online softmax, O = P V.
//
// A unit is 256 packed rows of one KV head (two 128-row tiles of (token, head of the group) rows), or with 64 dims 128
// rows, over a segment's keys or a part of them. All rows of a unit see the same keys, so the only mask is the end of
// the last 128-key tile: its scores past the end become -inf, and its V rows there zeros, because what lies behind a
// segment's keys may be anything (0 x NaN would reach the output).
//
// Warp roles: four warps a tile for softmax and epilogue (TMEM lane = row: row max and sum need no shuffles); then the
// TMA producer, which also announces the units; then an MMA issuer a tile (a converged warp, one elected lane), the first
// of which also allocates tensor memory. Tensor memory: tile i keeps S in two halves of 64 keys, with P as packed bf16
// over the first 32 columns of its half, and O behind the tiles' S. For a tile and half the MMAs run
// S(t) -> P(t) -> P V(t) -> S(t + 1). O is rescaled only when a row's maximum has grown by more than 2^8 since the last
// time, which keeps P <= 256.
//
// The grid has one CTA per unit, most keys first; a running one takes over units not yet launched (cluster launch
// control). Where the planner cut the steps into equal runs, each CTA has a list of units. The next unit's queries and
// first scores come under the last one's output. A unit of at most 128 rows is run by tile 0's warps alone.
// Every wait is bounded; a wait that runs out records an error, all roles leave their loops, the issuers wait for
// their MMAs, the producer for its copies, and tensor memory is released.
//
// What bounds it: with 128 dims the MMAs and, over a long call, the chip's power (32768 rows over 8 x 2560 states of 16
// query heads: 426 us, 1613 TFLOP/s, 93% of what a library product of this type sustains; a step of both tiles 1.40 us, 1.23
// of them without any softmax: the MMAs take 2048 cycles, and 2560 with their operands' way from shared memory, where
// Q is read for each half of the keys). With 64 dims the chain through the softmax: a key costs half the MMAs and the same
// exponentials and conversions (1.27 us a step of two CTAs, 0.74 without; 9 pages of 16 heads 57 us), with the tensor pipe
// 31% and the issue slots 44% busy. One CTA with two tiles took 63 us there, sixteen softmax warps 75. Few steps an item:
// its start and end, some 3 us. Pairs of CTAs that share K and V by cta_group::2 were slower with 128 dims (434 -> 459 us,
// one more hand-over a step).
#include <math.h>

#include "cross.cuh"
#include "tc.cuh"

namespace {

constexpr int kPanel = 128 * 128;      // [128 rows][64 bf16]
constexpr int kBlk = PADOC_CROSS_BLOCK;
constexpr int kKT = PADOC_CROSS_KEY_TILE;
// V tails that may have landed before a softmax warp has waited for the first of them: of the unit that it is in and,
// as a unit is announced once every warp has read the one two before it, of two more.
constexpr int kTails = 3;

template <int D>
struct Cfg {
    static constexpr int kPanels = D / 64;
    static constexpr int kTile = kPanels * kPanel;
    static constexpr int kTiles = D == 64 ? 1 : 2;   // 128-row tiles of a unit; with 64 dims two CTAs share an SM
    static constexpr int kCtas = D == 64 ? 2 : 1;
    static constexpr int kSoft = 4 * kTiles;         // softmax warps
    static constexpr int kThreads = 32 * (kSoft + kTiles + (kTiles == 2 ? 2 : 1));
    static constexpr uint32_t kTmemCols = 256 * kTiles;
    static constexpr int kStages = 2;
    static constexpr int kKPanel = kPanel / 2;       // 64 dims of the keys of one half
    static constexpr int kOutBytes = kSoft * 4096;   // [32 rows][64 dims] a softmax warp
    enum {
        B_QFULL = 0,                    // [tile]
        B_QEMPTY = 2,                   // [tile]
        B_SFULL = 4,                    // [tile][half]
        B_PFULL = 8,                    // [tile][half], one arrival per warp of the tile
        B_PVDONE = 12,                  // [tile][half]
        B_OFREE = 16,                   // [tile], one arrival per warp of the tile
        B_UFULL = 18,                   // [slot]: the announced unit
        B_UEMPTY = 20,                  // [slot], one arrival per reading warp
        B_NEXT = 22,                    // the launch control's answer
        B_FINAL = 23,                   // [tile]
        B_VTAIL = 25,                   // [tail % 3]: a unit's last V tile, where keys end inside it
        B_KFULL = 28,                   // [stage]
        B_KEMPTY = B_KFULL + kStages,   // [stage], one arrival per tile
        B_VFULL = B_KEMPTY + kStages,   // [stage]
        B_VEMPTY = B_VFULL + kStages,   // [stage], one arrival per tile
        B_COUNT = B_VEMPTY + kStages
    };
    static constexpr int kReaders = kSoft + kTiles;   // softmax and MMA warps
    static constexpr size_t kSmemBytes = 1024 + kTiles * (size_t)kTile + 2 * (size_t)kStages * kTile + kOutBytes + 96 + B_COUNT * 8 + 16;
    static_assert(kCtas * (kSmemBytes + 1024) <= 228 * 1024, "");
};

// A unit as the producer announces it; tiles < 0 ends the CTA.
struct Unit {
    int32_t tok, ntok, k0, nk;
    int32_t g, slot, tiles, two;   // tiles: 128-key tiles; two: whether the second tile has rows
};

__device__ __forceinline__ bool wait_or_abort(uint32_t bar, uint32_t parity, int *err, int site, volatile int *abort_flag)
{
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (mbar_wait_bounded(bar, parity, err, site)) return true;
    *abort_flag = 1;
    return false;
}

template <int D>
__global__ void __launch_bounds__(Cfg<D>::kThreads, Cfg<D>::kCtas)
cross_tc_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                const __grid_constant__ CUtensorMap vmap, const padoc_cross_args a)
{
    using C = Cfg<D>;
    constexpr int kStages = C::kStages, kTile = C::kTile, kThreads = C::kThreads, kSoft = C::kSoft;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sq = smem;                       // [tile][panel][128 rows]
    uint8_t *sk = sq + C::kTiles * kTile;             // [kStages][key half][panel]
    uint8_t *sv = sk + kStages * kTile;    // [kStages][panel]
    uint8_t *so = sv + kStages * kTile;    // [softmax warp][32][128 bytes]
    Unit *units = (Unit *)(so + C::kOutBytes);   // [2]
    uint8_t *answer = (uint8_t *)(units + 2); // 16 bytes
    uint64_t *bars = (uint64_t *)(so + C::kOutBytes + 96);
    uint32_t *tmem_slot = (uint32_t *)(bars + C::B_COUNT);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // (a value the compiler knows to be warp-uniform)
    const int tile_tokens = 2 * a.block_tokens;
    pdl_launch_dependents();   // the joining of split rows, where there is one, may take the SMs that run out of work
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    if (tid < C::B_COUNT) {
        const int i = tid;
        int n = 1;
        if (i >= C::B_PFULL && i < C::B_PFULL + 4) n = 4;
        if (i == C::B_OFREE || i == C::B_OFREE + 1) n = 4;
        if (i >= C::B_KEMPTY && i < C::B_KEMPTY + kStages) n = C::kTiles;
        if (i >= C::B_VEMPTY && i < C::B_VEMPTY + kStages) n = C::kTiles;
        if (i == C::B_UEMPTY || i == C::B_UEMPTY + 1) n = C::kReaders;
        mbar_init(bar(i), n);
        if (i == 0) *abort_flag = 0;
        fence_barrier_init();
    }
    // items of this CTA: x and, of a list, those up to xe; the first one is on its way while the barriers are set
    // up (a small call waits for each global read in turn)
    int x = 0, xe = 0;
    padoc_cross_unit item = {};
    if (warp == kSoft && lane == 0) {
        x = (int)blockIdx.x;
        tma_prefetch_desc(&qmap);
        tma_prefetch_desc(&kmap);
        tma_prefetch_desc(&vmap);
        pdl_wait_prerequisite();   // nothing in global memory is touched before (the other roles' work follows from this)
        if (a.ctas) {
            xe = a.ctas[x + 1];
            x = a.ctas[x];
        }
        item = a.units[x];
    }
    // rows of a block that hold no (token, head): no copy writes them
    const int used = a.block_tokens * a.group;
    if (used < kBlk) {
        for (int i = tid; i < 2 * C::kTiles * C::kPanels * (kBlk - used) * 8; i += kThreads) {
            const int r = i / 8 % (kBlk - used) + used, b = i / 8 / (kBlk - used);
            *reinterpret_cast<uint4 *>(sq + b * kBlk * 128 + r * 128 + i % 8 * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
    }
    if (warp == kSoft + 1) {
        tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    // the n-th unit, as every lane of a reading warp sees it
    auto read_unit = [&](int n, Unit &u, int site) {
        const bool r = wait_or_abort(bar(C::B_UFULL + (n & 1)), (n >> 1) & 1, a.err, site, abort_flag);
        if (!__all_sync(0xffffffffu, r)) return false;
        const Unit v = units[n & 1];
        u.tok = __shfl_sync(0xffffffffu, v.tok, 0);
        u.ntok = __shfl_sync(0xffffffffu, v.ntok, 0);
        u.nk = __shfl_sync(0xffffffffu, v.nk, 0);
        u.g = __shfl_sync(0xffffffffu, v.g, 0);
        u.slot = __shfl_sync(0xffffffffu, v.slot, 0);
        u.tiles = __shfl_sync(0xffffffffu, v.tiles, 0);
        u.two = __shfl_sync(0xffffffffu, v.two, 0);
        __syncwarp();   // (every lane's read has returned before the arrival lets the slot be written again)
        if (lane == 0) mbar_arrive(bar(C::B_UEMPTY + (n & 1)));
        return true;
    };
    // the next unit that tile i takes part in; ring: K and V tiles so far, of all units
    auto next_unit = [&](int i, int &n, Unit &u, int &ring, int site) {
        for (;;) {
            if (!read_unit(n++, u, site)) return false;
            if (u.tiles < 0 || C::kTiles == 1 || i == 0 || u.two) return true;
            ring += u.tiles;
        }
    };

    if (warp >= kSoft) {
        if (warp == kSoft && lane == 0) {
            // ------------------------------------------------------------ TMA producer
            auto wait = [&](int b, uint32_t parity, int site) {
                return wait_or_abort(bar(b), parity, a.err, site, abort_flag);
            };
            int tk = 0, tv = 0, nq[2] = {0, 0}, tails = 0;   // K and V tiles, queries per tile, V tails issued so far
            bool ok = true, more = true, asked = false;
            // asked with the unit's last tile, a few tiles ahead of the MMAs: early enough for the answer,
            // and late enough that no CTA holds a second unit while others run out of work
            auto ask = [&]() {
                if (a.ctas) return;
                mbar_arrive_expect_tx(bar(C::B_NEXT), 16);
                launch_control_ask(smem_u32(answer), bar(C::B_NEXT));
                asked = true;
            };
            auto load_q = [&](int i, const Unit &u) {
                if (nq[i] && !wait(C::B_QEMPTY + i, (nq[i] - 1) & 1, 120)) return false;
                const int t0 = u.tok + i * tile_tokens;
                mbar_arrive_expect_tx(bar(C::B_QFULL + i), 2 * C::kPanels * used * 128);
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int p = 0; p < C::kPanels; ++p) {
                        const uint32_t dst = smem_u32(sq + i * kTile + p * kPanel + b * kBlk * 128);
                        tma_load_3d(dst, &qmap, 64 * p, u.g * a.group, t0 + b * a.block_tokens, bar(C::B_QFULL + i));
                    }
                ++nq[i];
                return true;
            };
            int n = 0, asks = 0;   // units announced, questions answered
            for (;; ++n) {
                Unit u = {0, 0, 0, 0, 0, 0, -1, 0};
                if (n >= 2 && !wait(C::B_UEMPTY + (n & 1), ((n >> 1) - 1) & 1, 124)) break;
                if (more) {
                    u = {item.tok, item.ntok, item.k0, item.nk, item.g, item.slot, (item.nk + kKT - 1) / kKT,
                         C::kTiles == 2 && item.ntok > tile_tokens};
                    if (a.ctas && (more = ++x < xe)) item = a.units[x];   // (a list's next item is known at once)
                }
                units[n & 1] = u;
                mbar_arrive(bar(C::B_UFULL + (n & 1)));
                if (u.tiles < 0) break;
                for (int j = 0; j < u.tiles; ++j) {
                    if (j + 1 == u.tiles) ask();
                    // (the first K tile between the two tiles' queries: S_0 needs it first)
                    if (j == 0 && !(ok = load_q(0, u))) break;
                    const int s = tk % kStages, row = u.k0 + j * kKT;
                    if (tk >= kStages && !(ok = wait(C::B_KEMPTY + s, (tk / kStages - 1) & 1, 121))) break;
                    uint8_t *kb = sk + s * kTile;
                    mbar_arrive_expect_tx(bar(C::B_KFULL + s), kTile);
                    if (C::kTiles == 2 && !u.two) mbar_arrive(bar(C::B_KEMPTY + s));   // (for the second tile, which has no part)
#pragma unroll
                    for (int b = 0; b < 2 * C::kPanels; ++b)   // [key half][panel]
                        tma_load_2d(smem_u32(kb + b * C::kKPanel), &kmap, u.g * D + 64 * (b % C::kPanels), row + 64 * (b / C::kPanels),
                                    bar(C::B_KFULL + s));
                    ++tk;
                    if (j == 0 && u.two && !(ok = load_q(1, u))) break;
                    if (tv >= kStages && !(ok = wait(C::B_VEMPTY + s, (tv / kStages - 1) & 1, 123))) break;
                    uint8_t *vb = sv + s * kTile;
                    // a tail completes on a barrier of its own: the softmax warps zero its rows past the end
                    const bool tail = u.nk - j * kKT < kKT;
                    const uint32_t vbar = bar(tail ? C::B_VTAIL + tails % kTails : C::B_VFULL + s);
                    if (tail) {
                        mbar_arrive(bar(C::B_VFULL + s));
                        ++tails;
                    }
                    mbar_arrive_expect_tx(vbar, kTile);
                    if (C::kTiles == 2 && !u.two) mbar_arrive(bar(C::B_VEMPTY + s));
#pragma unroll
                    for (int p = 0; p < C::kPanels; ++p) tma_load_2d(smem_u32(vb + p * kPanel), &vmap, u.g * D + 64 * p, row, vbar);
                    ++tv;
                }
                if (!ok) break;
                if (!a.ctas) {
                    if (!wait(C::B_NEXT, asks & 1, 126)) break;
                    ++asks;
                    asked = false;
                    int y;
                    more = launch_control_answer(smem_u32(answer), x, y);
                    if (more) item = a.units[x];
                    fence_proxy_async_smem();   // the answer is read before the next one may be written
                }
            }
            // copies still in flight must land before the CTA's shared memory is released
            if (asked) mbar_wait_bounded(bar(C::B_NEXT), asks & 1, a.err, 127);
            for (int i = 0; i < C::kTiles; ++i)
                if (nq[i]) mbar_wait_bounded(bar(C::B_QFULL + i), (nq[i] - 1) & 1, a.err, 127);
            for (int t = max(tk - kStages, 0); t < tk; ++t)
                mbar_wait_bounded(bar(C::B_KFULL + t % kStages), (t / kStages) & 1, a.err, 128);
            for (int t = max(tails - kTails, 0); t < tails; ++t)
                mbar_wait_bounded(bar(C::B_VTAIL + t % kTails), (t / kTails) & 1, a.err, 127);
            for (int t = max(tv - kStages, 0); t < tv; ++t)
                mbar_wait_bounded(bar(C::B_VFULL + t % kStages), (t / kStages) & 1, a.err, 129);
        } else if (warp > kSoft && warp <= kSoft + C::kTiles) {
            // ------------------------------------------------------------ MMA issuers (a whole warp per tile)
            const int i = warp - kSoft - 1;
            constexpr uint32_t idS = umma_idesc_bf16(128, 64, false);
            constexpr uint32_t idPV = umma_idesc_bf16(128, D, true);
            const uint64_t dq = umma_desc_sw128(smem_u32(sq + i * kTile), 16, 1024);
            const uint64_t dk = umma_desc_sw128(smem_u32(sk), 16, 1024), dv = umma_desc_sw128(smem_u32(sv), kPanel, 1024);
            const uint32_t tS = tmem + 128 * i, tO = tmem + 128 * (C::kTiles + i);
            auto wait = [&](int b, uint32_t parity, int site) {
                return mbar_wait_warp(bar(b), parity, a.err, site, abort_flag);
            };
            auto commit = [&](int b) { umma_commit_warp(bar(b)); };
            // S_i over half h of the tile in the given stage; the last tile of a unit frees Q_i
            auto issue_s = [&](int stage, int h, bool last) {
                const uint64_t b = dk + ((stage * kTile + h * C::kPanels * C::kKPanel) >> 4);
                if constexpr (D == 128) umma_bf16_ss_k128_warp<1, kPanel, C::kKPanel>(tS + 64 * h, dq, b, idS);
                else umma_bf16_ss_k64_warp(tS + 64 * h, dq, b, idS);
                commit(C::B_SFULL + 2 * i + h);
                if (h == 1) {
                    if (last) commit(C::B_QEMPTY + i);
                    commit(C::B_KEMPTY + stage);
                }
            };
            int n = 0, ring = 0, t = 0;   // units read; K and V tiles of all units, and of this tile's
            Unit u;
            bool ok = next_unit(i, n, u, ring, 130);
            auto first_s = [&](int w) {
                const int s = ring % kStages;
                if (!wait(C::B_KFULL + s, (ring / kStages) & 1, 131) || !wait(C::B_QFULL + i, w & 1, 132)) return false;
                tc_fence_after();
                issue_s(s, 0, u.tiles == 1);
                issue_s(s, 1, u.tiles == 1);
                return true;
            };
            // O_i += P_i V over half h of the tile
            auto issue_pv = [&](int s, int h, bool first) {
                if (!wait(C::B_PFULL + 2 * i + h, t & 1, 135)) return false;
                tc_fence_after();
                umma_bf16_ts_k64_mn_warp<1>(tO, tS + 64 * h, dv + ((s * kTile + h * 8192) >> 4), idPV, !first);
                commit(C::B_PVDONE + 2 * i + h);
                if (h == 1) commit(C::B_VEMPTY + s);
                return true;
            };
            if (ok && u.tiles > 0) ok = first_s(0);
            for (int w = 0; ok && u.tiles > 0; ++w) {
                if (w > 0) ok = wait(C::B_OFREE + i, (w - 1) & 1, 134);
                const int ne = u.tiles;
                for (int j = 0; ok && j + 1 < ne; ++j, ++t, ++ring) {
                    const int s = ring % kStages, sn = (ring + 1) % kStages;
                    // (while the tensor cores still run the S of this tile)
                    ok = wait(C::B_VFULL + s, (ring / kStages) & 1, 133) && wait(C::B_KFULL + sn, ((ring + 1) / kStages) & 1, 136);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (ok && (ok = issue_pv(s, h, j == 0 && h == 0))) issue_s(sn, h, j + 2 == ne);
                }
                if (!ok) break;
                // the unit's last tile, then the first S of the next unit, under this one's epilogue
                const int s = ring % kStages;
                ok = wait(C::B_VFULL + s, (ring / kStages) & 1, 133) && issue_pv(s, 0, ne == 1) && issue_pv(s, 1, false);
                if (!ok) break;
                ++t;
                ++ring;
                ok = next_unit(i, n, u, ring, 130);
                if (!ok || u.tiles < 0) break;
                ok = first_s(w + 1);
            }
            // every MMA issued above must complete before TMEM is released
            umma_commit_warp(bar(C::B_FINAL + i));
            mbar_wait_bounded(bar(C::B_FINAL + i), 0, a.err, 138);
        }
    } else {
        // ---------------------------------------------------------------- softmax + epilogue
        const int hi = warp / 4;                    // tile inside the unit
        const int row = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lanes + 128 * hi, tO = tmem + lanes + 128 * (C::kTiles + hi);
        const float c = a.scale_log2;
        // every decision below is warp-uniform: the TMEM loads and stores are warp-collective
        auto wait_all = [&](int b, uint32_t parity, int site) {
            return mbar_wait_warp(bar(b), parity, a.err, site, abort_flag);
        };
        int t_tile = 0, ring = 0, n = 0, tails = 0;   // this tile's K tiles, all units', units read, V tails passed
        auto wait_tail = [&](int site) {
            const int t = tails++;
            return wait_all(C::B_VTAIL + t % kTails, (t / kTails) & 1, site);
        };
        Unit next = {};
        auto next_of_tile = [&]() {
            for (;;) {
                if (!read_unit(n++, next, 139)) return false;
                if (next.tiles < 0 || C::kTiles == 1 || hi == 0 || next.two) return true;
                ring += next.tiles;
                // (its V tail comes by the same barriers, whose phases are waited for one by one)
                if (next.nk % kKT != 0 && !wait_tail(144)) return false;
            }
        };
        bool ok = next_of_tile();
        while (ok && next.tiles > 0) {
            const Unit u = next;
            int token, head;
            const bool in = cross_row(a, u.tok, u.ntok, hi * 128 + row, token, head);
            const bool idle = !__any_sync(0xffffffffu, in);   // a warp without rows only keeps the others' pace
            float m_ref = -INFINITY, l = 0.f;   // m_ref in raw score units
            for (int j = 0; j < u.tiles; ++j, ++t_tile, ++ring) {
                const int left = u.nk - j * kKT;   // keys from this tile on
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t tB = tS + 64 * half;
                    if (!wait_all(C::B_SFULL + 2 * hi + half, t_tile & 1, 140)) { ok = false; break; }
                    tc_fence_after();
                    if (!idle) {
                        // the row's scores are read from tensor memory once and stay in registers
                        uint32_t sr[2][32];
                        tmem_ld32(tB, sr[0]);
                        tmem_ld32(tB + 32, sr[1]);
                        tmem_ld_wait();
                        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const int base = 64 * half + 32 * q;
                            if (left < base + 32) {
                                const uint32_t vis = interval_bits(0, left, base);
#pragma unroll
                                for (int i = 0; i < 32; ++i) sr[q][i] = (vis >> i) & 1u ? sr[q][i] : 0xff800000u;   // -inf
                            }
#pragma unroll
                            for (int i = 0; i < 32; i += 8) {
                                mx4[0] = fmax3f(mx4[0], __uint_as_float(sr[q][i]), __uint_as_float(sr[q][i + 1]));
                                mx4[1] = fmax3f(mx4[1], __uint_as_float(sr[q][i + 2]), __uint_as_float(sr[q][i + 3]));
                                mx4[2] = fmax3f(mx4[2], __uint_as_float(sr[q][i + 4]), __uint_as_float(sr[q][i + 5]));
                                mx4[3] = fmax3f(mx4[3], __uint_as_float(sr[q][i + 6]), __uint_as_float(sr[q][i + 7]));
                            }
                        }
                        const float mx = fmaxf(fmax3f(mx4[0], mx4[1], mx4[2]), mx4[3]);
                        const float m_new = fmaxf(m_ref, mx);
                        // a row with nothing accumulated yet (O holds zeros) adopts the new maximum directly;
                        // otherwise the reference only moves when the maximum grew by more than 2^8
                        const bool rescale = m_ref != -INFINITY && (m_new - m_ref) * c > 8.f;
                        if (m_ref == -INFINITY) m_ref = m_new;
                        if (__any_sync(0xffffffffu, rescale)) {
                            // O_i is quiescent once the previous half's PV is done: the next one waits for this P
                            // (the one before that was done before this half's S)
                            if (!wait_all(C::B_PVDONE + 2 * hi + (half ^ 1), (half ? t_tile : t_tile - 1) & 1, 141)) { ok = false; break; }
                            tc_fence_after();
                            const float alpha = rescale ? fast_exp2((m_ref - m_new) * c) : 1.f;
#pragma unroll 1   // (rare; unrolled it takes registers from every tile)
                            for (int q = 0; q < D / 16; ++q) {
                                uint32_t o[16];
                                tmem_ld16(tO + q * 16, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                tmem_st16(tO + q * 16, o);
                            }
                            if (rescale) { l *= alpha; m_ref = m_new; }
                        }
                        const float moff = m_ref == -INFINITY ? 0.f : m_ref * c;
                        // P = exp2(S * c - m * c) as packed bf16 over the first 32 columns of this half's S: the MMA's
                        // operand type, half a step (2^-9 of a weight on average), where l adds the unrounded weights
                        const uint64_t c2 = f2_pack(c, c), moff2 = f2_pack(-moff, -moff);
                        uint64_t rs[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            uint32_t pk[16];
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                float x0, x1;
                                f2_unpack(f2_fma(f2_pack(__uint_as_float(sr[q][i]), __uint_as_float(sr[q][i + 1])), c2, moff2), x0, x1);
                                const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
                                rs[(i >> 1) & 3] = f2_add(rs[(i >> 1) & 3], f2_pack(p0, p1));
                                pk[i >> 1] = pack_bf16x2(p0, p1);
                            }
                            tmem_st16(tB + q * 16, pk);
                        }
                        float r0, r1;
                        f2_unpack(f2_add(f2_add(rs[0], rs[1]), f2_add(rs[2], rs[3])), r0, r1);
                        l += r0 + r1;
                    }
                    const bool tail = half == 0 && left < kKT;
                    if (tail) {   // V's rows past the end (both tiles' warps write the same zeros)
                        if (!wait_tail(142)) { ok = false; break; }
                        uint8_t *vb = sv + ring % kStages * kTile + row * 128;
                        if (row >= left)
#pragma unroll
                            for (int p = 0; p < C::kPanels; ++p)
#pragma unroll
                                for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4 *>(vb + p * kPanel + 16 * i) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::B_PFULL + 2 * hi + half));
                }
                if (!ok) break;
            }
            const int last_tile = t_tile - 1;
            if (!ok || !(ok = wait_all(C::B_PVDONE + 2 * hi + 1, last_tile & 1, 143))) break;
            tc_fence_after();
            // O / l: through shared memory, so that eight lanes write a row's 128 bytes, or, as a part of the row's
            // keys, in fp32 with the part's log-sum-exp. O_i is free for the next unit's PV as soon as it is read.
            const float inv = l == 0.f ? 0.f : 1.f / l, lse2 = l == 0.f ? -INFINITY : m_ref * c + log2f(l);
            const int64_t at = in ? ((int64_t)token * a.hq + u.g * a.group + head) * D : -1;
            const size_t pr = (size_t)max(u.slot, 0) * (C::kTiles * 128) + hi * 128 + row;
            uint8_t *stage = so + warp * 4096;
#pragma unroll
            for (int half = 0; half < C::kPanels; ++half) {
                uint32_t o[2][32];
                tmem_ld32(tO + 64 * half, o[0]);
                tmem_ld32(tO + 64 * half + 32, o[1]);
                tmem_ld_wait();
                if (half == C::kPanels - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::B_OFREE + hi));
                }
                auto v = [&](int i) { return __uint_as_float(o[i >> 5][i & 31]) * inv; };
                if (u.slot >= 0) {
                    if (in) {
#pragma unroll
                        for (int i = 0; i < 64; i += 8)
                            st_global_v8(a.part + pr * D + 64 * half + i, v(i), v(i + 1), v(i + 2), v(i + 3), v(i + 4), v(i + 5),
                                         v(i + 6), v(i + 7));
                    }
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 64; i += 8)
                    *reinterpret_cast<uint4 *>(stage + lane * 128 + (((i / 8) ^ (lane & 7)) << 4)) =
                        make_uint4(pack_bf16x2(v(i), v(i + 1)), pack_bf16x2(v(i + 2), v(i + 3)), pack_bf16x2(v(i + 4), v(i + 5)),
                                   pack_bf16x2(v(i + 6), v(i + 7)));
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 4 * i + (lane >> 3), k = lane & 7;
                    const int64_t to = __shfl_sync(0xffffffffu, at, r);
                    const uint4 w = *reinterpret_cast<const uint4 *>(stage + r * 128 + ((k ^ (r & 7)) << 4));
                    if (to >= 0) *reinterpret_cast<uint4 *>((__nv_bfloat16 *)a.o + to + 64 * half + 8 * k) = w;
                }
                __syncwarp();
            }
            if (in) {
                if (u.slot < 0) a.lse[at / D] = lse2 * PADOC_LN2;
                else a.part_lse[pr] = lse2;
            }
            ok = next_of_tile();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kSoft + 1) {
        tc_fence_after();
        tmem_dealloc(tmem, C::kTmemCols);
    }
}

template <int D>
padoc_status launch(const padoc_cross_args &a, cudaStream_t stream)
{
    auto kernel = cross_tc_kernel<D>;
    constexpr size_t bytes = Cfg<D>::kSmemBytes;
    if (const padoc_status st = padoc_set_max_smem((const void *)kernel, (int)bytes)) return st;
    CUtensorMap qmap, kmap, vmap;
    if (!padoc_make_tmap_bf16_heads(&qmap, a.q, D, a.hq, a.query_rows, a.q_stride * 2, a.group, a.block_tokens) ||
        !padoc_make_tmap_bf16(&kmap, a.k, (uint64_t)a.hkv * D, a.key_rows, a.k_stride * 2, 64, 64) ||
        !padoc_make_tmap_bf16(&vmap, a.v, (uint64_t)a.hkv * D, a.key_rows, a.v_stride * 2, 64, kKT))
        return PADOC_ERR_CUDA;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(a.ctas ? a.num_ctas : a.num_units));
    lc.blockDim = dim3(Cfg<D>::kThreads);
    lc.dynamicSmemBytes = bytes;
    lc.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // set up behind the last kernel's end
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    PADOC_CUDA_TRY(cudaLaunchKernelEx(&lc, kernel, qmap, kmap, vmap, a));
    return padoc_launch_status();
}

}  // namespace

padoc_status padoc_cross_launch_tc(const padoc_cross_args &args, int head_dim, cudaStream_t stream)
{
    padoc_cross_args a = args;
    a.err = padoc_device_error_word();
    if (!a.err) return PADOC_ERR_CUDA;
    return head_dim == 64 ? launch<64>(a, stream) : launch<128>(a, stream);
}
