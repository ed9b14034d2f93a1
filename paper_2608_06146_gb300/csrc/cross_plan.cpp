// cross_plan.cpp -- the host planner of cross attention (integers only).
//
// Forward: every segment's rows are cut into units of 256 packed rows (512 for CTA pairs), each with the segment's
// whole key range, or, where that leaves the chip idle, with parts of it whose results are joined. Backward: the dq
// pass has units of 128 rows cut the same way; the dk/dv pass has key tiles. The key axis is cut at every
// segment's ends, so that a tile's keys are all seen by the same segments and its steps need no mask.
#include <string.h>

#include <algorithm>
#include <functional>
#include <queue>
#include <vector>

#include "cross_internal.h"
#include "plan_internal.h"

int32_t padoc_default_ctas();

namespace {

typedef padoc_cross_segment Segment;

// Time of a set of pieces, each run once per KV head, heaviest first on `lanes` SMs (or pairs): the greedy schedule
// that the hardware's launch order and the kernels' taking over of pending units come close to.
float makespan(std::vector<float> cost, int hkv, int lanes)
{
    if (cost.empty()) return 0.f;
    std::sort(cost.begin(), cost.end(), std::greater<float>());
    double total = 0;
    for (float c : cost) total += c;
    total *= hkv;
    if ((double)cost.size() * hkv > 16.0 * lanes) return (float)(total / lanes) + 0.5f * cost[0];
    std::priority_queue<float, std::vector<float>, std::greater<float>> free;
    for (int i = 0; i < lanes; ++i) free.push(0.f);
    float end = 0.f;
    for (float c : cost)
        for (int g = 0; g < hkv; ++g) {
            const float t = free.top() + c;
            free.pop();
            free.push(t);
            end = std::max(end, t);
        }
    return end;
}

// Costs in units of one 128-key step of two 128-row tiles (forward) or one 64-key step of a tile (dq).
struct Costs {
    float start;    // a unit's start and end
    float part;     // ... and what a partial result's traffic adds
    float merge;    // the launch that joins them
    float half;     // a step of a unit whose second tile is empty (forward)
};

struct Chunk {
    int32_t tok, ntok, k0, nk, steps;
    float step_cost;
};

struct Cut {
    int32_t longest;    // most steps of a piece; chunks are cut into equal pieces no longer than this
    float time;
};

int32_t pieces_of(const Chunk &c, int32_t longest) { return (c.steps + longest - 1) / longest; }

// The cut with the shortest estimated time: none, or pieces that give each SM one to eight of them.
Cut choose_cut(const std::vector<Chunk> &chunks, int hkv, int lanes, const Costs &k)
{
    double work = 0;
    int32_t most = 1;
    for (const Chunk &c : chunks) {
        work += c.steps;
        most = std::max(most, c.steps);
    }
    std::vector<int32_t> tries = {most};
    static const int waves[] = {1, 2, 3, 4, 6, 8};
    for (int w : waves) {
        const int32_t l = (int32_t)std::max(1.0, work * hkv / ((double)lanes * w) + 0.999);
        if (l < most) tries.push_back(l);
    }
    Cut best = {most, 0.f};
    bool first = true;
    for (int32_t longest : tries) {
        std::vector<float> cost;
        bool split = false;
        for (const Chunk &c : chunks) {
            const int32_t n = pieces_of(c, longest);
            split |= n > 1;
            for (int32_t i = 0; i < n; ++i) {
                const int32_t steps = (int32_t)((int64_t)c.steps * (i + 1) / n - (int64_t)c.steps * i / n);
                cost.push_back((float)steps * c.step_cost + k.start + (n > 1 ? k.part : 0.f));
            }
        }
        const float t = makespan(cost, hkv, lanes) + (split ? k.merge : 0.f);
        if (first || t < best.time) best = {longest, t};
        first = false;
    }
    return best;
}

// Units and merges of these chunks, heavier units first.
void cut_units(const std::vector<Chunk> &chunks, int32_t longest, int32_t step, std::vector<padoc_cross_unit> &units,
               std::vector<padoc_cross_merge> &merges, int32_t &slots, const std::function<int32_t(size_t)> &sub)
{
    slots = 0;
    for (size_t i = 0; i < chunks.size(); ++i) {
        const Chunk &c = chunks[i];
        const int32_t n = pieces_of(c, longest);
        if (n > 1) merges.push_back({c.tok, c.ntok, slots, n});
        for (int32_t p = 0; p < n; ++p) {
            const int32_t a = (int32_t)((int64_t)c.steps * p / n) * step;
            const int32_t b = std::min(c.nk, (int32_t)((int64_t)c.steps * (p + 1) / n) * step);
            units.push_back({c.tok, c.ntok, c.k0 + a, b - a, n > 1 ? slots + p : -1, p == 0 ? sub(i) : -1, {0, 0}});
        }
        if (n > 1) slots += n;
    }
    std::stable_sort(units.begin(), units.end(),
                     [](const padoc_cross_unit &x, const padoc_cross_unit &y) { return x.nk > y.nk; });
}

struct Built {
    std::vector<padoc_cross_unit> units, dq_units;
    std::vector<padoc_cross_merge> merges, dq_merges;
    std::vector<padoc_cross_key_tile> tiles;
    std::vector<padoc_cross_cover> covers;
    padoc_cross_plan info;
};

padoc_status check(const Segment *seg, int32_t n, const padoc_cross_config *cfg)
{
    if (!cfg || n < 0 || (n > 0 && !seg)) return PADOC_ERR_INVALID_ARGUMENT;
    if (cfg->num_q_heads < 1 || cfg->num_kv_heads < 1 || cfg->num_q_heads % cfg->num_kv_heads || cfg->ctas < 0 ||
        cfg->backward < 0 || cfg->backward > 1)
        return PADOC_ERR_INVALID_ARGUMENT;
    if (cfg->dtype != PADOC_DTYPE_F32 && cfg->dtype != PADOC_DTYPE_BF16) return PADOC_ERR_UNSUPPORTED;
    if (cfg->head_dim != 64 && cfg->head_dim != 128) return PADOC_ERR_UNSUPPORTED;
    if (cfg->num_q_heads / cfg->num_kv_heads > PADOC_CROSS_BLOCK || cfg->num_q_heads > 4096) return PADOC_ERR_UNSUPPORTED;
    const int64_t limit = (int64_t)INT32_MAX - 1024;   // (a tile's rows past the end still count in 32 bits)
    int64_t end = 0;
    for (int32_t i = 0; i < n; ++i) {
        const Segment &s = seg[i];
        if (s.q_begin < 0 || s.q_len < 0 || s.k_begin < 0 || s.k_len < 0) return PADOC_ERR_INVALID_ARGUMENT;
        if ((int64_t)s.q_begin + s.q_len > limit || (int64_t)s.k_begin + s.k_len > limit) return PADOC_ERR_INVALID_ARGUMENT;
        if (s.q_begin < end) return PADOC_ERR_INVALID_ARGUMENT;
        end = (int64_t)s.q_begin + s.q_len;
    }
    return PADOC_OK;
}

int32_t ceil_div(int64_t a, int64_t b) { return (int32_t)((a + b - 1) / b); }

padoc_status make(const Segment *seg, int32_t n, const padoc_cross_config *cfg, Built &b)
{
    const padoc_status st = check(seg, n, cfg);
    if (st != PADOC_OK) return st;
    memset(&b.info, 0, sizeof(b.info));
    padoc_cross_plan &info = b.info;
    info.cfg = *cfg;
    info.num_segments = n;
    const int32_t hkv = cfg->num_kv_heads, group = cfg->num_q_heads / hkv, block = PADOC_CROSS_BLOCK / group;
    // fp32 runs a CTA per 64 rows, a few of them on an SM: about two units' worth at a time
    const int32_t sms = cfg->ctas ? cfg->ctas : padoc_default_ctas();
    const int32_t lanes = cfg->dtype == PADOC_DTYPE_F32 ? std::max(1, sms / 2) : sms;

    int64_t q_end = 0, k_end = 0, subs = 0, blocks = 0;
    std::vector<int32_t> first_sub((size_t)n, 0);
    for (int32_t i = 0; i < n; ++i) {
        if (seg[i].q_len == 0) continue;
        q_end = std::max(q_end, (int64_t)seg[i].q_begin + seg[i].q_len);
        if (seg[i].k_len) k_end = std::max(k_end, (int64_t)seg[i].k_begin + seg[i].k_len);
        info.pairs += (int64_t)seg[i].q_len * seg[i].k_len;
        first_sub[i] = (int32_t)subs;
        blocks += ceil_div(seg[i].q_len, block);
        if (seg[i].k_len) subs += ceil_div(seg[i].q_len, block);
    }
    info.query_rows = (int32_t)q_end;
    info.key_rows = (int32_t)k_end;
    // blocks, and steps over them, are counted in 32 bits on the device
    if (blocks * hkv > (int64_t)1 << 24 || k_end > (int64_t)1 << 29) return PADOC_ERR_UNSUPPORTED;

    auto chunks_of = [&](int32_t unit_blocks, int32_t step, float half, std::vector<int32_t> *sub) {
        std::vector<Chunk> c;
        const int32_t per = unit_blocks * block;
        for (int32_t i = 0; i < n; ++i) {
            if (seg[i].q_len == 0 || seg[i].k_len == 0) continue;
            for (int32_t t = 0; t < seg[i].q_len; t += per) {
                const int32_t m = std::min(per, seg[i].q_len - t);
                c.push_back({seg[i].q_begin + t, m, seg[i].k_begin, seg[i].k_len, ceil_div(seg[i].k_len, step),
                             m <= per / 2 ? half : 1.f});
                if (sub) sub->push_back(first_sub[i] + t / block);
            }
        }
        return c;
    };
    auto empty_rows = [&](int32_t unit_blocks, std::vector<padoc_cross_merge> &merges) {
        const int32_t per = unit_blocks * block;
        for (int32_t i = 0; i < n; ++i)
            if (seg[i].k_len == 0)
                for (int32_t t = 0; t < seg[i].q_len; t += per)
                    merges.push_back({seg[i].q_begin + t, std::min(per, seg[i].q_len - t), 0, 0});
    };

    // forward (a step of two tiles lasts about 1.5 us)
    const Costs fwd = {1.5f, 0.5f, 2.0f, 0.65f};
    std::vector<Chunk> chunks = chunks_of(PADOC_CROSS_UNIT_BLOCKS, PADOC_CROSS_KEY_TILE, fwd.half, nullptr);
    Cut cut = choose_cut(chunks, hkv, lanes, fwd);
    b.info.pair = 0;
    cut_units(chunks, cut.longest, PADOC_CROSS_KEY_TILE, b.units, b.merges, info.num_slots, [](size_t) { return -1; });
    empty_rows(PADOC_CROSS_UNIT_BLOCKS, b.merges);

    if (cfg->backward) {
        const Costs bwd = {6.f, 1.f, 4.f, 1.f};   // (a step of a tile lasts about 0.55 us)
        std::vector<int32_t> sub;
        chunks = chunks_of(PADOC_CROSS_DQ_BLOCKS, PADOC_CROSS_DQ_STEP, 1.f, &sub);
        cut = choose_cut(chunks, hkv, lanes, bwd);
        cut_units(chunks, cut.longest, PADOC_CROSS_DQ_STEP, b.dq_units, b.dq_merges, info.num_dq_slots,
                  [&](size_t i) { return sub[i]; });
        empty_rows(PADOC_CROSS_DQ_BLOCKS, b.dq_merges);

        // key intervals between neighbouring ends of the segments' key ranges
        std::vector<int32_t> ends = {0};
        std::vector<int32_t> order;   // segments by their first key
        for (int32_t i = 0; i < n; ++i)
            if (seg[i].q_len && seg[i].k_len) {
                ends.push_back(seg[i].k_begin);
                ends.push_back(seg[i].k_begin + seg[i].k_len);
                order.push_back(i);
            }
        std::sort(ends.begin(), ends.end());
        ends.erase(std::unique(ends.begin(), ends.end()), ends.end());
        std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return seg[x].k_begin < seg[y].k_begin; });
        std::vector<int32_t> live;   // segments that see the interval, in their own order
        size_t next = 0;
        for (size_t e = 0; e + 1 < ends.size(); ++e) {
            const int32_t k0 = ends[e], k1 = ends[e + 1];
            live.erase(std::remove_if(live.begin(), live.end(), [&](int32_t i) { return seg[i].k_begin + seg[i].k_len <= k0; }),
                       live.end());
            for (; next < order.size() && seg[order[next]].k_begin <= k0; ++next)
                live.insert(std::lower_bound(live.begin(), live.end(), order[next]), order[next]);
            const int32_t cover = (int32_t)b.covers.size();
            int64_t steps = 0;
            for (int32_t i : live) {
                const int32_t m = ceil_div(seg[i].q_len, block);
                b.covers.push_back({seg[i].q_begin, seg[i].q_len, first_sub[i], m});
                steps += m;
            }
            if (b.covers.size() > (size_t)1 << 24) return PADOC_ERR_UNSUPPORTED;
            for (int32_t k = k0; k < k1; k += PADOC_CROSS_KEY_TILE)
                b.tiles.push_back({k, std::min(PADOC_CROSS_KEY_TILE, k1 - k), cover, (int32_t)live.size(), (int32_t)steps, {0, 0, 0}});
            info.max_steps = std::max(info.max_steps, (int32_t)steps);
        }
        std::stable_sort(b.tiles.begin(), b.tiles.end(),
                         [](const padoc_cross_key_tile &x, const padoc_cross_key_tile &y) { return x.steps > y.steps; });
        info.num_subs = (int32_t)subs;

        // The CTAs that share a key tile's steps: few tiles seen by many rows leave most of the chip idle, but each
        // sharing costs its exchange (in steps of 0.8 us).
        static const float start[] = {6.f, 12.f, 13.f, 16.f};
        float best = 0.f;
        for (int i = 0; i < (cfg->head_dim == 128 ? 4 : 3); ++i) {
            const int nc = 1 << i;
            std::vector<float> cost;
            for (const padoc_cross_key_tile &t : b.tiles)
                if (t.steps) cost.push_back((float)ceil_div(t.steps, nc) + start[i]);
            const float time = makespan(cost, hkv, std::max(1, lanes / nc));
            if (i == 0 || time < best) {
                best = time;
                info.cluster = nc;
            }
        }
    }
    if ((int64_t)std::max(b.units.size(), std::max(b.dq_units.size(), b.tiles.size())) * hkv * 8 > INT32_MAX ||
        (int64_t)std::max(b.merges.size(), b.dq_merges.size()) * hkv * 64 > INT32_MAX)
        return PADOC_ERR_UNSUPPORTED;   // (grid sizes)

    int64_t at = 0;
    auto place = [&](size_t items, size_t bytes) {
        const int64_t off = at;
        at += (int64_t)(items * bytes / 4 + 31) / 32 * 32;
        return off;
    };
    info.num_units = (int32_t)b.units.size();
    info.num_merges = (int32_t)b.merges.size();
    info.num_dq_units = (int32_t)b.dq_units.size();
    info.num_dq_merges = (int32_t)b.dq_merges.size();
    info.num_key_tiles = (int32_t)b.tiles.size();
    info.num_covers = (int32_t)b.covers.size();
    info.off_units = place(b.units.size(), sizeof(padoc_cross_unit));
    info.off_merges = place(b.merges.size(), sizeof(padoc_cross_merge));
    info.off_dq_units = place(b.dq_units.size(), sizeof(padoc_cross_unit));
    info.off_dq_merges = place(b.dq_merges.size(), sizeof(padoc_cross_merge));
    info.off_key_tiles = place(b.tiles.size(), sizeof(padoc_cross_key_tile));
    info.off_covers = place(b.covers.size(), sizeof(padoc_cross_cover));
    info.plan_ints = at;
    return PADOC_OK;
}

padoc_status guarded(const Segment *seg, int32_t n, const padoc_cross_config *cfg, Built &b)
{
    try {
        return make(seg, n, cfg, b);
    } catch (...) {   // (out of memory: nothing leaves a C entry)
        return PADOC_ERR_CAPACITY;
    }
}

}  // namespace

extern "C" padoc_status padoc_cross_plan_size(const padoc_cross_segment *segments, int32_t num_segments,
                                              const padoc_cross_config *cfg, int64_t *plan_ints)
{
    if (!plan_ints) return PADOC_ERR_INVALID_ARGUMENT;
    Built b;
    const padoc_status st = guarded(segments, num_segments, cfg, b);
    if (st == PADOC_OK) *plan_ints = b.info.plan_ints;
    return st;
}

extern "C" padoc_status padoc_build_cross_plan(const padoc_cross_segment *segments, int32_t num_segments,
                                               const padoc_cross_config *cfg, int32_t *plan, int64_t capacity_ints,
                                               padoc_cross_plan *info)
{
    if (!info || capacity_ints < 0 || (capacity_ints > 0 && !plan)) return PADOC_ERR_INVALID_ARGUMENT;
    Built b;
    const padoc_status st = guarded(segments, num_segments, cfg, b);
    if (st != PADOC_OK) return st;
    if (capacity_ints < b.info.plan_ints) {
        *info = b.info;   // (its plan_ints says what is needed)
        return PADOC_ERR_CAPACITY;
    }
    if (b.info.plan_ints) memset(plan, 0, (size_t)b.info.plan_ints * 4);
    auto put = [&](int64_t off, const void *src, size_t bytes) {
        if (bytes) memcpy(plan + off, src, bytes);
    };
    put(b.info.off_units, b.units.data(), b.units.size() * sizeof(padoc_cross_unit));
    put(b.info.off_merges, b.merges.data(), b.merges.size() * sizeof(padoc_cross_merge));
    put(b.info.off_dq_units, b.dq_units.data(), b.dq_units.size() * sizeof(padoc_cross_unit));
    put(b.info.off_dq_merges, b.dq_merges.data(), b.dq_merges.size() * sizeof(padoc_cross_merge));
    put(b.info.off_key_tiles, b.tiles.data(), b.tiles.size() * sizeof(padoc_cross_key_tile));
    put(b.info.off_covers, b.covers.data(), b.covers.size() * sizeof(padoc_cross_cover));
    *info = b.info;
    return PADOC_OK;
}

extern "C" padoc_status padoc_cross_workspace_size(const padoc_cross_plan *info, size_t *bytes)
{
    if (!info || !bytes || info->num_slots < 0) return PADOC_ERR_INVALID_ARGUMENT;
    // partial outputs [slots][Hkv][256][d] and their log-sum-exps [slots][Hkv][256], fp32
    const size_t rows = (size_t)info->num_slots * info->cfg.num_kv_heads * (PADOC_CROSS_UNIT_BLOCKS * PADOC_CROSS_BLOCK);
    *bytes = rows * (info->cfg.head_dim + 1) * sizeof(float);
    return PADOC_OK;
}

extern "C" padoc_status padoc_cross_bwd_workspace_size(const padoc_cross_plan *info, size_t *bytes)
{
    if (!info || !bytes || !info->cfg.backward || info->num_dq_slots < 0 || info->num_subs < 0) return PADOC_ERR_INVALID_ARGUMENT;
    // -lse2 and D, [Hkv][subs][64] each, then partial dq [slots][Hkv][128][d], fp32
    const size_t stats = (size_t)info->num_subs * info->cfg.num_kv_heads * PADOC_CROSS_BLOCK;
    const size_t rows = (size_t)info->num_dq_slots * info->cfg.num_kv_heads * (PADOC_CROSS_DQ_BLOCKS * PADOC_CROSS_BLOCK);
    *bytes = (2 * stats + rows * info->cfg.head_dim) * sizeof(float);
    return PADOC_OK;
}
