// cross_plan.cpp -- the host planner of cross attention. Plans hold integers alone; the choices between them compare
// estimated times.
//
// Forward: every segment's rows are cut into chunks of 256 packed rows (128 with 64 dims), each with the segment's whole
// key range for every KV head. They are work items as they are, or those of the last round are cut, or the sequence of
// all steps is cut into runs of equal time, one for each SM; the parts of a chunk are joined. Backward: the dq pass has
// chunks of 128 rows cut the same way; the dk/dv pass has key tiles with the segments that see them, in equal runs too.
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

int32_t ceil_div(int64_t a, int64_t b) { return (int32_t)((a + b - 1) / b); }

// Costs of a pass, in units of one step of a full item.
struct Costs {
    float start;    // an item's start and end
    float part;     // what writing a partial result adds
    float merge;    // the launch that joins them, and ...
    float read;     // ... what reading a partial result adds to it
    float half;     // a step of an item that is at most half full
    int32_t step;   // keys of a step
    int32_t least;  // fewest steps of a piece that is cut off
};

// Rows of one segment that are worked on together, for every KV head.
struct Chunk {
    int32_t tok, ntok, k0, nk, steps, sub;
    float step_cost;
};

struct Work {
    std::vector<padoc_cross_unit> units;
    std::vector<padoc_cross_merge> merges;
    std::vector<int32_t> ctas;   // first item of each CTA's list, and the end; empty: no lists
    int32_t slots = 0, max_parts = 0;
};

// Time of items, longest first on `lanes` SMs: the greedy schedule that the launch order and the kernels'
// taking over of pending items come close to.
float makespan(std::vector<float> cost, int lanes)
{
    if (cost.empty()) return 0.f;
    std::sort(cost.begin(), cost.end(), std::greater<float>());
    if (cost.size() > (size_t)16 * lanes) {
        double total = 0;
        for (float c : cost) total += c;
        return (float)(total / lanes) + 0.5f * cost[0];
    }
    std::priority_queue<float, std::vector<float>, std::greater<float>> free;
    for (int i = 0; i < lanes; ++i) free.push(0.f);
    float end = 0.f;
    for (float c : cost) {
        const float t = free.top() + c;
        free.pop();
        free.push(t);
        end = std::max(end, t);
    }
    return end;
}

bool longer(const padoc_cross_unit &x, const padoc_cross_unit &y) { return x.nk > y.nk; }

struct Piece {
    int32_t chunk, g, first, steps, cta;
};

// The (chunk, KV head, step) sequence cut into runs of equal time, one for each CTA; false when `lanes` do not suffice
// for a time of `most` each.
bool cut_runs(const std::vector<Chunk> &chunks, int hkv, int lanes, const Costs &k, float most, std::vector<Piece> *out)
{
    int cta = 0;
    float used = 0.f;
    for (size_t c = 0; c < chunks.size(); ++c)
        for (int32_t g = 0; g < hkv; ++g)
            for (int32_t at = 0; at < chunks[c].steps;) {
                const Chunk &ch = chunks[c];
                const int32_t rem = ch.steps - at;
                const float whole = used + k.start + (at ? k.part : 0.f) + rem * ch.step_cost;
                int32_t take = rem;
                if (whole > most) {
                    take = (int32_t)((most - used - k.start - k.part) / ch.step_cost);
                    take = std::min(take, rem - std::min(rem, k.least));   // (what is left is a piece, too)
                    if (take < std::min(k.least, rem)) {
                        if (used == 0.f) return false;
                        ++cta;
                        used = 0.f;
                        if (cta >= lanes) return false;
                        continue;
                    }
                }
                if (out) out->push_back({(int32_t)c, g, at, take, cta});
                used += k.start + (take < ch.steps ? k.part : 0.f) + take * ch.step_cost;
                at += take;
            }
    return true;
}

void make_work(const std::vector<Chunk> &chunks, const std::vector<Piece> &pieces, const Costs &k, Work &w)
{
    for (size_t i = 0; i < pieces.size();) {
        size_t n = i + 1;
        while (n < pieces.size() && pieces[n].chunk == pieces[i].chunk && pieces[n].g == pieces[i].g) ++n;
        const Chunk &c = chunks[pieces[i].chunk];
        const int32_t parts = (int32_t)(n - i);
        if (parts > 1) w.merges.push_back({c.tok, c.ntok, w.slots, parts, pieces[i].g, {0, 0, 0}});
        w.max_parts = std::max(w.max_parts, parts > 1 ? parts : 0);
        for (size_t p = i; p < n; ++p) {
            const int32_t a = pieces[p].first * k.step, b = std::min(c.nk, (pieces[p].first + pieces[p].steps) * k.step);
            w.units.push_back({c.tok, c.ntok, c.k0 + a, b - a, pieces[p].g, parts > 1 ? w.slots + (int32_t)(p - i) : -1,
                               p == i ? c.sub : -1, 0});
        }
        if (parts > 1) w.slots += parts;
        i = n;
    }
}

// Whole chunks but for the shortest, those of the last round, cut so that they fill it (164 items of 8 steps on 152 SMs:
// 36.0 -> 33.5 us; not where the last round matters little: 2048 items of 20 steps 447 -> 457). Returns the time, which
// is `plain` where nothing is cut (out is empty then).
float cut_ends(const std::vector<Chunk> &chunks, const std::vector<Piece> &whole, const std::vector<float> &cost, int lanes,
               const Costs &k, double total, float plain, std::vector<Piece> &out)
{
    const size_t tail = whole.size() % (size_t)lanes;
    if (whole.size() <= (size_t)lanes || whole.size() > (size_t)16 * lanes || !tail || (float)(total / lanes) >= 0.95f * plain) return plain;
    std::vector<size_t> order(whole.size());
    for (size_t i = 0; i < order.size(); ++i) order[i] = i;
    std::stable_sort(order.begin(), order.end(), [&](size_t x, size_t y) { return cost[x] > cost[y]; });
    auto parts_of = [&](size_t i, int32_t p) { return std::min(p, std::max(1, whole[i].steps / k.least)); };
    float best = 0.97f * plain;
    int32_t into = 0;
    for (const int32_t p : {2, 3, 4, 6, 8, 12, 16}) {
        std::vector<float> time = cost;
        size_t cuts = 0;
        double sum = total;
        for (size_t o = order.size() - tail; o < order.size(); ++o) {
            const size_t i = order[o];
            const int32_t parts = parts_of(i, p);
            if (parts == 1) continue;
            sum -= time[i];
            const float part = ceil_div(whole[i].steps, parts) * chunks[whole[i].chunk].step_cost + k.start + k.part;
            time[i] = part;
            time.insert(time.end(), parts - 1, part);
            cuts += parts;
            sum += parts * part;
        }
        const float join = k.merge + k.read * (float)cuts;
        if (!cuts || (float)(sum / lanes) + join >= best) break;   // (more parts cost more)
        const float t = makespan(time, lanes) + join;
        if (t < best) {
            best = t;
            into = p;
        }
    }
    if (!into) return plain;
    std::vector<char> cut(whole.size(), 0);
    for (size_t o = order.size() - tail; o < order.size(); ++o) cut[order[o]] = 1;
    for (size_t i = 0; i < whole.size(); ++i) {
        const int32_t steps = whole[i].steps, parts = cut[i] ? parts_of(i, into) : 1;
        for (int32_t q = 0; q < parts; ++q) {
            const int32_t a = (int32_t)((int64_t)steps * q / parts), b = (int32_t)((int64_t)steps * (q + 1) / parts);
            out.push_back({whole[i].chunk, whole[i].g, a, b - a, 0});
        }
    }
    return best;
}

// The items of a pass: whole chunks, taken as SMs get free, the last ones perhaps cut, or, where that leaves the chip idle,
// equal runs of the sequence of all steps, a list for each CTA, with chunks cut where a run ends. kPieces (fp32, whose kernels run a
// CTA per 64 rows): the runs' pieces without the lists.
enum Cuts { kPieces, kLists };
float plan_work(const std::vector<Chunk> &chunks, int hkv, int lanes, const Costs &k, Cuts cuts_allowed, Work &w)
{
    std::vector<float> cost;
    std::vector<Piece> whole;
    double total = 0;
    float longest = 0.f;
    for (size_t c = 0; c < chunks.size(); ++c)
        for (int32_t g = 0; g < hkv; ++g) {
            cost.push_back(chunks[c].steps * chunks[c].step_cost + k.start);
            whole.push_back({(int32_t)c, g, 0, chunks[c].steps, 0});
            total += cost.back();
            longest = std::max(longest, cost.back());
        }
    if (chunks.empty()) return 0.f;
    float plain = makespan(cost, lanes);
    const float lowest = (float)(total / lanes);
    std::vector<Piece> ends;
    plain = cut_ends(chunks, whole, cost, lanes, k, total, plain, ends);
    float lo = lowest, hi = std::max(longest, 2.f * lo) + 4.f * (k.start + k.part);
    if (lo < 0.97f * plain && cut_runs(chunks, hkv, lanes, k, hi, nullptr)) {
        for (int i = 0; i < 16 && hi - lo > 0.01f * hi; ++i) {
            const float mid = 0.5f * (lo + hi);
            (cut_runs(chunks, hkv, lanes, k, mid, nullptr) ? hi : lo) = mid;
        }
        std::vector<Piece> pieces;
        cut_runs(chunks, hkv, lanes, k, hi, &pieces);
        // (the merge's reads: two parts or more of each row block that was cut)
        const size_t cuts = pieces.size() - whole.size();
        const float time = hi + (cuts ? k.merge + k.read * (float)(cuts + std::min(cuts, whole.size())) : 0.f);
        if (time < 0.97f * plain) {
            make_work(chunks, pieces, k, w);
            if (cuts_allowed == kLists) {
                for (size_t i = 0; i < pieces.size(); ++i)
                    while ((int32_t)w.ctas.size() <= pieces[i].cta) w.ctas.push_back((int32_t)i);
                w.ctas.push_back((int32_t)pieces.size());
            } else {
                std::stable_sort(w.units.begin(), w.units.end(), longer);
            }
            return time;
        }
    }
    make_work(chunks, ends.empty() ? whole : ends, k, w);
    std::stable_sort(w.units.begin(), w.units.end(), longer);
    return plain;
}

struct Built {
    Work fwd, dq;
    std::vector<padoc_cross_key_tile> tiles;
    std::vector<padoc_cross_cover> covers;
    std::vector<padoc_cross_dkv> dkv;
    std::vector<int32_t> dkv_ctas;
    std::vector<padoc_cross_dkv_sum> sums;
    padoc_cross_plan info;
};

// The dk/dv pass's items: key tiles, or parts of their steps, in a list for each CTA. Costs in steps (0.7 us with 128
// dims, 0.6 with 64, where cheaper cuts were better: 2 pages of 1500 rows over 400 states 19.5 -> 17.2 us). More tiles
// than CTAs: whole ones, those of the last round cut where that pays, longest first to the CTA that is free first. They
// all begin with a segment's first rows, which the CTAs thus fetch at about the same time: equal runs of all steps, in
// which every CTA begins elsewhere, took 1750 us instead of 1640 for 320 tiles of 512 steps. Else equal runs, where they
// are shorter (120 tiles of up to 184 steps, 9510 in all, by clusters of CTAs 82 us, in runs 69 and their sums 8).
void plan_dkv(Built &b, int hkv, int lanes, int head_dim)
{
    const Costs k = head_dim == 128 ? Costs{5.f, 2.f, 5.f, 0.02f, 1.f, 1, 4} : Costs{4.f, 1.f, 5.f, 0.01f, 1.f, 1, 4};
    std::vector<Chunk> chunks;
    std::vector<Piece> pieces;
    std::vector<float> cost;
    double total = 0;
    for (const padoc_cross_key_tile &t : b.tiles)
        if (t.steps) {
            for (int32_t g = 0; g < hkv; ++g) {
                pieces.push_back({(int32_t)chunks.size(), g, 0, t.steps, 0});
                cost.push_back(t.steps + k.start);
                total += t.steps + k.start;
            }
            chunks.push_back({t.k0, t.nk, t.cover, 0, t.steps, 0, 1.f});
        }
    if (pieces.empty()) return;
    float plain = makespan(cost, lanes);
    bool runs = false;
    if (pieces.size() > (size_t)lanes) {
        std::vector<Piece> ends;
        cut_ends(chunks, pieces, cost, lanes, k, total, plain, ends);
        if (!ends.empty()) pieces = ends;
    } else {
        float lo = (float)(total / lanes), hi = std::max(plain, 2.f * lo) + 4.f * (k.start + k.part);
        if (lo < 0.97f * plain && cut_runs(chunks, hkv, lanes, k, hi, nullptr)) {
            for (int i = 0; i < 16 && hi - lo > 0.01f * hi; ++i) {
                const float mid = 0.5f * (lo + hi);
                (cut_runs(chunks, hkv, lanes, k, mid, nullptr) ? hi : lo) = mid;
            }
            std::vector<Piece> cut;
            cut_runs(chunks, hkv, lanes, k, hi, &cut);
            const size_t cuts = cut.size() - pieces.size();
            if (hi + (cuts ? k.merge + k.read * (float)(cuts + std::min(cuts, pieces.size())) : 0.f) < 0.97f * plain) {
                pieces = cut;
                runs = true;
            }
        }
    }
    std::vector<int32_t> place(pieces.size());   // the lists' order
    for (size_t i = 0; i < pieces.size(); ++i) place[i] = (int32_t)i;
    if (!runs) {
        std::stable_sort(place.begin(), place.end(), [&](int32_t x, int32_t y) { return pieces[x].steps > pieces[y].steps; });
        std::priority_queue<std::pair<float, int32_t>, std::vector<std::pair<float, int32_t>>, std::greater<std::pair<float, int32_t>>> free;
        for (int32_t c = 0; c < lanes; ++c) free.push({0.f, c});
        for (const int32_t i : place) {
            const std::pair<float, int32_t> f = free.top();
            free.pop();
            pieces[i].cta = f.second;
            free.push({f.first + pieces[i].steps + k.start, f.second});
        }
    }
    // slots in the order of the tiles' steps, then the lists
    std::vector<padoc_cross_dkv> items;
    for (size_t i = 0; i < pieces.size();) {
        size_t n = i + 1;
        while (n < pieces.size() && pieces[n].chunk == pieces[i].chunk && pieces[n].g == pieces[i].g) ++n;
        const Chunk &c = chunks[pieces[i].chunk];
        const int32_t parts = (int32_t)(n - i);
        if (parts > 1) b.sums.push_back({c.tok, c.ntok, pieces[i].g, b.info.num_dkv_slots, parts, {0, 0, 0}});
        for (size_t p = i; p < n; ++p)
            items.push_back({c.tok, c.ntok, c.k0, pieces[p].first, pieces[p].steps, pieces[p].g,
                             parts > 1 ? b.info.num_dkv_slots++ : -1, 0});
        i = n;
    }
    std::stable_sort(place.begin(), place.end(), [&](int32_t x, int32_t y) { return pieces[x].cta < pieces[y].cta; });
    for (size_t i = 0; i < place.size(); ++i) {
        if (i == 0 || pieces[place[i]].cta != pieces[place[i - 1]].cta) b.dkv_ctas.push_back((int32_t)i);
        b.dkv.push_back(items[place[i]]);
    }
    b.dkv_ctas.push_back((int32_t)b.dkv.size());
}

padoc_status check(const Segment *seg, int32_t n, const padoc_cross_config *cfg)
{
    if (!cfg || n < 0 || (n > 0 && !seg)) return PADOC_ERR_INVALID_ARGUMENT;
    if (cfg->num_q_heads < 1 || cfg->num_kv_heads < 1 || cfg->num_q_heads % cfg->num_kv_heads || cfg->ctas < 0 || cfg->ctas > 65535 ||
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

// The forward's items for few rows, where that is faster than `time` (us): 16 or 32 rows an item, by clusters of 1 to 8
// CTAs that join their parts of the keys themselves, or keys cut into parts.
//
// Both sides, in us (these items / those of 256 rows, with 64 dims 128):
//                                                   16 + 2 of 128     8 + 8 of 128     16 + 16 of 64
//   672 streams, each over 100 to 500 states           36 / 64          128 / 228        143 / 187
//   ... over 300 to 1200                               56 / 97          244 / 354        257 / 316
//   32 pages of up to 1201 states, 2 streams each      11 / 16           26 / 33          27 / 31
//   ... 8 streams                                      20 / 16           25 / 31          27 / 31
//   ... 30 streams                                     43 / 25           34 / 32          35 / 30
//   ... 64 rows                                        81 / 25           46 / 34          49 / 32
// The estimate takes the faster side but for 128 dims with a token an item and some 200 states and more (56 / 97 and
// 244 / 354: it counts the keys' bytes at the memory's rate, while crops of one page come from L2) and pages of up to 16
// streams under 8 + 8 heads (25 / 31).
template <typename F>
void plan_few(const Segment *seg, int32_t n, int32_t group, int32_t head_dim, int32_t hkv, int32_t sms, float time,
              const F &chunks_of, Work &fwd, padoc_cross_plan &info, int32_t &per)
{
    int32_t most = 0;   // rows of the largest segment
    for (int32_t i = 0; i < n; ++i)
        if (seg[i].k_len) most = std::max(most, std::min(seg[i].q_len, 2 * PADOC_CROSS_FEW_ROWS) * group);
    const int32_t rows = most <= 16 ? 16 : PADOC_CROSS_FEW_ROWS;
    const int32_t an_sm = head_dim == 64 ? 3 : 2, lanes = sms * an_sm;   // CTAs
    // Many blocks of rows, each reading the keys anew, do not win (32 pages of 128 rows over up to 1201 states: 149 us against
    // 37, over up to 60 states 56 against 16, 16 heads of 64 dims 84 against 32). Items of a token each would (2500 streams
    // of 16 heads of 64 dims over 60 to 200 states: 326 us against 510), but planning these 40000 takes 12 ms instead of 4.
    int64_t items = 0;
    for (int32_t i = 0; i < n; ++i)
        if (seg[i].k_len) items += ((int64_t)seg[i].q_len * group + rows - 1) / rows * hkv;
    if (items > (most > PADOC_CROSS_FEW_ROWS ? 4 : 64) * (int64_t)lanes) return;
    const float step = (float)an_sm * PADOC_CROSS_FEW_STEP * head_dim * 4 / 45e3f;
    const Costs k = {3.f / step, 0.3f / step, 3.f / step, 0.001f / step, 1.f, PADOC_CROSS_FEW_STEP, 2};
    const std::vector<Chunk> chunks = chunks_of(rows / group, k);
    Work w;
    int few = 1;
    float best = step * plan_work(chunks, hkv, lanes, k, kPieces, w);
    bool parts = w.slots > 0;
    for (int nc = 1; nc <= 8; nc *= 2) {
        std::vector<float> cost;
        for (const Chunk &c : chunks)
            for (int32_t g = 0; g < hkv; ++g) cost.push_back(ceil_div(c.steps, nc) + (nc > 1 ? 1.f / step : 0.f) + k.start);
        const float t = step * makespan(cost, std::max(1, lanes / nc));
        if (t < best) {
            best = t;
            few = nc;
            parts = false;
        }
    }
    if (best >= time) return;
    if (!parts) {
        w = Work();
        std::vector<Piece> whole;
        for (size_t c = 0; c < chunks.size(); ++c)
            for (int32_t g = 0; g < hkv; ++g) whole.push_back({(int32_t)c, g, 0, chunks[c].steps, 0});
        make_work(chunks, whole, k, w);
        std::stable_sort(w.units.begin(), w.units.end(), longer);
    }
    fwd = w;
    info.few = few;
    info.unit_rows = rows;
    per = rows / group;
}

padoc_status make(const Segment *seg, int32_t n, const padoc_cross_config *cfg, Built &b)
{
    const padoc_status st = check(seg, n, cfg);
    if (st != PADOC_OK) return st;
    memset(&b.info, 0, sizeof(b.info));
    padoc_cross_plan &info = b.info;
    info.cfg = *cfg;
    info.num_segments = n;
    const int32_t hkv = cfg->num_kv_heads, group = cfg->num_q_heads / hkv, block = PADOC_CROSS_BLOCK / group;
    const int32_t sms = cfg->ctas ? cfg->ctas : padoc_default_ctas();
    const bool f32 = cfg->dtype == PADOC_DTYPE_F32;

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

    auto chunks_of = [&](int32_t per, const Costs &k) {   // of `per` tokens
        std::vector<Chunk> c;
        for (int32_t i = 0; i < n; ++i) {
            if (seg[i].q_len == 0 || seg[i].k_len == 0) continue;
            for (int32_t t = 0; t < seg[i].q_len; t += per) {
                const int32_t m = std::min(per, seg[i].q_len - t);
                c.push_back({seg[i].q_begin + t, m, seg[i].k_begin, seg[i].k_len, ceil_div(seg[i].k_len, k.step),
                             first_sub[i] + t / block, m <= per / 2 ? k.half : 1.f});
            }
        }
        return c;
    };
    auto empty_rows = [&](int32_t per, std::vector<padoc_cross_merge> &merges) {
        for (int32_t i = 0; i < n; ++i)
            if (seg[i].k_len == 0)
                for (int32_t t = 0; t < seg[i].q_len; t += per)
                    for (int32_t g = 0; g < hkv; ++g)
                        merges.push_back({seg[i].q_begin + t, std::min(per, seg[i].q_len - t), 0, 0, g, {0, 0, 0}});
    };
    const Cuts cuts = f32 ? kPieces : kLists;
    // fp32: a CTA per 64 rows, 5 us a 64-key step with 64 dims and 8 with 128 (the backward's half as long again)
    const Costs simt = {0.5f, 0.2f, 0.6f, 0.002f, 1.f, 64, 1};

    // Forward. Times in us: of two 128-row tiles' steps of 128 keys, and for few rows of a 64-key tile's bytes at the
    // SM's share of the memory bandwidth (45 KB a us), which its CTAs share.
    // With 64 dims an item is one tile and two CTAs share an SM.
    const int32_t an_sm = !f32 && cfg->head_dim == 64 ? 2 : 1, unit_blocks = PADOC_CROSS_UNIT_BLOCKS / an_sm;
    int32_t per = unit_blocks * block;
    {
        const Costs tc = {1.8f, 1.5f, 2.f, 0.012f / an_sm, an_sm == 2 ? 1.f : 0.65f, PADOC_CROSS_KEY_TILE, 1};
        const Costs &k = f32 ? simt : tc;
        const int32_t lanes = f32 ? std::max(1, sms / PADOC_CROSS_UNIT_BLOCKS) : sms * an_sm;
        const float time = 1.65f * plan_work(chunks_of(per, k), hkv, lanes, k, cuts, b.fwd);
        info.unit_rows = unit_blocks * PADOC_CROSS_BLOCK;
        if (!f32 && group <= PADOC_CROSS_FEW_ROWS && !b.fwd.units.empty())
            plan_few(seg, n, group, cfg->head_dim, hkv, sms, time, chunks_of, b.fwd, info, per);
    }
    empty_rows(per, b.fwd.merges);

    if (cfg->backward) {
        const Costs bwd = {6.f, 2.f, 6.f, 0.018f, 1.f, PADOC_CROSS_DQ_STEP, 4};   // (a step of a tile lasts about 0.55 us)
        const Costs &k = f32 ? simt : bwd;
        const int32_t lanes = f32 ? std::max(1, sms / PADOC_CROSS_DQ_BLOCKS) : sms;
        plan_work(chunks_of(PADOC_CROSS_DQ_BLOCKS * block, k), hkv, lanes, k, cuts, b.dq);
        empty_rows(PADOC_CROSS_DQ_BLOCKS * block, b.dq.merges);

        // Key tiles: ranges that overlap are tiled together, from the first one's begin; between them lie keys that
        // nobody sees.
        std::vector<int32_t> order;   // segments by their first key
        for (int32_t i = 0; i < n; ++i)
            if (seg[i].q_len && seg[i].k_len) order.push_back(i);
        std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return seg[x].k_begin < seg[y].k_begin; });
        std::vector<int32_t> live;    // segments that may see the tile, in their own order
        auto end_of = [&](int32_t i) { return seg[i].k_begin + seg[i].k_len; };
        size_t next = 0;
        auto add_tile = [&](int32_t k0, int32_t k1) {
            live.erase(std::remove_if(live.begin(), live.end(), [&](int32_t i) { return end_of(i) <= k0; }), live.end());
            for (; next < order.size() && seg[order[next]].k_begin < k1; ++next)
                live.insert(std::lower_bound(live.begin(), live.end(), order[next]), order[next]);
            int64_t steps = 0;
            const int32_t cover = (int32_t)b.covers.size();
            for (int32_t i : live) {
                const int32_t m = ceil_div(seg[i].q_len, block), c0 = std::max(k0, seg[i].k_begin);
                b.covers.push_back({seg[i].q_begin, seg[i].q_len, first_sub[i], m, c0, std::min(k1, end_of(i)) - c0, {0, 0}});
                steps += m;
            }
            b.tiles.push_back({k0, k1 - k0, cover, (int32_t)live.size(), (int32_t)steps, {0, 0, 0}});
        };
        int32_t at = 0;               // keys tiled so far
        for (size_t i = 0; i < order.size();) {
            const int32_t begin = seg[order[i]].k_begin;
            int32_t end = end_of(order[i]);
            for (++i; i < order.size() && seg[order[i]].k_begin < end; ++i) end = std::max(end, end_of(order[i]));
            for (; at < begin; at = std::min(begin, at + PADOC_CROSS_KEY_TILE)) add_tile(at, std::min(begin, at + PADOC_CROSS_KEY_TILE));
            for (; at < end; at = std::min(end, at + PADOC_CROSS_KEY_TILE)) {
                add_tile(at, std::min(end, at + PADOC_CROSS_KEY_TILE));
                if (b.covers.size() > (size_t)1 << 24) return PADOC_ERR_UNSUPPORTED;
            }
        }
        std::stable_sort(b.tiles.begin(), b.tiles.end(),
                         [](const padoc_cross_key_tile &x, const padoc_cross_key_tile &y) { return x.steps > y.steps; });
        info.num_subs = (int32_t)subs;

        for (const padoc_cross_key_tile &t : b.tiles) info.num_gap_tiles += t.steps == 0;
        if (f32) {
            // The CTAs that share a key tile's steps: few tiles seen by many rows leave most of the chip idle, but each
            // sharing costs its exchange (in steps of 12 us; two clusters a tile).
            static const float start[] = {0.4f, 0.6f, 0.6f, 0.7f};
            float best = 0.f;
            for (int i = 0; i < 4; ++i) {
                const int nc = 1 << i;
                std::vector<float> cost;
                for (const padoc_cross_key_tile &t : b.tiles)
                    for (int32_t g = 0; g < hkv && t.steps; ++g) cost.push_back((float)ceil_div(t.steps, nc) + start[i]);
                const float time = makespan(cost, std::max(1, lanes / nc));
                if (i == 0 || time < best) {
                    best = time;
                    info.cluster = nc;
                }
            }
        } else {
            plan_dkv(b, hkv, sms, cfg->head_dim);
        }
    }
    if ((int64_t)b.sums.size() * PADOC_CROSS_KEY_TILE * cfg->head_dim > INT32_MAX ||
        (int64_t)std::max(b.fwd.units.size(), b.dq.units.size()) * 4 > INT32_MAX || (int64_t)b.tiles.size() * hkv * 8 > INT32_MAX ||
        (int64_t)std::max(b.fwd.merges.size(), b.dq.merges.size()) * 512 > INT32_MAX)
        return PADOC_ERR_UNSUPPORTED;   // (grid sizes)

    int64_t at = 0;
    auto place = [&](size_t items, size_t bytes) {
        const int64_t off = at;
        at += (int64_t)(items * bytes / 4 + 31) / 32 * 32;
        return off;
    };
    info.num_units = (int32_t)b.fwd.units.size();
    info.num_ctas = b.fwd.ctas.empty() ? 0 : (int32_t)b.fwd.ctas.size() - 1;
    info.num_merges = (int32_t)b.fwd.merges.size();
    info.num_slots = b.fwd.slots;
    info.max_parts = b.fwd.max_parts;
    info.num_dq_units = (int32_t)b.dq.units.size();
    info.num_dq_ctas = b.dq.ctas.empty() ? 0 : (int32_t)b.dq.ctas.size() - 1;
    info.num_dq_merges = (int32_t)b.dq.merges.size();
    info.num_dq_slots = b.dq.slots;
    info.max_dq_parts = b.dq.max_parts;
    info.num_key_tiles = (int32_t)b.tiles.size();
    info.num_covers = (int32_t)b.covers.size();
    info.off_units = place(b.fwd.units.size(), sizeof(padoc_cross_unit));
    info.off_ctas = place(b.fwd.ctas.size(), sizeof(int32_t));
    info.off_merges = place(b.fwd.merges.size(), sizeof(padoc_cross_merge));
    info.off_dq_units = place(b.dq.units.size(), sizeof(padoc_cross_unit));
    info.off_dq_ctas = place(b.dq.ctas.size(), sizeof(int32_t));
    info.off_dq_merges = place(b.dq.merges.size(), sizeof(padoc_cross_merge));
    info.off_key_tiles = place(b.tiles.size(), sizeof(padoc_cross_key_tile));
    info.off_covers = place(b.covers.size(), sizeof(padoc_cross_cover));
    info.num_dkv_units = (int32_t)b.dkv.size();
    info.num_dkv_ctas = b.dkv_ctas.empty() ? 0 : (int32_t)b.dkv_ctas.size() - 1;
    info.num_dkv_sums = (int32_t)b.sums.size();
    info.off_dkv = place(b.dkv.size(), sizeof(padoc_cross_dkv));
    info.off_dkv_ctas = place(b.dkv_ctas.size(), sizeof(int32_t));
    info.off_dkv_sums = place(b.sums.size(), sizeof(padoc_cross_dkv_sum));
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
    put(b.info.off_units, b.fwd.units.data(), b.fwd.units.size() * sizeof(padoc_cross_unit));
    put(b.info.off_ctas, b.fwd.ctas.data(), b.fwd.ctas.size() * sizeof(int32_t));
    put(b.info.off_merges, b.fwd.merges.data(), b.fwd.merges.size() * sizeof(padoc_cross_merge));
    put(b.info.off_dq_units, b.dq.units.data(), b.dq.units.size() * sizeof(padoc_cross_unit));
    put(b.info.off_dq_ctas, b.dq.ctas.data(), b.dq.ctas.size() * sizeof(int32_t));
    put(b.info.off_dq_merges, b.dq.merges.data(), b.dq.merges.size() * sizeof(padoc_cross_merge));
    put(b.info.off_key_tiles, b.tiles.data(), b.tiles.size() * sizeof(padoc_cross_key_tile));
    put(b.info.off_covers, b.covers.data(), b.covers.size() * sizeof(padoc_cross_cover));
    put(b.info.off_dkv, b.dkv.data(), b.dkv.size() * sizeof(padoc_cross_dkv));
    put(b.info.off_dkv_ctas, b.dkv_ctas.data(), b.dkv_ctas.size() * sizeof(int32_t));
    put(b.info.off_dkv_sums, b.sums.data(), b.sums.size() * sizeof(padoc_cross_dkv_sum));
    *info = b.info;
    return PADOC_OK;
}

extern "C" padoc_status padoc_cross_workspace_size(const padoc_cross_plan *info, size_t *bytes)
{
    if (!info || !bytes || info->num_slots < 0 || info->unit_rows < 0) return PADOC_ERR_INVALID_ARGUMENT;
    // partial outputs [slots][unit_rows][d] and their log-sum-exps [slots][unit_rows], fp32
    const size_t rows = (size_t)info->num_slots * info->unit_rows;
    *bytes = rows * (info->cfg.head_dim + 1) * sizeof(float);
    return PADOC_OK;
}

extern "C" padoc_status padoc_cross_bwd_workspace_size(const padoc_cross_plan *info, size_t *bytes)
{
    if (!info || !bytes || !info->cfg.backward || info->num_dq_slots < 0 || info->num_subs < 0 || info->num_dkv_slots < 0)
        return PADOC_ERR_INVALID_ARGUMENT;
    // -lse2 and D (bf16: four words), [Hkv][subs][64] each, partial dq [slots][128][d], partial dv and dk [slots][128][2 d], fp32
    const bool f32 = info->cfg.dtype == PADOC_DTYPE_F32;
    const size_t stats = (size_t)info->num_subs * info->cfg.num_kv_heads * PADOC_CROSS_BLOCK;
    const size_t rows = (size_t)info->num_dq_slots * (PADOC_CROSS_DQ_BLOCKS * PADOC_CROSS_BLOCK);
    const size_t keys = (size_t)info->num_dkv_slots * PADOC_CROSS_KEY_TILE * 2;
    *bytes = ((f32 ? 2 : 5) * stats + (rows + keys) * info->cfg.head_dim) * sizeof(float);
    return PADOC_OK;
}
