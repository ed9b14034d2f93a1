// rotary.cuh -- rotary positions with several axes and the per-head RMS norm before them, as device
// helpers shared by the packed forward and backward, the append into the paged pool and the E4M3 append.
//
// A head of d dims is taken in chunks of 2 V dims, one lane each, as two vectors of V: chunk c holds the dims from
// c V and from R/2 + c V on (R rotated dims), or, behind the rotated ones, the same of the remaining d - R. So the
// lanes' vectors lie behind one another (side by side in a lane, each access would touch every sector for half of
// it: the packed backward with norms 96 us instead of 62 for 26041 rows). Of pairs (i, i + R/2) a lane holds both
// members, V pairs from c V on; of adjacent pairs V/2 from c V/2 and V/2 from R/4 + c V/2 on. A lane's V angles serve
// every head of its row.
#pragma once

#include "common.cuh"
#include "tc.cuh"

namespace padoc_rotary_dev {

// Arguments of a head's norm and rotation.
struct Spec {
    const uint64_t *freq;        // [rot / 2]
    const void *q_weight, *k_weight;
    float eps, cos_amplitude, sin_amplitude;   // (the sine's negated: the rotation back)
    int32_t d, rot, axes;
};

// The cosine and sine of one pair's angle, times their amplitudes. A table entry holds the fraction of a
// turn per position unit as a 64-bit integer, its axis in the two lowest bits; times a 32-bit position it
// wraps modulo a whole turn. The product is cut at 2^-32 of a turn, and the entry is at most 2^-54 of a turn off
// (frequencies from 0 to 1 radian a position: two fp64 roundings, then 62 bits), so an angle a million tokens away is
// 2^-31.7 of a turn off, one at 2^31 2^-23 (a product in fp32 would be off by 0.06 rad at 10^6).
__device__ __forceinline__ float half_turns(uint64_t f, const int32_t *__restrict__ pos, int32_t axes)
{
    const int32_t p = pos[min((int32_t)(f & 3u), axes - 1)];   // (a table of more axes than the rows have stays in the row)
    const int32_t t = (int32_t)(((f & ~(uint64_t)3) * (uint64_t)(int64_t)p) >> 32);
    return (float)t * 0x1p-31f;   // in [-1, 1], 24 bits (the last 64 values of t round up to 1): the angle is pi times this
}
// kFast (outputs of 16 bits or fewer): the hardware's sine and cosine, each 2^-20.5 off at most (absolute, on [-pi, pi]; at
// half a turn the fp32 pi lies 2^-23.5 past it, where a test holds the same bound). A turned value u c - v s is off by
// that times |u| + |v|: 2^-11.5 or less of the half step by which a bf16 value of that size is rounded, and more than a
// half step where the two terms cancel to less than 2^-11.5 of it. Else CUDA's sincospif, within 2 units of the last place, which
// takes some 40 instructions more a pair.
template <bool kFast>
__device__ __forceinline__ void cos_sin(uint64_t f, const int32_t *__restrict__ pos, const Spec &sp, float &c, float &s)
{
    const float t = half_turns(f, pos, sp.axes);
    if constexpr (kFast) __sincosf(t * 3.14159265358979f, &s, &c);
    else sincospif(t, &s, &c);
    c *= sp.cos_amplitude;
    s *= sp.sin_amplitude;
}

// V consecutive elements, as they are stored and as fp32.
template <typename T, int V>
struct Raw;
template <>
struct Raw<__nv_bfloat16, 8> {
    uint4 w;
};
template <>
struct Raw<__nv_bfloat16, 4> {
    uint2 w;
};
template <>
struct Raw<float, 4> {
    float4 w;
};
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> load_raw(const T *p)
{
    Raw<T, V> r;
    r.w = *reinterpret_cast<const decltype(r.w) *>(p);
    return r;
}
__device__ __forceinline__ void widen(uint32_t w, float &lo, float &hi)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16, 8> &r, float (&x)[8])
{
    widen(r.w.x, x[0], x[1]), widen(r.w.y, x[2], x[3]), widen(r.w.z, x[4], x[5]), widen(r.w.w, x[6], x[7]);
}
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16, 4> &r, float (&x)[4])
{
    widen(r.w.x, x[0], x[1]), widen(r.w.y, x[2], x[3]);
}
__device__ __forceinline__ void unpack(const Raw<float, 4> &r, float (&x)[4])
{
    x[0] = r.w.x, x[1] = r.w.y, x[2] = r.w.z, x[3] = r.w.w;
}
// The same as packed pairs of fp32 (f2_*: one instruction for two values).
template <typename T, int V>
__device__ __forceinline__ void unpack2(const Raw<T, V> &r, uint64_t (&x)[V / 2])
{
    float f[V];
    unpack(r, f);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) x[j] = f2_pack(f[2 * j], f[2 * j + 1]);
}
template <int V>
__device__ __forceinline__ void store_vec(__nv_bfloat16 *p, const float (&x)[V])
{
    uint32_t w[V / 2];
#pragma unroll
    for (int j = 0; j < V / 2; ++j) w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
    if constexpr (V == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}
template <int V>
__device__ __forceinline__ void store_vec(float *p, const float (&x)[V])
{
    *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
template <int V, typename T>
__device__ __forceinline__ void store_vec2(T *p, const uint64_t (&x)[V / 2])
{
    float f[V];
#pragma unroll
    for (int j = 0; j < V / 2; ++j) f2_unpack(x[j], f[2 * j], f[2 * j + 1]);
    store_vec<V>(p, f);
}

// The lanes of a warp: `group` lanes share a head (kGroup of them where known at compile time, a power of two), as many
// heads as fit side by side; lanes behind the last one hold no dims.
struct Lane {
    int group, heads, sub, chunk;
    bool used;
};
template <int kGroup>
__device__ __forceinline__ Lane warp_lane(int group)
{
    const int lane = threadIdx.x & 31;
    Lane l;
    l.group = kGroup ? kGroup : group;
    l.heads = 32 / l.group;
    l.sub = lane / l.group;
    l.used = kGroup || l.sub < l.heads;
    if (!l.used) l.sub = 0;
    l.chunk = l.used ? lane - l.sub * l.group : 0;
    return l;
}
// Sum over the lanes that share a head, the same bits in each of them.
template <int kGroup>
__device__ __forceinline__ float group_sum(float v, const Lane &l)
{
    if constexpr (kGroup != 0) {
#pragma unroll
        for (int m = kGroup / 2; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    } else {   // after step m a lane has the sum of its own and the 2 m - 1 lanes behind it in the head
#pragma unroll
        for (int m = 1; m < 32; m <<= 1)
            if (m < l.group) {
                const float t = __shfl_down_sync(0xffffffffu, v, m);
                if (l.chunk + m < l.group) v += t;
            }
        v = __shfl_sync(0xffffffffu, v, (threadIdx.x & 31) - l.chunk);
    }
    return v;
}

// A lane's place in a head: the element offsets of its two vectors (lanes without dims: the first lane's), whether
// they are its own and are rotated.
struct Place {
    int a, b;
    bool active, turned;
};
template <int V>
__device__ __forceinline__ Place lane_place(int chunk, bool used, int d, int rot)
{
    Place p;
    p.active = used;
    p.turned = chunk * 2 * V < rot;
    p.a = p.turned ? chunk * V : rot / 2 + chunk * V;   // (R + (c - R / 2V) V)
    p.b = p.a + (p.turned ? rot : d - rot) / 2;
    return p;
}
// The pair that a lane's angle j belongs to.
template <int V, bool kAdjacent>
__device__ __forceinline__ int lane_pair(int chunk, int j, int rot)
{
    if constexpr (!kAdjacent) return chunk * V + j;
    else return chunk * (V / 2) + (j < V / 2 ? j : rot / 4 + j - V / 2);
}

// The rotation of a lane's V pairs by its angles; pairs (i, i + R / 2) on packed values, adjacent ones one by one.
template <int V, bool kAdjacent>
__device__ __forceinline__ void turn_pairs(uint64_t (&a)[V / 2], uint64_t (&b)[V / 2], const uint64_t (&c)[V / 2], const uint64_t (&s)[V / 2])
{
    if constexpr (!kAdjacent) {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            const uint64_t x = f2_sub(f2_mul(a[j], c[j]), f2_mul(b[j], s[j]));
            b[j] = f2_fma(b[j], c[j], f2_mul(a[j], s[j]));
            a[j] = x;
        }
    } else {
        float fa[V], fb[V], fc[V], fs[V];
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            f2_unpack(a[j], fa[2 * j], fa[2 * j + 1]);
            f2_unpack(b[j], fb[2 * j], fb[2 * j + 1]);
            f2_unpack(c[j], fc[2 * j], fc[2 * j + 1]);
            f2_unpack(s[j], fs[2 * j], fs[2 * j + 1]);
        }
        auto turn = [](float &x, float &y, float cc, float ss) {
            const float x0 = x, y0 = y;
            x = fmaf(x0, cc, -(y0 * ss));
            y = fmaf(y0, cc, x0 * ss);
        };
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            turn(fa[2 * j], fa[2 * j + 1], fc[j], fs[j]);
            turn(fb[2 * j], fb[2 * j + 1], fc[V / 2 + j], fs[V / 2 + j]);
        }
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            a[j] = f2_pack(fa[2 * j], fa[2 * j + 1]);
            b[j] = f2_pack(fb[2 * j], fb[2 * j + 1]);
        }
    }
}
__device__ __forceinline__ float f2_sum(uint64_t v)
{
    float lo, hi;
    f2_unpack(v, lo, hi);
    return lo + hi;
}

// RMS norm of a head spread over `group` lanes: x r w with r = 1 / sqrt(mean x^2 + eps), sums in fp32. `here`:
// the lane holds dims of a head.
template <int V, int kGroup>
__device__ __forceinline__ float norm_scale(const uint64_t (&a)[V / 2], const uint64_t (&b)[V / 2], bool here, const Spec &sp, const Lane &l)
{
    uint64_t ss = 0;
#pragma unroll
    for (int j = 0; j < V / 2; ++j) ss = f2_fma(a[j], a[j], f2_fma(b[j], b[j], ss));
    return rsqrtf(group_sum<kGroup>(here ? f2_sum(ss) : 0.f, l) * (1.f / (float)sp.d) + sp.eps);
}
template <int V, typename T>
__device__ __forceinline__ void scale_head(uint64_t (&a)[V / 2], uint64_t (&b)[V / 2], float r, const Raw<T, V> &rwa, const Raw<T, V> &rwb)
{
    uint64_t wa[V / 2], wb[V / 2];
    unpack2(rwa, wa);
    unpack2(rwb, wb);
    const uint64_t r2 = f2_pack(r, r);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        a[j] = f2_mul(a[j], f2_mul(r2, wa[j]));
        b[j] = f2_mul(b[j], f2_mul(r2, wb[j]));
    }
}

// The cosines and sines of a lane's V pairs at a row's positions; for the whole warp. The lanes that hold the same chunk
// of different heads share the work where there are enough of them: each computes kOwn pairs and hands them to the
// others.
template <int V, bool kAdjacent, bool kFast, int kOwn>
__device__ __forceinline__ void shared_angles(const Spec &sp, const int32_t *__restrict__ pos, const Lane &l, bool turned, float (&cj)[V], float (&sj)[V])
{
    float co[kOwn], so[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
        co[j] = so[j] = 0.f;
        if (turned && l.sub * kOwn < V) cos_sin<kFast>(sp.freq[lane_pair<V, kAdjacent>(l.chunk, l.sub * kOwn + j, sp.rot)], pos, sp, co[j], so[j]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int from = j / kOwn * l.group + l.chunk;
        cj[j] = __shfl_sync(0xffffffffu, co[j % kOwn], from);
        sj[j] = __shfl_sync(0xffffffffu, so[j % kOwn], from);
    }
}
// The same at row `row`, as packed pairs, shared or not.
template <int V, bool kAdjacent, bool kFast, int kGroup>
__device__ __forceinline__ void lane_angles(const Spec &sp, const int32_t *__restrict__ pos, int64_t row, const Lane &l, bool turned,
                                            uint64_t (&c)[V / 2], uint64_t (&s)[V / 2])
{
    pos += row * sp.axes;
    float cj[V], sj[V];
    if constexpr (kGroup * V >= 32) {
        shared_angles<V, kAdjacent, kFast, kGroup * V / 32>(sp, pos, l, turned, cj, sj);
    } else if (kGroup == 0 && l.heads * 2 >= V) {
        shared_angles<V, kAdjacent, kFast, 2>(sp, pos, l, turned, cj, sj);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            cj[j] = sj[j] = 0.f;
            if (turned) cos_sin<kFast>(sp.freq[lane_pair<V, kAdjacent>(l.chunk, j, sp.rot)], pos, sp, cj[j], sj[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        c[j] = f2_pack(cj[2 * j], cj[2 * j + 1]);
        s[j] = f2_pack(sj[2 * j], sj[2 * j + 1]);
    }
}
// The same where every head of the warp has a row of its own.
template <int V, bool kAdjacent, bool kFast>
__device__ __forceinline__ void own_angles(const Spec &sp, const int32_t *__restrict__ pos, int64_t row, int chunk, uint64_t (&c)[V / 2], uint64_t (&s)[V / 2])
{
    pos += row * sp.axes;
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        float c0, c1, s0, s1;
        cos_sin<kFast>(sp.freq[lane_pair<V, kAdjacent>(chunk, 2 * j, sp.rot)], pos, sp, c0, s0);
        cos_sin<kFast>(sp.freq[lane_pair<V, kAdjacent>(chunk, 2 * j + 1, sp.rot)], pos, sp, c1, s1);
        c[j] = f2_pack(c0, c1);
        s[j] = f2_pack(s0, s1);
    }
}

// Arguments of a call's rows.
struct Args {
    Spec sp;
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;   // elements
    const int32_t *pos;
    int64_t rows;                           // source rows
    int32_t hq, hkv;
    void *q_out, *k_out;
    int64_t q_out_stride, k_out_stride;
    int32_t group, steps;                   // lanes per head; steps of a part
    // append
    void *v_out;                            // with k_out: the pool's arrays
    const int32_t *src_rows, *slots;
    int64_t count, pool_slots;
    int32_t block_size;
    int *err;
};

// What a call does with its rows: writes the query and key heads to rows of their own; appends to the paged
// pool (row i of the call is source row src_rows[i]; its K and V heads go to pool slot slots[i], its query heads
// to row i of q_out); or writes an append's query heads only.
enum { kPacked = 0, kAppend = 1, kQueries = 2 };

// Most steps of a part. 5: the 16 + 2 heads of 128 dims in bf16, four at a time, in one part. An append's rows are
// few and its loads wait for their row number: two parts on more warps an SM hide more of it. Own choice of registers
// and 5 steps / 7 CTAs an SM and 3 steps, with the norm: one row 2.2 / 2.5 us, 672 rows 3.7 / 3.6, 2000 5.1 / 5.2, 4001
// 12.3 / 11.1; without it 672 3.2 / 2.7, 4001 10.3 / 9.0. Adjacent pairs, at 28 spilled bytes: 672 3.9 / 3.7, 2000 5.4 /
// 5.4, 4001 12.7 / 11.3; 64 dims 672 3.1 / 3.0, 4001 6.6 / 5.3; 80 dims (the general form) 672 3.6 / 3.6, 4001 8.7 /
// 8.2. (3 steps at the compiler's own registers are faster while the grid is one round, 672 rows 3.3, and slower behind
// it, 2000 6.2.) fp32 rows and 8-byte vectors need fewer registers: no difference.
constexpr int steps_of(int mode) { return mode == kAppend ? 3 : 5; }

// One warp's work: part `part` of row i, p.steps steps of as many heads as fit a warp, at most kSteps. All of the part's loads
// are issued before its angles are computed. Bound by HBM in large calls: every element is read once and written
// once.
// kGroup: see Lane.
template <typename T, int V, bool kAdjacent, bool kNorm, int kMode, int kGroup>
__device__ __forceinline__ void row_part(const Args &p, int64_t i, int part)
{
    constexpr int kSteps = steps_of(kMode);
    const int lane = threadIdx.x & 31;
    int64_t row = i;
    uint32_t slot = 0;
    if constexpr (kMode != kPacked) {
        if (p.src_rows) row = p.src_rows[i];
        const int32_t at = p.slots[i];
        if (at < 0 || at >= p.pool_slots || row < 0 || row >= p.rows) {
            if (kMode == kAppend && lane == 0 && part == 0)
                padoc_record_error(p.err, PADOC_DEVERR_BLOCK_ID, (at < 0 || at >= p.pool_slots) ? at : (int)row);
            return;
        }
        slot = (uint32_t)at;
    }
    const Lane l = warp_lane<kGroup>(p.group);
    const int heads = l.heads, sub = l.sub;
    const Place pl = lane_place<V>(l.chunk, l.used, p.sp.d, p.sp.rot);
    const int nq = p.q ? p.hq : 0, turned = kMode == kQueries ? nq : nq + p.hkv, total = kMode == kAppend ? turned + p.hkv : turned;
    const int first = part * p.steps * heads, lane_at = sub * p.sp.d + pl.a, to_b = pl.b - pl.a;
    // heads first + u heads + sub; a step of query heads alone has one address for the warp and the lane's place in it
    const T *q = static_cast<const T *>(p.q) + row * p.q_stride + lane_at;
    Raw<T, V> ra[kSteps], rb[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        if (u >= p.steps) break;
        const int h0 = first + u * heads;
        const T *src = q + h0 * p.sp.d;
        if (h0 + heads > nq) {
            // Lanes past the last head load what another lane does and store nothing: the steps have no divergent
            // branch but the stores'.
            const int h = min(h0 + sub, total - 1) - sub;
            if (h + sub < nq) src = q + h * p.sp.d;
            else if (kMode != kAppend || h + sub < turned) src = static_cast<const T *>(p.k) + row * p.k_stride + lane_at + (h - nq) * p.sp.d;
            else src = static_cast<const T *>(p.v) + row * p.v_stride + lane_at + (h - turned) * p.sp.d;
        }
        ra[u] = load_raw<T, V>(src);
        rb[u] = load_raw<T, V>(src + to_b);
    }
    uint64_t c[V / 2], s[V / 2];
    lane_angles<V, kAdjacent, sizeof(T) == 2, kGroup>(p.sp, p.pos, row, l, pl.turned, c, s);
    T *q_out = static_cast<T *>(p.q_out) + i * p.q_out_stride + lane_at;
    // where the row's KV heads go, and the distance from one to the next
    int64_t k_at = 0, k_step = p.sp.d;
    if constexpr (kMode == kAppend) {
        const uint32_t bs = (uint32_t)p.block_size;
        k_at = ((int64_t)(slot / bs) * p.hkv * bs + slot % bs) * p.sp.d;
        k_step = (int64_t)bs * p.sp.d;
    } else if constexpr (kMode == kPacked) {
        k_at = i * p.k_out_stride;
    }
    const bool whole = p.sp.rot == p.sp.d;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        if (u >= p.steps) break;
        const int h0 = first + u * heads, h = h0 + sub;
        if (kMode == kAppend && h0 + heads > turned) {   // value heads: as they are
            if (h >= turned && h < total && pl.active) {
                T *dst = static_cast<T *>(p.v_out) + k_at + (h - turned) * k_step + pl.a;
                *reinterpret_cast<Raw<T, V> *>(dst) = ra[u];
                *reinterpret_cast<Raw<T, V> *>(dst + to_b) = rb[u];
            }
            if (h0 >= turned) continue;
        }
        uint64_t a[V / 2], b[V / 2];
        unpack2(ra[u], a);
        unpack2(rb[u], b);
        if constexpr (kNorm) {
            const float r = norm_scale<V, kGroup>(a, b, pl.active, p.sp, l);
            const T *w = static_cast<const T *>(h < nq ? p.sp.q_weight : p.sp.k_weight) + pl.a;
            scale_head<V, T>(a, b, r, load_raw<T, V>(w), load_raw<T, V>(w + to_b));
        }
        if (whole) turn_pairs<V, kAdjacent>(a, b, c, s);
        else if (pl.turned) turn_pairs<V, kAdjacent>(a, b, c, s);
        T *dst = q_out + h0 * p.sp.d;
        bool here = pl.active;
        if (h0 + heads > nq) {
            here = here && h < turned;
            if (h >= nq) dst = static_cast<T *>(p.k_out) + k_at + (h - nq) * k_step + pl.a;
        }
        if (here) {
            store_vec2<V>(dst, a);
            store_vec2<V>(dst + to_b, b);
        }
    }
}

// Elements of a lane's vectors: 16 bytes where the rotated and the other dims come in whole chunks of
// them, else 8 bytes (bf16 heads whose dims are an odd multiple of 8).
int vec_of(const padoc_rotary *rot, padoc_dtype dtype);
// Lanes that share a head.
inline int group_of(int head_dim, int vec) { return head_dim / (2 * vec); }
// Sets group and steps; returns the parts of a row: as few as most_steps allows when the rows give every SM 8 warps,
// else as many as it takes to have them (at 5 steps a part, 672 rows of 20 heads: 3.9 us in two parts, 4.6 in one,
// 4.3 in three; 2617 rows: 5.4 in one, 5.6 in two; one row: 2.3 in five, 3.9 in one).
int split_rows(Args &p, int vec, int heads_total, int most_steps);

// Host checks of a padoc_rotary (defined in rotary.cu), and its device form.
padoc_status check_spec(const padoc_rotary *rot);
inline Spec make_spec(const padoc_rotary *r)
{
    return Spec{r->freq, r->q_weight, r->k_weight, r->eps, r->amplitude, r->amplitude, r->head_dim, r->rotary_dim, r->num_axes};
}
// Host checks of a call's source rows: strides and alignment of q (when given), k and, with_v, v.
padoc_status check_rows(const padoc_qkv_rows *in, const padoc_rotary *rot, bool with_v);

}  // namespace padoc_rotary_dev
