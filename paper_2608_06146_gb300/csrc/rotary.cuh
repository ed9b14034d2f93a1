// rotary.cuh -- rotary positions with several axes and the per-head RMS norm before them, as device
// helpers shared by the packed forward and backward, the append into the paged pool and the E4M3 append.
//
// A head of d dims is taken in chunks of 2 V dims, one lane each: V pairs of the rotated part, or 2 V
// consecutive dims behind it. Lane chunk c holds two vectors of V elements: of pairs (i, i + R/2) the
// dims c V and R/2 + c V, of adjacent pairs and of dims past R the dims 2 c V and 2 c V + V. In both
// layouts its pairs are c V .. c V + V - 1, so a lane's V angles serve every head of its row.
#pragma once

#include "common.cuh"

namespace padoc_rotary_dev {

// Arguments of a head's norm and rotation.
struct Spec {
    const uint64_t *freq;        // [rot / 2]
    const void *q_weight, *k_weight;
    float eps, amplitude;
    int32_t d, rot, axes;
};

// The cosine and sine of one pair's angle, times the amplitude. A table entry holds the fraction of a
// turn per position unit as a 64-bit integer, its axis in the two lowest bits; times a 32-bit position it
// wraps modulo a whole turn, so the angle of a position a million tokens away is as exact as that of the
// first ones (its fraction is cut at 2^-32 of a turn; a product in fp32 would be off by 0.06 rad at 10^6).
__device__ __forceinline__ float half_turns(uint64_t f, const int32_t *__restrict__ pos)
{
    const int32_t p = pos[f & 3u];
    const int32_t t = (int32_t)(((f & ~(uint64_t)3) * (uint64_t)(int64_t)p) >> 32);
    return (float)t * 0x1p-31f;   // in [-1, 1): the angle is pi times this
}
__device__ __forceinline__ void cos_sin(uint64_t f, const int32_t *__restrict__ pos, float amplitude, float &c, float &s)
{
    sincospif(half_turns(f, pos), &s, &c);
    c *= amplitude;
    s *= amplitude;
}

// V consecutive elements as fp32.
template <int V>
__device__ __forceinline__ void load_vec(const __nv_bfloat16 *p, float (&x)[V])
{
    static_assert(V == 8 || V == 4 || V == 2, "8, 4 or 2 elements");
    uint32_t w[V / 2];
    if constexpr (V == 8) {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    } else if constexpr (V == 4) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        w[0] = u.x, w[1] = u.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t *>(p);
    }
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
}
template <int V>
__device__ __forceinline__ void load_vec(const float *p, float (&x)[V])
{
    static_assert(V == 4, "4 elements");
    const float4 u = *reinterpret_cast<const float4 *>(p);
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
}
template <int V>
__device__ __forceinline__ void store_vec(__nv_bfloat16 *p, const float (&x)[V])
{
    uint32_t w[V / 2];
#pragma unroll
    for (int j = 0; j < V / 2; ++j) w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
    if constexpr (V == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (V == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t *>(p) = w[0];
}
template <int V>
__device__ __forceinline__ void store_vec(float *p, const float (&x)[V])
{
    *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
}

// Sum over the `group` lanes (a power of two) that share a head.
__device__ __forceinline__ float group_sum(float v, int group)
{
    for (int m = group >> 1; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}

// A lane's place in a head: its chunk, the element offsets of its two vectors, whether its dims are rotated.
struct Place {
    int a, b;
    bool active, turned;
};
template <int V, bool kAdjacent>
__device__ __forceinline__ Place lane_place(int chunk, int d, int rot)
{
    Place p;
    p.active = chunk * 2 * V < d;
    p.turned = chunk * 2 * V < rot;
    const bool split = !kAdjacent && p.turned;
    p.a = split ? chunk * V : chunk * 2 * V;
    p.b = split ? rot / 2 + chunk * V : chunk * 2 * V + V;
    return p;
}

// The rotation of a lane's V pairs by its angles (kBack: by the opposite ones, the gradient's).
template <int V, bool kAdjacent, bool kBack>
__device__ __forceinline__ void turn_pairs(float (&a)[V], float (&b)[V], const float (&c)[V], const float (&s)[V])
{
    auto turn = [](float &x, float &y, float cc, float ss) {
        const float x0 = x, y0 = y;
        x = kBack ? fmaf(x0, cc, y0 * ss) : fmaf(x0, cc, -(y0 * ss));
        y = kBack ? fmaf(y0, cc, -(x0 * ss)) : fmaf(y0, cc, x0 * ss);
    };
    if constexpr (!kAdjacent) {
#pragma unroll
        for (int j = 0; j < V; ++j) turn(a[j], b[j], c[j], s[j]);
    } else {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) turn(a[2 * j], a[2 * j + 1], c[j], s[j]);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) turn(b[2 * j], b[2 * j + 1], c[V / 2 + j], s[V / 2 + j]);
    }
}

// RMS norm of a head spread over `group` lanes: x r w with r = 1 / sqrt(mean x^2 + eps), sums in fp32.
template <typename T, int V>
__device__ __forceinline__ void norm_head(float (&a)[V], float (&b)[V], const T *w, const Place &pl, const Spec &sp, int group)
{
    float ss = 0.f;
    if (pl.active) {
#pragma unroll
        for (int j = 0; j < V; ++j) ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
    }
    const float r = rsqrtf(group_sum(ss, group) / (float)sp.d + sp.eps);
    if (pl.active) {
        float wa[V], wb[V];
        load_vec<V>(w + pl.a, wa);
        load_vec<V>(w + pl.b, wb);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            a[j] *= r * wa[j];
            b[j] *= r * wb[j];
        }
    }
}

// Host checks of a padoc_rotary (defined in rotary.cu), and its device form.
padoc_status check_spec(const padoc_rotary *rot);
inline Spec make_spec(const padoc_rotary *r)
{
    return Spec{r->freq, r->q_weight, r->k_weight, r->eps, r->amplitude, r->head_dim, r->rotary_dim, r->num_axes};
}
// Host checks of a call's source rows: strides and alignment of q (when given), k and, with_v, v.
padoc_status check_rows(const padoc_qkv_rows *in, const padoc_rotary *rot, bool with_v);

}  // namespace padoc_rotary_dev
