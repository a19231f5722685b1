// Norms of heads with the rotation in the same pass: what the norm kernels and the kernel that appends to packed pages share.
// Not part of the C ABI, and not exported.
#ifndef HPS_SEQ_NORM_H
#define HPS_SEQ_NORM_H

#include "hps_seq_common.h"

// One tensor of heads, and how work-groups share it.
struct NormTensor {
    const char *in, *back;                             // back: gradients of the outputs
    char *out;
    const float *weight;
    int64_t in_token, in_head, back_token, back_head, out_token, out_head;  // strides in bytes
    uint32_t heads, heads_beside, tokens_beside, groups;                    // side by side in a work-group; work-groups
};

struct NormArgs {
    NormTensor x[2];                                   // queries, keys
    const int32_t *positions;
    const float *table;
    float *parts, *weight_grad[2];
    float eps, eps_small, per_value;                   // eps_small: eps * 2^200; 1 / head_dim
    uint32_t n_tokens, head_dim, half, max_pos, lane_bits;                  // half = rot_dim / 2; lanes of a head: 1 << lane_bits
    uint32_t first_group;                              // of this launch
    int16_t interleaved, norm;                         // of 16 bits: a call whose arguments are over 272 bytes takes 0.2 us more
};

constexpr uint32_t kNormThreads = 256;

// E values as they are loaded and stored: 16 bytes, or one value.
template <typename T, int E> struct NormVec {
    typedef uint32_t raw __attribute__((ext_vector_type(4)));
    struct V { T v[E]; };
};
template <typename T> struct NormVec<T, 1> {
    typedef T raw;
    struct V { T v[1]; };
};

// Sum over the 1 << bits lanes that hold a head; every lane gets it, the same bits.
template <int kCtrl> __device__ __forceinline__ float norm_dpp(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, false));
}
__device__ __forceinline__ float norm_sum(float x, uint32_t bits) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    if (bits > 0) x += norm_dpp<0xB1>(x);              // lane ^ 1
    if (bits > 1) x += norm_dpp<0x4E>(x);              // lane ^ 2
    if (bits > 2) x += norm_dpp<0x141>(x);             // 7 - lane of 8, whose quads are alike by now
    if (bits > 3) x += norm_dpp<0x140>(x);             // 15 - lane of 16
    if (bits > 4) {
        const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r.x) + __uint_as_float(r.y);
    }
    if (bits > 5) {
        const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r.x) + __uint_as_float(r.y);
    }
    return x;
}

// 1 / sqrt(m), to the last bit but one.  (The instruction takes numbers below 2^-126 for 0.)
__device__ __forceinline__ float norm_inverse(float m) {
    const bool low = m < 0x1p-126f;
    return __builtin_amdgcn_rsqf(low ? m * 0x1p64f : m) * (low ? 0x1p32f : 1.f);
}

// Heads whose squares 32 bits do not hold, small ones (with an eps as small: their mean m = mean(x^2) + eps lost bits) and large ones (m is infinite): they
// are multiplied by a power of two, and m is formed anew.  Any other head keeps its m, bit for bit, and a wave of such heads pays for the question alone (0 to 1.5 % of a call).
struct NormFit {
    float by, eps;
    static __device__ __forceinline__ bool needed(float m) { return !(m >= 0x1p-90f && m < __builtin_inff()); }
    __device__ __forceinline__ NormFit(const NormArgs &a, float m)
        : by(m < 0x1p-90f ? 0x1p100f : m == __builtin_inff() ? 0x1p-72f : 1.f), eps(m < 0x1p-90f ? a.eps_small : m == __builtin_inff() ? a.eps * 0x1p-72f * 0x1p-72f : a.eps) {}
};

// E floats from an address of 4 bytes.
template <int E> struct NormFloats { float v[E]; };
template <int E> __device__ __forceinline__ NormFloats<E> norm_floats(const float *from) {
    NormFloats<E> x;
    if constexpr (E % 4 == 0) {
        typedef float quad __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const quad y = *(const quad *)(from + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) x.v[i + j] = y[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) x.v[i] = from[i];
    }
    return x;
}

// The values that a lane has of a head, two vectors of E: for halves the two that hold E pairs, for neighbours (kWithin) two that
// lie side by side.
template <typename T, int E, bool kWithin> struct NormSpan {
    typedef typename NormVec<T, E>::V V;
    typedef typename NormVec<T, E>::raw raw;
    uint32_t o0, o1;                                   // the two vectors, in values
    bool has0, has1, turn0, turn1;
    float cs[E], sn[E];                                // of the pairs: across the two vectors E, within them E / 2 each
    float w[2 * E];

    __device__ __forceinline__ void place(const NormArgs &a, uint32_t s) {
        if (kWithin || a.interleaved) {
            o0 = 2 * s * E;
            o1 = o0 + E;
        } else {
            const uint32_t split = a.half / E;         // behind the pairs, two neighbours to a span
            o0 = s < split ? s * E : 2 * a.half + 2 * (s - split) * E;
            o1 = s < split ? a.half + s * E : o0 + E;
        }
        has0 = o0 < a.head_dim;
        has1 = o1 < a.head_dim;
        turn0 = a.table && o0 < 2 * a.half;
        turn1 = a.table && o1 < 2 * a.half;
    }
    __device__ __forceinline__ void weights(const float *weight) {
#pragma unroll
        for (int j = 0; j < 2 * E; ++j) w[j] = 1.f;
        if (!weight) return;
        if (has0) {
            const NormFloats<E> x = norm_floats<E>(weight + o0);
#pragma unroll
            for (int j = 0; j < E; ++j) w[j] = x.v[j];
        }
        if (has1) {
            const NormFloats<E> x = norm_floats<E>(weight + o1);
#pragma unroll
            for (int j = 0; j < E; ++j) w[E + j] = x.v[j];
        }
    }
    // Cosines and sines (those times `sign`) of a position; NaN behind the table's last one.
    __device__ __forceinline__ void angles(const NormArgs &a, uint32_t s, int32_t pos, float sign) {
        const bool known = (uint32_t)pos < a.max_pos;
        const float *row = a.table + (size_t)(known ? pos : 0) * (2 * a.half);
        constexpr int kFirst = kWithin ? E / 2 : E;    // pairs of the first vector, or of both
#pragma unroll
        for (int j = 0; j < E; ++j) {
            cs[j] = 1.f;
            sn[j] = 0.f;
        }
        if (turn0) {
            const NormFloats<2 * kFirst> x = norm_floats<2 * kFirst>(row + 2 * (kWithin || a.interleaved ? s * E : o0));
#pragma unroll
            for (int j = 0; j < kFirst; ++j) {
                cs[j] = x.v[2 * j];
                sn[j] = x.v[2 * j + 1];
            }
        }
        if (kWithin && turn1) {
            const NormFloats<E> x = norm_floats<E>(row + 2 * s * E + E);
#pragma unroll
            for (int j = 0; j < E / 2; ++j) {
                cs[E / 2 + j] = x.v[2 * j];
                sn[E / 2 + j] = x.v[2 * j + 1];
            }
        }
#pragma unroll
        for (int j = 0; j < E; ++j) {
            cs[j] = known ? cs[j] : __builtin_nanf("");
            sn[j] = known ? sn[j] * sign : __builtin_nanf("");
        }
    }
    struct Raw { raw u, v; };
    __device__ __forceinline__ Raw request(const char *from) const {
        Raw r{};
        if (has0) r.u = *(const raw *)(from + o0 * sizeof(T));
        if (has1) r.v = *(const raw *)(from + o1 * sizeof(T));
        return r;
    }
    static __device__ __forceinline__ void take(const Raw &r, float (&x)[2 * E]) {
        const V u = __builtin_bit_cast(V, r.u), v = __builtin_bit_cast(V, r.v);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            x[j] = (float)u.v[j];
            x[E + j] = (float)v.v[j];
        }
    }
    __device__ __forceinline__ void store(char *to, const float (&x)[2 * E]) const {
        V u, v;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            u.v[j] = (T)x[j];
            v.v[j] = (T)x[E + j];
        }
        if (has0) *(raw *)(to + o0 * sizeof(T)) = __builtin_bit_cast(raw, u);
        if (has1) *(raw *)(to + o1 * sizeof(T)) = __builtin_bit_cast(raw, v);
    }
    static __device__ __forceinline__ void pair(float &p, float &q, float c, float s) {
        const float qs = q * s, qc = q * c, u = __builtin_fmaf(p, c, -qs), v = __builtin_fmaf(p, s, qc);
        p = u;
        q = v;
    }
    __device__ __forceinline__ void turn(float (&x)[2 * E]) const {
        if constexpr (kWithin) {
            if (turn0)
#pragma unroll
                for (int j = 0; j < E / 2; ++j) pair(x[2 * j], x[2 * j + 1], cs[j], sn[j]);
            if (turn1)
#pragma unroll
                for (int j = 0; j < E / 2; ++j) pair(x[E + 2 * j], x[E + 2 * j + 1], cs[E / 2 + j], sn[E / 2 + j]);
        } else {
            if (turn0)
#pragma unroll
                for (int j = 0; j < E; ++j) pair(x[j], x[E + j], cs[j], sn[j]);
        }
    }
};

// A work-group's heads of one tensor: y = turn(w x / sqrt(mean(x^2) + eps)).  A lane's place in its head stays the same from head to
// head, so weights, cosines and sines are read once for all of its heads; the next head is under way while one is computed.  E = 1 is
// for rows that are not in whole 16-byte vectors.  Bound by HBM where there are many tokens (8,192 of 40 heads of 128 of 16 bits, 170 MB moved:
// 38 us, 4.5 TB/s), else by the chain position, angles, row, store (26 tokens 3.5 us).
template <typename T, int E, bool kWithin> __device__ __forceinline__ void norm_forward(const NormArgs &a, const NormTensor &g, uint32_t group) {
    constexpr int kPer = E == 1 ? 4 : 1;
    typedef NormSpan<T, E, kWithin> Span;
    const uint32_t l = threadIdx.x & ((1u << a.lane_bits) - 1u), row = threadIdx.x >> a.lane_bits;
    const uint32_t beside = row / g.heads_beside, t = group * g.tokens_beside + beside;
    if (beside >= g.tokens_beside || t >= a.n_tokens) return;               // all lanes of a head, or none
    uint32_t h = row - beside * g.heads_beside;
    if (h >= g.heads) return;
    const int32_t pos = a.table ? a.positions[t] : 0;
    Span sp[kPer];
    typename Span::Raw next[kPer];
    const char *from = g.in + (int64_t)t * g.in_token;
    char *to = g.out + (int64_t)t * g.out_token;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        sp[i].place(a, l + ((uint32_t)i << a.lane_bits));
        next[i] = sp[i].request(from + (int64_t)h * g.in_head);
        sp[i].weights(a.norm ? g.weight : nullptr);
    }
    if (pos < 0) return;
    if (a.table)
#pragma unroll
        for (int i = 0; i < kPer; ++i) sp[i].angles(a, l + ((uint32_t)i << a.lane_bits), pos, 1.f);
    for (;;) {
        float x[kPer][2 * E], r = 1.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) Span::take(next[i], x[i]);
        const uint32_t after = h + g.heads_beside;
        if (after < g.heads)
#pragma unroll
            for (int i = 0; i < kPer; ++i) next[i] = sp[i].request(from + (int64_t)after * g.in_head);
        if (a.norm) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
#pragma unroll
                for (int j = 0; j < 2 * E; ++j) sum = __builtin_fmaf(x[i][j], x[i][j], sum);
            float m = __builtin_fmaf(norm_sum(sum, a.lane_bits), a.per_value, a.eps);
            if (__builtin_expect(__ballot(NormFit::needed(m)) != 0, 0)) {
                const NormFit fit(a, m);
                sum = 0.f;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
#pragma unroll
                    for (int j = 0; j < 2 * E; ++j) {
                        x[i][j] *= fit.by;
                        sum = __builtin_fmaf(x[i][j], x[i][j], sum);
                    }
                m = __builtin_fmaf(norm_sum(sum, a.lane_bits), a.per_value, fit.eps);
            }
            r = norm_inverse(m);
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (a.norm)
#pragma unroll
                for (int j = 0; j < 2 * E; ++j) x[i][j] = x[i][j] * r * sp[i].w[j];
            sp[i].turn(x[i]);
            sp[i].store(to + (int64_t)h * g.out_head, x[i]);
        }
        h = after;
        if (h >= g.heads) return;
    }
}

// In 32 bits, and not 0 where it is not.
inline float norm_eps(double eps) { return eps > 0 ? std::fmax((float)eps, __FLT_DENORM_MIN__) : 0.f; }
inline void norm_set_eps(NormArgs &a, double eps) {
    a.eps = norm_eps(eps);
    a.eps_small = norm_eps(std::fmin(eps, 0x1p-80) * 0x1p200);              // not read where eps is larger
}
// Puts a tensor's heads into place i.  false if it is not there or not aligned to its values.
SEQ_HIDDEN bool norm_put(NormArgs &a, int i, uint32_t heads, const hps_seq_heads_t &in, const hps_seq_heads_t &out, const hps_seq_heads_t *back, int size);
// Whether every row starts on 16 bytes, no vector holds pairs of two kinds, and `more`; sets the lanes of a head for either.
SEQ_HIDDEN bool norm_whole(NormArgs &a, uint32_t rot_dim, int size, bool more = true);
// Shares a tensor's rows between work-groups: with enough of them a lane gets several heads of a token, and a work-group several tokens.
SEQ_HIDDEN void norm_share(NormArgs &a, int i, uint32_t most_groups, uint32_t most_each);
SEQ_HIDDEN hps_status_t norm_check(int dtype, uint32_t head_dim, uint32_t rot_dim, const float *table, const int32_t *positions, uint32_t max_pos, uint32_t n_tokens, double eps,
                        const float *q_weight, const float *k_weight);

#endif  // HPS_SEQ_NORM_H
