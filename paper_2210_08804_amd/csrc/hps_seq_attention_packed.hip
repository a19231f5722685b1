// Attention over pages that hold keys and values in 4 bits (hps_seq.h), for gfx950.
//
// What it computes, and how the work is cut and joined, is as in attention over 16-bit pages.  Here a key and its value are 17/32
// of a byte a number, so that the conversion to 16 bits, not memory, is what few rows have to be fast at:
//
//   few rows (Few)    Every wave reads codes straight into the registers that the matrix instructions read, converted there; nothing
//                     goes through LDS.  Scores are S^T = K Q^T with 16x16x32 instructions: lane (m = l % 16, g = l / 16) of the first
//                     operand holds 8 * G neighbours of one key (G = head_dim / 32), which is one load; which key a row m stands for is
//                     free, and chosen so that a lane ends with the scores of keys 8 g .. 8 g + 7 of its row, which are
//                     its share of the second operand of O^T = V^T W^T as they are.  The pages' values lie so that a lane's
//                     2 G numbers of 8 tokens are 8 * G adjacent bytes; two conversions (of a pair of numbers of two tokens) and two
//                     byte permutations give a register of either number of both.
//   many rows (Wide)  Keys and values are converted once for 128 rows on their way to LDS, where they lie as rows of 16-bit
//                     pages do, and the loop is theirs.
#include <hip/hip_runtime.h>

#include <cmath>

#include "hps_seq_attend.h"
#include "hps_seq_packed.h"

namespace {

template <typename T> struct Type16;
template <> struct Type16<__bf16> {
    static __device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Type16<_Float16> {
    static __device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// Over the four lanes that share a row.
__device__ __forceinline__ float row_max(float x) {
    const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return both_max(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)));
}
__device__ __forceinline__ float row_sum(float x) {
    const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return both_sum(__uint_as_float(r.x) + __uint_as_float(r.y));
}

// Two codes, byte `at` of x (known when compiled), as numbers of 16 bits each.
template <typename T> __device__ __forceinline__ uint32_t two(uint32_t x, float s, int at) {
    typedef Packed<T> P;
    return __builtin_bit_cast(uint32_t, at == 0 ? P::template values<0>(x, s) : at == 1 ? P::template values<1>(x, s) : at == 2 ? P::template values<2>(x, s) : P::template values<3>(x, s));
}
template <typename T, typename F> __device__ __forceinline__ F eight(uint32_t x, float s) {
    return __builtin_bit_cast(F, u32x4{two<T>(x, s, 0), two<T>(x, s, 1), two<T>(x, s, 2), two<T>(x, s, 3)});
}

// The highest bit of each byte of x that is the scale of no number.
template <typename T> __device__ __forceinline__ uint32_t odd_bytes(uint32_t x) {
    constexpr uint32_t k = (0x7Fu - (kPackedMost<T> & 0x7Fu)) * 0x01010101u;
    return ((x & 0x7F7F7F7Fu) + k) & x & 0x80808080u;
}

// How many scales a lane's numbers have: of 8 G neighbours of a key, of 2 G of a value.
template <int G> constexpr int kKeyScales = G == 3 ? 3 : G == 8 ? 2 : 1;
template <int G> constexpr int kValueScales = G == 3 ? 3 : 1;
// Which 32 numbers of a head scale x of lane part g of four (c of 16) is of; and which scale dword s (pair p) has.
template <int G> __device__ __forceinline__ uint32_t key_group(uint32_t g, int x) { return G == 3 ? (3 * g + x) / 4 : G == 8 ? 2 * g + x : G * g / 4; }
template <int G> __device__ __forceinline__ uint32_t value_group(uint32_t c, int x) { return G == 3 ? (6 * c + 2 * x) / 32 : 2 * G * c / 32; }
template <int G> constexpr int key_scale(int s) { return G == 3 ? s : G == 8 ? s / 4 : 0; }
template <int G> constexpr int value_scale(int p) { return G == 3 ? p : 0; }

// kWords dwords of a tile from an address that is a multiple of kAlign bytes, in the widest loads that allows.
template <int kWords, int kAlign> __device__ __forceinline__ void load_words(const char *from, uint32_t (&to)[kWords]) {
    constexpr int kEach = kAlign >= 16 && kWords % 4 == 0 ? 4 : kAlign >= 8 && kWords % 2 == 0 ? 2 : 1;
    typedef uint32_t piece __attribute__((ext_vector_type(kEach)));
#pragma unroll
    for (int i = 0; i < kWords; i += kEach) {
        if constexpr (kEach == 1) to[i] = *(const uint32_t *)(from + 4 * i);
        else {
            const piece x = *(const piece *)(from + 4 * i);
#pragma unroll
            for (int j = 0; j < kEach; ++j) to[i + j] = x[j];
        }
    }
}

// ---- few rows

template <typename T, int G, int NT> struct Few {
    typedef typename Type<T>::frag frag;
    static constexpr int KS = kKeyScales<G>, VS = kValueScales<G>;
    static constexpr uint32_t kLds = 4 * 2 * G * 64 * 16 * NT, kSums = 4 * 16 * NT * sizeof(float2);
    // The codes and scales of 32 keys and values, as loaded.
    struct Raw {
        uint32_t k[2][G], ks[2][KS], v[2 * G];
        uint32_t vs[VS][2];
        bool bad0, bad1;                               // of the first and of the second 16: their block is none
    };
    // Where 32 keys begin, and their blocks.  Beyond the end: the first ones again, so that there always are loads under way to count.
    struct Where { uint32_t at; int32_t id0, id1; };

    const Args &a;
    const Item it;
    const uint32_t lane, n, g;
    const char *const tiles;                           // of the head
    frag q[NT][G];
    f32x4 o[NT][2 * G];
    float m[NT], l[NT];
    int32_t limit[NT];
    uint32_t poison[NT];                               // bit 4 x + j: the row saw a value that is no number in the lane's scale x, numbers j
    uint32_t k_off, v_off, ks_off[KS], vs_off[VS];

    __device__ __forceinline__ Few(const Args &args, const Item &item)
        : a(args), it(item), lane(threadIdx.x & 63u), n(lane & 15u), g(lane >> 4), tiles(args.k + (int64_t)item.head * args.page_head) {
        const uint32_t place = 8 * (n >> 2 & 1u) + (n & 3u);               // of the lane's first key, in its 16
        k_off = place * (16 * G) + g * (4 * G);
        v_off = (g & 1u) * (128 * G) + n * (8 * G);
#pragma unroll
        for (int x = 0; x < KS; ++x) ks_off[x] = place * G + key_group<G>(g, x);
#pragma unroll
        for (int x = 0; x < VS; ++x) vs_off[x] = (g & 1u) * (8 * G) + value_group<G>(n, x) * 8;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t row = it.row0 + 16 * t + n, i = a.by_ratio.quotient(row);
            const bool there = row < it.rows;
            limit[t] = !there ? kAll : it.causal_from == kAll ? (int32_t)it.end : min((int32_t)it.end, it.causal_from + (int32_t)i);
            const char *src = a.q + (int64_t)(it.token0 + i) * a.q_token + (int64_t)(it.head * a.ratio + (row - i * a.ratio)) * a.q_head + g * (16 * G);
#pragma unroll
            for (int s = 0; s < G; ++s) {
                u32x4 x = {0, 0, 0, 0};
                if (there) x = *(const u32x4 *)(src + 16 * s);
                q[t][s] = __builtin_bit_cast(frag, x);
            }
#pragma unroll
            for (int i2 = 0; i2 < 2 * G; ++i2) o[t][i2] = f32x4{0, 0, 0, 0};
            m[t] = -kInf;
            l[t] = 0.f;
            poison[t] = 0;
        }
    }

    __device__ __forceinline__ Where where(uint32_t x, uint32_t from) const {
        const uint32_t at = x < it.end ? x : from, second = at + 16 < it.end ? at + 16 : at;
        return {at, scalar(it.table, at >> a.sh), scalar(it.table, second >> a.sh)};
    }

    // Requests 32 keys and values (from a multiple of 16 below the end).  Behind the end of the keys, and in the place of a block that is
    // none, something else of the pages comes: hidden, or made zeros, in front of its use.
    __device__ __forceinline__ void load(Raw &r, const Where &w) const {
        const bool more = w.at + 16 < it.end;
        r.bad0 = (uint32_t)w.id0 >= a.n_blocks;
        r.bad1 = (uint32_t)w.id1 >= a.n_blocks;        // without a second 16: the first one's
        const uint32_t block = 1u << a.sh, p0 = w.at & (block - 1u), p1 = more ? (w.at + 16) & (block - 1u) : p0;
        const char *t0 = tiles + (uint64_t)(uint32_t)(r.bad0 ? 0 : w.id0) * (uint64_t)a.packed_block, *t1 = tiles + (uint64_t)(uint32_t)(r.bad1 ? 0 : w.id1) * (uint64_t)a.packed_block;
        const char *c0 = t0 + p0 * (16 * G), *c1 = t1 + p1 * (16 * G), *s0 = t0 + block * (32 * G) + p0 * G, *s1 = t1 + block * (32 * G) + p1 * G;
        const char *kc = (n & 8u ? c1 : c0) + k_off, *vc = (g & 2u ? c1 : c0) + block * (16 * G) + v_off;
        const char *ks = n & 8u ? s1 : s0, *vs = (g & 2u ? s1 : s0) + block * G;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            load_words<G, (G % 4 == 0 ? 16 : 4 * (G & 3))>(kc + j * (64 * G), r.k[j]);
#pragma unroll
            for (int x = 0; x < KS; ++x) r.ks[j][x] = *(const uint8_t *)(ks + ks_off[x] + j * (4 * G));
        }
        load_words<2 * G, (G % 2 == 0 ? 16 : 8)>(vc, r.v);
#pragma unroll
        for (int x = 0; x < VS; ++x) load_words<2, 8>(vs + vs_off[x], r.vs[x]);
    }

    // A block that is none stands for zeros.
    __device__ __forceinline__ void zeros(Raw &r) const {
        if (lane == 0) atomicOr(a.flags, HPS_SEQ_FLAG_BLOCK);
        const bool no_key = n & 8u ? r.bad1 : r.bad0, no_value = g & 2u ? r.bad1 : r.bad0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int x = 0; x < G; ++x) r.k[j][x] = no_key ? 0u : r.k[j][x];
#pragma unroll
            for (int x = 0; x < KS; ++x) r.ks[j][x] = no_key ? 0u : r.ks[j][x];
        }
#pragma unroll
        for (int x = 0; x < 2 * G; ++x) r.v[x] = no_value ? 0u : r.v[x];
#pragma unroll
        for (int x = 0; x < VS; ++x) {
            r.vs[x][0] = no_value ? 0u : r.vs[x][0];
            r.vs[x][1] = no_value ? 0u : r.vs[x][1];
        }
    }

    __device__ __forceinline__ void move(int t, float top) {
        const float next = fmaxf(m[t], top - Type<T>::kBelow), ref = next == -kInf ? 0.f : next, f = exp2_(m[t] - ref);
        l[t] *= f;
#pragma unroll
        for (int i = 0; i < 2 * G; ++i) o[t][i] *= f;
        m[t] = next;
    }

    // 32 keys and values from `at` on.
    __device__ __forceinline__ void step(Raw &r, uint32_t at, uint32_t least) {
        if (__builtin_expect(r.bad0 || r.bad1, 0)) zeros(r);
        f32x4 s[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float f[KS];
#pragma unroll
            for (int x = 0; x < KS; ++x) f[x] = packed_scale<T>(r.ks[j][x]);
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const frag k = eight<T, frag>(r.k[j][i], f[key_scale<G>(i)]);
#pragma unroll
                for (int t = 0; t < NT; ++t) s[t][j] = Type16<T>::mfma(k, q[t][i], s[t][j]);
            }
        }
        const bool edge = at + 32 > least;             // uniform: some rows do not see some keys
        uint32_t seen[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) seen[t] = 255u;
        if (edge) hide(s, r, at, seen);
        uint32_t odd[VS][2], any = 0;
#pragma unroll
        for (int x = 0; x < VS; ++x)
#pragma unroll
            for (int i = 0; i < 2; ++i) any |= odd[x][i] = odd_bytes<T>(r.vs[x][i]);
        if (__builtin_expect(__ballot(any != 0) != 0, 0)) spoil(r, odd, edge, seen);
        frag w[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float top = s[t][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, s[t][i / 4][i % 4]);
            top = row_max(top) * a.c;
            if (__ballot(top > m[t] + Type<T>::kSlack)) move(t, top);      // also the first time: m is -inf
            const float ref = m[t] == -kInf ? 0.f : m[t];
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = exp2_(__builtin_fmaf(s[t][i / 4][i % 4], a.c, -ref));
                sum += x;
                w[t][i] = (T)x;
            }
            l[t] += sum;
        }
        float f[VS][8];
#pragma unroll
        for (int x = 0; x < VS; ++x)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[x][i] = __uint_as_float((r.vs[x][i / 4] >> 8 * (i % 4) & 255u) << 23);
#pragma unroll
        for (int p = 0; p < G; ++p) {                  // the lane's numbers 2 p and 2 p + 1 of its eight tokens
            u32x4 even, odd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int b0 = 2 * i * G + p, b1 = b0 + G;
                const uint32_t x = two<T>(r.v[b0 / 4], f[value_scale<G>(p)][2 * i], b0 % 4), y = two<T>(r.v[b1 / 4], f[value_scale<G>(p)][2 * i + 1], b1 % 4);
                even[i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                odd[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                o[t][2 * p] = Type16<T>::mfma(__builtin_bit_cast(frag, even), w[t], o[t][2 * p]);
                o[t][2 * p + 1] = Type16<T>::mfma(__builtin_bit_cast(frag, odd), w[t], o[t][2 * p + 1]);
            }
        }
    }

    // Hides the scores that a row does not see, and values behind the end: their scales become 0, as the weights that they meet are.
    __device__ __forceinline__ void hide(f32x4 (&s)[NT][2], Raw &r, uint32_t at, uint32_t (&seen)[NT]) const {
        const int32_t first = (int32_t)(at + 8 * g);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int32_t many = min(max(limit[t] - first, 0), 8);
            seen[t] = (1u << many) - 1u;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[t][i / 4][i % 4] = i < many ? s[t][i / 4][i % 4] : -kInf;
        }
        const int32_t there = min(max((int32_t)it.end - first, 0), 8);
        const uint32_t low = there >= 4 ? ~0u : (1u << 8 * there) - 1u, high = there >= 8 ? ~0u : there <= 4 ? 0u : (1u << 8 * (there - 4)) - 1u;
#pragma unroll
        for (int x = 0; x < VS; ++x) {
            r.vs[x][0] &= low;
            r.vs[x][1] &= high;
        }
    }

    // Some values are no numbers.  Where all rows see all keys the product shows it, from a scale that is NaN.  A hidden value must not meet
    // its weight 0 like that: there the product takes a 0, and the rows that see the value are told by `poison`.
    __device__ __forceinline__ void spoil(Raw &r, const uint32_t (&odd)[VS][2], bool edge, const uint32_t (&seen)[NT]) {
#pragma unroll
        for (int x = 0; x < VS; ++x)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t bytes = (odd[x][i] >> 7) * 255u;
                r.vs[x][i] = edge ? r.vs[x][i] & ~bytes : r.vs[x][i] | bytes;
            }
        if (!edge) return;
#pragma unroll
        for (int x = 0; x < VS; ++x)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t left = odd[x][i] >> 7;
#pragma unroll 1
                for (int e = 4 * i; e < 4 * i + 4; ++e, left >>= 8) {       // token e of each eight
                    const uint64_t who = __ballot(left & 1u);               // lanes that hold values: number c of 16, eight tokens g
                    if (!who) continue;
#pragma unroll
                    for (int oct = 0; oct < 4; ++oct)
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const bool see = __shfl(seen[t], 16 * oct + (int)n) >> e & 1u;
                            poison[t] |= see ? ((uint32_t)(who >> (16 * oct + 4 * g)) & 15u) << 4 * x : 0u;
                        }
                }
            }
    }
    __device__ __forceinline__ void poisoned() {
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (__builtin_expect(__ballot(poison[t] != 0) != 0, 0))
#pragma unroll
                for (int i = 0; i < 2 * G; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (poison[t] >> (4 * value_scale<G>(i / 2) + j) & 1u) o[t][i][j] = __builtin_nanf("");
    }

    __device__ __forceinline__ uint32_t least_limit() const {               // over the wave's rows
        int32_t x = max(limit[0], 0);
#pragma unroll
        for (int t = 1; t < NT; ++t) x = min(x, max(limit[t], 0));
        for (int d = 1; d < 16; d <<= 1) x = min(x, __shfl_xor(x, d));
        return uniform((uint32_t)x);
    }

    // Every `stride`-th 32 keys from `from` on, the next ones' codes under way, the blocks of those behind them too.  Bound by reading: 4 tokens behind
    // 200,003 keys (8 heads of 128, 218 MB) 43 us, 5.1 TB/s, 64 behind up to 8,001 of their own (279 MB) 70 us, where a kernel that only reads as much
    // takes 35 and 45.
    __device__ __forceinline__ void run(uint32_t from, uint32_t stride) {
        if (from >= it.end) return;
        const uint32_t least = least_limit();
        Raw here, there;
        load(here, Where{from, it.id0, from + 16 < it.end ? it.id1 : it.id0});
        Where next = where(from + stride, from);
        uint32_t at = from, left = (it.end - from + stride - 1) / stride;
        // Two steps a turn, with one way out: a second one in the middle has the compiler wait there for loads that are to stay under way.
#pragma unroll 1
        for (; left >= 2; left -= 2) {
            load(there, next);
            next = where(at + 2 * stride, from);
            step(here, at, least);
            at += stride;
            load(here, next);
            next = where(at + 2 * stride, from);
            step(there, at, least);
            at += stride;
        }
        if (left) step(here, at, least);
        poisoned();
    }

    // The lane's 8 G neighbours of a row, from number 8 G g on.
    template <typename F> static __device__ __forceinline__ f32x4 quad(int y, F of) { return f32x4{of(4 * y), of(4 * y + 1), of(4 * y + 2), of(4 * y + 3)}; }
    __device__ __forceinline__ f32x4 quad(int t, int y) const {
        return quad(y, [&](int x) { return o[t][x % (2 * G)][x / (2 * G)]; });
    }

    struct Place {
        char *to;
        bool direct;
        float f;
        __device__ __forceinline__ void put4(uint32_t dim, f32x4 x) const {
            if (direct) {
                typedef T t4 __attribute__((ext_vector_type(4)));
                t4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = f == 0.f ? (T)0.f : (T)(x[j] * f);
                *(t4 *)(to + dim * 2) = y;
            } else {
                *(f32x4 *)(to + dim * 4) = x;
            }
        }
    };
    __device__ __forceinline__ Place place(uint32_t row, float ref, float sum, bool first) const {
        const uint32_t i = a.by_ratio.quotient(row), h = it.head * a.ratio + (row - i * a.ratio), t = it.token0 + i;
        const size_t at = (size_t)t * a.q_heads + h, part = (size_t)it.part * a.n_tokens * a.q_heads + at;
        if (first) {
            if (!a.direct) a.part_ml[part] = make_float2(ref, sum);
            else if (a.lse) a.lse[at] = sum == 0.f ? -kInf : (ref + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
        }
        return {a.direct ? a.out + (int64_t)t * a.out_token + (int64_t)h * a.out_head : (char *)(a.part_o + part * (32 * G)), a.direct != 0, sum == 0.f ? 0.f : 1.f / sum};
    }
    // The wave's own rows, as they are.
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t row = it.row0 + 16 * t + n;
            const float sum = row_sum(l[t]);
            if (row >= it.rows) continue;
            const Place p = place(row, m[t], sum, g == 0);
#pragma unroll
            for (int y = 0; y < 2 * G; ++y) p.put4(8 * G * g + 4 * y, quad(t, y));
        }
    }
    // The four waves have the same rows and different keys: joined through LDS, each wave a quarter of the values.
    __device__ __forceinline__ void finish_split(char *shared) {
        const uint32_t wave = uniform(threadIdx.x >> 6);
        f32x4 *l_o = (f32x4 *)shared;                  // [wave][NT * 2 G][64]
        float2 *l_ml = (float2 *)(shared + kLds);      // [wave][NT * 16]
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float sum = row_sum(l[t]);
#pragma unroll
            for (int y = 0; y < 2 * G; ++y) l_o[(wave * (NT * 2 * G) + t * 2 * G + y) * 64 + lane] = quad(t, y);
            if (g == 0) l_ml[(wave * NT + t) * 16 + n] = make_float2(m[t], sum);
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t row = it.row0 + 16 * t + n;
            float ref = -kInf, total = 0.f, f[kWaves];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) ref = fmaxf(ref, l_ml[(w * NT + t) * 16 + n].x);
            const float at = ref == -kInf ? 0.f : ref;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float2 x = l_ml[(w * NT + t) * 16 + n];
                f[w] = exp2_(x.x - at);
                total += f[w] * x.y;
            }
            if (row >= it.rows) continue;
            const Place p = place(row, ref, total, wave == 0 && g == 0);
            for (uint32_t y = wave; y < 2 * G; y += kWaves) {
                f32x4 x{};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) x += f[w] * l_o[(w * (NT * 2 * G) + t * 2 * G + y) * 64 + lane];
                p.put4(8 * G * g + 4 * y, x);
            }
        }
    }
};

// ---- many rows

template <typename T, int G> struct Wide : Engine<T, G, true, false> {
    typedef Engine<T, G, true, false> E;
    typedef typename E::frag frag;
    typedef __attribute__((address_space(3))) uint32_t lds1;
    typedef __attribute__((address_space(3))) u32x2 lds2;
    typedef __attribute__((address_space(3))) u32x4 lds4;
    static constexpr int KS = kKeyScales<G>, VS = kValueScales<G>;
    // A wave's share of a step as the pages hold it, 16 keys and 16 values: codes of keys, of values, scales of keys, of values.
    static constexpr uint32_t kCodes = 256 * G, kKeyScalesAt = 2 * kCodes, kValueScalesAt = kKeyScalesAt + 16 * G, kRaw = kValueScalesAt + 16 * G;
    static constexpr uint32_t kLds = E::kLds + 4 * kRaw;

    const char *const tiles;
    const uint32_t raw;
    bool has_key, has_value;                           // whether what is under way is there: its block is one

    __device__ __forceinline__ Wide(const Args &args, const Item &item, uint32_t lds_base, uint32_t wave)
        : E(args, item, lds_base, 32 * wave), tiles(args.k + (int64_t)item.head * args.page_head), raw(lds_base + E::kLds + wave * kRaw), has_key(false), has_value(false) {}

    // Block of the 16 tokens from `at` on: true if it is one, false (and a flag, within the length) if not.
    __device__ __forceinline__ bool valid(uint32_t at, int32_t id) const {
        if (__builtin_expect((uint32_t)id < this->a.n_blocks, 1)) return true;
        if (at < this->it.end && this->lane == 0) atomicOr(this->a.flags, HPS_SEQ_FLAG_BLOCK);
        return false;
    }
    // kBytes, a multiple of 16, from an address that all lanes share to LDS.
    template <uint32_t kBytes> __device__ __forceinline__ void fetch(const char *from, uint32_t to) const {
#pragma unroll
        for (uint32_t i = 0; i < kBytes; i += 1024)
            if (kBytes - i >= 1024 || this->lane * 16 < kBytes - i) load_to_lds(from + i, this->lane * 16, to + i);
    }
    __device__ __forceinline__ void fetch_keys(uint32_t at, int32_t id) {
        has_key = valid(at, id);
        if (!has_key) return;
        const uint32_t block = 1u << this->a.sh, p = at & (block - 1u);
        const char *t = tiles + (uint64_t)(uint32_t)id * (uint64_t)this->a.packed_block;
        fetch<kCodes>(t + p * (16 * G), raw);
        fetch<16 * G>(t + block * (32 * G) + p * G, raw + kKeyScalesAt);
    }
    __device__ __forceinline__ void fetch_values(uint32_t at, int32_t id) {
        has_value = valid(at, id);
        if (!has_value) return;
        const uint32_t block = 1u << this->a.sh, p = at & (block - 1u);
        const char *t = tiles + (uint64_t)(uint32_t)id * (uint64_t)this->a.packed_block;
        fetch<kCodes>(t + block * (16 * G) + p * (16 * G), raw + kCodes);
        fetch<16 * G>(t + block * (33 * G) + p * G, raw + kValueScalesAt);
    }
    template <int kWords> static __device__ __forceinline__ void read_words(uint32_t from, uint32_t (&to)[kWords]) {
        if constexpr (kWords % 4 == 0) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const u32x4 x = *(const lds4 *)(lds_char *)(uintptr_t)(from + 4 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) to[i + j] = x[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) to[i] = *(const lds1 *)(lds_char *)(uintptr_t)(from + 4 * i);
        }
    }
    // To rows of 16 bits, as Engine::load16 leaves them: a lane has 8 G neighbours of a key.  Zeros for a block that is none.
    __device__ __forceinline__ void put_keys(uint32_t to) const {
        const uint32_t key = this->lane >> 2, part = this->lane & 3u, row = to + key * E::kRow, sw = E::sw_k(key);
        uint32_t k[G];
        float f[KS];
        read_words(raw + key * (16 * G) + part * (4 * G), k);
#pragma unroll
        for (int x = 0; x < KS; ++x)
            f[x] = packed_scale<T>(*(const __attribute__((address_space(3))) uint8_t *)(lds_char *)(uintptr_t)(raw + kKeyScalesAt + key * G + key_group<G>(part, x)));
        if (!has_key)
#pragma unroll
            for (int s = 0; s < G; ++s) k[s] = 0, f[key_scale<G>(s)] = 1.f;
#pragma unroll
        for (int s = 0; s < G; ++s) *(lds4 *)(lds_char *)(uintptr_t)(row + ((G * part + s) ^ sw) * 16) = __builtin_bit_cast(u32x4, eight<T, frag>(k[s], f[key_scale<G>(s)]));
    }
    // And 2 G numbers of four values.  Zeros behind the end too.
    __device__ __forceinline__ void put_values(uint32_t at, uint32_t to) const {
        const uint32_t c = this->lane >> 1 & 15u, first = 8 * (this->lane >> 5) + 4 * (this->lane & 1u);
        uint32_t v[G], vs[VS], odd = 0;
        read_words(raw + kCodes + (this->lane >> 5) * (128 * G) + c * (8 * G) + (this->lane & 1u) * (4 * G), v);
#pragma unroll
        for (int x = 0; x < VS; ++x) {
            vs[x] = *(const lds1 *)(lds_char *)(uintptr_t)(raw + kValueScalesAt + (this->lane >> 5) * (8 * G) + value_group<G>(c, x) * 8 + 4 * (this->lane & 1u));
            odd |= odd_bytes<T>(vs[x]);
        }
        const bool careful = !has_value || at + 16 > this->it.end;          // uniform
        if (__builtin_expect(careful || __ballot(odd != 0) != 0, 0)) {
            const int32_t there = has_value ? min(max((int32_t)this->it.end - (int32_t)(at + first), 0), 4) : 0;
#pragma unroll
            for (int x = 0; x < VS; ++x) vs[x] |= (odd_bytes<T>(vs[x]) >> 7) * 255u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i < there) continue;
#pragma unroll
                for (int x = 0; x < VS; ++x) vs[x] &= ~(255u << 8 * i);
#pragma unroll
                for (int p = 0; p < G; ++p) v[(i * G + p) / 4] &= ~(255u << 8 * ((i * G + p) % 4));
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {                  // tokens
            const uint32_t t = first + i, row = to + t * E::kRow, sw = E::sw_v(t);
            uint32_t x[G];
#pragma unroll
            for (int p = 0; p < G; ++p) {
                const int b = i * G + p;
                x[p] = two<T>(v[b / 4], __uint_as_float((vs[value_scale<G>(p)] >> 8 * i & 255u) << 23), b % 4);
            }
            // 4 G bytes from byte 4 G c of the row on; chunks of 16 bytes change places
            if constexpr (G % 4 == 0) {
#pragma unroll
                for (int p = 0; p < G; p += 4) *(lds4 *)(lds_char *)(uintptr_t)(row + ((G / 4 * c + p / 4) ^ sw) * 16) = u32x4{x[p], x[p + 1], x[p + 2], x[p + 3]};
            } else if constexpr (G == 2) {
                *(lds2 *)(lds_char *)(uintptr_t)(row + ((c >> 1) ^ sw) * 16 + (c & 1u) * 8) = u32x2{x[0], x[1]};
            } else {
#pragma unroll
                for (int p = 0; p < G; ++p) {
                    const uint32_t at4 = G * c + p;
                    *(lds1 *)(lds_char *)(uintptr_t)(row + ((at4 >> 2) ^ sw) * 16 + (at4 & 3u) * 4) = x[p];
                }
            }
        }
    }

    // (512 rows of 4 heads each behind 32,768 keys of 8 heads of 128: 305 us of which matrix instructions alone take 210; from 16-bit pages, whose
    // rows need no conversion, 312.)
    // Engine::wide, with a step's keys and values brought to LDS one step earlier, as they are, and converted there at the start of the step in
    // front of theirs.
    __device__ __forceinline__ void run() {
        const uint32_t wave = uniform(threadIdx.x >> 6), least = this->least_limit(), mine = 16 * wave;
        const Item &it = this->it;
        if (it.first >= it.end) return;                // uniform in the work-group, as are all meetings
        uint32_t at = it.first;                        // the step's first value; its first key is 32 further on
        uint32_t keys_to = this->lds + mine * E::kRow, values_to = keys_to + E::kWideValues, flip = E::kStage;
        // keys `first` .. + 32 go to the second half of the other place, as if they were the end of a step in front
        if (wave >= 2) {
            fetch_keys(at + mine - 32, block_at(at + mine - 32));
            wait_loads<0>();
            put_keys(keys_to + E::kStage);
            wait_lds();
        }
        fetch_keys(at + 32 + mine, block_at(at + 32 + mine));
        fetch_values(at + mine, block_at(at + mine));
        wait_loads<0>();
        put_keys(keys_to);
        put_values(at + mine, values_to);
        wait_lds();
        fetch_keys(at + 96 + mine, block_at(at + 96 + mine));
        fetch_values(at + 64 + mine, block_at(at + 64 + mine));
        int32_t key_id = block_at(at + 160 + mine), value_id = block_at(at + 128 + mine);
        meet();
        this->k_row += E::kStage;
        f32x16 s = this->template scores<32 * E::kRow>(), t;
        this->k_row -= E::kStage;
        auto start = [&] {                             // everybody is done with the last step's keys and values
            wait_loads<0>();
            meet();
            if (at + 96 < it.end) put_keys(keys_to + flip);
            if (at + 64 < it.end) put_values(at + 64 + mine, values_to + flip);
            wait_lds();                                // the wave has read its share: the next one may come
            if (at + 160 < it.end) fetch_keys(at + 160 + mine, key_id);
            if (at + 128 < it.end) fetch_values(at + 128 + mine, value_id);
            key_id = block_at(at + 224 + mine);
            value_id = block_at(at + 192 + mine);
            this->fresh();
        };
        auto end = [&] {                               // the places change
            keys_to += flip;
            values_to += flip;
            this->k_row += flip;
            this->v_row += flip;
            this->here += flip;
            flip = 0u - flip;
            at += 64;
        };
        frag w[2];
        for (;;) {
            uint32_t left = 2;                         // stretches of 32 keys that the step has left
            bool ahead = false;                        // t has the next stretch's scores
            for (;;) {
                start();
                if (at + 64 > least) break;
                t = this->template scores<0>();
                float sum = this->weights(s, w, this->m);   // infinite, or NaN, the first time: m is -inf
                if (__ballot(!(sum < Type<T>::kMost))) {
                    ahead = true;
                    break;
                }
                this->l += sum;
                this->template add_values<E::kWideValues>(w);
                s = this->template scores<32 * E::kRow>();
                sum = this->weights(t, w, this->m);
                if (__ballot(!(sum < Type<T>::kMost))) {
                    ahead = true;
                    left = 1;
                    const f32x16 x = s;
                    s = t;
                    t = x;
                    break;
                }
                this->l += sum;
                this->template add_values<E::kWideValues + 32 * E::kRow>(w);
                end();
                if (at >= it.end) return;
            }
            if (left == 2) {
                this->template rest<E::kWideValues>(s, w, at, least);
                s = ahead ? t : this->template scores<0>();
                t = this->template scores<32 * E::kRow>();
            }
            this->template rest<E::kWideValues + 32 * E::kRow>(s, w, at + 32, least);
            s = t;
            end();
            if (at >= it.end) return;
        }
    }
    __device__ __forceinline__ int32_t block_at(uint32_t at) const { return at < this->it.end ? scalar(this->it.table, at >> this->a.sh) : -1; }
};

// Reads the blocks of the first 32 keys that a wave of few rows has.
__device__ __forceinline__ void first_blocks(const Args &a, Item &it, uint32_t width, uint32_t wave) {
    if (width == 0) {
        it.id0 = it.id1 = -1;
        return;
    }
    const uint32_t at = it.first + 32 * wave, last = width - 1;
    it.id0 = scalar(it.table, min(at >> a.sh, last));
    it.id1 = scalar(it.table, min((at + 16) >> a.sh, last));
}

// The work of one work-group, or of one of its waves where each has its own (solo).  false: none, and what it would leave is marked.
// (The loops over pages of 16 bits have no registers left for what this reads ahead, nor for how the compiler joins its ends: taken as it is it spills 49
// scalars there and costs 1 % at 512 rows behind 32,768 keys, 4 % at small calls.)
template <uint32_t kNarrow>                            // rows of a work-group of few
__device__ __forceinline__ bool item_of(const Args &a, uint32_t group, uint32_t wave, uint32_t lane, Item &it, bool &is_wide, bool &solo) {
    solo = false;
    if (group < a.history_groups) {
        // Work-groups of one (group, chunk, head) read the same keys: they go to one XCD (workgroups are dealt to the eight in turn).
        uint32_t combo, tile;
        if (a.history_combos >= 8) {
            const uint32_t y = group >> 3, q = a.by_history_tiles.quotient(y);
            combo = (group & 7u) + 8 * q;
            tile = y - q * a.history_tiles;
            if (combo >= a.history_combos) return false;
        } else {
            tile = a.by_history_combos.quotient(group);
            combo = group - tile * a.history_combos;
        }
        // From chunk to chunk the heads go round, so that an XCD has different ones at a time: where the heads of a token lie
        // side by side, one head's rows are in few of the L2's channels.
        // From group to group the chunks do: where histories end at different lengths, the last chunks have little to do, and must not
        // all be one XCD's (26 groups of 187 to 3,000 keys, two heads of 64, 4 chunks 50.6 -> 42.8 us, 8 chunks 51.7 -> 48.6).
        const uint32_t rest = a.by_kv_heads.quotient(combo), g = a.by_history_chunks.quotient(rest), turned = rest + g, chunk = turned - a.by_history_chunks.quotient(turned) * a.history_chunks;
        it.head = combo + rest - a.by_kv_heads.quotient(combo + rest) * a.kv_heads;
        it.table = a.prefix_table + (size_t)g * a.prefix_width;
        it.first = chunk * a.history_chunk;
        first_blocks(a, it, a.prefix_width, a.history_wide ? 0 : wave);
        const int32_t prefix = scalar(a.prefix_lens, g);
        const uint32_t r0 = clamp_to(scalar(a.group_offsets, g), a.n_requests), r1 = clamp_to(scalar(a.group_offsets, g + 1), a.n_requests);
        const uint32_t t0 = clamp_to(scalar(a.token_offsets, r0), a.n_tokens), t1 = clamp_to(scalar(a.token_offsets, r1), a.n_tokens);
        const uint32_t n = t1 > t0 ? t1 - t0 : 0;
        if (n > a.max_group) atomicOr(a.flags, HPS_SEQ_FLAG_LENGTH);
        is_wide = a.history_wide;
        it.token0 = t0;
        it.rows = min(n, a.max_group) * a.ratio;
        it.row0 = tile * (is_wide ? kWideRows : kNarrow);
        if (it.row0 >= it.rows) return false;
        it.end = min(length(a, prefix, a.prefix_width, a.max_prefix), it.first + a.history_chunk);
        it.causal_from = kAll;
        it.part = chunk;
    } else {
        uint32_t x = group - a.history_groups;
        is_wide = a.own_mode == kOwnWide;
        solo = a.own_mode == kOwnSolo;
        if (solo) {
            x = x * kWaves + wave;
            if (x >= a.own_items) return false;              // no wave of a solo work-group waits for another
        }
        const uint32_t rest = a.by_kv_heads.quotient(x), tiles = a.by_own_chunks.quotient(rest), r = a.by_own_tiles.quotient(tiles), turn = rest - tiles * a.own_chunks, tile = tiles - r * a.own_tiles;
        it.head = x - rest * a.kv_heads;
        // The chunks are dealt anew to each request: where lengths differ, the last ones have little to do, and work-groups a fixed number
        // apart share a CU.
        const uint32_t dealt = turn + (r * 0x9E3779B9u >> 24), chunk = dealt - a.by_own_chunks.quotient(dealt) * a.own_chunks;
        it.table = a.block_table + (size_t)r * a.table_width;
        it.first = chunk * a.own_chunk;
        first_blocks(a, it, a.table_width, solo || is_wide ? 0 : wave);
        const int32_t own = scalar(a.lens, r);
        const uint32_t t0 = clamp_to(scalar(a.token_offsets, r), a.n_tokens), t1 = clamp_to(scalar(a.token_offsets, r + 1), a.n_tokens);
        const uint32_t n = t1 > t0 ? t1 - t0 : 0, tile_rows = is_wide ? kWideRows : kNarrow;
        if (n > a.max_new) atomicOr(a.flags, HPS_SEQ_FLAG_LENGTH);
        it.token0 = t0;
        it.rows = min(n, a.max_new) * a.ratio;
        it.row0 = tile * tile_rows;
        if (it.row0 >= it.rows) return false;
        const uint32_t len = length(a, own, a.table_width, a.max_len);
        // places by all of the request's new tokens: queries may end inside it
        const int32_t from = (int32_t)len - (scalar(a.token_offsets, r + 1) - (int32_t)t0) + 1, last = from + (int32_t)(a.by_ratio.quotient(min(it.rows, it.row0 + tile_rows) - 1));        // keys that the tile's last row sees
        it.causal_from = n > 1 ? from : kAll;
        it.end = min((uint32_t)max(last, 0), it.first + a.own_chunk);
        it.part = a.history_chunks + chunk;
        if (a.history_chunks && chunk == 0 && ((int32_t)r < scalar(a.group_offsets, 0) || (int32_t)r >= scalar(a.group_offsets, a.n_groups)))
            for (uint32_t p = 0; p < a.history_chunks; ++p) mark_empty(a, it, p, tile_rows, solo ? lane : threadIdx.x, solo ? 64 : kThreads);
    }
    if (it.first >= it.end && !a.direct) {
        mark_empty(a, it, it.part, is_wide ? kWideRows : kNarrow, solo ? lane : threadIdx.x, solo ? 64 : kThreads);
        return false;
    }
    return true;
}

// Waves of a SIMD that the registers of few rows leave room for: work-groups of a CU (the registers that the compiler takes: one tile of 16 rows 88, 118, 158,
// 145 and 228 for 32 .. 256 values a head, two tiles 126, 156, 219 and 218).
template <int G, int NT> constexpr int kFewBeside = NT == 1 ? (G == 8 ? 2 : G >= 3 ? 3 : 4) : G >= 3 ? 2 : G == 2 ? 3 : 4;

// Work-groups of few rows alone: 16 * NT of an item.
template <typename T, int G, int NT> __global__ void __launch_bounds__(kThreads, (kFewBeside<G, NT>)) packed_few_kernel(const Args a) {
    typedef Few<T, G, NT> F;
    extern __shared__ __align__(16) char shared[];
    const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    Item it;
    bool is_wide, solo;
    if (!item_of<16 * NT>(a, a.first_group + blockIdx.x, wave, lane, it, is_wide, solo)) return;
    F e(a, it);
    e.run(solo ? it.first : it.first + 32 * wave, solo ? 32 : 32 * kWaves);
    if (solo) e.finish();
    else e.finish_split(shared);
}

// Either kind, where a history or the own tokens have many rows.
template <typename T, int G, int NT> __global__ void __launch_bounds__(kThreads, G <= 4 ? 2 : 1) packed_kernel(const Args a) {
    typedef Wide<T, G> W;
    typedef Few<T, G, NT> F;
    extern __shared__ __align__(16) char shared[];
    const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    Item it;
    bool is_wide, solo;
    if (!item_of<16 * NT>(a, a.first_group + blockIdx.x, wave, lane, it, is_wide, solo)) return;
    if (is_wide) {
        W e(a, it, (uint32_t)(uintptr_t)(lds_char *)shared, wave);
        e.run();
        e.finish(32 * wave);
    } else {
        F e(a, it);
        e.run(solo ? it.first : it.first + 32 * wave, solo ? 32 : 32 * kWaves);
        if (solo) e.finish();
        else e.finish_split(shared);
    }
}

// ---- host ---------------------------------------------------------------------------------

template <typename T, int G, int NT> constexpr uint32_t kFewLds = Few<T, G, NT>::kLds + Few<T, G, NT>::kSums;
template <typename T, int G, int NT> constexpr uint32_t kMixedLds = Wide<T, G>::kLds > kFewLds<T, G, NT> ? Wide<T, G>::kLds : kFewLds<T, G, NT>;

// Kernels of either kind, or of few rows alone, with 16 or 32 rows to a tile of few.
template <typename T, int G, typename F> hipError_t with_kernel(bool mixed, bool two, F f) {
    if constexpr (G <= 4) {
        if (mixed && two) return f(&packed_kernel<T, G, 2>, kMixedLds<T, G, 2>);
        if (two) return f(&packed_few_kernel<T, G, 2>, kFewLds<T, G, 2>);
    }
    if (mixed) return f(&packed_kernel<T, G, 1>, kMixedLds<T, G, 1>);
    return f(&packed_few_kernel<T, G, 1>, kFewLds<T, G, 1>);
}

template <typename T, int G> hipError_t allow_lds() {
    static_assert(kMixedLds<T, G, 1> <= 160 * 1024 && (G > 4 || (kMixedLds<T, G, 2> <= 80 * 1024 && kFewLds<T, G, 2> <= 80 * 1024)), "LDS of a CU");
    for (int kind = 0; kind < (G <= 4 ? 4 : 2); ++kind) {
        const hipError_t e = with_kernel<T, G>((kind & 1) != 0, (kind & 2) != 0, [](auto kernel, uint32_t lds) {
            return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        });
        if (e) return e;
    }
    return hipSuccess;
}
template <typename T> hipError_t allow_lds() {
    if (hipError_t e = allow_lds<T, 3>()) return e;
    if (hipError_t e = allow_lds<T, 4>()) return e;
    return allow_lds<T, 8>();
}

template <typename T, int G> hipError_t launch(Args &a, bool mixed, bool two, uint32_t groups, hipStream_t st) {
    return with_kernel<T, G>(mixed, two, [&](auto kernel, uint32_t lds) {
        return seq_launches(groups, [&](uint32_t first, uint32_t n) {
            a.first_group = first;
            hipLaunchKernelGGL(kernel, dim3(n), dim3(kThreads), lds, st, a);
        });
    });
}

template <typename T> hipError_t launch(Args &a, bool mixed, bool two, uint32_t groups, hipStream_t st) {
    switch (a.head_dim) {
    case 32: return launch<T, 1>(a, mixed, two, groups, st);
    case 64: return launch<T, 2>(a, mixed, two, groups, st);
    case 96: return launch<T, 3>(a, mixed, two, groups, st);
    case 128: return launch<T, 4>(a, mixed, two, groups, st);
    default: return launch<T, 8>(a, mixed, two, groups, st);
    }
}

// Many rows pay where what they save is more than their longer start, 7 us: a row of 32 takes 0.76 us for a million keys and heads, one of 128,
// of which all have to be filled, 0.66 (0.45 and 0.27 at 64 values a head).  (Measured, us a call, few / many, 8 heads of 128: 192 rows, 65,536 keys 89 / 99, 256
// rows 110 / 106, 512 rows 203 / 187; 512 rows, 8,192 keys 39 / 45, 1,024 rows 64 / 64; heads of 64 34 / 37, 49 / 46.  128 rows, 65,536 keys, heads of 32 / 64 / 96 / 256:
// 40 / 38, 45 / 42, 58 / 51, 126 / 123; 512 rows 132 / 103, 149 / 119, 192 / 148, 450 / 382; 256 rows, 8,192 keys 18 / 22, 21 / 25, 30 / 30, 48 / 60; 512 rows 28 / 29, 32 / 37, 38 / 42,
// 72 / 77, where the rule takes the slower one at 256 values alone; 2,048 rows 69 / 58, 78 / 68, 104 / 86, 245 / 223.)
bool wide_rows(bool, uint64_t rows, uint32_t keys, uint64_t stretches, uint32_t head_dim) {
    const double size = head_dim / 128.0, work = (double)keys * (double)stretches * 1e-6;
    const double few = head_dim > 128 ? 0.95 * size : 0.14 + 0.62 * size, many = head_dim > 128 ? 0.82 * size : std::fmax(0.12, 0.77 * size - 0.12);      // 16 rows a tile beyond 128 values
    return work * (few * (double)((rows + 31) / 32 * 32) - many * (double)((rows + 127) / 128 * 128)) > 7.0;
}
uint32_t beside(bool wide, uint32_t head_dim) { return head_dim > 128 ? (wide ? 1u : 2u) : wide ? 2u : 3u; }
// A step of a work-group of few rows (128 keys) takes 1.0 us alone on its CU, which is its chain of loads, conversions and products, and 0.87 for each
// that shares a CU, which is memory: 5.1 TB/s, at 128 values a head; 0.66 and 0.52 at 64.  (Measured, us a call: 16 rows, 200,003 keys,
// 8 heads: 32 / 48 / 64 / 80 / 96 / 128 chunks 58.5 / 54.5 / 51.2 / 56.5 / 54.0 / 58.8; with 64 values 39.5 / 40.0 / 33.6 / 37.0 / 33.7 / 34.8; 60,000 keys of
// 128: 21.5 / 23.2 / 22.4 / 24.9 / 25.0 / 27.8.)
double step_time(bool wide, double n, double beside, uint32_t cus, double size) {
    return wide ? (n <= cus ? 1.33 : 1.9) * (0.35 + 0.65 * size) : std::fmax(0.32 + 0.68 * size, std::ceil(beside / cus) * (0.17 + 0.7 * size));
}
// Rows of a tile of few: 16 where all that are served so fit one, else 32 (heads up to 128, whose registers suffice).  (Measured, us a call, 16 / 32: 16 rows,
// 200,003 keys 50.8 / 55.6, of 64 values 32.3 / 40.1; 32 rows, 65,536 keys 30.0 / 27.1, 96 rows 59.9 / 49.8; 512 rows, 8,192 keys 45.0 / 38.2; where there are few
// keys 16 can be ahead too: 192 rows, 1,000 keys 13.3 / 15.3.)
uint32_t narrow_rows(uint64_t most, uint32_t head_dim) { return head_dim <= 128 && most > 16 ? 32u : 16u; }

constexpr SeqAttendShape kShape = {kWideRows, kWideKeys, 32, narrow_rows, 512, wide_rows, beside, step_time};

}  // namespace

hipError_t seq_packed_allow_lds() {
    if (hipError_t e = allow_lds<_Float16>()) return e;
    return allow_lds<__bf16>();
}

extern "C" {

hps_status_t hps_seq_attention_packed(hps_seq_attention_t *s, const hps_seq_attention_packed_args_t *args, void *stream) {
    Args a{};
    bool work = false;
    if (hps_status_t st = seq_attend_args(s, args, a, work)) return st;
    const hps_seq_attention_packed_args_t &r = *args;
    if (hps_status_t st = seq_check_packed(r.pages, r.head_dim)) return st;
    if (!work) return HPS_OK;
    a.k = reinterpret_cast<const char *>(r.pages.data);
    a.packed_block = r.pages.block_stride;
    a.page_head = r.pages.head_stride;
    if (r.pages.n_blocks == 0) {                       // no block number is one; what is read in their place is thrown away, and has to be somewhere
        static_assert(65536u * 32 * 4 >= HPS_SEQ_MAX_BLOCK * 256 / 16 * 17, "a tile lies within any session's memory");
        a.k = reinterpret_cast<const char *>(s->part_o);
        a.packed_block = a.page_head = 0;
    }
    SeqAttendCut cut;
    if (hps_status_t st = seq_attend_cut(a, kShape, *s, cut)) return st;
    const bool mixed = a.own_mode == kOwnWide || a.history_wide, two = cut.narrow_rows == 32;
    hipStream_t st = static_cast<hipStream_t>(stream);
    SEQ_TRY(seq_attend_check(a, st));
    SEQ_TRY(r.dtype == HPS_SEQ_F16 ? launch<_Float16>(a, mixed, two, cut.groups, st) : launch<__bf16>(a, mixed, two, cut.groups, st));
    SEQ_TRY(seq_attend_join(a, r.dtype, cut.parts, st));
    return HPS_OK;
}

}  // extern "C"
