// Keys and values of new tokens to pages that hold them in 4 bits, and back (hps_seq.h), for gfx950.
#include <hip/hip_runtime.h>

#include "hps_seq_norm.h"
#include "hps_seq_packed.h"

namespace {

// Where a token's values lie in its tile.
struct Tile {
    uint32_t dim, groups, block;
    __device__ __forceinline__ uint32_t key(uint32_t place, uint32_t d) const { return place * (dim / 2) + d / 2; }
    __device__ __forceinline__ uint32_t key_scale(uint32_t place, uint32_t d) const { return block * dim + place * groups + d / 32; }
    // of values d, d + 1, d even
    __device__ __forceinline__ uint32_t value(uint32_t place, uint32_t d) const {
        return block * (dim / 2) + place / 8 * (4 * dim) + d / (2 * groups) * (8 * groups) + place % 8 * groups + d % (2 * groups) / 2;
    }
    __device__ __forceinline__ uint32_t value_scale(uint32_t place, uint32_t d) const { return block * (dim + groups) + (place / 8 * groups + d / 32) * 8 + place % 8; }
};

struct PackedArgs {
    NormArgs norm;                                     // of the queries
    const char *k, *v;
    int64_t k_token, k_head, v_token, v_head;          // strides in bytes
    char *k_out, *v_out;                               // of a reading
    uint8_t *pages;
    int64_t page_block, page_head;
    const int32_t *slots;
    const float *k_weight;
    double eps, per_value;                             // 1 / head_dim
    uint32_t kv_heads, n_slots, sh, lane_bits, heads_each, head_groups;     // lanes of a head: 1 << lane_bits, 8 values each; heads of a work-group
    uint32_t first_group, kv_groups;
    Tile tile;
};

constexpr uint32_t kThreads = 256;

template <int kCtrl> __device__ __forceinline__ uint32_t moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xf, 0xf, false); }
template <int kCtrl> __device__ __forceinline__ double moved(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)moved<kCtrl>((uint32_t)(u >> 32)) << 32 | moved<kCtrl>((uint32_t)u));
}
// Over the four lanes that hold 32 neighbours.
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
    x = max(x, moved<0xB1>(x));
    return max(x, moved<0x4E>(x));
}
// Over the 1 << bits lanes, four at least, that hold a head; every lane gets it, the same bits.
__device__ __forceinline__ double head_sum(double x, uint32_t bits) {
    x += moved<0xB1>(x);
    x += moved<0x4E>(x);
    if (bits > 2) x += moved<0x141>(x);                // 7 - lane of 8, whose quads are alike by now
    if (bits > 3) x += moved<0x140>(x);                // 15 - lane of 16
    if (bits > 4) x += __shfl_xor(x, 16);
    return x;
}

template <typename T> struct Eight { T v[8]; };
template <bool kWhole, typename T> __device__ __forceinline__ Eight<T> load8(const char *from) {
    typedef uint32_t raw __attribute__((ext_vector_type(2 * sizeof(T)), aligned(16)));
    if constexpr (kWhole) return __builtin_bit_cast(Eight<T>, *(const raw *)from);
    Eight<T> x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x.v[j] = ((const T *)from)[j];
    return x;
}

// The scale byte of 32 values, of which the largest in size is `top` (as bits of 32): the least power of two s with a <= 7 s, 7 being 1.75 * 2^2.
template <typename T> __device__ __forceinline__ uint32_t scale_of(uint32_t top) {
    if (top >= 0x7F800000u) return 255u;               // infinite or NaN
    const int b = (int)(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x600000u);  // numbers below 2^-126 get the least scale either way
    return (uint32_t)min(max(b, kPackedLeast<T>), (int)kPackedMost<T>);
}

// Numbers in 32 bits that are cut off, the last bit set where anything was: what is rounded to few bits afterwards is rounded as if from 64
// bits, and compared with a number of few bits as if it had them all.  (Conversions in the mode that cuts off, which is left again at once.)
__device__ __forceinline__ void odd_floats(const double (&y)[8], float (&x)[8]) {
    asm("s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 4), 15\n\t"
        "v_cvt_f32_f64 %0, %8\n\tv_cvt_f32_f64 %1, %9\n\tv_cvt_f32_f64 %2, %10\n\tv_cvt_f32_f64 %3, %11\n\t"
        "v_cvt_f32_f64 %4, %12\n\tv_cvt_f32_f64 %5, %13\n\tv_cvt_f32_f64 %6, %14\n\tv_cvt_f32_f64 %7, %15\n\t"
        "s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 4), 0"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(y[0]), "v"(y[1]), "v"(y[2]), "v"(y[3]), "v"(y[4]), "v"(y[5]), "v"(y[6]), "v"(y[7]));
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(__float_as_uint(x[j]) | (uint32_t)((double)x[j] != y[j]));     // below 2^-126 too, where more than 29 bits are cut
}

// 1 / sqrt(x): the instruction's 2^-26 or so, and a step that leaves the third power of it.  (0 for infinity, which the step would make no number.)
__device__ __forceinline__ double inverse_root(double x) {
    const double y = __builtin_amdgcn_rsq(x), e = __builtin_fma(-x * y, y, 1.0), z = __builtin_fma(y * e, __builtin_fma(e, 0.375, 0.5), y);
    return y == 0.0 ? 0.0 : z;
}

// Eight values' codes.  The conversion takes 32 bits, rounds to the nearest, of two to the even code, and ends at 6.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], float s) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
}

// Eight codes of values: runs of `groups` bytes, 8 * groups apart.
__device__ __forceinline__ void put_values(uint8_t *to, const Tile &tile, uint32_t place, uint32_t d, uint32_t codes) {
    if ((tile.groups & 3u) == 0) {
        *(uint32_t *)(to + tile.value(place, d)) = codes;
    } else if (tile.groups == 2) {
        *(uint16_t *)(to + tile.value(place, d)) = (uint16_t)codes;
        *(uint16_t *)(to + tile.value(place, d + 4)) = (uint16_t)(codes >> 16);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) to[tile.value(place, d + 2 * j)] = (uint8_t)(codes >> 8 * j);
    }
}
__device__ __forceinline__ uint32_t get_values(const uint8_t *from, const Tile &tile, uint32_t place, uint32_t d) {
    if ((tile.groups & 3u) == 0) return *(const uint32_t *)(from + tile.value(place, d));
    if (tile.groups == 2) return *(const uint16_t *)(from + tile.value(place, d)) | (uint32_t)*(const uint16_t *)(from + tile.value(place, d + 4)) << 16;
    uint32_t codes = 0;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) codes |= (uint32_t)from[tile.value(place, d + 2 * j)] << 8 * j;
    return codes;
}

// A lane's place: one of a work-group's rows, half of which are keys', half values', of as many tokens.
struct Place {
    uint32_t d, token, head0, heads;
    bool values, live;
    __device__ __forceinline__ Place(const PackedArgs &a, uint32_t group) {
        const uint32_t row = threadIdx.x >> a.lane_bits, tokens = (kThreads >> a.lane_bits) / 2, chunk = group / a.head_groups;
        d = (threadIdx.x & ((1u << a.lane_bits) - 1u)) * 8;
        values = row >= tokens;
        token = chunk * tokens + (values ? row - tokens : row);
        head0 = group % a.head_groups * a.heads_each;
        heads = min(head0 + a.heads_each, a.kv_heads);
        live = token < a.norm.n_tokens;
    }
};

// A lane's eight keys in 64 bits, normed and turned.  Codes are steps of up to half a value's size, so a difference in the last bit of a
// sum can change a key by as much: in 64 bits that does not happen, and it costs nothing here (its operations run at the rate of
// 32 bits on this device).
template <typename T, bool kWhole, bool kWithin> struct Keys {
    double own[8], other[8];                           // factors of the lane's values, and of their partners in the turning
    uint32_t d;
    bool in, turns;
    struct Raw { Eight<T> x, p; };
    static __device__ __forceinline__ bool neighbours(const NormArgs &n) { return kWhole ? kWithin : n.interleaved != 0; }
    __device__ __forceinline__ uint32_t partner(const NormArgs &n, uint32_t x) const { return neighbours(n) ? x ^ 1u : x < n.half ? x + n.half : x - n.half; }
    __device__ __forceinline__ Keys(const PackedArgs &a, uint32_t first, bool plain) : d(first) {
        in = d < a.norm.head_dim;
        turns = !plain && a.norm.table && in && d < 2 * a.norm.half;
    }
    __device__ __forceinline__ void factors(const PackedArgs &a, int32_t pos) {
        const NormArgs &n = a.norm;
        const float *weight = n.norm ? a.k_weight : nullptr;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            own[j] = 1.0;
            other[j] = 0.0;
        }
        if (!in) return;
        NormFloats<8> w{{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}}, wp = w;
        if (weight) w = norm_floats<8>(weight + d);
        const bool known = (uint32_t)pos < n.max_pos, leads = d < n.half;
        const float *row = n.table + (size_t)(known ? pos : 0) * (2 * n.half);
        if (!turns) {
#pragma unroll
            for (int j = 0; j < 8; ++j) own[j] = (double)w.v[j];
        } else if (kWhole && !kWithin) {               // eight of one half
            if (weight) wp = norm_floats<8>(weight + partner(n, d));
            const NormFloats<16> f = norm_floats<16>(row + 2 * (leads ? d : d - n.half));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                own[j] = (double)w.v[j] * (double)f.v[2 * j];
                other[j] = (double)wp.v[j] * (double)(leads ? -f.v[2 * j + 1] : f.v[2 * j + 1]);      // a cos - b sin; b cos + a sin
            }
        } else if (kWhole) {                           // four pairs of neighbours
            const NormFloats<8> f = norm_floats<8>(row + d);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                own[j] = (double)w.v[j] * (double)f.v[j & ~1];
                other[j] = (double)w.v[j ^ 1] * (double)(j & 1 ? f.v[j] : -f.v[j + 1]);
            }
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                own[j] = (double)w.v[j];
                if (d + j >= 2 * n.half) continue;
                const uint32_t at = d + j, pair = n.interleaved ? at / 2 : at < n.half ? at : at - n.half;
                const bool first = n.interleaved ? (at & 1u) == 0 : at < n.half;
                own[j] *= (double)row[2 * pair];
                other[j] = (weight ? (double)weight[partner(n, at)] : 1.0) * (double)(first ? -row[2 * pair + 1] : row[2 * pair + 1]);
            }
        }
        if (turns && !known)
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j)
                if (d + j < 2 * n.half) own[j] = __builtin_nan("");
    }
    __device__ __forceinline__ Raw request(const PackedArgs &a, const char *from) const {
        const NormArgs &n = a.norm;
        Raw r{};
        if (!in) return r;
        r.x = load8<kWhole, T>(from + d * sizeof(T));
        if (!turns || neighbours(n)) return r;
        if constexpr (kWhole) r.p = load8<true, T>(from + partner(n, d) * sizeof(T));
        else
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j)
                if (d + j < 2 * n.half) r.p.v[j] = ((const T *)from)[partner(n, d + j)];
        return r;
    }
    __device__ __forceinline__ void values(const PackedArgs &a, const Raw &r, float (&out)[8]) const {
        const NormArgs &n = a.norm;
        double scale = 1.0;
        if (n.norm) {
            double sum = 0.0;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)(float)r.x.v[j], (double)(float)r.x.v[j], sum);
            scale = inverse_root(__builtin_fma(head_sum(sum, a.lane_bits), a.per_value, a.eps));
        }
        double y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double x = (double)(float)r.x.v[j] * own[j];
            y[j] = turns ? __builtin_fma((double)(float)(neighbours(n) ? r.x.v[j ^ 1] : r.p.v[j]), other[j], x) : x;
            if (n.norm) y[j] *= scale;
        }
        odd_floats(y, out);
    }
};

// Work-groups of the launch: the queries' (as in the norm kernels) and those of keys and values, in turn.  Bound by HBM where there are many
// tokens (8,192 of 32 and 8 heads of 128, 178 MB moved: 44 us, 4.0 TB/s), else by the chain slot, position, row, largest value, store (64
// tokens 4.4 us).
template <typename T, int E, bool kWithin> __global__ void __launch_bounds__(kThreads) append_kernel(const PackedArgs a) {
    // one kind's arithmetic runs beside the other's loads
    const uint32_t group = a.first_group + blockIdx.x, pairs = 2 * min(a.norm.x[0].groups, a.kv_groups);
    const bool queries = group < pairs ? (group & 1u) == 0 : a.norm.x[0].groups > a.kv_groups;
    const uint32_t mine = group < pairs ? group / 2 : group - pairs / 2;
    if (queries) return norm_forward<T, E, kWithin>(a.norm, a.norm.x[0], mine);
    const Place at(a, mine);
    if (!at.live) return;
    const int32_t pos = a.norm.table ? a.norm.positions[at.token] : 0;
    const uint32_t slot = (uint32_t)a.slots[at.token];
    if (pos < 0 || slot >= a.n_slots) return;          // all lanes of a row
    const uint32_t place = slot & (a.tile.block - 1u);
    uint8_t *const block = a.pages + (int64_t)(slot >> a.sh) * a.page_block;
    const bool in = at.d < a.tile.dim;
    const char *from = at.values ? a.v + (int64_t)at.token * a.v_token : a.k + (int64_t)at.token * a.k_token;
    const int64_t step = at.values ? a.v_head : a.k_head;
    typedef Keys<T, (E > 1), kWithin> K;
    K keys(a, at.d, at.values);
    typename K::Raw next = keys.request(a, from + (int64_t)at.head0 * step);
    if (!at.values) keys.factors(a, pos);
    for (uint32_t h = at.head0; h < at.heads; ++h) {
        float x[8];
        const typename K::Raw raw = next;
        if (h + 1 < at.heads) next = keys.request(a, from + (int64_t)(h + 1) * step);
        if (at.values)                                 // uniform in a wave, of heads up to 128
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (float)raw.x.v[j];
        else keys.values(a, raw, x);
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
        top = group_max(top);
        if (!in) continue;
        const uint32_t b = scale_of<T>(top), codes = codes_of(x, __uint_as_float(b << 23));
        uint8_t *to = block + (int64_t)h * a.page_head;
        if (at.values) put_values(to, a.tile, place, at.d, codes);
        else *(uint32_t *)(to + a.tile.key(place, at.d)) = codes;
        if ((at.d & 31u) == 0) to[at.values ? a.tile.value_scale(place, at.d) : a.tile.key_scale(place, at.d)] = (uint8_t)b;
    }
}

// A place's row of codes and its scale to 16 or 32 bits: bound by HBM (8,448 tokens of 8 heads of 128, 44 MB moved: 10.5 us one call behind the other, 4.2 TB/s), else
// by a chain of three reads (64 tokens 3.4 us).
template <typename T, bool kWhole> __global__ void __launch_bounds__(kThreads) read_kernel(const PackedArgs a) {
    const Place at(a, a.first_group + blockIdx.x);
    if (!at.live || at.d >= a.tile.dim) return;
    const uint32_t slot = (uint32_t)a.slots[at.token], place = slot & (a.tile.block - 1u);
    char *out = at.values ? a.v_out : a.k_out;
    if (slot >= a.n_slots || !out) return;
    out += (int64_t)at.token * (at.values ? a.v_token : a.k_token) + at.d * sizeof(T);
    const uint8_t *const block = a.pages + (int64_t)(slot >> a.sh) * a.page_block;
    for (uint32_t h = at.head0; h < at.heads; ++h) {
        const uint8_t *from = block + (int64_t)h * a.page_head;
        const uint32_t codes = at.values ? get_values(from, a.tile, place, at.d) : *(const uint32_t *)(from + a.tile.key(place, at.d));
        const float s = packed_scale<T>(from[at.values ? a.tile.value_scale(place, at.d) : a.tile.key_scale(place, at.d)]);
        typedef typename Packed<T>::pair pair;
        const pair p[4] = {Packed<T>::template values<0>(codes, s), Packed<T>::template values<1>(codes, s), Packed<T>::template values<2>(codes, s), Packed<T>::template values<3>(codes, s)};
        Eight<T> x;
#pragma unroll
        for (int j = 0; j < 8; ++j) x.v[j] = p[j / 2][j % 2];
        char *to = out + (int64_t)h * (at.values ? a.v_head : a.k_head);
        typedef uint32_t raw __attribute__((ext_vector_type(2 * sizeof(T)), aligned(16)));
        if constexpr (kWhole) *(raw *)to = __builtin_bit_cast(raw, x);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) ((T *)to)[j] = x.v[j];
    }
}

int size_of(int dtype) { return dtype == HPS_SEQ_F32 ? 4 : 2; }

// Lanes, and the heads that a work-group goes through, which share the token's factors: several where there are work-groups enough.  (us, keys and values alone,
// one head / two / four / eight: 8,192 tokens of 8 heads of 128 33.2 / 23.3 / 17.7 / 14.9, with their queries 65.3 / 53.6 / 44.1 / 46.0; 4,000 tokens 17.6 / 13.2 / 10.0 / 12.9;
// 8,192 of 4 heads 17.8 / 13.3 / 10.4.)
constexpr uint32_t kFill = 512;
void share(PackedArgs &a, uint32_t n_tokens) {
    a.lane_bits = 2;
    while ((8u << a.lane_bits) < a.tile.dim) ++a.lane_bits;
    const uint32_t tokens = (kThreads >> a.lane_bits) / 2, chunks = (n_tokens + tokens - 1) / tokens;
    const uint64_t full = (uint64_t)chunks * a.kv_heads;
    a.heads_each = full >= 4 * kFill ? 4 : full >= 2 * kFill ? 2 : 1;
    if (a.heads_each > a.kv_heads) a.heads_each = a.kv_heads;
    a.head_groups = (a.kv_heads + a.heads_each - 1) / a.heads_each;
}

void put_pages(PackedArgs &a, const hps_seq_packed_t &p, uint32_t head_dim) {
    a.pages = p.data;
    a.page_block = p.block_stride;
    a.page_head = p.head_stride;
    a.n_slots = p.n_blocks * p.block_size;
    a.sh = (uint32_t)__builtin_ctz(p.block_size);
    a.tile = Tile{head_dim, head_dim / 32, p.block_size};
}

template <typename T> hipError_t launch_append(PackedArgs &a, bool whole, hipStream_t st) {
    return seq_launches((uint64_t)a.norm.x[0].groups + a.kv_groups, [&](uint32_t first, uint32_t n) {
        a.first_group = first;
        if (whole && a.norm.interleaved) hipLaunchKernelGGL((append_kernel<T, 16 / sizeof(T), true>), dim3(n), dim3(kThreads), 0, st, a);
        else if (whole) hipLaunchKernelGGL((append_kernel<T, 16 / sizeof(T), false>), dim3(n), dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL((append_kernel<T, 1, false>), dim3(n), dim3(kThreads), 0, st, a);
    });
}

template <typename T> hipError_t launch_read(PackedArgs &a, bool whole, hipStream_t st) {
    return seq_launches(a.kv_groups, [&](uint32_t first, uint32_t n) {
        a.first_group = first;
        if (whole) hipLaunchKernelGGL((read_kernel<T, true>), dim3(n), dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL((read_kernel<T, false>), dim3(n), dim3(kThreads), 0, st, a);
    });
}

bool heads16(const void *p, int64_t token, int64_t head) { return seq_aligned(p, 16) && ((token | head) & 15) == 0; }

}  // namespace

hps_status_t seq_check_packed(const hps_seq_packed_t &p, uint32_t head_dim) {
    SEQ_REQUIRE(seq_packed_dim(head_dim), "head_dim must be 32, 64, 96, 128 or 256");
    SEQ_REQUIRE(seq_packed_block(p.block_size), "block_size must be a power of two in 16 .. 1024");
    SEQ_REQUIRE((uint64_t)p.n_blocks * p.block_size < (1ull << 31), "n_blocks * block_size must be < 2^31");
    SEQ_REQUIRE(p.n_blocks == 0 || (p.data && seq_aligned(p.data, 16)), "the pages must be a device pointer, 16-byte aligned");
    SEQ_REQUIRE(p.block_stride >= 0 && p.head_stride >= 0 && ((p.block_stride | p.head_stride) & 15) == 0, "the pages' strides must be multiples of 16 bytes and not negative");
    return HPS_OK;
}

extern "C" {

size_t hps_seq_packed_bytes(uint32_t block_size, uint32_t head_dim) {
    return seq_packed_block(block_size) && seq_packed_dim(head_dim) ? (size_t)block_size * head_dim / 16 * 17 : 0;
}

hps_status_t hps_seq_append_packed(const hps_seq_append_packed_args_t *args, void *stream) {
    SEQ_REQUIRE(args, "args must not be NULL");
    const hps_seq_append_packed_args_t &r = *args;
    if (hps_status_t st = norm_check(r.dtype, r.head_dim, r.rot_dim, r.table, r.positions, r.max_pos, r.n_tokens, r.norm ? r.eps : 0.0, r.q_weight, r.k_weight)) return st;
    if (hps_status_t st = seq_check_packed(r.pages, r.head_dim)) return st;
    SEQ_REQUIRE(r.kv_heads > 0 && (uint64_t)r.q_heads + 2ull * r.kv_heads <= 65536, "kv_heads must be > 0, and at most 65536 heads in all");
    if (r.n_tokens == 0) return HPS_OK;
    SEQ_REQUIRE(seq_words(r.slots), "slots must be a 4-byte aligned device pointer");
    const int size = size_of(r.dtype);
    PackedArgs a{};
    NormArgs &n = a.norm;
    n.positions = r.positions;
    n.table = r.table;
    n.x[0].weight = r.q_weight;
    norm_set_eps(n, r.eps);
    n.per_value = 1.f / (float)r.head_dim;
    n.n_tokens = r.n_tokens;
    n.head_dim = r.head_dim;
    n.half = r.table ? r.rot_dim / 2 : 0;
    n.max_pos = r.max_pos;
    n.interleaved = r.table && r.interleaved;
    n.norm = r.norm != 0;
    SEQ_REQUIRE(norm_put(n, 0, r.q_heads, r.q, r.q_out, nullptr, size) && r.k.data && r.v.data && seq_aligned(r.k.data, size) && seq_aligned(r.v.data, size),
                "q, q_out, k and v must be device pointers aligned to their type");
    a.k = static_cast<const char *>(r.k.data);
    a.v = static_cast<const char *>(r.v.data);
    a.k_token = r.k.token_stride * size;
    a.k_head = r.k.head_stride * size;
    a.v_token = r.v.token_stride * size;
    a.v_head = r.v.head_stride * size;
    a.slots = r.slots;
    a.k_weight = r.k_weight;
    a.eps = r.eps;
    a.per_value = 1.0 / r.head_dim;
    a.kv_heads = r.kv_heads;
    put_pages(a, r.pages, r.head_dim);
    // vectors of eight keys, none of which holds pairs of two kinds
    const bool whole = norm_whole(n, 2 * n.half, size, heads16(a.k, a.k_token, a.k_head) && heads16(a.v, a.v_token, a.v_head) && (n.interleaved ? 2 * n.half : n.half) % 8 == 0);
    norm_share(n, 0, 0xFFFFFFFFu, 4);
    share(a, r.n_tokens);
    const uint32_t tokens = (kThreads >> a.lane_bits) / 2;
    const uint64_t kv_groups = a.n_slots ? (uint64_t)((r.n_tokens + tokens - 1) / tokens) * a.head_groups : 0;
    SEQ_REQUIRE(kv_groups + n.x[0].groups < (1ull << 32), "too many tokens and heads for one call");
    a.kv_groups = (uint32_t)kv_groups;
    hipStream_t st = static_cast<hipStream_t>(stream);
    SEQ_TRY(r.dtype == HPS_SEQ_F32 ? launch_append<float>(a, whole, st) : r.dtype == HPS_SEQ_F16 ? launch_append<_Float16>(a, whole, st) : launch_append<__bf16>(a, whole, st));
    return HPS_OK;
}

hps_status_t hps_seq_read_packed(const hps_seq_packed_t *pages, const int32_t *slots, uint32_t n_tokens, uint32_t kv_heads, uint32_t head_dim,
                                 const hps_seq_heads_t *k_out, const hps_seq_heads_t *v_out, int dtype, void *stream) {
    SEQ_REQUIRE(pages && k_out && v_out, "pages, k_out and v_out must not be NULL");
    SEQ_REQUIRE(dtype == HPS_SEQ_F32 || dtype == HPS_SEQ_F16 || dtype == HPS_SEQ_BF16, "dtype must be HPS_SEQ_F32, HPS_SEQ_F16 or HPS_SEQ_BF16");
    if (hps_status_t st = seq_check_packed(*pages, head_dim)) return st;
    SEQ_REQUIRE(n_tokens < (1u << 31), "n_tokens must be < 2^31");
    SEQ_REQUIRE(kv_heads > 0 && kv_heads <= 65536, "kv_heads must be in 1 .. 65536");
    if (n_tokens == 0 || pages->n_blocks == 0 || (!k_out->data && !v_out->data)) return HPS_OK;
    const int size = size_of(dtype);
    SEQ_REQUIRE(seq_words(slots), "slots must be a 4-byte aligned device pointer");
    SEQ_REQUIRE(seq_aligned(k_out->data, size) && seq_aligned(v_out->data, size), "k_out and v_out must be aligned to their type");
    PackedArgs a{};
    a.norm.n_tokens = n_tokens;
    a.k_out = static_cast<char *>(k_out->data);
    a.v_out = static_cast<char *>(v_out->data);
    a.k_token = k_out->token_stride * size;
    a.k_head = k_out->head_stride * size;
    a.v_token = v_out->token_stride * size;
    a.v_head = v_out->head_stride * size;
    a.slots = slots;
    a.kv_heads = kv_heads;
    put_pages(a, *pages, head_dim);
    const bool whole = heads16(a.k_out, a.k_token, a.k_head) && heads16(a.v_out, a.v_token, a.v_head);
    share(a, n_tokens);
    const uint32_t tokens = (kThreads >> a.lane_bits) / 2;
    const uint64_t groups = (uint64_t)((n_tokens + tokens - 1) / tokens) * a.head_groups;
    SEQ_REQUIRE(groups < (1ull << 32), "too many tokens and heads for one call");
    a.kv_groups = (uint32_t)groups;
    hipStream_t st = static_cast<hipStream_t>(stream);
    SEQ_TRY(dtype == HPS_SEQ_F32 ? launch_read<float>(a, whole, st) : dtype == HPS_SEQ_F16 ? launch_read<_Float16>(a, whole, st) : launch_read<__bf16>(a, whole, st));
    return HPS_OK;
}

}  // extern "C"
