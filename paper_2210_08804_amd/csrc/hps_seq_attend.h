// What attention over pages of 16-bit and of packed values shares: the arguments, how work-groups find their work, and the
// arithmetic of a step.  Not part of the C ABI, and not exported.
#ifndef HPS_SEQ_ATTEND_H
#define HPS_SEQ_ATTEND_H

#include <cmath>

#include "hps_seq_common.h"

// Division of a number below 2^31 by one that the host knows: one of the device's own takes some 40 instructions, and a work-group has five
// in front of its first load.
struct SeqDivisor {
    uint32_t d, m, s;
    static SeqDivisor of(uint32_t d) {
        uint32_t s = 0;
        while (s < 31 && (1u << s) < d) ++s;
        return {d, (uint32_t)((((1ull << s) - d) << 32) / d + 1), s};
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t x) const { return (__umulhi(m, x) + x) >> s; }
};

struct SeqAttendArgs {
    const char *q, *k, *v;
    char *out;
    float *lse, *part_o;
    float2 *part_ml;                                   // reference and sum of each part's row; sum 0: nothing attended
    uint32_t *flags;
    const int32_t *prefix_table, *prefix_lens, *group_offsets, *block_table, *lens, *token_offsets;
    int64_t q_token, q_head, out_token, out_head, page_head;            // strides in bytes
    uint32_t page_block, page_token;
    uint32_t n_tokens, n_requests, n_groups, table_width, prefix_width, max_new, max_group, max_len, max_prefix;
    uint32_t q_heads, kv_heads, ratio, head_dim, n_blocks, sh;
    uint32_t history_groups, history_tiles, history_chunks, history_chunk, history_combos; // work-groups; row tiles; chunks, keys of one; (group, chunk, head)
    uint32_t own_tiles, own_chunks, own_chunk, own_items;
    uint32_t first_group;                              // of this launch
    int32_t history_wide, own_mode, direct;            // direct: one part only, results go straight out
    float c;                                           // scale * log2(e)
    SeqDivisor by_kv_heads, by_ratio, by_history_tiles, by_history_combos, by_history_chunks, by_own_chunks, by_own_tiles;
    int64_t packed_block;                              // packed pages: block stride in bytes; page_head is the heads', k the tiles
};

struct hps_seq_attention_session {
    uint64_t magic;
    size_t max_rows, part_rows;
    uint32_t max_head_dim, cus;
    int device;
    float *part_o;
    float2 *part_ml;
    uint32_t *flags;
};

// What the host goes by where it cuts a call into work-groups.
struct SeqAttendShape {
    uint32_t wide_rows, wide_keys, narrow_keys;        // rows of a wide work-group; keys of a step: of a wide work-group, of a narrow one's wave
    uint32_t (*narrow_rows)(uint64_t most, uint32_t head_dim);              // rows of a narrow work-group, where the most rows that such ones serve behind a stretch are `most`
    uint32_t solo_keys;                                // own keys up to which a wave takes a request where there are many
    bool (*wide)(bool own, uint64_t rows, uint32_t keys, uint64_t stretches, uint32_t head_dim);              // whether rows share keys: `rows` behind each of so many stretches of keys
    uint32_t (*beside)(bool wide, uint32_t head_dim);  // work-groups of a CU at a time
    double (*step)(bool wide, double groups, double beside, uint32_t cus, double size);     // us; size: head_dim / 128
};

// A launch: its work-groups, the parts that they leave, the rows of narrow ones.
struct SeqAttendCut { uint32_t groups, parts, narrow_rows; };

// Sets the launch's sizes in `a` and `cut`.  What kind of work-groups histories and own tokens have is decided here and nowhere else: a.history_wide, a.own_mode.
SEQ_HIDDEN hps_status_t seq_attend_cut(SeqAttendArgs &a, const SeqAttendShape &shape, const hps_seq_attention_session &s, SeqAttendCut &cut);
// In front of the attention: flags histories that a bound of 0 keeps out of the launch.  Behind it: joins the parts.
SEQ_HIDDEN hipError_t seq_attend_check(const SeqAttendArgs &a, hipStream_t st);
SEQ_HIDDEN hipError_t seq_attend_join(const SeqAttendArgs &a, int dtype, uint32_t parts, hipStream_t st);
// Kernels that use more LDS than 64 KiB have to be told so once a device: those of packed pages.
SEQ_HIDDEN hipError_t seq_packed_allow_lds();

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;
typedef const __attribute__((address_space(4))) int32_t scalar_i32;

constexpr uint64_t kMagic = 0x4850535345514154ull;
constexpr float kInf = __builtin_inff();
constexpr uint32_t kMaxParts = 1024;
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr uint32_t kWideRows = 128, kNarrowRows = 32;  // rows of a work-group
constexpr uint32_t kWideKeys = 64, kNarrowKeys = 32;   // keys of a step: of the work-group, of a wave
// A row's reference m need not be its maximum.  Where it moves it goes to kBelow below the largest score (in powers of two), and it
// moves when a score is kSlack ahead of it, or 16 weights of a lane sum to kMost, far within the type's range: most steps need
// no rescaling then.  bf16 has the exponents of 32 bits, so its weights lose the same few bits wherever the reference is.  f16 has
// none below 2^-14 and loses weights of 2^-25 whole, which a long history has many of behind one large weight: its reference stays 8
// below the largest score, which leaves weights of 2^-22 of the largest their bits (15,000 keys of which 31 in 32 have a weight of
// 2^-26: with the largest score for a reference all of those were lost, now they are 1 % off at most).

typedef SeqAttendArgs Args;
enum { kOwnSplit = 0, kOwnSolo = 1, kOwnWide = 2 };    // a work-group's waves share the keys; have an item each; share the rows

template <typename T> struct Type;
template <> struct Type<__bf16> {
    typedef bf16x8 frag;
    static __device__ __forceinline__ f32x16 mfma(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static constexpr uint32_t kExp = 0x7F80u;
    static constexpr float kBelow = 0.f, kSlack = 8.f, kMost = 0x1p12f;
};
template <> struct Type<_Float16> {
    typedef f16x8 frag;
    static __device__ __forceinline__ f32x16 mfma(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static constexpr uint32_t kExp = 0x7C00u;
    static constexpr float kBelow = 8.f, kSlack = 15.f, kMost = 0x1p15f;    // weights stay below 2^15, f16 ends at 2^16
};

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ int32_t scalar(const int32_t *p, size_t i) { return ((scalar_i32 *)(uintptr_t)p)[i]; }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// maximum and sum with the lane that holds the row's other keys
__device__ __forceinline__ float both_max(float x) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float both_sum(float x) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// 64 lanes' 16 bytes from base + off (or from an address of each lane) to LDS at `to` + 16 * lane.  The caller waits for vmcnt;
// lanes that are switched off leave their place in LDS alone.  (Not the builtin: the compiler then waits for every such
// load in front of any read of LDS, and the next step's loads are what is to stay in flight.)
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, uint32_t to) {
    uint32_t kept;                                     // m0 is the compiler's: it gets it back (which costs no time beside the load)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(to), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t to) {
    uint32_t kept;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(to), "v"(from) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Keeps x in its 16 adjacent registers.  Where a loop's vector starts as a constant or is put together from elements, the
// compiler takes it to pieces for the loop, and moves them into place in front of every matrix instruction.
__device__ __forceinline__ void whole(f32x16 &x) { asm("" : "+v"(x)); }

// What a wave attends with: 32 rows against keys first .. end of one table.
struct Item {
    const int32_t *table;
    uint32_t first, end;
    uint32_t token0, row0, rows;                       // the tile's rows are row0 .. of `rows` (token, head) pairs from token0 on
    uint32_t head, part;                               // key/value head; part that the result is
    int32_t causal_from;                               // row's query i sees keys below causal_from + i; or kAll
    int32_t id0, id1;                                  // blocks of the first 32 keys of the wave, read ahead of the lengths (a place that the table holds)
};
constexpr int32_t kAll = 0x7FFFFFFF;

// kCleared: places of LDS rows that no load fills are zeros.
template <typename T, int DT, bool kExact, bool kCleared = true> struct Engine {            // head_dim <= 32 * DT, or just that
    typedef typename Type<T>::frag frag;
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    static constexpr int kRow = DT <= 2 ? 128 : DT <= 4 ? 256 : 512;        // bytes of a row in LDS
    static constexpr int kChunks = kRow / 16, kSteps = 2 * DT;
    static constexpr bool kFull = kExact && 64 * DT == kRow;                // every chunk of a row in LDS is one of the head's
    static constexpr int kLoads = 16 * kRow / 1024, kLoadRows = 1024 / kRow;        // wave loads of 16 rows, rows of one
    static constexpr uint32_t kLds = 256 * kRow;       // wide: 2 stages of 64 keys and values; narrow: 4 waves of 32
    static constexpr uint32_t kWaveLds = 64 * kRow;    // of a narrow wave
    static constexpr uint32_t kStage = 128 * kRow, kWideValues = 64 * kRow, kNarrowValues = 32 * kRow;

    const Args &a;
    const Item it;
    const uint32_t lane, half, lds;
    const char *const k_head, *const v_head;
    frag q[kSteps];
    f32x16 o[DT];
    float m, l;
    int32_t limit;                                     // the lane's row sees keys below it
    // The lane's places, as a row's offset and a chunk's within the row: the operands of both products in LDS, and the 16
    // bytes that it loads.  The other chunks are reached by an exclusive or, one instruction each (`fresh` keeps the
    // compiler from holding all of them in registers instead, which cost spills in the middle of the loop).
    uint32_t k_row, k_chunk, v_row, v_chunk, load_row, load_k, load_v;
    uint32_t here;                                     // LDS address of the keys at hand

    static __device__ __forceinline__ uint32_t sw_k(uint32_t t) { return t & (kRow == 128 ? 7u : 15u); }
    static __device__ __forceinline__ uint32_t sw_v(uint32_t t) { return ((kRow == 128 ? (t >> 1) & 1u : t & 3u) << 2) | ((t >> 2) & 3u); }
    template <bool kValues> static __device__ __forceinline__ uint32_t sw(uint32_t t) { return kValues ? sw_v(t) : sw_k(t); }

    __device__ __forceinline__ Engine(const Args &args, const Item &item, uint32_t lds_base, uint32_t first_row)
        : a(args), it(item), lane(threadIdx.x & 63u), half(lane >> 5), lds(lds_base), k_head(args.k + (int64_t)item.head * args.page_head),
          v_head(args.v + (int64_t)item.head * args.page_head) {
        const uint32_t n = lane & 31u, g = lane & 15u;
        here = lds;
        k_row = lds + n * kRow;
        k_chunk = (half ^ sw_k(n)) << 4;
        const uint32_t t = 4 * half + (g >> 2), r = lane / kChunks;
        v_row = lds + t * kRow;
        v_chunk = ((2 * ((lane >> 4) & 1u) + ((g & 3u) >> 1)) ^ sw_v(t)) << 4 | (g & 1u) << 3;
        load_row = r * a.page_token;
        load_k = (lane % kChunks ^ sw_k(r)) << 4;
        load_v = (lane % kChunks ^ sw_v(r)) << 4;
        const uint32_t row = it.row0 + first_row + n, i = row / a.ratio;
        const bool there = row < it.rows;
        limit = it.causal_from == kAll ? (int32_t)it.end : min((int32_t)it.end, it.causal_from + (int32_t)i);
        const char *src = a.q + (int64_t)(it.token0 + i) * a.q_token + (int64_t)(it.head * a.ratio + (row - i * a.ratio)) * a.q_head;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            u32x4 x = {0, 0, 0, 0};
            if (there && (kExact || (uint32_t)(16 * s + 8 * half) < a.head_dim)) x = *(const u32x4 *)(src + (16 * s + 8 * half) * 2);
            q[s] = __builtin_bit_cast(frag, x);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            o[d] = f32x16{};
            whole(o[d]);
        }
        m = -kInf;
        l = 0.f;
        if (!there) limit = kAll;                      // their results go nowhere
    }

    __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(k_chunk), "+v"(v_chunk), "+v"(load_k), "+v"(load_v)); }
    // of key operand i; of value operand d, its second half 8 rows on
    __device__ __forceinline__ lds_char *k_at(int i) const { return (lds_char *)(uintptr_t)(k_row + (k_chunk ^ (uint32_t)(i << 5))); }
    __device__ __forceinline__ lds_char *v_at(int j, int d) const { return (lds_char *)(uintptr_t)(v_row + (v_chunk ^ (uint32_t)(d << 6) ^ (uint32_t)(j << 5))) + j * 8 * kRow; }

    // Block of the 16 keys from `at` on; -1 where there are none, or where blocks are smaller.
    __device__ __forceinline__ int32_t block_of(uint32_t at) const { return a.sh >= 4 && at < it.end ? scalar(it.table, at >> a.sh) : -1; }

    // Rows of 16 keys (or values) from token `at` on to LDS.  Whole ones of a block: returns true, the loads are under way,
    // kLoads of them.  At the end of the keys, for small blocks and for a block number that is none: each lane by itself,
    // zeros in the place of what is not there.  (Blocks of fewer than 16 tokens always come this way, and wait for it: 256 requests behind
    // 8,192 keys 83 us instead of 38, 4 behind 200,003 718 instead of 156.)
    template <bool kValues> __device__ __forceinline__ bool load16(uint32_t at, int32_t id, uint32_t to) {
        const char *head = kValues ? v_head : k_head;
        if (__builtin_expect(at + 16 <= it.end && (uint32_t)id < a.n_blocks, 1)) {
            const char *base = head + (uint64_t)(uint32_t)id * a.page_block + (uint64_t)(at & ((1u << a.sh) - 1u)) * a.page_token;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const uint32_t chunk = (kValues ? load_v : load_k) ^ sw<kValues>(i * kLoadRows) << 4;
                if (kFull || chunk < 2 * a.head_dim) load_to_lds(base + (uint64_t)a.page_token * (i * kLoadRows), load_row + chunk, to + i * 1024);
            }
            return true;
        }
#pragma unroll 1
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t t = i * kLoadRows + lane / kChunks, chunk = (lane % kChunks) ^ sw<kValues>(t), key = at + t;
            if (!kFull && chunk * 8 >= a.head_dim) continue;               // nothing ever lies there
            const char *from = nullptr;
            if (key < it.end) {
                const uint32_t b = (uint32_t)it.table[key >> a.sh];
                if (b < a.n_blocks) from = head + (uint64_t)b * a.page_block + (uint64_t)(key & ((1u << a.sh) - 1u)) * a.page_token + chunk * 16;
                else atomicOr(a.flags, HPS_SEQ_FLAG_BLOCK);
            }
            if (from) load_to_lds(from, to + i * 1024);
            else *(lds_u32x4 *)(lds_char *)(uintptr_t)(to + i * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
        }
        return false;
    }

    template <bool kValues> __device__ __forceinline__ bool load32(uint32_t at, int32_t id0, int32_t id1, uint32_t to) {
        const bool x = load16<kValues>(at, id0, to), y = load16<kValues>(at + 16, id1, to + 16 * kRow);
        return x && y;
    }

    // Scores of 32 keys, kAt bytes behind the first ones.
    template <int kAt> __device__ __forceinline__ f32x16 scores() const {
        f32x16 s{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) s = Type<T>::mfma(*(__attribute__((address_space(3))) frag *)(k_at(i) + kAt), q[i], s);
        return s;
    }
    static __device__ __forceinline__ uint32_t key_of(int i, uint32_t half) { return 8 * (i >> 2) + 4 * half + (i & 3); }

    // Hides what the lane's row does not see; a bit for each key that it sees.
    __device__ __forceinline__ uint32_t hide(f32x16 &s, uint32_t at) const {
        uint32_t seen = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const bool see = (int32_t)(at + key_of(i, half)) < limit;
            seen |= see ? 1u << i : 0u;
            s[i] = see ? s[i] : -kInf;
        }
        return seen;
    }

    // The row's largest score, in powers of two.
    __device__ __forceinline__ float largest(const f32x16 &s) const {
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        return both_max(top) * a.c;
    }
    // Moves the reference to the largest score so far (or kBelow below it), and what was summed with it.
    __device__ __forceinline__ void move(float top) {
        const float next = fmaxf(m, top - Type<T>::kBelow), ref = next == -kInf ? 0.f : next, f = exp2_(m - ref);
        l *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            o[d] *= f;
            whole(o[d]);
        }
        m = next;
    }
    __device__ __forceinline__ float reference() const { return m == -kInf ? 0.f : m; }       // -inf: nothing but -inf so far
    // Weights of 32 keys' scores, rounded for the second product, and their sum (of the lane's keys) before that.
    __device__ __forceinline__ float weights(const f32x16 &s, frag (&w)[2], float ref) const {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float x = exp2_(__builtin_fmaf(s[i], a.c, -ref));
            sum += x;
            w[i / 8][i % 8] = (T)x;
        }
        return sum;
    }

    template <int kAt> __device__ __forceinline__ frag values(int d) const {
        s16x4 x[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
            x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(v_at(j, d) + kAt));
        return __builtin_bit_cast(frag, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }

    // o += weights x values of 32 keys, kAt bytes behind the first ones.
    template <int kAt> __device__ __forceinline__ void add_values(const frag (&w)[2]) {
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = Type<T>::mfma(values<kAt>(d), w[0], o[d]);
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = Type<T>::mfma(values<kAt + 16 * kRow>(d), w[1], o[d]);
    }
    // Whether any value of 32 keys, kAt bytes behind the first ones, is not finite.  (Where places that the head does not
    // fill are not cleared they hold what an earlier kernel left, and have no say.)
    template <int kAt> __device__ __forceinline__ bool any_odd() const {
        constexpr uint32_t e = Type<T>::kExp;
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < 2 * kLoads; ++i) {
            if (!kCleared && !kFull && (lane % kChunks ^ sw_v(i * kLoadRows + lane / kChunks)) >= 4 * DT) continue;
            const u32x4 y = *(lds_u32x4 *)((lds_char *)(uintptr_t)(here + lane * 16) + kAt + i * 1024);
#pragma unroll
            for (int j = 0; j < 4; ++j) odd |= (uint32_t)((y[j] & e) == e) | (uint32_t)((y[j] >> 16 & e) == e);
        }
        return __ballot(odd) != 0;
    }
    // o += weights x values where some rows do not see some keys.  A hidden value that is not finite must not meet the
    // weight 0: where there is any that is not finite, the products are formed one by one, with the same rounding.
    template <int kAt> __device__ __forceinline__ void add_values_hidden(const frag (&w)[2], uint32_t seen) {
        if (!__builtin_expect(any_odd<kAt>(), 0)) return add_values<kAt>(w);
#pragma unroll 1
        for (int i = 0; i < 32; ++i) {                 // keys; the lane holds the weights of those with bit 2 as its half
            const int mine = (i >> 3) * 4 + (i & 3);
            float x = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) x = j == mine ? (float)w[j / 8][j % 8] : x;
            const u32x2 both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
            const u32x2 sees = __builtin_amdgcn_permlane32_swap(seen >> mine & 1u, seen >> mine & 1u, false, false);
            const float wi = __uint_as_float(i & 4 ? both.y : both.x);
            const bool see = i & 4 ? sees.y : sees.x;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint32_t dim = 32 * d + key_of(j, half);
                    const float v = (float)*(__attribute__((address_space(3))) T *)((lds_char *)(uintptr_t)(here + i * kRow + ((dim / 8 ^ sw_v(i)) << 4) + dim % 8 * 2) + kAt);
                    o[d][j] += see ? wi * v : 0.f;
                }
        }
    }

    __device__ __forceinline__ uint32_t least_limit() const {               // over the wave's rows
        int32_t x = max(limit, 0);
        for (int d = 1; d < 32; d <<= 1) x = min(x, __shfl_xor(x, d));
        return uniform((uint32_t)x);
    }

    // A work-group's four waves have 32 rows each and share keys and values: 64 of either a step, two places for either, one
    // meeting a step.  The scores of the next 32 keys are formed beside the weights of these, so that a wave's matrix
    // instructions run while it computes exponentials: the keys of a step are 32 ahead of its values.
    // The inner loop has the steps of which every row sees all keys and whose reference can stay: weights may be large, they
    // only must not overflow (kMost), which their sum shows.  The others leave it for the end of the step.
    // Bound by the matrix instructions and what they wait for: 512 requests of 32 / 8 heads of 128 behind 32,768 keys take 285 to
    // 298 us in this kernel by device (964 to 924 TFLOP/s; of 307 at the time matrix instructions alone took 210, all but the loads 249, all
    // but the exponentials 287).  The matrix pipes are busy 48 % of all cycles, LDS 24 % without a bank conflict (waves wait 3 % of
    // their time to issue to it), the clock is 1.86 to 2.0 GHz.  Two meetings a step 318 us instead of 307; eight waves to a work-group 292 instead of 299, but 42.5 instead of 40.2 for 256 requests behind 8,192 keys.
    __device__ __forceinline__ void wide() {
        const uint32_t wave = uniform(threadIdx.x >> 6), least = least_limit(), mine = 16 * wave;
        if (it.first >= it.end) return;                // uniform in the work-group, as are all meetings
        uint32_t at = it.first;                        // the step's first value; its first key is 32 further on
        uint32_t keys_to = lds + mine * kRow, values_to = keys_to + kWideValues, flip = kStage;
        // keys `first` .. + 32 go to the second half of the other place, as if they were the end of a step in front
        if (wave >= 2) load16<false>(at + mine - 32, block_of(at + mine - 32), keys_to + kStage);
        if (at + 32 < it.end) load16<false>(at + 32 + mine, block_of(at + 32 + mine), keys_to);
        int32_t value_id = block_of(at + mine), key_id = block_of(at + 96 + mine);          // of the values and of the keys that are fetched next
        load16<true>(at + mine, value_id, values_to);
        value_id = block_of(at + 64 + mine);
        wait_loads<0>();
        meet();
        k_row += kStage;
        f32x16 s = scores<32 * kRow>(), t;
        k_row -= kStage;
        auto start = [&] {                             // everybody is done with the last step's keys and values
            wait_loads<0>();
            meet();
            if (at + 96 < it.end) load16<false>(at + 96 + mine, key_id, keys_to + flip);
            if (at + 64 < it.end) load16<true>(at + 64 + mine, value_id, values_to + flip);
            key_id = block_of(at + 160 + mine);
            value_id = block_of(at + 128 + mine);
            fresh();
        };
        auto end = [&] {                               // the places change
            keys_to += flip;
            values_to += flip;
            k_row += flip;
            v_row += flip;
            here += flip;
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
                t = scores<0>();
                float sum = weights(s, w, m);       // infinite, or NaN, the first time: m is -inf
                if (__ballot(!(sum < Type<T>::kMost))) {
                    ahead = true;
                    break;
                }
                l += sum;
                add_values<kWideValues>(w);
                s = scores<32 * kRow>();
                sum = weights(t, w, m);
                if (__ballot(!(sum < Type<T>::kMost))) {
                    ahead = true;
                    left = 1;
                    const f32x16 x = s;
                    s = t;
                    t = x;
                    break;
                }
                l += sum;
                add_values<kWideValues + 32 * kRow>(w);
                end();
                if (at >= it.end) return;
            }
            if (left == 2) {
                rest<kWideValues>(s, w, at, least);
                s = ahead ? t : scores<0>();
                t = scores<32 * kRow>();
            }
            rest<kWideValues + 32 * kRow>(s, w, at + 32, least);
            s = t;
            end();
            if (at >= it.end) return;
        }
    }
    // 32 keys of which some may be hidden, and whose scores may be far above the reference.
    template <int kAt> __device__ __forceinline__ void rest(f32x16 &s, frag (&w)[2], uint32_t at, uint32_t least) {
        const bool hidden = at + 32 > least;           // uniform
        uint32_t seen = 0xFFFFu;
        if (hidden) seen = hide(s, at);
        const float top = largest(s);
        if (__ballot(top > m + Type<T>::kSlack)) move(top);
        l += weights(s, w, reference());
        if (hidden && it.causal_from != kAll) add_values_hidden<kAt>(w, seen);
        else add_values<kAt>(w);
    }

    // One wave, 32 rows, every `stride`-th 32 keys from `from` on, in its own part of LDS: the next keys are fetched as soon
    // as the scores are there, the next values behind the product with these.  Bound by HBM where histories are long (4 requests of
    // 32 / 8 heads of 128 behind 200,003 keys: 146 to 153 us, 5.4 to 5.6 TB/s; a kernel that only reads as much takes 153 to 160), else by the chain offsets, block, keys, scores, values.
    __device__ __forceinline__ void narrow(uint32_t from, uint32_t stride) {
        const uint32_t least = least_limit();
        if (from >= it.end) return;
        int32_t id0 = block_of(from), id1 = block_of(from + 16);
        // whether the last keys and the last values asked for are under way, as 2 * kLoads loads each
        bool keys_fly = load32<false>(from, id0, id1, lds), values_fly = load32<true>(from, id0, id1, lds + kNarrowValues);
        for (uint32_t at = from;;) {
            f32x16 s;
            frag w[2];
            float top;
            bool full, more;
            uint32_t next;
            auto next_values = [&] {
                if (more) {
                    wait_lds();
                    values_fly = load32<true>(next, id0, id1, lds + kNarrowValues);
                }
                at = next;
            };
            auto wait_values = [&] {
                if (more && keys_fly && values_fly) wait_loads<2 * kLoads>();
                else wait_loads<0>();
            };
            for (;;) {
                if (at >= it.end) return;
                next = at + stride;
                more = next < it.end;
                fresh();
                id0 = block_of(next);
                id1 = block_of(next + 16);
                if (keys_fly && values_fly) wait_loads<2 * kLoads>();
                else wait_loads<0>();
                s = scores<0>();
                if (more) {
                    wait_lds();
                    keys_fly = load32<false>(next, id0, id1, lds);
                }
                full = at + 32 <= least;
                if (!full) break;
                top = largest(s);
                if (__ballot(top > m + Type<T>::kSlack)) break;                      // also the first time: m is -inf
                l += weights(s, w, reference());
                wait_values();
                add_values<kNarrowValues>(w);
                next_values();
            }
            uint32_t seen = 0xFFFFu;
            if (!full) {
                seen = hide(s, at);
                top = largest(s);
            }
            move(top);
            l += weights(s, w, reference());
            wait_values();
            if (!full && it.causal_from != kAll) add_values_hidden<kNarrowValues>(w, seen);
            else add_values<kNarrowValues>(w);
            next_values();
        }
    }

    // Where a row's values go: final, or as a part.
    struct Place {
        char *to;
        bool direct;
        float f;
        uint32_t dims;
        __device__ __forceinline__ void put4(uint32_t dim, f32x4 x) const {
            if (!kExact && dim >= dims) return;
            if (direct) {
                typedef T t4 __attribute__((ext_vector_type(4)));
                t4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = f == 0.f ? (T)0.f : (T)(x[j] * f);      // nothing attended: 0, though weights of 0 met values that are not finite
                *(t4 *)(to + dim * 2) = y;
            } else {
                *(f32x4 *)(to + dim * 4) = x;
            }
        }
    };
    // Stores the row's reference and sum (one lane of it), and returns its place.
    __device__ __forceinline__ Place place(uint32_t row, float ref, float sum, bool first) const {
        const uint32_t i = row / a.ratio, h = it.head * a.ratio + (row - i * a.ratio), t = it.token0 + i;
        const size_t at = (size_t)t * a.q_heads + h, part = (size_t)it.part * a.n_tokens * a.q_heads + at;
        if (first) {
            if (!a.direct) a.part_ml[part] = make_float2(ref, sum);
            else if (a.lse) a.lse[at] = sum == 0.f ? -kInf : (ref + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
        }
        return {a.direct ? a.out + (int64_t)t * a.out_token + (int64_t)h * a.out_head : (char *)(a.part_o + part * a.head_dim), a.direct != 0, sum == 0.f ? 0.f : 1.f / sum,
                a.head_dim};
    }
    // The wave's own rows, as they are.
    __device__ __forceinline__ void finish(uint32_t first_row) {
        const uint32_t row = it.row0 + first_row + (lane & 31u);
        const float sum = both_sum(l);
        if (row >= it.rows) return;
        const Place p = place(row, m, sum, half == 0);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) p.put4(32 * d + 8 * i + 4 * half, f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]});
    }
    // The four waves have the same rows and different keys: joined through LDS, each wave a quarter of the values.
    __device__ __forceinline__ void finish_split(char *shared) {
        const uint32_t wave = uniform(threadIdx.x >> 6), row = it.row0 + (lane & 31u);
        const float sum = both_sum(l);
        float2 *l_ml = (float2 *)(shared + kLds);
        __syncthreads();
        f32x4 *l_o = (f32x4 *)shared;                  // [wave][DT * 4][64]
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                l_o[(wave * DT * 4 + d * 4 + i) * 64 + lane] = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
        if (half == 0) l_ml[wave * 32 + lane] = make_float2(m, sum);
        __syncthreads();
        float ref = -kInf, total = 0.f, f[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) ref = fmaxf(ref, l_ml[w * 32 + (lane & 31u)].x);
        const float at = ref == -kInf ? 0.f : ref;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2 x = l_ml[w * 32 + (lane & 31u)];
            f[w] = exp2_(x.x - at);
            total += f[w] * x.y;
        }
        if (row >= it.rows) return;
        const Place p = place(row, ref, total, wave == 0 && half == 0);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const uint32_t x = wave * DT + i;
            f32x4 y{};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) y += f[w] * l_o[(w * DT * 4 + x) * 64 + lane];
            p.put4(8 * x + 4 * half, y);
        }
    }
};

// Rows of a tile whose part has nothing.
__device__ __forceinline__ void mark_empty(const Args &a, const Item &it, uint32_t part, uint32_t n, uint32_t lane, uint32_t lanes) {
    for (uint32_t x = lane; x < n && it.row0 + x < it.rows; x += lanes) {
        const uint32_t row = it.row0 + x, i = row / a.ratio, h = it.head * a.ratio + (row - i * a.ratio);
        a.part_ml[((size_t)part * a.n_tokens + it.token0 + i) * a.q_heads + h] = make_float2(-kInf, 0.f);
    }
}

__device__ __forceinline__ uint32_t clamp_to(int32_t x, uint32_t most) { return min((uint32_t)max(x, 0), most); }

// A length as the tables and the launch hold it.
__device__ __forceinline__ uint32_t length(const Args &a, int32_t x, uint32_t width, uint32_t most) {
    const uint32_t n = (uint32_t)max(x, 0), fits = min(width << a.sh, most);
    if (n > fits) atomicOr(a.flags, HPS_SEQ_FLAG_LENGTH);
    return min(n, fits);
}

inline bool seq_multiple16(int64_t stride) { return (stride * 2 & 15) == 0; }
inline bool seq_heads16(const hps_seq_heads_t &h) { return h.data && seq_aligned(h.data, 16) && seq_multiple16(h.token_stride) && seq_multiple16(h.head_stride); }

// The checks that calls over either kind of pages share, and what they put into the arguments.  work: whether there are any rows.
template <typename R> hps_status_t seq_attend_args(const hps_seq_attention_t *s, const R *args, Args &a, bool &work) {
    SEQ_REQUIRE(s && s->magic == kMagic, "not a live attention session");
    SEQ_REQUIRE(args, "args must not be NULL");
    const R &r = *args;
    int device = -1;
    SEQ_TRY(hipGetDevice(&device));
    SEQ_REQUIRE(device == s->device, "the session is of another device than the current one");
    SEQ_REQUIRE(r.dtype == HPS_SEQ_F16 || r.dtype == HPS_SEQ_BF16, "dtype must be HPS_SEQ_F16 or HPS_SEQ_BF16");
    SEQ_REQUIRE(r.head_dim > 0 && r.head_dim <= 256, "head_dim must be in 1 .. 256");
    SEQ_REQUIRE(r.head_dim <= s->max_head_dim, "head_dim exceeds the session's max_head_dim");
    SEQ_REQUIRE(r.kv_heads > 0 && r.q_heads > 0 && r.q_heads % r.kv_heads == 0 && r.q_heads <= 65536, "q_heads must be a multiple of kv_heads, at most 65536");
    SEQ_REQUIRE(std::isfinite(r.scale) && r.scale > 0, "scale must be finite and > 0");
    SEQ_REQUIRE((uint64_t)r.n_tokens * r.q_heads <= s->max_rows, "n_tokens * q_heads exceeds the session's max_rows");
    SEQ_REQUIRE(seq_block_size(r.pages.block_size), "block_size must be a power of two in 1 .. 1024");
    SEQ_REQUIRE((uint64_t)r.pages.n_blocks * r.pages.block_size < (1ull << 31), "n_blocks * block_size must be < 2^31");
    SEQ_REQUIRE((uint64_t)r.table_width * r.pages.block_size < (1ull << 31) && (uint64_t)r.prefix_width * r.pages.block_size < (1ull << 31),
                "table_width and prefix_width times block_size must be < 2^31");
    SEQ_REQUIRE(r.max_len < (1u << 30) && r.max_prefix < (1u << 30), "max_len and max_prefix must be < 2^30");
    SEQ_REQUIRE(r.n_requests <= (1u << 24) && r.n_groups <= (1u << 24), "n_requests and n_groups must be <= 2^24");
    work = r.n_tokens != 0 && r.n_requests != 0;
    if (!work) return HPS_OK;
    SEQ_REQUIRE(seq_heads16(r.q) && seq_heads16(r.out), "q and out must be device pointers, 16-byte aligned, their strides multiples of 16 bytes");
    SEQ_REQUIRE(seq_words(r.token_offsets) && seq_words(r.lens), "token_offsets and lens must be 4-byte aligned device pointers");
    SEQ_REQUIRE(r.table_width == 0 || seq_words(r.block_table), "block_table must be a 4-byte aligned device pointer");
    SEQ_REQUIRE(r.n_groups == 0 || (seq_words(r.prefix_lens) && seq_words(r.group_offsets) && (r.prefix_width == 0 || seq_words(r.prefix_table))),
                "prefix_table, prefix_lens and group_offsets must be 4-byte aligned device pointers");
    SEQ_REQUIRE(r.lse == nullptr || seq_aligned(r.lse, 4), "lse must be 4-byte aligned");
    a.q = static_cast<const char *>(r.q.data);
    a.out = static_cast<char *>(r.out.data);
    a.lse = r.lse;
    a.part_o = s->part_o;
    a.part_ml = s->part_ml;
    a.flags = s->flags;
    a.prefix_table = r.prefix_table;
    a.prefix_lens = r.prefix_lens;
    a.group_offsets = r.group_offsets;
    a.block_table = r.block_table;
    a.lens = r.lens;
    a.token_offsets = r.token_offsets;
    a.q_token = r.q.token_stride * 2;
    a.q_head = r.q.head_stride * 2;
    a.out_token = r.out.token_stride * 2;
    a.out_head = r.out.head_stride * 2;
    a.n_tokens = r.n_tokens;
    a.n_requests = r.n_requests;
    a.n_groups = r.n_groups;
    a.table_width = r.table_width;
    a.prefix_width = r.prefix_width;
    a.max_new = r.max_new < r.n_tokens ? r.max_new : r.n_tokens;
    a.max_group = r.max_group < r.n_tokens ? r.max_group : r.n_tokens;
    a.max_len = r.max_len;
    a.max_prefix = r.max_prefix;
    a.q_heads = r.q_heads;
    a.kv_heads = r.kv_heads;
    a.ratio = r.q_heads / r.kv_heads;
    a.head_dim = r.head_dim;
    a.n_blocks = r.pages.n_blocks;
    a.sh = (uint32_t)__builtin_ctz(r.pages.block_size);
    a.c = r.scale * 1.4426950408889634f;
    return HPS_OK;
}

}  // namespace

#endif  // HPS_SEQ_ATTEND_H
