// Attention of new tokens over a history that their group shares and over their request's own tokens (hps_seq.h), for
// gfx950.
//
//   o_t = sum_j w_tj v_j / sum_j w_tj,   w_tj = exp(scale * q_t . k_j - m_t)
//
// Sums over disjoint sets of keys join: with (m, l, o) = (reference, sum of weights, weighted sum) of each,
// m = max m_i, l = sum 2^(m_i - m) l_i, o = sum 2^(m_i - m) o_i (in powers of two).  So the history is attended once for
// all rows of its group - the rows of a matrix product are the (token, query head) pairs that share a key/value head -
// and a request's own tokens separately; long stretches of keys are cut into chunks where there are few rows; and a
// second kernel joins what the parts left behind.
//
// Scores are computed transposed, S^T = K Q^T, with 32x32x16 matrix instructions: lane l holds 16 of the 32 keys' scores
// of row l % 32, so a row's maximum and sum are almost wholly within a lane, and the weights, rounded, are at once the
// second operand of O^T = V^T W^T.  Both products read their first operand from LDS: keys 16 bytes along a row, values
// transposed on the way (ds_read_b64_tr_b16).  Rows of keys and values go from memory to LDS without registers between; chunks of 16
// bytes change places within their row there (sw_k, sw_v), so that the lanes of one read meet all banks.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "hps_seq_common.h"

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
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr uint32_t kWideRows = 128, kNarrowRows = 32;  // rows of a work-group
constexpr uint32_t kWideKeys = 64, kNarrowKeys = 32;   // keys of a step: of the work-group, of a wave
// A row's reference m need not be its maximum.  Where it moves it goes to kBelow below the largest score (in powers of two), and it
// moves when a score is kSlack ahead of it, or 16 weights of a lane sum to kMost, far within the type's range: most steps need
// no rescaling then.  bf16 has the exponents of 32 bits, so its weights lose the same few bits wherever the reference is.  f16 has
// none below 2^-14 and loses weights of 2^-25 whole, which a long history has many of behind one large weight: its reference stays 8
// below the largest score, which leaves weights of 2^-22 of the largest their bits (15,000 keys of which 31 in 32 have a weight of
// 2^-26: with the largest score for a reference all of those were lost, now they are 1 % off at most).

struct Args {
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
};
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
};
constexpr int32_t kAll = 0x7FFFFFFF;

template <typename T, int DT, bool kExact> struct Engine {                  // head_dim <= 32 * DT, or just that
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
    // Whether any value of 32 keys, kAt bytes behind the first ones, is not finite.
    template <int kAt> __device__ __forceinline__ bool any_odd() const {
        constexpr uint32_t e = Type<T>::kExp;
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < 2 * kLoads; ++i) {
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

template <typename T, int DT, bool kExact> __global__ void __launch_bounds__(kThreads, DT <= 4 ? 2 : 1) attend_kernel(const Args a) {
    typedef Engine<T, DT, kExact> E;
    extern __shared__ __align__(16) char shared[];
    const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_char *)shared;
    if (!E::kFull) {                                   // places of LDS rows that no load fills
        for (uint32_t x = threadIdx.x * 16; x < E::kLds; x += kThreads * 16) *(u32x4 *)(shared + x) = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    const uint32_t group = a.first_group + blockIdx.x;
    Item it;
    bool is_wide, solo = false;
    if (group < a.history_groups) {
        // Work-groups of one (group, chunk, head) read the same keys: they go to one XCD (workgroups are dealt to the eight in turn).
        uint32_t combo, tile;
        if (a.history_combos >= 8) {
            const uint32_t y = group >> 3;
            combo = (group & 7u) + 8 * (y / a.history_tiles);
            tile = y % a.history_tiles;
            if (combo >= a.history_combos) return;
        } else {
            combo = group % a.history_combos;
            tile = group / a.history_combos;
        }
        // From chunk to chunk the heads go round, so that an XCD has different ones at a time: where the heads of a token lie
        // side by side, one head's rows are in few of the L2's channels.
        // From group to group the chunks do: where histories end at different lengths, the last chunks have little to do, and must not
        // all be one XCD's (26 groups of 187 to 3,000 keys, two heads of 64, 4 chunks 50.6 -> 42.8 us, 8 chunks 51.7 -> 48.6).
        const uint32_t rest = combo / a.kv_heads, g = rest / a.history_chunks, chunk = (rest + g) % a.history_chunks;
        it.head = (combo + rest) % a.kv_heads;
        const uint32_t r0 = clamp_to(scalar(a.group_offsets, g), a.n_requests), r1 = clamp_to(scalar(a.group_offsets, g + 1), a.n_requests);
        const uint32_t t0 = clamp_to(scalar(a.token_offsets, r0), a.n_tokens), t1 = clamp_to(scalar(a.token_offsets, r1), a.n_tokens);
        const uint32_t n = t1 > t0 ? t1 - t0 : 0;
        if (n > a.max_group) atomicOr(a.flags, HPS_SEQ_FLAG_LENGTH);
        is_wide = a.history_wide;
        it.token0 = t0;
        it.rows = min(n, a.max_group) * a.ratio;
        it.row0 = tile * (is_wide ? kWideRows : kNarrowRows);
        if (it.row0 >= it.rows) return;
        it.table = a.prefix_table + (size_t)g * a.prefix_width;
        it.first = chunk * a.history_chunk;
        it.end = min(length(a, scalar(a.prefix_lens, g), a.prefix_width, a.max_prefix), it.first + a.history_chunk);
        it.causal_from = kAll;
        it.part = chunk;
    } else {
        uint32_t x = group - a.history_groups;
        is_wide = a.own_mode == kOwnWide;
        solo = a.own_mode == kOwnSolo;
        if (solo) {
            x = x * kWaves + wave;
            if (x >= a.own_items) return;              // no wave of a solo work-group waits for another
        }
        it.head = x % a.kv_heads;
        uint32_t rest = x / a.kv_heads;
        const uint32_t chunk = rest % a.own_chunks;
        rest /= a.own_chunks;
        const uint32_t tile = rest % a.own_tiles, r = rest / a.own_tiles;
        const uint32_t t0 = clamp_to(scalar(a.token_offsets, r), a.n_tokens), t1 = clamp_to(scalar(a.token_offsets, r + 1), a.n_tokens);
        const uint32_t n = t1 > t0 ? t1 - t0 : 0, tile_rows = is_wide ? kWideRows : kNarrowRows;
        if (n > a.max_new) atomicOr(a.flags, HPS_SEQ_FLAG_LENGTH);
        it.token0 = t0;
        it.rows = min(n, a.max_new) * a.ratio;
        it.row0 = tile * tile_rows;
        if (it.row0 >= it.rows) return;
        const uint32_t len = length(a, scalar(a.lens, r), a.table_width, a.max_len);
        it.table = a.block_table + (size_t)r * a.table_width;
        it.first = chunk * a.own_chunk;
        // places by all of the request's new tokens: queries may end inside it
        const int32_t from = (int32_t)len - (scalar(a.token_offsets, r + 1) - (int32_t)t0) + 1, last = from + (int32_t)((min(it.rows, it.row0 + tile_rows) - 1) / a.ratio);        // keys that the tile's last row sees
        it.causal_from = n > 1 ? from : kAll;
        it.end = min((uint32_t)max(last, 0), it.first + a.own_chunk);
        it.part = a.history_chunks + chunk;
        if (a.history_chunks && chunk == 0 && ((int32_t)r < scalar(a.group_offsets, 0) || (int32_t)r >= scalar(a.group_offsets, a.n_groups)))
            for (uint32_t p = 0; p < a.history_chunks; ++p) mark_empty(a, it, p, tile_rows, solo ? lane : threadIdx.x, solo ? 64 : kThreads);
    }
    if (it.first >= it.end && !a.direct) {
        mark_empty(a, it, it.part, is_wide ? kWideRows : kNarrowRows, solo ? lane : threadIdx.x, solo ? 64 : kThreads);
        return;
    }
    if (is_wide) {
        E e(a, it, lds_base, 32 * wave);
        e.wide();
        e.finish(32 * wave);
    } else {
        E e(a, it, lds_base + wave * E::kWaveLds, 0);
        e.narrow(solo ? it.first : it.first + 32 * wave, solo ? 32 : 32 * kWaves);
        if (solo) e.finish(0);
        else e.finish_split(shared);
    }
}

// Joins the parts of a row.  A work-group has kRows rows, kLanes lanes with four values each of every kWays-th part.  First
// every lane computes one part's share of one row (the references and sums of all parts are read side by side), then the
// values are read, several parts under way at a time.  Bound by the round trips where rows are few (64 rows: 4 us), else by
// reading the parts (16,384 rows of 5 parts of 128 values: 10 us, 4.2 TB/s).  Done in the launch in front, by the work-group that ends
// last, it costs more: with the fences that its reading needs 8 candidates behind 500 keys take 24 us instead of 14.
constexpr int kJoin = 256, kMaxParts = 1024;
template <typename T, int kLanes, int kWays> __global__ void __launch_bounds__(kJoin) join_kernel(const Args a, uint32_t parts, uint32_t first_group) {
    constexpr uint32_t kRows = kJoin / (kLanes * kWays), kPerRow = kJoin / kRows;
    extern __shared__ __align__(16) char shared[];
    float *l_share = (float *)shared;                  // [kRows][parts]
    const uint32_t tid = threadIdx.x, r = tid / kPerRow, i = tid % kPerRow, x = i % kLanes, way = i / kLanes;
    const size_t rows = (size_t)a.n_tokens * a.q_heads, row = ((size_t)first_group + blockIdx.x) * kRows + r, near = row < rows ? row : rows - 1;
    const uint32_t t = (uint32_t)(near / a.q_heads), h = (uint32_t)(near - (size_t)t * a.q_heads);
    // only rows of requests have parts of this call; others are not the call's to write
    const bool live = row < rows && (int32_t)t >= scalar(a.token_offsets, 0) && (int32_t)t < scalar(a.token_offsets, a.n_requests);
    float ref = -kInf, sum = 0.f;
    constexpr uint32_t kEach = (kMaxParts + kPerRow - 1) / kPerRow;
    float2 ml[kEach > 4 ? 4 : kEach];
    constexpr uint32_t kHeld = kEach > 4 ? 4 : kEach;  // a lane's parts that it holds; what is beyond is read again
#pragma unroll
    for (uint32_t j = 0; j < kHeld; ++j) {
        const uint32_t p = i + j * kPerRow;
        ml[j] = p < parts ? a.part_ml[p * rows + near] : make_float2(-kInf, 0.f);
    }
#pragma unroll
    for (uint32_t j = 0; j < kHeld; ++j)
        if (ml[j].y != 0.f) ref = fmaxf(ref, ml[j].x);
    for (uint32_t p = i + kHeld * kPerRow; p < parts; p += kPerRow) {
        const float2 y = a.part_ml[p * rows + near];
        if (y.y != 0.f) ref = fmaxf(ref, y.x);
    }
    // over the row's kPerRow lanes, which are a part of a wave or whole waves
    __shared__ float l_wave[2][kJoin / 64];
    constexpr uint32_t kIn = kPerRow < 64 ? kPerRow : 64;
    for (uint32_t d = 1; d < kIn; d <<= 1) ref = fmaxf(ref, __shfl_xor(ref, d));
    if (kPerRow > 64) {
        if ((tid & 63u) == 0) l_wave[0][tid >> 6] = ref;
        __syncthreads();
        for (uint32_t w = 0; w < kPerRow / 64; ++w) ref = fmaxf(ref, l_wave[0][r * (kPerRow / 64) + w]);
    }
    const float at = ref == -kInf ? 0.f : ref;
#pragma unroll
    for (uint32_t j = 0; j < kHeld; ++j) {
        const uint32_t p = i + j * kPerRow;
        if (p >= parts) break;
        const float f = ml[j].y == 0.f ? 0.f : exp2_(ml[j].x - at);
        l_share[r * parts + p] = ml[j].y == 0.f ? -1.f : f;                 // -1: nothing attended, what lies there is no number of this call
        sum += f * ml[j].y;
    }
    for (uint32_t p = i + kHeld * kPerRow; p < parts; p += kPerRow) {
        const float2 y = a.part_ml[p * rows + near];
        const float f = y.y == 0.f ? 0.f : exp2_(y.x - at);
        l_share[r * parts + p] = y.y == 0.f ? -1.f : f;
        sum += f * y.y;
    }
    for (uint32_t d = 1; d < kIn; d <<= 1) sum += __shfl_xor(sum, d);
    if (kPerRow > 64 && (tid & 63u) == 0) l_wave[1][tid >> 6] = sum;
    __syncthreads();
    if (kPerRow > 64) {
        sum = 0.f;
        for (uint32_t w = 0; w < kPerRow / 64; ++w) sum += l_wave[1][r * (kPerRow / 64) + w];
    }
    f32x4 y{};
    if (x * 4 < a.head_dim) {
        const float *from = a.part_o + near * a.head_dim + x * 4;
        const size_t step = rows * a.head_dim;
#pragma unroll 4
        for (uint32_t p = way; p < parts; p += kWays) {
            const f32x4 v = *(const f32x4 *)(from + p * step);
            const float f = l_share[r * parts + p];
            if (f != -1.f) y += f * v;
        }
    }
    if constexpr (kWays > 1) {
        __shared__ f32x4 l_y[kJoin];
        l_y[tid] = y;
        __syncthreads();
        if (way) return;
#pragma unroll
        for (int w = 1; w < kWays; ++w) y += l_y[tid + w * kLanes];
    }
    if (!live) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if (x * 4 < a.head_dim) {
        typedef T t4 __attribute__((ext_vector_type(4)));
        t4 z;
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = (T)(y[j] * inv);
        *(t4 *)(a.out + (int64_t)t * a.out_token + (int64_t)h * a.out_head + x * 8) = z;
    }
    if (a.lse && i == 0) a.lse[row] = sum == 0.f ? -kInf : (ref + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
}

// Where a bound of 0 keeps all histories out of the launch: whether there are any all the same.
__global__ void __launch_bounds__(kThreads) check_kernel(const Args a) {
    const uint32_t g = blockIdx.x * kThreads + threadIdx.x;
    if (g >= a.n_groups) return;
    const uint32_t r0 = clamp_to(a.group_offsets[g], a.n_requests), r1 = clamp_to(a.group_offsets[g + 1], a.n_requests);
    const uint32_t t0 = clamp_to(a.token_offsets[r0], a.n_tokens), t1 = clamp_to(a.token_offsets[r1], a.n_tokens);
    if (t1 <= t0) return;
    if (t1 - t0 > a.max_group) atomicOr(a.flags, HPS_SEQ_FLAG_LENGTH);
    length(a, a.prefix_lens[g], a.prefix_width, a.max_prefix);
}

__global__ void clear_kernel(uint32_t *p) { *p = 0u; }

// ---- host ---------------------------------------------------------------------------------

uint32_t div_up(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

// How many chunks a stretch of `keys` keys is cut into, where one chunk gives `tiles` work-groups: the least of an estimate in
// microseconds.  A step of a wide work-group (64 keys) takes 1.33 us alone on its CU and 1.9 beside another at 128 values
// a head; one of a narrow one (128 keys) 2.2, or what reading takes at 5.4 TB/s for all work-groups together; 4 us go to a
// round's start and end; each part of `rows` rows is written and read at 4 TB/s.  (Measured: 4,096 rows, 8,192 keys, 32 tiles:
// 4 / 8 / 12 / 16 chunks 55 / 39 / 43 / 49 us; 16,384 rows, 32,768 keys, 128 tiles: 2 / 3 / 4 / 5 / 6 chunks 373 / 342 / 311 / 347 / 323;
// 128 rows, 200,003 keys, 8 tiles: 16 / 32 / 64 / 128 chunks 197 / 159 / 168 / 186.)
uint32_t choose_chunks(uint64_t tiles, uint32_t keys, bool wide, uint64_t rows, uint32_t head_dim, uint32_t cus, uint64_t most) {
    const uint32_t step = wide ? kWideKeys : kNarrowKeys * kWaves, limit = div_up(keys, step), slots = cus * (head_dim <= 128 ? 2 : 1);
    const double size = head_dim / 128.0, part = rows * (head_dim * 8.0 + 16.0) / 4e6;
    uint32_t best = 1;
    double least = 0;
    for (uint32_t s = 1; s <= limit && s <= most && s < kMaxParts / 2; ++s) {
        const uint32_t chunk = div_up(limit, s);       // in steps
        if (s > 1 && div_up(limit, chunk) != s) continue;
        const double n = (double)(tiles * s), beside = n < slots ? n : slots, all = n <= slots ? 1.0 : (n / slots + std::ceil(n / slots)) / 2;
        const double one = wide ? (n <= cus ? 1.33 : 1.9) * (0.35 + 0.65 * size) : std::fmax(2.2, beside * 0.0121 * size);
        const double cost = all * (chunk * one + 4.0) + s * part;
        if (s == 1 || cost < least) {
            best = s;
            least = cost;
        }
    }
    return best;
}

}  // namespace

struct hps_seq_attention_session {
    uint64_t magic;
    size_t max_rows, part_rows;
    uint32_t max_head_dim, cus;
    int device;
    float *part_o;
    float2 *part_ml;
    uint32_t *flags;
};

namespace {

template <typename T, int DT, bool kExact> constexpr uint32_t kAttendLds = Engine<T, DT, kExact>::kLds + kWaves * 32 * sizeof(float2);

// Kernels that use more LDS than 64 KiB have to be told so once a device.
template <typename T, int DT> hipError_t allow_lds() {
    static_assert(kAttendLds<T, DT, true> <= 160 * 1024, "LDS of a CU");
    if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&attend_kernel<T, DT, true>), hipFuncAttributeMaxDynamicSharedMemorySize, kAttendLds<T, DT, true>)) return e;
    return hipFuncSetAttribute(reinterpret_cast<const void *>(&attend_kernel<T, DT, false>), hipFuncAttributeMaxDynamicSharedMemorySize, kAttendLds<T, DT, false>);
}
template <typename T> hipError_t allow_lds() {
    if (hipError_t e = allow_lds<T, 3>()) return e;
    if (hipError_t e = allow_lds<T, 4>()) return e;
    return allow_lds<T, 8>();
}

template <typename T, int DT, bool kExact> hipError_t launch_attend(Args &a, uint32_t groups, hipStream_t st) {
    return seq_launches(groups, [&](uint32_t first, uint32_t n) {
        a.first_group = first;
        hipLaunchKernelGGL((attend_kernel<T, DT, kExact>), dim3(n), dim3(kThreads), (kAttendLds<T, DT, kExact>), st, a);
    });
}

template <typename T, int DT> hipError_t launch(Args &a, uint32_t groups, uint32_t parts, hipStream_t st) {
    if (hipError_t e = a.head_dim == 32 * DT ? launch_attend<T, DT, true>(a, groups, st) : launch_attend<T, DT, false>(a, groups, st)) return e;
    if (a.direct) return hipSuccess;
    constexpr int kLanes = DT == 1 ? 8 : DT == 2 ? 16 : DT <= 4 ? 32 : 64;
    const size_t rows = (size_t)a.n_tokens * a.q_heads;
    auto join = [&](auto ways) {
        constexpr int kWays = decltype(ways)::value, kRows = kJoin / (kLanes * kWays);
        return seq_launches(div_up(rows, kRows), [&](uint32_t first, uint32_t n) {
            hipLaunchKernelGGL((join_kernel<T, kLanes, kWays>), dim3(n), dim3(kJoin), kRows * parts * sizeof(float), st, a, parts, first);
        });
    };
    // Few rows: all lanes of a work-group to one, which read its parts side by side (a row each / several rows each, us of a whole
    // call, 16 heads of 128: 1 token behind 1,000 keys 13.0 / 13.8, 4 behind 32,768 21.6 / 36.6, 64 37.0 / 45.1, 256 behind 1,000 25.1 / 22.3).
    // Many parts too: a launch has 64 KiB of LDS unasked, and several rows of heads up to 32 would want more beyond 512.
    return rows * kLanes <= 65536 || kJoin / kLanes * parts * sizeof(float) > 65536 - 512 ? join(std::integral_constant<int, kJoin / kLanes>()) : join(std::integral_constant<int, 1>());
}

template <typename T> hipError_t launch(Args &a, uint32_t groups, uint32_t parts, hipStream_t st) {
    if (a.head_dim <= 32) return launch<T, 1>(a, groups, parts, st);
    if (a.head_dim <= 64) return launch<T, 2>(a, groups, parts, st);
    if (a.head_dim <= 96) return launch<T, 3>(a, groups, parts, st);
    if (a.head_dim <= 128) return launch<T, 4>(a, groups, parts, st);
    return launch<T, 8>(a, groups, parts, st);
}

bool multiple16(int64_t stride) { return (stride * 2 & 15) == 0; }
bool heads16(const hps_seq_heads_t &h) { return h.data && seq_aligned(h.data, 16) && multiple16(h.token_stride) && multiple16(h.head_stride); }

}  // namespace

extern "C" {

hps_status_t hps_seq_attention_create(size_t max_rows, uint32_t max_head_dim, hps_seq_attention_t **out) {
    SEQ_REQUIRE(out, "out must not be NULL");
    *out = nullptr;
    SEQ_REQUIRE(max_rows > 0 && max_rows < (1ull << 31), "max_rows must be in 1 .. 2^31 - 1");
    SEQ_REQUIRE(max_head_dim > 0 && max_head_dim <= 256, "max_head_dim must be in 1 .. 256");
    hps_seq_attention_session *s = new (std::nothrow) hps_seq_attention_session();
    if (!s) return hps_seq_fail(HPS_ERR_OOM, "host allocation failed");
    s->max_rows = max_rows;
    s->part_rows = 3 * max_rows + 65536;
    s->max_head_dim = (max_head_dim + 7) / 8 * 8;
    int cus = 0;
    hipError_t e = hipGetDevice(&s->device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, s->device);
    s->cus = cus > 0 ? (uint32_t)cus : 256u;
    if (e == hipSuccess) e = allow_lds<_Float16>();
    if (e == hipSuccess) e = allow_lds<__bf16>();
    // one piece: values (a multiple of 32 bytes a row), references and sums, the flag word
    const size_t o_bytes = s->part_rows * s->max_head_dim * sizeof(float), ml_bytes = s->part_rows * sizeof(float2);
    char *piece = nullptr;
    if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void **>(&piece), o_bytes + ml_bytes + 256);
    if (e == hipSuccess) {
        s->part_o = reinterpret_cast<float *>(piece);
        s->part_ml = reinterpret_cast<float2 *>(piece + o_bytes);
        s->flags = reinterpret_cast<uint32_t *>(piece + o_bytes + ml_bytes);
        hipLaunchKernelGGL(clear_kernel, dim3(1), dim3(1), 0, 0, s->flags);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipStreamSynchronize(0);
    if (e != hipSuccess) {
        (void)hipFree(piece);
        delete s;
        (void)hipGetLastError();
        return hps_seq_fail(e == hipErrorOutOfMemory ? HPS_ERR_OOM : HPS_ERR_DEVICE, "hps_seq_attention_create: ", hipGetErrorString(e));
    }
    s->magic = kMagic;
    *out = s;
    return HPS_OK;
}

hps_status_t hps_seq_attention_destroy(hps_seq_attention_t *s) {
    if (!s) return HPS_OK;
    SEQ_REQUIRE(s->magic == kMagic, "not a live attention session");
    int prev = -1;
    SEQ_TRY(hipGetDevice(&prev));
    SEQ_TRY(hipSetDevice(s->device));
    hipError_t e = hipDeviceSynchronize();
    (void)hipFree(s->part_o);
    s->magic = 0;
    delete s;
    (void)hipSetDevice(prev);
    if (e != hipSuccess) return hps_seq_fail(HPS_ERR_DEVICE, "hipDeviceSynchronize: ", hipGetErrorString(e));
    return HPS_OK;
}

hps_status_t hps_seq_attention_flags(hps_seq_attention_t *s, uint32_t *flags, int clear) {
    SEQ_REQUIRE(s && s->magic == kMagic, "not a live attention session");
    SEQ_REQUIRE(flags, "flags must not be NULL");
    SEQ_TRY(hipMemcpy(flags, s->flags, sizeof(uint32_t), hipMemcpyDeviceToHost));
    const uint32_t zero = 0u;
    if (clear) SEQ_TRY(hipMemcpy(s->flags, &zero, sizeof(uint32_t), hipMemcpyHostToDevice));
    return HPS_OK;
}

hps_status_t hps_seq_attention(hps_seq_attention_t *s, const hps_seq_attention_args_t *args, void *stream) {
    SEQ_REQUIRE(s && s->magic == kMagic, "not a live attention session");
    SEQ_REQUIRE(args, "args must not be NULL");
    const hps_seq_attention_args_t &r = *args;
    int device = -1;
    SEQ_TRY(hipGetDevice(&device));
    SEQ_REQUIRE(device == s->device, "the session is of another device than the current one");
    SEQ_REQUIRE(r.dtype == HPS_SEQ_F16 || r.dtype == HPS_SEQ_BF16, "dtype must be HPS_SEQ_F16 or HPS_SEQ_BF16");
    SEQ_REQUIRE(r.head_dim > 0 && r.head_dim % 8 == 0 && r.head_dim <= 256, "head_dim must be a multiple of 8 in 8 .. 256");
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
    if (r.n_tokens == 0 || r.n_requests == 0) return HPS_OK;
    SEQ_REQUIRE(heads16(r.q) && heads16(r.out), "q and out must be device pointers, 16-byte aligned, their strides multiples of 16 bytes");
    SEQ_REQUIRE(seq_words(r.token_offsets) && seq_words(r.lens), "token_offsets and lens must be 4-byte aligned device pointers");
    SEQ_REQUIRE(r.table_width == 0 || seq_words(r.block_table), "block_table must be a 4-byte aligned device pointer");
    SEQ_REQUIRE(r.pages.n_blocks == 0 || (r.pages.k && r.pages.v && seq_aligned(r.pages.k, 16) && seq_aligned(r.pages.v, 16)), "the pages must be device pointers, 16-byte aligned");
    SEQ_REQUIRE(multiple16(r.pages.block_stride) && multiple16(r.pages.token_stride) && multiple16(r.pages.head_stride), "the pages' strides must be multiples of 16 bytes");
    SEQ_REQUIRE(r.pages.token_stride >= 0 && r.pages.token_stride < (1 << 25), "the pages' token_stride must be in 0 .. 2^25 - 1");
    SEQ_REQUIRE(r.pages.block_stride >= 0 && r.pages.block_stride < (1ll << 31), "the pages' block_stride must be in 0 .. 2^31 - 1");
    SEQ_REQUIRE(r.n_groups == 0 || (seq_words(r.prefix_lens) && seq_words(r.group_offsets) && (r.prefix_width == 0 || seq_words(r.prefix_table))),
                "prefix_table, prefix_lens and group_offsets must be 4-byte aligned device pointers");
    SEQ_REQUIRE(r.lse == nullptr || seq_aligned(r.lse, 4), "lse must be 4-byte aligned");

    Args a{};
    a.q = static_cast<const char *>(r.q.data);
    a.k = static_cast<const char *>(r.pages.k);
    a.v = static_cast<const char *>(r.pages.v);
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
    a.page_block = (uint32_t)(r.pages.block_stride * 2);
    a.page_token = (uint32_t)(r.pages.token_stride * 2);
    a.page_head = r.pages.head_stride * 2;
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

    const uint64_t rows = (uint64_t)r.n_tokens * r.q_heads, part_limit = s->part_rows / rows;
    // own tokens: one part at least, so that every row has one
    const uint64_t own_rows = (uint64_t)a.max_new * a.ratio;
    uint32_t own_keys = r.max_len ? r.max_len : 1;
    const uint64_t requests_heads = (uint64_t)r.n_requests * r.kv_heads;
    if (own_rows > kNarrowRows) {
        a.own_mode = kOwnWide;
        a.own_tiles = div_up(own_rows, kWideRows);
        a.own_chunks = choose_chunks(requests_heads * a.own_tiles, own_keys, true, rows, r.head_dim, s->cus, part_limit / 2);
        a.own_chunk = div_up(div_up(own_keys, a.own_chunks), kWideKeys) * kWideKeys;
    } else {
        // A wave to a request where there are more requests than work-groups at a time, up to 512 keys (a wave / a work-group each, us, 4
        // key heads of 128: 64 requests of 64 / 256 / 512 keys 14.6, 21.9, 32.4 / 13.9, 14.9, 19.9; 512 of 64 / 256 / 512 / 1,024 keys 26.2, 38.0,
        // 63.2, 134.1 / 43.6, 50.6, 69.6, 129.2).
        a.own_mode = requests_heads > 2 * s->cus && own_keys <= 512 ? kOwnSolo : kOwnSplit;
        a.own_tiles = 1;
        const uint32_t step = a.own_mode == kOwnSolo ? kNarrowKeys : kNarrowKeys * kWaves;
        a.own_chunks = a.own_mode == kOwnSolo ? 1 : choose_chunks(requests_heads, own_keys, false, rows, r.head_dim, s->cus, part_limit / 2);
        a.own_chunk = div_up(div_up(own_keys, a.own_chunks), step) * step;
    }
    if (a.own_tiles == 0) a.own_tiles = 1;
    const uint64_t own_items = requests_heads * a.own_tiles * a.own_chunks, own_groups = a.own_mode == kOwnSolo ? (own_items + kWaves - 1) / kWaves : own_items;
    uint64_t history_groups = 0;
    if (r.n_groups && r.max_prefix && a.max_group) {
        const uint64_t group_rows = (uint64_t)a.max_group * a.ratio;
        // Up to 32 rows the waves share the keys; up to 64 too, in two work-groups, where reading a long history is what counts (waves share
        // keys / rows, us: 64 rows behind 4,096 keys 16.1 / 15.4, behind 65,536 36.9 / 41.1; 96 rows 53.1 / 37.7).
        a.history_wide = group_rows > (r.max_prefix >= 16384 ? 2 : 1) * kNarrowRows;
        a.history_tiles = div_up(group_rows, a.history_wide ? kWideRows : kNarrowRows);
        const uint32_t step = a.history_wide ? kWideKeys : kNarrowKeys * kWaves;
        a.history_chunks = choose_chunks((uint64_t)a.history_tiles * r.n_groups * r.kv_heads, r.max_prefix, a.history_wide, rows, r.head_dim, s->cus, part_limit - a.own_chunks);
        a.history_chunk = div_up(div_up(r.max_prefix, a.history_chunks), step) * step;
        const uint64_t combos = (uint64_t)r.n_groups * r.kv_heads * a.history_chunks;
        SEQ_REQUIRE(combos < (1u << 30), "too many groups, heads and chunks for one launch");
        a.history_combos = (uint32_t)combos;
        history_groups = (combos >= 8 ? (combos + 7) / 8 * 8 : combos) * a.history_tiles;
    }
    SEQ_REQUIRE(history_groups + own_groups < (1ull << 31) && own_items < (1ull << 31), "too many requests, heads and chunks for one launch");
    a.history_groups = (uint32_t)history_groups;
    a.own_items = (uint32_t)own_items;
    const uint32_t parts = a.history_chunks + a.own_chunks;
    a.direct = parts == 1;
    const uint32_t groups = (uint32_t)(history_groups + own_groups);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (r.n_groups && !history_groups) {
        hipLaunchKernelGGL(check_kernel, dim3(div_up(r.n_groups, kThreads)), dim3(kThreads), 0, st, a);
        SEQ_TRY(hipGetLastError());
    }
    SEQ_TRY(r.dtype == HPS_SEQ_F16 ? launch<_Float16>(a, groups, parts, st) : launch<__bf16>(a, groups, parts, st));
    return HPS_OK;
}

}  // extern "C"
