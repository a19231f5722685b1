// Pages of sequence models: block tables and slots from lengths, rotary positions, keys and values written to their
// pages (hps_seq.h), for gfx950.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "hps_seq_common.h"

namespace {

thread_local char g_err[256];

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// ---- extend and release -------------------------------------------------------------------
//
// Everything follows from two exclusive sums over the requests: of their new tokens, and of their new blocks.  A
// work-group takes a chunk of requests, four to a thread, adds up what all requests in front of it have (nobody waits for
// anybody: the lengths are few and in the caches, and reading them again costs less than a second launch or a chain of
// work-groups), scans its own into LDS, and writes its share of the chunk's tokens and blocks, each found by a binary
// search in LDS; some of its waves see to the blocks while the others see to the tokens.  Bound by the chain of round trips
// (arguments, lengths, table or free list): 64 requests of a token each 5.8 us, 8,192 requests with a million tokens 12 us (9 MB,
// which a copy moves in 2).  What reading the lengths again costs grows with the square of the requests: 65,536 of a token each 22 us,
// 262,144 62, a million 323.
constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;                // of a work-group (256 threads: the same times)
constexpr uint32_t kPer = 4, kChunk = kPer * kThreads; // requests of a thread, of a work-group
constexpr uint32_t kMaxSum = 0x7FFFFFFFu;

__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
template <int kCtrl, int kRows = 0xf> __device__ __forceinline__ uint32_t moved(uint32_t x) {     // 0 where nothing comes from
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, kRows, 0xf, false);
}
// Inclusive sums over 16 lanes, over a wave; saturating sums are associative, so they scan like any other.
__device__ __forceinline__ uint32_t scan16(uint32_t x) {
    x = add_sat(x, moved<0x111>(x));                   // one lane on, two, four, eight
    x = add_sat(x, moved<0x112>(x));
    x = add_sat(x, moved<0x114>(x));
    return add_sat(x, moved<0x118>(x));
}
__device__ __forceinline__ uint32_t scan64(uint32_t x) {
    x = scan16(x);
    x = add_sat(x, moved<0x142, 0xa>(x));              // the last lane of 16 to the next 16, of 32 to the next 32
    return add_sat(x, moved<0x143, 0xc>(x));
}
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

// One request: its kept tokens, and what it adds.
struct Request {
    uint32_t past, fresh, fit, kept, blocks;
    __device__ __forceinline__ Request(int32_t p, int32_t n, uint32_t cap, uint32_t sh) {
        const uint32_t round = (1u << sh) - 1u;
        past = min((uint32_t)max(p, 0), cap);
        fresh = (uint32_t)max(n, 0);
        fit = min(fresh, cap - past);
        kept = (past + round) >> sh;
        blocks = ((past + fit + round) >> sh) - kept;
    }
};

// The last i in lo .. hi - 1 with first[i] <= x, where first[lo] <= x < first[hi].
__device__ __forceinline__ uint32_t find(const uint32_t *first, uint32_t lo, uint32_t hi, uint32_t x) {
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// The same for a whole wave's x and n <= 4096 of them, in two looks.
__device__ __forceinline__ uint32_t find_together(const uint32_t *first, uint32_t n, uint32_t x) {
    const uint32_t lane = threadIdx.x & 63u, step = (n + 63) / 64;
    const uint32_t lo = ((uint32_t)__popcll(__ballot(lane * step < n && first[lane * step] <= x)) - 1u) * step, i = lo + lane;
    return lo + (uint32_t)__popcll(__ballot(lane < step && i < n && first[i] <= x)) - 1u;
}

struct ExtendArgs {
    hps_seq_extend_args_t a;
    uint32_t sh, cap;                                  // log2 of the block size; tokens that a table holds
};

// The place in the free list of the call's k-th new block; null where the list has none.
__device__ __forceinline__ const int32_t *new_block(const ExtendArgs &e, uint32_t n_free, uint32_t k) {
    return k < n_free ? e.a.free_blocks + (n_free - 1u - k) : nullptr;
}

__global__ void __launch_bounds__(kThreads) extend_kernel(const ExtendArgs e) {
    constexpr uint32_t kBlockWaves = kWaves / 4;       // waves that see to the blocks
    __shared__ uint32_t l_tok[kChunk + 1], l_blk[kChunk + 1], l_past[kChunk];
    __shared__ uint32_t l_wave[4][16];                 // tokens and blocks of the chunk's waves; of what is in front of the chunk
    __shared__ unsigned long long l_over;
    const hps_seq_extend_args_t &a = e.a;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, r0 = blockIdx.y * kChunk, mine = min(kChunk, a.n_requests - r0);
    const bool last_chunk = blockIdx.y == gridDim.y - 1;
    const int32_t free_now = *a.n_free;
    if (tid == 0) l_over = 0;

    uint32_t tok[kPer], blk[kPer], end[kPer], tokens = 0, blocks = 0, over = 0;
    int32_t p[kPer], n[kPer];
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) {
        const bool there = tid * kPer + i < mine;
        p[i] = there ? a.past_lens[r0 + tid * kPer + i] : 0;
        n[i] = there ? a.new_lens[r0 + tid * kPer + i] : 0;
    }
    uint32_t front_tokens = 0, front_blocks = 0;
    for (uint32_t r = tid; r < r0; r += kThreads) {
        const Request q(a.past_lens[r], a.new_lens[r], e.cap, e.sh);
        front_tokens = add_sat(front_tokens, q.fresh);
        front_blocks = add_sat(front_blocks, q.blocks);
        over = add_sat(over, q.fresh - q.fit);
    }
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) {
        const Request q(p[i], n[i], e.cap, e.sh);
        tok[i] = tokens;
        blk[i] = blocks;
        end[i] = q.past + q.fit;
        tokens = add_sat(tokens, q.fresh);
        blocks = add_sat(blocks, q.blocks);
        over = add_sat(over, q.fresh - q.fit);
        if (tid * kPer + i < mine) l_past[tid * kPer + i] = q.past;
    }
    const uint32_t inc_tokens = scan64(tokens), inc_blocks = scan64(blocks);
    if (lane == 63) {
        l_wave[0][wave] = inc_tokens;
        l_wave[1][wave] = inc_blocks;
    }
    if (r0) {                                          // uniform
        front_tokens = scan64(front_tokens);
        front_blocks = scan64(front_blocks);
        if (lane == 63) {
            l_wave[2][wave] = front_tokens;
            l_wave[3][wave] = front_blocks;
        }
    }
    __syncthreads();
    if (over) atomicAdd(&l_over, (unsigned long long)over);                 // seldom: a table too short
    uint32_t sums[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[i] = scan16(lane < kWaves && (i < 2 || r0) ? l_wave[i][lane] : 0);
    const uint32_t base_tokens = lane_of(sums[2], kWaves - 1), base_blocks = lane_of(sums[3], kWaves - 1);
    const uint32_t all_tokens = add_sat(base_tokens, lane_of(sums[0], kWaves - 1)), all_blocks = add_sat(base_blocks, lane_of(sums[1], kWaves - 1));
    uint32_t at_tokens = base_tokens, at_blocks = base_blocks;
    const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)wave);
    if (w) {
        at_tokens = add_sat(at_tokens, lane_of(sums[0], (int)w - 1));
        at_blocks = add_sat(at_blocks, lane_of(sums[1], (int)w - 1));
    }
    at_tokens = add_sat(at_tokens, moved<0x138>(inc_tokens));               // the lane below's
    at_blocks = add_sat(at_blocks, moved<0x138>(inc_blocks));
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) {
        const uint32_t j = tid * kPer + i;
        if (j < mine) {
            l_tok[j] = add_sat(at_tokens, tok[i]);
            l_blk[j] = add_sat(at_blocks, blk[i]);
            if (blockIdx.x == 0) {
                a.token_offsets[r0 + j] = (int32_t)min(add_sat(at_tokens, tok[i]), kMaxSum);
                a.total_lens[r0 + j] = (int32_t)end[i];
            }
        }
    }
    if (tid == 0) {
        l_tok[mine] = all_tokens;
        l_blk[mine] = all_blocks;
    }
    const uint32_t n_free = (uint32_t)min(max(free_now, 0), (int32_t)a.n_blocks);
    __syncthreads();
    if (tid == 0 && last_chunk && blockIdx.x == 0) {
        const uint32_t taken = min(all_blocks, n_free);
        a.token_offsets[a.n_requests] = (int32_t)min(all_tokens, kMaxSum);
        a.info[0] = (int32_t)(n_free - taken);
        a.info[1] = (int32_t)min(all_tokens, kMaxSum);
        a.info[2] = (int32_t)min(all_blocks - taken, kMaxSum);
        a.info[3] = (int32_t)min(l_over, (unsigned long long)kMaxSum);
    }

    const uint32_t round = (1u << e.sh) - 1u;
    if (wave >= kWaves - kBlockWaves) {
        constexpr uint32_t kFill = 64 * kBlockWaves;
        for (uint64_t k = l_blk[0] + (uint64_t)(blockIdx.x * kFill + tid - (kThreads - kFill)); k < l_blk[mine]; k += gridDim.x * kFill) {
            const uint32_t i = find(l_blk, 0, mine, (uint32_t)k), kept = (l_past[i] + round) >> e.sh;
            const int32_t *from = new_block(e, n_free, (uint32_t)k);
            const int32_t id = from ? *from : -1;
            a.block_table[(size_t)(r0 + i) * a.table_width + kept + ((uint32_t)k - l_blk[i])] = (uint32_t)id < a.n_blocks ? id : -1;
        }
        return;
    }
    // Tokens in fours, 16 bytes a store; the first and the last four of a chunk may belong to its neighbours in part.  A wave's
    // 256 tokens are of a few requests, which it finds together.
    constexpr uint32_t kFill = 64 * (kWaves - kBlockWaves);
    const uint32_t t_begin = min(l_tok[0], a.max_tokens), t_end = min(l_tok[mine], a.max_tokens), t_all = last_chunk ? a.max_tokens : t_end;
    const bool wide = (((uintptr_t)a.slots | (uintptr_t)a.positions) & 15u) == 0;
    for (uint64_t g0 = (t_begin >> 2) + (uint64_t)(blockIdx.x * kFill + 64 * w); g0 * 4 < t_all; g0 += gridDim.x * kFill) {        // uniform in a wave
        const uint32_t g = (uint32_t)g0 + lane, t0 = max((uint32_t)g0 * 4, t_begin), t1 = min((uint32_t)g0 * 4 + 256, t_end);       // max_tokens < 2^31
        uint32_t lo = 0, hi = 0;
        if (t0 < t1) {
            lo = find_together(l_tok, mine, t0);
            hi = find_together(l_tok, mine, t1 - 1) + 1;
        }
        uint32_t own[4];
        int32_t start[4], id[4];
        uint32_t i = lo, next = 0;
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) {             // all loads first
            const uint32_t t = g * 4 + c;
            own[c] = 0xFFFFFFFFu;
            start[c] = 0;
            id[c] = -1;
            if (t < t_begin || t >= t_end) continue;
            if (t >= next) {
                i = find(l_tok, i, hi, t);
                next = l_tok[i + 1];
            }
            const uint32_t past = l_past[i], kept = (past + round) >> e.sh, j = (past + (t - l_tok[i])) >> e.sh;
            own[c] = past + (t - l_tok[i]);
            if (a.start) start[c] = a.start[r0 + i];
            const int32_t *from = own[c] >= e.cap ? nullptr : j < kept ? a.block_table + (size_t)(r0 + i) * a.table_width + j : new_block(e, n_free, l_blk[i] + (j - kept));
            if (from) id[c] = *from;
        }
        i32x4 slot, pos;
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) {
            const uint32_t t = g * 4 + c;
            const bool inside = t >= t_begin && t < t_end;
            pos[c] = inside ? (int32_t)min((int64_t)start[c] + own[c], (int64_t)kMaxSum) : -1;
            slot[c] = inside && (uint32_t)id[c] < a.n_blocks ? (int32_t)(((uint32_t)id[c] << e.sh) | (own[c] & round)) : -1;
        }
        if (wide && g * 4 >= t_begin && g * 4 + 4 <= t_all) {
            *(i32x4 *)(a.slots + g * 4) = slot;
            *(i32x4 *)(a.positions + g * 4) = pos;
        } else {
            for (uint32_t c = 0; c < 4; ++c) {
                const uint32_t t = g * 4 + c;
                if (t < t_begin || t >= t_all) continue;
                a.slots[t] = slot[c];
                a.positions[t] = pos[c];
            }
        }
    }
}

struct ReleaseArgs {
    int32_t *lens;
    const int32_t *finished;
    int32_t *table, *free_blocks;
    const int32_t *n_free;
    int32_t *info;
    uint32_t n_requests, sh, cap, width, n_blocks;
};

// One work-group: the free list is one stack whose order the call fixes.  Bound by the round trips of a thousand blocks at a time, some
// 1.4 us: 64 requests of which 8 end with 63 blocks each 5.3 us, 1,040 that all end with a block each (candidates that were scored) 6, 8,192
// with a block each 14, with ten each 115.
__global__ void __launch_bounds__(kThreads) release_kernel(const ReleaseArgs a) {
    __shared__ uint32_t l_blk[kChunk + 1], l_wave[kWaves];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
    const uint32_t had = (uint32_t)min(max(*a.n_free, 0), (int32_t)a.n_blocks);
    uint32_t base = had, lost = 0;                     // the same in all threads
    // sum over the waves in front of this one, and over all, of what the waves' last lanes have
    auto over_waves = [&](uint32_t mine, uint32_t &all) {
        if (lane == 63) l_wave[wave] = mine;
        __syncthreads();
        const uint32_t sums = scan16(lane < kWaves ? l_wave[lane] : 0);
        __syncthreads();
        all = lane_of(sums, kWaves - 1);
        return wave ? lane_of(sums, (int)wave - 1) : 0u;
    };
    for (uint32_t r0 = 0; r0 < a.n_requests; r0 += kChunk) {
        const uint32_t mine = min(kChunk, a.n_requests - r0);
        uint32_t n[kPer], sum = 0, total;
        for (uint32_t i = 0; i < kPer; ++i) {
            const uint32_t j = tid * kPer + i, r = r0 + j;
            n[i] = 0;
            if (j < mine && a.finished[r]) {
                n[i] = (min((uint32_t)max(a.lens[r], 0), a.cap) + (1u << a.sh) - 1u) >> a.sh;
                a.lens[r] = 0;
            }
            sum = add_sat(sum, n[i]);
        }
        const uint32_t inc = scan64(sum);
        uint32_t at = add_sat(over_waves(inc, total), moved<0x138>(inc));
        for (uint32_t i = 0; i < kPer; ++i) {
            if (tid * kPer + i < mine) l_blk[tid * kPer + i] = at;
            at = add_sat(at, n[i]);
        }
        if (tid == 0) l_blk[mine] = total;
        __syncthreads();
        for (uint64_t k0 = 0; k0 < total; k0 += kThreads) {
            const uint32_t k = (uint32_t)k0 + tid;
            int32_t id = -1;
            if (k0 + tid < total) {
                const uint32_t i = find(l_blk, 0, mine, k);
                int32_t *entry = a.table + (size_t)(r0 + i) * a.width + (k - l_blk[i]);
                id = *entry;
                *entry = -1;
            }
            const bool valid = (uint32_t)id < a.n_blocks;
            const uint64_t m = __ballot(valid);
            uint32_t all;
            const uint32_t to = base + over_waves((uint32_t)__popcll(m), all) + (uint32_t)__popcll(m & ((1ull << lane) - 1ull));
            if (valid && to < a.n_blocks) a.free_blocks[to] = id;
            const uint32_t room = a.n_blocks - base;
            lost = add_sat(lost, all - min(all, room));
            base += min(all, room);
        }
        __syncthreads();
    }
    if (tid == 0) {
        a.info[0] = (int32_t)base;
        a.info[1] = (int32_t)(base - had);
        a.info[2] = (int32_t)min(lost, kMaxSum);
    }
}

// ---- rotary positions ---------------------------------------------------------------------

// Angles in 64 bits: in 32 bits one at position 131,071 would be off by up to 2^-8.  Bound by that arithmetic, once a model: 131,072 positions
// of 128 values 100 us, 4,096 positions 5 us.
__global__ void rope_table_kernel(float *table, uint32_t max_pos, uint32_t half, double base, int scale, double factor, double original,
                                  double low, double high, double magnitude) {
    const uint64_t n = (uint64_t)max_pos * half;
    for (uint64_t x = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x; x < n; x += (uint64_t)gridDim.x * blockDim.x) {
        const uint32_t pos = (uint32_t)(x / half), i = (uint32_t)(x % half);
        double w = pow(base, -(double)i / (double)half);
        if (scale == HPS_SEQ_SCALE_LINEAR) w /= factor;
        if (scale == HPS_SEQ_SCALE_PARTS) {
            const double turns = original * w / (2.0 * M_PI), g = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
            w *= g + (1.0 - g) / factor;
        }
        double s, c;
        sincos((double)pos * w, &s, &c);
        *(float2 *)(table + x * 2) = make_float2((float)(c * magnitude), (float)(s * magnitude));
    }
}

// The heads of a token, in the order queries, keys, values.  `out` of keys and values is an array like the input, or
// the pages.
struct RopeArgs {
    const char *in[3];
    char *out[3];
    int64_t in_token[3], in_head[3], out_token[3], out_head[3];         // strides in bytes
    int64_t page_block;                                                 // of the pages: block stride; out_token is the place's
    const int32_t *positions, *slots;
    const float *table;
    uint32_t heads[3], n_heads;                                         // of each, of all
    uint32_t head_dim, half, max_pos;                                   // half = rot_dim / 2
    uint32_t spans, per_pass, n_slots, sh;                              // spans: pairs of vectors of a head; per_pass: heads side by side
    uint32_t first_token;                                               // of this launch
    int32_t interleaved;
    float sign;
};

template <typename T, int E> struct alignas(E * sizeof(T) > 16 ? 16 : E * sizeof(T)) Vec { T v[E]; };

// One pair, in 32 bits, rounded once; the products are written out, so that every shape of the kernel gives the same bits.
template <typename T> __device__ __forceinline__ void turn(T &a, T &b, float c, float s) {
    const float p = (float)a, q = (float)b, qs = q * s, qc = q * c;
    a = (T)__builtin_fmaf(p, c, -qs);
    b = (T)__builtin_fmaf(p, s, qc);
}

// One work-group per token.  A lane has two vectors of 16 bytes of a head (for halves: the two that hold E pairs), which
// stay the same from head to head, so cosines and sines are read once for all of them.  Bound by HBM where tokens have many
// heads (8,192 tokens of 48 heads of 128: 37.5 us, 5.4 TB/s while the pages are in the Infinity Cache, 50 us, 4.0 TB/s, otherwise),
// else by the chain position, cosines, rows, store.  Two heads under way instead of one: 38.6 us, four 41.7; rows requested in front of
// the position 41.1.  E = 1 is for rows that are not in whole 16-byte vectors (67.9 us).
template <typename T, int E, bool kPages>
__global__ void __launch_bounds__(256) rope_kernel(const RopeArgs a) {
    typedef Vec<T, E> V;
    const uint32_t t = a.first_token + blockIdx.x, tid = threadIdx.x;
    const uint32_t lane_head = tid / a.spans, s = tid - lane_head * a.spans;
    if (lane_head >= a.per_pass) return;
    const bool turns = a.table != nullptr;

    // the two vectors (o0, o1, in values), and the pairs in them
    const bool within = a.interleaved && E > 1;        // pairs lie within a vector
    uint32_t o0, o1;
    if (a.interleaved) {
        o0 = 2 * s * E;
        o1 = o0 + E;
    } else {
        const uint32_t split = a.half / E;             // behind the pairs, two neighbours to a span
        o0 = s < split ? s * E : 2 * a.half + 2 * (s - split) * E;
        o1 = s < split ? a.half + s * E : o0 + E;
    }
    const bool has0 = o0 < a.head_dim, has1 = o1 < a.head_dim;
    const int32_t pos = turns ? a.positions[t] : 0;
    uint32_t slot = 0;
    if (kPages) slot = (uint32_t)a.slots[t];
    if (pos < 0) return;
    const bool stored = !kPages || slot < a.n_slots;
    const bool turn0 = turns && o0 < 2 * a.half, turn1 = turns && o1 < 2 * a.half;
    float cs[E], sn[E];                                // of the pairs: across the two vectors E, within them E / 2 each
#pragma unroll
    for (int j = 0; j < E; ++j) cs[j] = sn[j] = 0.f;
    if (turn0) {
        if ((uint32_t)pos < a.max_pos) {
            const float2 *row = (const float2 *)a.table + (size_t)pos * a.half;
            const uint32_t pair = within ? s * E : a.interleaved ? s : o0;
            const uint32_t n = within ? (turn1 ? E : E / 2) : E;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if ((uint32_t)j < n) {
                    const float2 f = row[pair + j];
                    cs[j] = f.x;
                    sn[j] = f.y * a.sign;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) cs[j] = sn[j] = __builtin_nanf("");
        }
    }

    for (uint32_t hh = lane_head; hh < a.n_heads; hh += a.per_pass) {
        const int seg = hh < a.heads[0] ? 0 : hh < a.heads[0] + a.heads[1] ? 1 : 2;
        if (seg > 0 && !stored) break;                 // keys and values come last
        const uint32_t h = hh - (seg > 0 ? a.heads[0] : 0) - (seg > 1 ? a.heads[1] : 0);
        const char *from = seg == 0 ? a.in[0] : seg == 1 ? a.in[1] : a.in[2];
        const int64_t it = seg == 0 ? a.in_token[0] : seg == 1 ? a.in_token[1] : a.in_token[2];
        const int64_t ih = seg == 0 ? a.in_head[0] : seg == 1 ? a.in_head[1] : a.in_head[2];
        from += (int64_t)t * it + (int64_t)h * ih;
        V x, y;
        if (has0) x = *(const V *)(from + o0 * sizeof(T));
        if (has1) y = *(const V *)(from + o1 * sizeof(T));
        char *to = seg == 0 ? a.out[0] : seg == 1 ? a.out[1] : a.out[2];
        const int64_t ot = seg == 0 ? a.out_token[0] : seg == 1 ? a.out_token[1] : a.out_token[2];
        const int64_t oh = seg == 0 ? a.out_head[0] : seg == 1 ? a.out_head[1] : a.out_head[2];
        if (kPages && seg > 0) to += (int64_t)(slot >> a.sh) * a.page_block + (int64_t)(slot & ((1u << a.sh) - 1u)) * ot;
        else to += (int64_t)t * ot;
        to += (int64_t)h * oh;
        if (seg < 2 && turn0) {
            if (within) {
                if constexpr (E > 1) {
#pragma unroll
                    for (int j = 0; j < E / 2; ++j) {
                        turn(x.v[2 * j], x.v[2 * j + 1], cs[j], sn[j]);
                        if (turn1) turn(y.v[2 * j], y.v[2 * j + 1], cs[E / 2 + j], sn[E / 2 + j]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) turn(x.v[j], y.v[j], cs[j], sn[j]);
            }
        }
        if (has0) *(V *)(to + o0 * sizeof(T)) = x;
        if (has1) *(V *)(to + o1 * sizeof(T)) = y;
    }
}

template <typename T, bool kPages>
hipError_t launch_rope(RopeArgs &a, uint32_t n_tokens, uint32_t rot_dim, hipStream_t st) {
    constexpr int E = 16 / sizeof(T);
    a.n_heads = a.heads[0] + a.heads[1] + a.heads[2];
    // whole vectors: every row starts on 16 bytes, and no vector holds pairs of two kinds
    bool whole = a.head_dim % E == 0 && (a.interleaved ? rot_dim % E : a.half % E) == 0 && (a.page_block & 15) == 0;
    for (int i = 0; i < 3; ++i)
        if (a.heads[i])
            whole = whole && seq_aligned(a.in[i], 16) && seq_aligned(a.out[i], 16) && ((a.in_token[i] | a.in_head[i] | a.out_token[i] | a.out_head[i]) & 15) == 0;
    const uint32_t e = whole ? E : 1, rest = a.head_dim - rot_dim;
    a.spans = a.interleaved ? (a.head_dim / e + 1) / 2 : a.half / e + (rest / e + 1) / 2;
    uint32_t threads = (a.n_heads * a.spans + 63) / 64 * 64;
    if (threads > 256) threads = 256;
    a.per_pass = threads / a.spans;
    return seq_launches(n_tokens, [&](uint32_t first, uint32_t n) {
        a.first_token = first;
        if (whole) hipLaunchKernelGGL((rope_kernel<T, E, kPages>), dim3(n), dim3(threads), 0, st, a);
        else hipLaunchKernelGGL((rope_kernel<T, 1, kPages>), dim3(n), dim3(threads), 0, st, a);
    });
}

template <bool kPages> hipError_t launch_rope(RopeArgs &a, int dtype, uint32_t n_tokens, uint32_t rot_dim, hipStream_t st) {
    if (dtype == HPS_SEQ_F32) return launch_rope<float, kPages>(a, n_tokens, rot_dim, st);
    if (dtype == HPS_SEQ_F16) return launch_rope<_Float16, kPages>(a, n_tokens, rot_dim, st);
    return launch_rope<__bf16, kPages>(a, n_tokens, rot_dim, st);
}

int size_of(int dtype) { return dtype == HPS_SEQ_F32 ? 4 : 2; }

hps_status_t check_rope(int dtype, uint32_t head_dim, uint32_t rot_dim, const float *table, const int32_t *positions, uint32_t max_pos, uint32_t n_tokens) {
    SEQ_REQUIRE(dtype == HPS_SEQ_F32 || dtype == HPS_SEQ_F16 || dtype == HPS_SEQ_BF16, "dtype must be HPS_SEQ_F32, HPS_SEQ_F16 or HPS_SEQ_BF16");
    SEQ_REQUIRE(head_dim > 0 && head_dim <= 512, "head_dim must be in 1 .. 512");
    SEQ_REQUIRE(n_tokens < (1u << 31), "n_tokens must be < 2^31");
    if (!table) return HPS_OK;
    SEQ_REQUIRE(rot_dim % 2 == 0 && rot_dim > 0 && rot_dim <= head_dim, "rot_dim must be even and in 2 .. head_dim");
    SEQ_REQUIRE(max_pos > 0 && max_pos <= (1u << 31), "max_pos must be in 1 .. 2^31");
    SEQ_REQUIRE(seq_aligned(table, 8), "table must be 8-byte aligned");
    SEQ_REQUIRE(n_tokens == 0 || seq_words(positions), "positions must be a 4-byte aligned device pointer");
    return HPS_OK;
}

// Puts an array of heads into the arguments' place i; false if it is not there or not aligned to its values.
bool put(RopeArgs &a, int i, uint32_t heads, const hps_seq_heads_t &in, const hps_seq_heads_t &out, int size) {
    a.heads[i] = heads;
    a.in[i] = static_cast<const char *>(in.data);
    a.out[i] = static_cast<char *>(out.data);
    a.in_token[i] = in.token_stride * size;
    a.in_head[i] = in.head_stride * size;
    a.out_token[i] = out.token_stride * size;
    a.out_head[i] = out.head_stride * size;
    return heads == 0 || (in.data && out.data && seq_aligned(in.data, size) && seq_aligned(out.data, size));
}

}  // namespace

hps_status_t hps_seq_fail(hps_status_t code, const char *what, const char *more) {
    snprintf(g_err, sizeof(g_err), "%s%s", what, more);
    return code;
}

extern "C" {

const char *hps_seq_last_error(void) { return g_err; }

hps_status_t hps_seq_extend(const hps_seq_extend_args_t *args, void *stream) {
    SEQ_REQUIRE(args, "args must not be NULL");
    const hps_seq_extend_args_t &a = *args;
    SEQ_REQUIRE(seq_block_size(a.block_size), "block_size must be a power of two in 1 .. 1024");
    SEQ_REQUIRE((uint64_t)a.n_blocks * a.block_size < (1ull << 31), "n_blocks * block_size must be < 2^31");
    SEQ_REQUIRE((uint64_t)a.table_width * a.block_size < (1ull << 31), "table_width * block_size must be < 2^31");
    SEQ_REQUIRE(a.n_requests <= (1u << 24), "n_requests must be <= 2^24");
    SEQ_REQUIRE(a.max_tokens < (1u << 31), "max_tokens must be < 2^31");
    SEQ_REQUIRE(seq_words(a.n_free) && seq_words(a.token_offsets) && seq_words(a.info), "n_free, token_offsets and info must be 4-byte aligned device pointers");
    SEQ_REQUIRE(a.n_blocks == 0 || seq_words(a.free_blocks), "free_blocks must be a 4-byte aligned device pointer");
    SEQ_REQUIRE(a.max_tokens == 0 || (seq_words(a.slots) && seq_words(a.positions)), "slots and positions must be 4-byte aligned device pointers");
    SEQ_REQUIRE(a.n_requests == 0 || (seq_words(a.past_lens) && seq_words(a.new_lens) && seq_words(a.total_lens)),
                "past_lens, new_lens and total_lens must be 4-byte aligned device pointers");
    SEQ_REQUIRE(a.n_requests == 0 || a.table_width == 0 || seq_words(a.block_table), "block_table must be a 4-byte aligned device pointer");
    SEQ_REQUIRE(a.start == nullptr || seq_aligned(a.start, 4), "start must be 4-byte aligned");
    SEQ_REQUIRE(a.n_free != a.info, "info must not be the array that n_free is read from");
    SEQ_REQUIRE(a.n_requests == 0 || (a.total_lens != a.past_lens && a.total_lens != a.new_lens), "total_lens must be an array of its own");
    ExtendArgs e{a, (uint32_t)__builtin_ctz(a.block_size), a.table_width * a.block_size};
    const uint32_t chunks = a.n_requests ? (a.n_requests + kChunk - 1) / kChunk : 1;
    // a store of each lane that sees to tokens, and one work-group per CU at most (1.2 million tokens of 8,192 requests: 64 / 128 / 256 / 512
    // work-groups 21.3 / 14.8 / 12.2 / 14.6 us)
    uint32_t parts = (a.max_tokens + 3 * kThreads - 1) / (3 * kThreads), most = 256u / chunks;
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    hipLaunchKernelGGL(extend_kernel, dim3(parts, chunks), dim3(kThreads), 0, static_cast<hipStream_t>(stream), e);
    SEQ_TRY(hipGetLastError());
    return HPS_OK;
}

hps_status_t hps_seq_release(int32_t *lens, const int32_t *finished, uint32_t n_requests, uint32_t block_size, int32_t *block_table,
                             uint32_t table_width, int32_t *free_blocks, uint32_t n_blocks, const int32_t *n_free, int32_t *info, void *stream) {
    SEQ_REQUIRE(seq_block_size(block_size), "block_size must be a power of two in 1 .. 1024");
    SEQ_REQUIRE((uint64_t)n_blocks * block_size < (1ull << 31), "n_blocks * block_size must be < 2^31");
    SEQ_REQUIRE((uint64_t)table_width * block_size < (1ull << 31), "table_width * block_size must be < 2^31");
    SEQ_REQUIRE(n_requests <= (1u << 24), "n_requests must be <= 2^24");
    SEQ_REQUIRE(seq_words(n_free) && seq_words(info), "n_free and info must be 4-byte aligned device pointers");
    SEQ_REQUIRE(n_blocks == 0 || seq_words(free_blocks), "free_blocks must be a 4-byte aligned device pointer");
    SEQ_REQUIRE(n_requests == 0 || (seq_words(lens) && seq_words(finished)), "lens and finished must be 4-byte aligned device pointers");
    SEQ_REQUIRE(n_requests == 0 || table_width == 0 || seq_words(block_table), "block_table must be a 4-byte aligned device pointer");
    const ReleaseArgs a{lens, finished, block_table, free_blocks, n_free, info, n_requests, (uint32_t)__builtin_ctz(block_size), table_width * block_size,
                        table_width, n_blocks};
    hipLaunchKernelGGL(release_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
    SEQ_TRY(hipGetLastError());
    return HPS_OK;
}

hps_status_t hps_seq_rope_table(float *table, uint32_t max_pos, uint32_t rot_dim, double base, int scale, double factor, double original, double low,
                                double high, double magnitude, void *stream) {
    SEQ_REQUIRE(rot_dim > 0 && rot_dim % 2 == 0 && rot_dim <= 512, "rot_dim must be even and in 2 .. 512");
    SEQ_REQUIRE(max_pos <= (1u << 31), "max_pos must be <= 2^31");
    SEQ_REQUIRE(std::isfinite(base) && base > 0, "base must be finite and > 0");
    SEQ_REQUIRE(std::isfinite(magnitude), "magnitude must be finite");
    SEQ_REQUIRE(scale >= HPS_SEQ_SCALE_NONE && scale <= HPS_SEQ_SCALE_PARTS, "scale must be HPS_SEQ_SCALE_NONE, _LINEAR or _PARTS");
    SEQ_REQUIRE(scale == HPS_SEQ_SCALE_NONE || (std::isfinite(factor) && factor > 0), "factor must be finite and > 0");
    SEQ_REQUIRE(scale != HPS_SEQ_SCALE_PARTS || (std::isfinite(original) && original > 0 && std::isfinite(low) && std::isfinite(high) && low < high),
                "original must be finite and > 0, and low < high");
    if (max_pos == 0) return HPS_OK;
    SEQ_REQUIRE(table && seq_aligned(table, 8), "table must be an 8-byte aligned device pointer");
    const uint64_t n = (uint64_t)max_pos * (rot_dim / 2), groups = (n + 255) / 256;
    hipLaunchKernelGGL(rope_table_kernel, dim3((uint32_t)(groups < 65536 ? groups : 65536)), dim3(256), 0, static_cast<hipStream_t>(stream), table, max_pos,
                       rot_dim / 2, base, scale, factor, original, low, high, magnitude);
    SEQ_TRY(hipGetLastError());
    return HPS_OK;
}

hps_status_t hps_seq_rope(const hps_seq_rope_args_t *args, void *stream) {
    SEQ_REQUIRE(args, "args must not be NULL");
    const hps_seq_rope_args_t &r = *args;
    SEQ_REQUIRE(r.table, "table must not be NULL");
    if (hps_status_t st = check_rope(r.dtype, r.head_dim, r.rot_dim, r.table, r.positions, r.max_pos, r.n_tokens)) return st;
    SEQ_REQUIRE((uint64_t)r.q_heads + r.k_heads <= 65536, "at most 65536 heads");
    if (r.n_tokens == 0 || r.q_heads + r.k_heads == 0) return HPS_OK;
    RopeArgs a{};
    SEQ_REQUIRE(put(a, 0, r.q_heads, r.q, r.q_out, size_of(r.dtype)) && put(a, 1, r.k_heads, r.k, r.k_out, size_of(r.dtype)),
                "q, k, q_out and k_out must be device pointers aligned to their type");
    a.positions = r.positions;
    a.table = r.table;
    a.head_dim = r.head_dim;
    a.half = r.rot_dim / 2;
    a.max_pos = r.max_pos;
    a.interleaved = r.interleaved != 0;
    a.sign = r.inverse ? -1.f : 1.f;
    SEQ_TRY(launch_rope<false>(a, r.dtype, r.n_tokens, r.rot_dim, static_cast<hipStream_t>(stream)));
    return HPS_OK;
}

hps_status_t hps_seq_append(const hps_seq_append_args_t *args, void *stream) {
    SEQ_REQUIRE(args, "args must not be NULL");
    const hps_seq_append_args_t &r = *args;
    if (hps_status_t st = check_rope(r.dtype, r.head_dim, r.rot_dim, r.table, r.positions, r.max_pos, r.n_tokens)) return st;
    SEQ_REQUIRE(seq_block_size(r.pages.block_size), "block_size must be a power of two in 1 .. 1024");
    SEQ_REQUIRE((uint64_t)r.pages.n_blocks * r.pages.block_size < (1ull << 31), "n_blocks * block_size must be < 2^31");
    SEQ_REQUIRE(r.kv_heads > 0 && (uint64_t)r.q_heads + 2ull * r.kv_heads <= 65536, "kv_heads must be > 0, and at most 65536 heads in all");
    if (r.n_tokens == 0) return HPS_OK;
    SEQ_REQUIRE(seq_words(r.slots), "slots must be a 4-byte aligned device pointer");
    const int size = size_of(r.dtype);
    const hps_seq_heads_t pk{r.pages.k, r.pages.token_stride, r.pages.head_stride}, pv{r.pages.v, r.pages.token_stride, r.pages.head_stride};
    RopeArgs a{};
    SEQ_REQUIRE(put(a, 0, r.q_heads, r.q, r.q_out, size) && put(a, 1, r.kv_heads, r.k, pk, size) && put(a, 2, r.kv_heads, r.v, pv, size),
                "q, q_out, k, v and the pages must be device pointers aligned to their type");
    a.page_block = r.pages.block_stride * size;
    a.positions = r.positions;
    a.slots = r.slots;
    a.table = r.table;
    a.head_dim = r.head_dim;
    a.half = r.table ? r.rot_dim / 2 : 0;
    a.max_pos = r.max_pos;
    a.n_slots = r.pages.n_blocks * r.pages.block_size;
    a.sh = (uint32_t)__builtin_ctz(r.pages.block_size);
    a.interleaved = r.table && r.interleaved;
    a.sign = 1.f;
    SEQ_TRY(launch_rope<true>(a, r.dtype, r.n_tokens, r.table ? r.rot_dim : 0, static_cast<hipStream_t>(stream)));
    return HPS_OK;
}

}  // extern "C"
