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

#include "hps_seq_attend.h"

namespace {

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
constexpr int kJoin = 256;
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
uint32_t choose_chunks(const SeqAttendShape &shape, uint64_t tiles, uint32_t keys, bool wide, uint64_t rows, uint32_t head_dim, uint32_t cus, uint64_t most) {
    const uint32_t step = wide ? shape.wide_keys : shape.narrow_keys * kWaves, limit = div_up(keys, step), slots = cus * shape.beside(wide, head_dim);
    const double size = head_dim / 128.0, part = rows * (head_dim * 8.0 + 16.0) / 4e6;
    uint32_t best = 1;
    double least = 0;
    for (uint32_t s = 1; s <= limit && s <= most && s < kMaxParts / 2; ++s) {
        const uint32_t chunk = div_up(limit, s);       // in steps
        if (s > 1 && div_up(limit, chunk) != s) continue;
        const double n = (double)(tiles * s), beside = n < slots ? n : slots, all = n <= slots ? 1.0 : (n / slots + std::ceil(n / slots)) / 2;
        const double cost = all * (chunk * shape.step(wide, n, beside, cus, size) + 4.0) + s * part;
        if (s == 1 || cost < least) {
            best = s;
            least = cost;
        }
    }
    return best;
}

// Up to 32 rows the waves share the keys; up to 64 too, in two work-groups, where reading a long history is what counts (waves share
// keys / rows, us: 64 rows behind 4,096 keys 16.1 / 15.4, behind 65,536 36.9 / 41.1; 96 rows 53.1 / 37.7).
// A wave to a request where there are more requests than work-groups at a time, up to 512 keys (a wave / a work-group each, us, 4
// key heads of 128: 64 requests of 64 / 256 / 512 keys 14.6, 21.9, 32.4 / 13.9, 14.9, 19.9; 512 of 64 / 256 / 512 / 1,024 keys 26.2, 38.0,
// 63.2, 134.1 / 43.6, 50.6, 69.6, 129.2).
constexpr SeqAttendShape kShape = {
    kWideRows, kWideKeys, kNarrowKeys,
    [](uint64_t, uint32_t) { return kNarrowRows; },
    512,
    [](bool own, uint64_t rows, uint32_t keys, uint64_t, uint32_t) { return rows > (!own && keys >= 16384 ? 2 : 1) * kNarrowRows; },
    [](bool, uint32_t head_dim) { return head_dim <= 128 ? 2u : 1u; },
    [](bool wide, double n, double beside, uint32_t cus, double size) { return wide ? (n <= cus ? 1.33 : 1.9) * (0.35 + 0.65 * size) : std::fmax(2.2, beside * 0.0121 * size); },
};

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

template <typename T, int DT> hipError_t launch(Args &a, uint32_t groups, hipStream_t st) {
    return a.head_dim == 32 * DT ? launch_attend<T, DT, true>(a, groups, st) : launch_attend<T, DT, false>(a, groups, st);
}

template <typename T> hipError_t launch(Args &a, uint32_t groups, hipStream_t st) {
    if (a.head_dim <= 32) return launch<T, 1>(a, groups, st);
    if (a.head_dim <= 64) return launch<T, 2>(a, groups, st);
    if (a.head_dim <= 96) return launch<T, 3>(a, groups, st);
    if (a.head_dim <= 128) return launch<T, 4>(a, groups, st);
    return launch<T, 8>(a, groups, st);
}

template <typename T, int kLanes> hipError_t launch_join(const Args &a, uint32_t parts, hipStream_t st) {
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

template <typename T> hipError_t launch_join(const Args &a, uint32_t parts, hipStream_t st) {
    if (a.head_dim <= 32) return launch_join<T, 8>(a, parts, st);
    if (a.head_dim <= 64) return launch_join<T, 16>(a, parts, st);
    if (a.head_dim <= 128) return launch_join<T, 32>(a, parts, st);
    return launch_join<T, 64>(a, parts, st);
}

}  // namespace

hps_status_t seq_attend_cut(SeqAttendArgs &a, const SeqAttendShape &shape, const hps_seq_attention_session &s, SeqAttendCut &cut) {
    const uint64_t rows = (uint64_t)a.n_tokens * a.q_heads, part_limit = s.part_rows / rows;
    // own tokens: one part at least, so that every row has one
    const uint64_t own_rows = (uint64_t)a.max_new * a.ratio, requests_heads = (uint64_t)a.n_requests * a.kv_heads;
    const uint64_t group_rows = a.n_groups && a.max_prefix ? (uint64_t)a.max_group * a.ratio : 0;
    const uint32_t own_keys = a.max_len ? a.max_len : 1;
    const bool own_wide = shape.wide(true, own_rows, own_keys, requests_heads, a.head_dim);
    a.history_wide = group_rows && shape.wide(false, group_rows, a.max_prefix, (uint64_t)a.n_groups * a.kv_heads, a.head_dim);
    const uint64_t own_narrow = own_wide ? 0 : own_rows, group_narrow = a.history_wide ? 0 : group_rows;
    const uint32_t narrow_rows = cut.narrow_rows = shape.narrow_rows(own_narrow > group_narrow ? own_narrow : group_narrow, a.head_dim);
    if (own_wide) {
        a.own_mode = kOwnWide;
        a.own_tiles = div_up(own_rows, shape.wide_rows);
        a.own_chunks = choose_chunks(shape, requests_heads * a.own_tiles, own_keys, true, rows, a.head_dim, s.cus, part_limit / 2);
        a.own_chunk = div_up(div_up(own_keys, a.own_chunks), shape.wide_keys) * shape.wide_keys;
    } else {
        a.own_mode = requests_heads > 2 * s.cus && own_keys <= shape.solo_keys ? kOwnSolo : kOwnSplit;
        a.own_tiles = div_up(own_rows, narrow_rows);
        const uint32_t step = a.own_mode == kOwnSolo ? shape.narrow_keys : shape.narrow_keys * kWaves;
        a.own_chunks = a.own_mode == kOwnSolo ? 1 : choose_chunks(shape, requests_heads * a.own_tiles, own_keys, false, rows, a.head_dim, s.cus, part_limit / 2);
        a.own_chunk = div_up(div_up(own_keys, a.own_chunks), step) * step;
    }
    if (a.own_tiles == 0) a.own_tiles = 1;
    const uint64_t own_items = requests_heads * a.own_tiles * a.own_chunks, own_groups = a.own_mode == kOwnSolo ? (own_items + kWaves - 1) / kWaves : own_items;
    uint64_t history_groups = 0;
    if (group_rows) {
        a.history_tiles = div_up(group_rows, a.history_wide ? shape.wide_rows : narrow_rows);
        const uint32_t step = a.history_wide ? shape.wide_keys : shape.narrow_keys * kWaves;
        a.history_chunks = choose_chunks(shape, (uint64_t)a.history_tiles * a.n_groups * a.kv_heads, a.max_prefix, a.history_wide, rows, a.head_dim, s.cus, part_limit - a.own_chunks);
        a.history_chunk = div_up(div_up(a.max_prefix, a.history_chunks), step) * step;
        const uint64_t combos = (uint64_t)a.n_groups * a.kv_heads * a.history_chunks;
        SEQ_REQUIRE(combos < (1u << 30), "too many groups, heads and chunks for one launch");
        a.history_combos = (uint32_t)combos;
        history_groups = (combos >= 8 ? (combos + 7) / 8 * 8 : combos) * a.history_tiles;
    }
    SEQ_REQUIRE(history_groups + own_groups < (1ull << 31) && own_items < (1ull << 31), "too many requests, heads and chunks for one launch");
    a.history_groups = (uint32_t)history_groups;
    a.own_items = (uint32_t)own_items;
    const auto divisor = [](uint32_t d) { return SeqDivisor::of(d ? d : 1); };
    a.by_kv_heads = divisor(a.kv_heads);
    a.by_ratio = divisor(a.ratio);
    a.by_history_tiles = divisor(a.history_tiles);
    a.by_history_combos = divisor(a.history_combos);
    a.by_history_chunks = divisor(a.history_chunks);
    a.by_own_chunks = divisor(a.own_chunks);
    a.by_own_tiles = divisor(a.own_tiles);
    cut.parts = a.history_chunks + a.own_chunks;
    a.direct = cut.parts == 1;
    cut.groups = (uint32_t)(history_groups + own_groups);
    return HPS_OK;
}

hipError_t seq_attend_check(const SeqAttendArgs &a, hipStream_t st) {
    if (!a.n_groups || a.history_groups) return hipSuccess;
    hipLaunchKernelGGL(check_kernel, dim3(div_up(a.n_groups, kThreads)), dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t seq_attend_join(const SeqAttendArgs &a, int dtype, uint32_t parts, hipStream_t st) {
    if (a.direct) return hipSuccess;
    return dtype == HPS_SEQ_F16 ? launch_join<_Float16>(a, parts, st) : launch_join<__bf16>(a, parts, st);
}

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
    if (e == hipSuccess) e = seq_packed_allow_lds();
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
    Args a{};
    bool work = false;
    if (hps_status_t st = seq_attend_args(s, args, a, work)) return st;
    const hps_seq_attention_args_t &r = *args;
    SEQ_REQUIRE(r.head_dim % 8 == 0, "head_dim must be a multiple of 8 in 8 .. 256");
    SEQ_REQUIRE(seq_block_size(r.pages.block_size), "block_size must be a power of two in 1 .. 1024");
    if (!work) return HPS_OK;
    SEQ_REQUIRE(r.pages.n_blocks == 0 || (r.pages.k && r.pages.v && seq_aligned(r.pages.k, 16) && seq_aligned(r.pages.v, 16)), "the pages must be device pointers, 16-byte aligned");
    SEQ_REQUIRE(seq_multiple16(r.pages.block_stride) && seq_multiple16(r.pages.token_stride) && seq_multiple16(r.pages.head_stride), "the pages' strides must be multiples of 16 bytes");
    SEQ_REQUIRE(r.pages.token_stride >= 0 && r.pages.token_stride < (1 << 25), "the pages' token_stride must be in 0 .. 2^25 - 1");
    SEQ_REQUIRE(r.pages.block_stride >= 0 && r.pages.block_stride < (1ll << 31), "the pages' block_stride must be in 0 .. 2^31 - 1");
    a.k = static_cast<const char *>(r.pages.k);
    a.v = static_cast<const char *>(r.pages.v);
    a.page_block = (uint32_t)(r.pages.block_stride * 2);
    a.page_token = (uint32_t)(r.pages.token_stride * 2);
    a.page_head = r.pages.head_stride * 2;
    SeqAttendCut cut;
    if (hps_status_t st = seq_attend_cut(a, kShape, *s, cut)) return st;
    hipStream_t st = static_cast<hipStream_t>(stream);
    SEQ_TRY(seq_attend_check(a, st));
    SEQ_TRY(r.dtype == HPS_SEQ_F16 ? launch<_Float16>(a, cut.groups, st) : launch<__bf16>(a, cut.groups, st));
    SEQ_TRY(seq_attend_join(a, r.dtype, cut.parts, st));
    return HPS_OK;
}

}  // extern "C"
