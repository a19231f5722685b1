// Norms of heads with the rotation in the same pass, and their gradients (hps_seq.h), for gfx950.
#include <hip/hip_runtime.h>

#include <cmath>

#include "hps_seq_norm.h"

namespace {

template <typename T, int E, bool kWithin> __global__ void __launch_bounds__(kNormThreads) norm_kernel(const NormArgs a) {
    const uint32_t group = a.first_group + blockIdx.x;
    if (group < a.x[0].groups) norm_forward<T, E, kWithin>(a, a.x[0], group);
    else norm_forward<T, E, kWithin>(a, a.x[1], group - a.x[0].groups);
}

// With n = r x, r = 1 / sqrt(mean(x^2) + eps), and y = turn(w n): dz = turn back(dy); dw = sum dz n; with g = w dz
//   dx = r (g - n mean(g n)),
// so a head takes one pass with two sums.  A work-group goes through tokens with its weights' sums in registers, joins its lanes' in
// LDS at the end, and a second kernel adds up the work-groups'.  Bound by HBM where there are many (16,384 tokens of 32 heads of 64 of 32 bits,
// 403 MB moved: 78 us, 5.2 TB/s, and 4.8 of the sums), else by the chain position, angles and rows, sums, store of each token, of which nothing is requested
// ahead (2,003 of 24 heads of 96 of 16 bits, 28 MB: 10.4 to 11.4 and 3.9).
template <typename T, int E, bool kWithin> __device__ __forceinline__ void norm_backward(const NormArgs &a, const NormTensor &g, uint32_t which, uint32_t group) {
    constexpr int kPer = E == 1 ? 4 : 1;
    __shared__ float l_sum[kNormThreads][kPer * 2 * E + 1];
    const uint32_t l = threadIdx.x & ((1u << a.lane_bits) - 1u), row = threadIdx.x >> a.lane_bits, beside = row / g.heads_beside;
    NormSpan<T, E, kWithin> sp[kPer];
    float sum[kPer][2 * E];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        sp[i].place(a, l + ((uint32_t)i << a.lane_bits));
        sp[i].weights(g.weight);
#pragma unroll
        for (int j = 0; j < 2 * E; ++j) sum[i][j] = 0.f;
    }
    for (uint64_t at = (uint64_t)group * g.tokens_beside; at < a.n_tokens; at += (uint64_t)g.groups * g.tokens_beside) {
        const uint64_t t = at + beside;
        if (beside >= g.tokens_beside || t >= a.n_tokens) break;
        const int32_t pos = a.table ? a.positions[t] : 0;
        if (pos < 0) continue;
        if (a.table)
#pragma unroll
            for (int i = 0; i < kPer; ++i) sp[i].angles(a, l + ((uint32_t)i << a.lane_bits), pos, -1.f);
        const char *from = g.in + (int64_t)t * g.in_token, *back = g.back + (int64_t)t * g.back_token;
        char *to = g.out + (int64_t)t * g.out_token;
        for (uint32_t h = row % g.heads_beside; h < g.heads; h += g.heads_beside) {
            float x[kPer][2 * E], z[kPer][2 * E], squares = 0.f, products = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                NormSpan<T, E, kWithin>::take(sp[i].request(from + (int64_t)h * g.in_head), x[i]);
                NormSpan<T, E, kWithin>::take(sp[i].request(back + (int64_t)h * g.back_head), z[i]);
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                sp[i].turn(z[i]);
#pragma unroll
                for (int j = 0; j < 2 * E; ++j) {
                    squares = __builtin_fmaf(x[i][j], x[i][j], squares);
                    products = __builtin_fmaf(z[i][j] * sp[i].w[j], x[i][j], products);
                }
            }
            const float m = __builtin_fmaf(norm_sum(squares, a.lane_bits), a.per_value, a.eps);
            products = norm_sum(products, a.lane_bits);
            float r = norm_inverse(m), c = products * r * a.per_value;
            // products alone may be beyond what 32 bits hold, or below: then their sum is formed of n, as for a head that does not fit
            const bool odd = NormFit::needed(m) || !(__builtin_fabsf(products) >= 0x1p-100f && __builtin_fabsf(products) < __builtin_inff());
            if (__builtin_expect(__ballot(odd) != 0, 0)) {
                const NormFit fit(a, m);
                squares = products = 0.f;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
#pragma unroll
                    for (int j = 0; j < 2 * E; ++j) {
                        const float y = x[i][j] * fit.by;
                        squares = __builtin_fmaf(y, y, squares);
                    }
                r = norm_inverse(__builtin_fmaf(norm_sum(squares, a.lane_bits), a.per_value, fit.eps));
#pragma unroll
                for (int i = 0; i < kPer; ++i)
#pragma unroll
                    for (int j = 0; j < 2 * E; ++j) {
                        float y = x[i][j], w = sp[i].w[j];                  // nothing that the other way has: kept for here it costs a wave of a SIMD
                        asm("" : "+v"(y), "+v"(w));
                        products = __builtin_fmaf(z[i][j] * w, y * fit.by * r, products);
                    }
                products = norm_sum(products, a.lane_bits) * a.per_value;
                c = odd ? products : c;                // a head that fits keeps its bits beside one that does not
                // back to the head as it is, whose r may itself be beyond 32 bits: with r / k, k dz and k^2 c for r, dz and c the gradients are what they were
                const float k = fit.by > 1.f && r > 0x1p20f ? 0x1p28f : fit.by < 1.f && r < 0x1p-48f ? 0x1p-4f : 1.f;
                r *= fit.by / k;
                c *= k * k;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
#pragma unroll
                    for (int j = 0; j < 2 * E; ++j) z[i][j] *= k;
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
#pragma unroll
                for (int j = 0; j < 2 * E; ++j) {
                    const float n = x[i][j] * r;
                    sum[i][j] = __builtin_fmaf(z[i][j], n, sum[i][j]);
                    x[i][j] = r * __builtin_fmaf(z[i][j], sp[i].w[j], -n * c);
                }
                sp[i].store(to + (int64_t)h * g.out_head, x[i]);
            }
        }
    }
    if (!a.weight_grad[which]) return;                 // uniform
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int j = 0; j < 2 * E; ++j) l_sum[threadIdx.x][i * 2 * E + j] = sum[i][j];
    __syncthreads();
    const uint32_t rows = min(kNormThreads >> a.lane_bits, g.heads_beside * g.tokens_beside);
    float *to = a.parts + ((size_t)which * HPS_SEQ_NORM_PARTS + group) * a.head_dim;
    for (uint32_t x = threadIdx.x; x < (uint32_t)(kPer * 2 * E) << a.lane_bits; x += kNormThreads) {
        const uint32_t lane = x & ((1u << a.lane_bits) - 1u), at = x >> a.lane_bits, j = at % (2 * E);
        NormSpan<T, E, kWithin> of;
        of.place(a, lane + (at / (2 * E) << a.lane_bits));
        if (!(j < E ? of.has0 : of.has1)) continue;
        float y = 0.f;
        for (uint32_t r = 0; r < rows; ++r) y += l_sum[(r << a.lane_bits) + lane][at];
        to[j < E ? of.o0 + j : of.o1 + j - E] = y;
    }
}

template <typename T, int E, bool kWithin> __global__ void __launch_bounds__(kNormThreads) norm_grad_kernel(const NormArgs a) {
    const uint32_t group = blockIdx.x;
    if (group < a.x[0].groups) norm_backward<T, E, kWithin>(a, a.x[0], 0, group);
    else norm_backward<T, E, kWithin>(a, a.x[1], 1, group - a.x[0].groups);
}

// Sums of the work-groups' parts, 16 values of a weight to a work-group, 64 threads to a value.
constexpr uint32_t kJoinWays = 64;
__global__ void __launch_bounds__(16 * kJoinWays) norm_join_kernel(const NormArgs a) {
    __shared__ float l_sum[kJoinWays][17];
    const uint32_t which = blockIdx.y, d = blockIdx.x * 16 + (threadIdx.x & 15u), way = threadIdx.x >> 4, n = a.x[which].groups;
    float *to = a.weight_grad[which];
    if (!to) return;
    const float *from = a.parts + (size_t)which * HPS_SEQ_NORM_PARTS * a.head_dim + d;
    float sum = 0.f;
    if (d < a.head_dim) {
        constexpr uint32_t kEach = HPS_SEQ_NORM_PARTS / kJoinWays;
        float x[kEach];
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) x[i] = way + i * kJoinWays < n ? from[(size_t)(way + i * kJoinWays) * a.head_dim] : 0.f;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) sum += x[i];
    }
    l_sum[way][threadIdx.x & 15u] = sum;
    __syncthreads();
    for (uint32_t w = kJoinWays / 2; w; w >>= 1) {
        if (way < w) l_sum[way][threadIdx.x & 15u] += l_sum[way + w][threadIdx.x & 15u];
        __syncthreads();
    }
    if (way == 0 && d < a.head_dim) to[d] = l_sum[0][threadIdx.x];
}

int size_of(int dtype) { return dtype == HPS_SEQ_F32 ? 4 : 2; }

template <typename T> hipError_t launch_norm(NormArgs &a, bool whole, hipStream_t st) {
    return seq_launches((uint64_t)a.x[0].groups + a.x[1].groups, [&](uint32_t first, uint32_t n) {
        a.first_group = first;
        if (whole && a.interleaved) hipLaunchKernelGGL((norm_kernel<T, 16 / sizeof(T), true>), dim3(n), dim3(kNormThreads), 0, st, a);
        else if (whole) hipLaunchKernelGGL((norm_kernel<T, 16 / sizeof(T), false>), dim3(n), dim3(kNormThreads), 0, st, a);
        else hipLaunchKernelGGL((norm_kernel<T, 1, false>), dim3(n), dim3(kNormThreads), 0, st, a);
    });
}

template <typename T> hipError_t launch_grad(const NormArgs &a, bool whole, hipStream_t st) {
    const uint32_t n = a.x[0].groups + a.x[1].groups;
    if (n) {
        if (whole && a.interleaved) hipLaunchKernelGGL((norm_grad_kernel<T, 16 / sizeof(T), true>), dim3(n), dim3(kNormThreads), 0, st, a);
        else if (whole) hipLaunchKernelGGL((norm_grad_kernel<T, 16 / sizeof(T), false>), dim3(n), dim3(kNormThreads), 0, st, a);
        else hipLaunchKernelGGL((norm_grad_kernel<T, 1, false>), dim3(n), dim3(kNormThreads), 0, st, a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (!a.weight_grad[0] && !a.weight_grad[1]) return hipSuccess;
    hipLaunchKernelGGL(norm_join_kernel, dim3((a.head_dim + 15) / 16, 2), dim3(16 * kJoinWays), 0, st, a);
    return hipGetLastError();
}

// Work-groups of a tensor's gradients: fewer leave the device idle, more have more sums to join (us with 256 / 512 / 1,024: 8,192 tokens of 20
// heads of 128 42.1 / 33.4 / 34.2, of 40 heads 68.0 / 56.4 / 58.1; 16,384 of 32 heads of 64 in 32 bits 85.7 / 87.0 / 89.0; 2,003 of 24 heads of 96
// 17.4 / 16.4 / 16.9).
constexpr uint32_t kGradGroups = 512;
static_assert(kGradGroups <= HPS_SEQ_NORM_PARTS, "a part each");

NormArgs args_of(const hps_seq_norm_args_t &r) {
    NormArgs a{};
    a.positions = r.positions;
    a.table = r.table;
    a.x[0].weight = r.q_weight;
    a.x[1].weight = r.k_weight;
    norm_set_eps(a, r.eps);
    a.per_value = 1.f / (float)r.head_dim;
    a.n_tokens = r.n_tokens;
    a.head_dim = r.head_dim;
    a.half = r.table ? r.rot_dim / 2 : 0;
    a.max_pos = r.max_pos;
    a.interleaved = r.table && r.interleaved;
    a.norm = 1;
    return a;
}

}  // namespace

bool norm_put(NormArgs &a, int i, uint32_t heads, const hps_seq_heads_t &in, const hps_seq_heads_t &out, const hps_seq_heads_t *back, int size) {
    NormTensor &x = a.x[i];
    x.heads = heads;
    x.in = static_cast<const char *>(in.data);
    x.out = static_cast<char *>(out.data);
    x.in_token = in.token_stride * size;
    x.in_head = in.head_stride * size;
    x.out_token = out.token_stride * size;
    x.out_head = out.head_stride * size;
    if (back) {
        x.back = static_cast<const char *>(back->data);
        x.back_token = back->token_stride * size;
        x.back_head = back->head_stride * size;
    }
    return heads == 0 || (in.data && out.data && seq_aligned(in.data, size) && seq_aligned(out.data, size) && (!back || (back->data && seq_aligned(back->data, size))));
}

bool norm_whole(NormArgs &a, uint32_t rot_dim, int size, bool more) {
    const uint32_t most = 16 / size;
    bool whole = more && a.head_dim % most == 0 && (a.interleaved ? rot_dim % most : a.half % most) == 0;
    for (const NormTensor &x : a.x)
        if (x.heads)
            whole = whole && seq_aligned(x.in, 16) && seq_aligned(x.out, 16) && seq_aligned(x.back, 16) &&
                    ((x.in_token | x.in_head | x.out_token | x.out_head | x.back_token | x.back_head) & 15) == 0;
    const uint32_t e = whole ? most : 1, spans = a.interleaved ? (a.head_dim / e + 1) / 2 : a.half / e + ((a.head_dim - 2 * a.half) / e + 1) / 2;
    a.lane_bits = 0;
    while (a.lane_bits < 6 && (1u << a.lane_bits) < spans) ++a.lane_bits;
    return whole;
}

// A lane gets two heads of a token where there still are eight work-groups to a CU, so that weights and angles are read half as often.  (us, one to a lane /
// two, 8,192 tokens: 20 heads of 128 22.1 / 20.2, 40 heads 38.3 / 36.0, four to a lane 38.7; 24 heads of 96 23.6 / 20.3.  Beside keys and values in one
// launch four are better, where there are enough: 8,192 tokens of 32 and 8 heads 50.6 -> 44.)  A work-group gets several tokens
// where there is one for each CU: below that a token each has the shorter chain.  (16 heads of 64, 8,192 tokens: a token at a time 15.1, four 10.5.)
constexpr uint32_t kFull = 2048, kCus = 256;

void norm_share(NormArgs &a, int i, uint32_t most_groups, uint32_t most_each) {
    NormTensor &x = a.x[i];
    x.heads_beside = x.tokens_beside = 1;
    x.groups = 0;
    if (x.heads == 0 || a.n_tokens == 0) return;
    const uint32_t rows = kNormThreads >> a.lane_bits;
    const uint64_t full = ((uint64_t)a.n_tokens * x.heads + rows - 1) / rows;                  // work-groups with a head to a lane
    uint32_t each = most_each >= 4 && full >= 4 * kFull ? 4 : full >= kFull ? 2 : 1;
    if (x.heads > each * rows) each = (x.heads + rows - 1) / rows;
    x.heads_beside = (x.heads + each - 1) / each;
    const uint64_t spare = full / kCus + 1;
    x.tokens_beside = rows / x.heads_beside;
    if (most_groups > HPS_SEQ_NORM_PARTS && x.tokens_beside > spare) x.tokens_beside = (uint32_t)spare;
    x.groups = (a.n_tokens + x.tokens_beside - 1) / x.tokens_beside;
    if (x.groups > most_groups) x.groups = most_groups;
}

hps_status_t norm_check(int dtype, uint32_t head_dim, uint32_t rot_dim, const float *table, const int32_t *positions, uint32_t max_pos, uint32_t n_tokens, double eps,
                        const float *q_weight, const float *k_weight) {
    if (hps_status_t st = seq_check_rope(dtype, head_dim, rot_dim, table, positions, max_pos, n_tokens)) return st;
    SEQ_REQUIRE(eps >= 0 && eps <= __FLT_MAX__, "eps must be finite and >= 0");
    SEQ_REQUIRE(seq_aligned(q_weight, 4) && seq_aligned(k_weight, 4), "q_weight and k_weight must be 4-byte aligned");
    return HPS_OK;
}

extern "C" {

hps_status_t hps_seq_norm_rope(const hps_seq_norm_args_t *args, void *stream) {
    SEQ_REQUIRE(args, "args must not be NULL");
    const hps_seq_norm_args_t &r = *args;
    if (hps_status_t st = norm_check(r.dtype, r.head_dim, r.rot_dim, r.table, r.positions, r.max_pos, r.n_tokens, r.eps, r.q_weight, r.k_weight)) return st;
    SEQ_REQUIRE((uint64_t)r.q_heads + r.k_heads <= 65536, "at most 65536 heads");
    if (r.n_tokens == 0 || r.q_heads + r.k_heads == 0) return HPS_OK;
    NormArgs a = args_of(r);
    SEQ_REQUIRE(norm_put(a, 0, r.q_heads, r.q, r.q_out, nullptr, size_of(r.dtype)) && norm_put(a, 1, r.k_heads, r.k, r.k_out, nullptr, size_of(r.dtype)),
                "q, k, q_out and k_out must be device pointers aligned to their type");
    const bool whole = norm_whole(a, 2 * a.half, size_of(r.dtype));
    norm_share(a, 0, 0xFFFFFFFFu, 2);
    norm_share(a, 1, 0xFFFFFFFFu, 2);
    hipStream_t st = static_cast<hipStream_t>(stream);
    SEQ_TRY(r.dtype == HPS_SEQ_F32 ? launch_norm<float>(a, whole, st) : r.dtype == HPS_SEQ_F16 ? launch_norm<_Float16>(a, whole, st) : launch_norm<__bf16>(a, whole, st));
    return HPS_OK;
}

hps_status_t hps_seq_norm_rope_grad(const hps_seq_norm_args_t *args, const hps_seq_heads_t *q_grad, const hps_seq_heads_t *k_grad, float *q_weight_grad,
                                    float *k_weight_grad, float *parts, void *stream) {
    SEQ_REQUIRE(args, "args must not be NULL");
    const hps_seq_norm_args_t &r = *args;
    if (hps_status_t st = norm_check(r.dtype, r.head_dim, r.rot_dim, r.table, r.positions, r.max_pos, r.n_tokens, r.eps, r.q_weight, r.k_weight)) return st;
    SEQ_REQUIRE((uint64_t)r.q_heads + r.k_heads <= 65536, "at most 65536 heads");
    SEQ_REQUIRE(seq_aligned(q_weight_grad, 4) && seq_aligned(k_weight_grad, 4) && seq_aligned(parts, 4), "q_weight_grad, k_weight_grad and parts must be 4-byte aligned");
    SEQ_REQUIRE(parts || (!q_weight_grad && !k_weight_grad), "parts must not be NULL where a weight's gradient is wanted");
    NormArgs a = args_of(r);
    const hps_seq_heads_t none{nullptr, 0, 0};
    if (r.n_tokens) {
        SEQ_REQUIRE(norm_put(a, 0, r.q_heads, r.q, q_grad ? *q_grad : none, &r.q_out, size_of(r.dtype)) &&
                    norm_put(a, 1, r.k_heads, r.k, k_grad ? *k_grad : none, &r.k_out, size_of(r.dtype)),
                    "q, k, q_out, k_out, q_grad and k_grad must be device pointers aligned to their type");
    }
    a.parts = parts;
    a.weight_grad[0] = q_weight_grad;
    a.weight_grad[1] = k_weight_grad;
    const bool whole = norm_whole(a, 2 * a.half, size_of(r.dtype));
    norm_share(a, 0, kGradGroups, 2);
    norm_share(a, 1, kGradGroups, 2);
    hipStream_t st = static_cast<hipStream_t>(stream);
    SEQ_TRY(r.dtype == HPS_SEQ_F32 ? launch_grad<float>(a, whole, st) : r.dtype == HPS_SEQ_F16 ? launch_grad<_Float16>(a, whole, st) : launch_grad<__bf16>(a, whole, st));
    return HPS_OK;
}

}  // extern "C"
