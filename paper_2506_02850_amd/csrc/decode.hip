// Attention of one new token per video over the dense or paged KV cache that stage 3 leaves (Sec. 3.3), with the token's own row
// appended and, if asked, the attention weight of every cached row accumulated (what metok_kv_evict ranks the rows by).
//
//   decode_attention_kernel  (decode_attention.h) every wave's tiles of the rows of all (video, kv head, block of query heads): scores,
//                            running maximum and sum of the softmax, weighted sum of the values, in one pass over K and V
//   decode_join_kernel       joins the parts of a (video, query head) whose rows several waves had; and, with weights, turns the
//                            scores that the first kernel kept into probabilities and adds their mean over the heads to the rows' weights
//
// What bounds it is the stream of K and V: 4 Hq dh operations a row on 2 Hkv dh elements, 7 operations a byte with seven query
// heads to a kv head in bf16.  The query heads of a kv head are the columns of one MFMA, so a row is read once for all of them.
// 8 videos of 36992 rows, 28 heads on 4 of 128 in bf16, 606 MB: 95.5 us a call, 6.35 TB/s (the join 4.5 us of it; a copy of 1 GiB moves
// 6.65 TB/s).  One of 2306 rows 8.8 us: two launches and their latency.
#include "decode_attention.h"

namespace metok {

constexpr int kJoinThreads = 256;
constexpr int kWeightRows = kJoinThreads;       // cache rows a workgroup adds up at a time: four to a lane
// Up to so many workgroups a head's elements are spread over several of them, 32 each: with few heads every one has many parts (one
// video of 2307 rows, 28 heads: 10.1 us a call with one workgroup a head, 9.0 with four).
constexpr int kJoinSpread = 512;
// (m, l) stands for the sum l 2^(m scale).
__device__ __forceinline__ void add_sum(float& m, float& l, float m2, float l2, float scale) {
    const float to = fmaxf(m, m2), ref = to == -INFINITY ? 0.f : to;
    l = l * exp2_from(m, ref, scale) + l2 * exp2_from(m2, ref, scale);
    m = to;
}

// The parts of a query head's result, and the place of each among all query rows of all parts.
struct HeadParts {
    PairParts pair;
    int n, rows, row;
    __device__ __forceinline__ int64_t slot(int p) const { return static_cast<int64_t>(pair.slot(p)) * rows + row; }
};
__device__ __forceinline__ HeadParts parts_of(const DecodeArgs& a, int b, int head) {
    const int kvh = head / a.group, qi = head - kvh * a.group, rb = qi / a.block_rows;
    const int2 w = a.pair_workers[(static_cast<int64_t>(b) * a.Hkv + kvh) * a.row_blocks + rb];
    const PairParts pair = pair_parts(w.x, w.y, a.teams != 0);
    return {pair, pair.n, a.rows, qi - rb * a.block_rows};
}

template <typename T, int DH>
__global__ __launch_bounds__(kJoinThreads) void decode_join_kernel(const DecodeArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
    const float scale = score_scale(a);
    if (static_cast<int>(blockIdx.x) < a.join_blocks) {
        // One (video, query head), or 4 join_lanes of its elements.  Every wave sums up the parts' statistics for itself; the parts of the output
        // are on their way meanwhile, the first kAhead of every group of lanes.
        constexpr int kAhead = 4;
        __shared__ float4 s_part[kJoinThreads];
        const int lanes = a.join_lanes, groups = kJoinThreads / lanes, pieces = DH / 4 / lanes;
        const int unit = blockIdx.x / pieces, piece = blockIdx.x - unit * pieces;
        const int b = unit / a.Hq, head = unit - b * a.Hq;
        const HeadParts parts = parts_of(a, b, head);
        if (parts.n == 1) return;
        const int g = threadIdx.x / lanes, x = threadIdx.x - g * lanes;
        const float* part = a.part_o + (piece * lanes + x) * 4;
        float4 ahead[kAhead];
        float ahead_m[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t slot = parts.slot(min(g + k * groups, parts.n - 1));
            ahead[k] = *reinterpret_cast<const float4*>(part + slot * DH);
            ahead_m[k] = ml[slot].x;
        }
        float m = -INFINITY, l = 0.f;
#pragma unroll 4
        for (int p = lane; p < parts.n; p += 64) {
            const float2 v = ml[parts.slot(p)];
            add_sum(m, l, v.x, v.y, scale);
        }
        const float top = score_of_key(wave_extreme<true>(ordered_key(m))), ref = top == -INFINITY ? 0.f : top;
        // The parts are added up relative to the largest maximum and divided by the sum, not scaled by 2^(m - log2 of the sum): that logarithm, rounded
        // at its full size, is off by a common factor of the result (fp32, 3000 rows with scores around 700: 1.9e-5 off, 1e-7 so).
        l = wave_sum(l * exp2_from(m, ref, scale));
        const float inv = l == 0.f ? 0.f : 1.f / l;                           // 0: no row counts
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](const float4& v, float f) { o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w); };
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (g + k * groups < parts.n) add(ahead[k], exp2_from(ahead_m[k], ref, scale));
#pragma unroll 4
        for (int p = g + kAhead * groups; p < parts.n; p += groups) {
            const int64_t slot = parts.slot(p);
            add(*reinterpret_cast<const float4*>(part + slot * DH), exp2_from(ml[slot].x, ref, scale));
        }
        s_part[threadIdx.x] = o;
        __syncthreads();
        if (g == 0) {
#pragma unroll 8
            for (int k = 1; k < groups; ++k) {
                const float4 v = s_part[k * lanes + x];
                o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
            }
            o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
            const int64_t at = static_cast<int64_t>(b) * a.Hq + head, to = at * DH + (piece * lanes + x) * 4;
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(a.out + to * 2) = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
            else *reinterpret_cast<float4*>(a.out + to * 4) = o;
        }
        if (threadIdx.x == 0 && piece == 0) {
            const int64_t at = static_cast<int64_t>(b) * a.Hq + head;
            if (a.lse) a.lse[at] = fmaf(ref, scale, log2_of(l)) * 0.693147180559945309f;       // log2(0) is -inf
        }
        return;
    }
    // Rows of one video: every lane has four neighbouring rows, the waves share the heads.
    __shared__ float2 s_norm[1024];
    __shared__ float4 s_sum[kJoinThreads];
    const int w = static_cast<int>(blockIdx.x) - a.join_blocks, b = w / a.weight_blocks, first = w - b * a.weight_blocks;
    const int fresh = a.k_new != nullptr, n_cache = rows_before(a, b), n = min(n_cache + fresh, a.S_cap);       // rows that have a place
    if (static_cast<int64_t>(first) * kWeightRows >= n) return;
    // Maximum and 1 / sum of every head (0 and 0 where no row counts): a.head_lanes neighbouring lanes to a head.  Apart, not as the rounded logarithm
    // of the sum, and the scores unscaled, as the sums were taken of them: a step's weights add up to 1 (fp32, 20000 rows with scores around
    // 700, one head: 2.7e-5 off through the logarithm, 9e-8 so).
    for (int h0 = 0; h0 < a.Hq; h0 += kJoinThreads / a.head_lanes) {
        const int h = min(h0 + static_cast<int>(threadIdx.x) / a.head_lanes, a.Hq - 1), part = threadIdx.x % a.head_lanes;
        const HeadParts parts = parts_of(a, b, h);
        float m = -INFINITY, l = 0.f;
#pragma unroll 8
        for (int p = part; p < (parts.n > 1 ? parts.n : 0); p += a.head_lanes) {
            const float2 v = ml[parts.slot(p)];
            add_sum(m, l, v.x, v.y, scale);
        }
        for (int off = a.head_lanes / 2; off; off >>= 1) add_sum(m, l, __shfl_xor(m, off, 64), __shfl_xor(l, off, 64), scale);
        const float2 norm = parts.n == 1 ? a.norm[static_cast<int64_t>(b) * a.Hq + h] : l == 0.f ? make_float2(0.f, 0.f) : make_float2(m, 1.f / l);
        if (part == 0) s_norm[h] = norm;
    }
    __syncthreads();
    const float inv = 1.f / static_cast<float>(a.Hq);
    for (int64_t j0 = static_cast<int64_t>(first) * kWeightRows; j0 < n; j0 += static_cast<int64_t>(a.weight_blocks) * kWeightRows) {
        const int64_t j = j0 + 4 * lane;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j < n) {
            const float* p = a.logits + static_cast<int64_t>(b) * a.Hq * a.logit_stride + j;
#pragma unroll 8
            for (int h = wave; h < a.Hq; h += kJoinThreads / 64) {
                const float4 x = *reinterpret_cast<const float4*>(p + h * a.logit_stride);
                const float2 z = s_norm[h];
                sum.x = fmaf(exp2_from(x.x, z.x, scale), z.y, sum.x); sum.y = fmaf(exp2_from(x.y, z.x, scale), z.y, sum.y);
                sum.z = fmaf(exp2_from(x.z, z.x, scale), z.y, sum.z); sum.w = fmaf(exp2_from(x.w, z.x, scale), z.y, sum.w);
            }
        }
        s_sum[threadIdx.x] = sum;
        __syncthreads();
        const int64_t mine = j0 + threadIdx.x;
        if (mine < n) {
            float total = 0.f;
#pragma unroll
            for (int k = 0; k < kJoinThreads / 64; ++k) total += reinterpret_cast<const float*>(s_sum + 64 * k)[threadIdx.x];
            float* out = a.weight + static_cast<int64_t>(b) * a.weight_stride + mine;
            *out = (mine < n_cache ? *out : 0.f) + total * inv;
        }
        __syncthreads();
    }
}

// Caches of more than this many bytes are read with the streaming hint: 375 MB (4 x 4571 rows, 40 heads of 128) 91 us without, 81 with; 606 MB
// 109 and 98; a tenth of them, that the memory-side cache still holds from the call before, 16.5 and 18.1 (67 MB).  Row by row (8 x 36990 rows in pages of 7 / 8 / 1)
// 116 / 112 / 123 without, 112 / 110 / 124 with.
constexpr int64_t kStreamBytes = 128 << 20;

template <typename T, int DH>
static int launch_attend(const DecodeArgs& a, const AttendPlan& plan, hipStream_t st) {
    const int64_t bytes = static_cast<int64_t>(a.B) * a.Hkv * a.S_cap * DH * static_cast<int64_t>(sizeof(T)) * 2;
    const unsigned groups = static_cast<unsigned>(plan.grid);
    const bool stream = bytes > kStreamBytes;
    if (plan.whole) {
        launch_short_attention(a, sizeof(T) == 2 ? METOK_BF16 : METOK_F32, DH, static_cast<unsigned>(plan.pairs), st);
        return check_launch("decode attention");
    }
    if (plan.wide) launch_wide_attention(a, sizeof(T) == 2 ? METOK_BF16 : METOK_F32, DH, stream, groups, st);
    else if (!a.table) stream ? launch_attention<T, DH, kDense, true, 1>(a, groups, st) : launch_attention<T, DH, kDense, false, 1>(a, groups, st);
    else if (a.page_size % 16 != 0) stream ? launch_attention<T, DH, kRows, true, 1>(a, groups, st) : launch_attention<T, DH, kRows, false, 1>(a, groups, st);
    else stream ? launch_attention<T, DH, kBlocks, true, 1>(a, groups, st) : launch_attention<T, DH, kBlocks, false, 1>(a, groups, st);
    return check_launch("decode attention");
}
static int launch_decode(const DecodeArgs& a, const AttendPlan& plan, int dtype, int dh, hipStream_t st) {
    if (dtype == METOK_BF16) {
        if (dh == 32) return launch_attend<bf16_t, 32>(a, plan, st);
        if (dh == 64) return launch_attend<bf16_t, 64>(a, plan, st);
        if (dh == 128) return launch_attend<bf16_t, 128>(a, plan, st);
        return launch_attend<bf16_t, 256>(a, plan, st);
    }
    if (dh == 32) return launch_attend<float, 32>(a, plan, st);
    if (dh == 64) return launch_attend<float, 64>(a, plan, st);
    return launch_attend<float, 128>(a, plan, st);
}

template <typename T, int DH>
static int launch_join(DecodeArgs& a, const AttendPlan& plan, hipStream_t st) {
    const int64_t units = plan.joined ? static_cast<int64_t>(a.B) * a.Hq : 0;
    // few heads have many parts each: their elements over several workgroups
    a.join_lanes = units * (DH / 4 / 8) <= kJoinSpread ? 8 : DH / 4;
    a.join_blocks = static_cast<int>(units * (DH / 4 / a.join_lanes));
    const int64_t blocks = a.join_blocks + (a.weight ? static_cast<int64_t>(a.B) * a.weight_blocks : 0);
    if (blocks == 0) return METOK_OK;
    a.head_lanes = 64;
    while (a.head_lanes > 1 && a.Hq * a.head_lanes > kJoinThreads) a.head_lanes /= 2;
    hipLaunchKernelGGL((decode_join_kernel<T, DH>), dim3(static_cast<unsigned>(blocks)), dim3(kJoinThreads), 0, st, a);
    return check_launch("decode join");
}

const char* bad_attend_heads(int B, int Hq, int Hkv, int dh, int dtype) {
    if (dtype != METOK_F32 && dtype != METOK_BF16) return "unknown dtype";
    if (B < 1 || B > METOK_MAX_DECODE_BATCH) return "B must be in [1, METOK_MAX_DECODE_BATCH]";
    if (Hkv < 1 || Hq < 1 || Hq > 1024 || Hq % Hkv != 0) return "Hq must be a multiple of Hkv and at most 1024";
    if (dh != 32 && dh != 64 && dh != 128 && !(dh == 256 && dtype == METOK_BF16)) return "dh must be 32, 64, 128 or (bf16) 256";
    return nullptr;
}
// The shapes that the calls and the workspace query take, NULL or the reason why not.
static const char* bad_shape(int B, int Hq, int Hkv, int64_t S_cap, int dh, int dtype) {
    if (const char* why = bad_attend_heads(B, Hq, Hkv, dh, dtype)) return why;
    if (S_cap < 1 || S_cap >= INT32_MAX - 64) return "the capacity must be in [1, 2^31 - 64)";
    const int64_t pairs = static_cast<int64_t>(B) * Hkv * ((Hq / Hkv + kAttendRows - 1) / kAttendRows);      // at most
    if (pairs * (S_cap / 16 + 4) > INT32_MAX) return "too many rows";
    return nullptr;
}

int attend_call(const AttendCall& c, const AttendPlan& plan, int (*launch)(const DecodeArgs& a, const AttendPlan& plan, int dtype, int dh, hipStream_t st)) {
    const auto& [q, B, Hq, Hkv, dh, dtype, k, v, S_cap, cache_bytes, table, n_pages, page_size, pages_per_seq, len, k_new, v_new, scale, logit_cap,
                 out, lse, weight, weight_stride, workspace, workspace_bytes, stream] = c;
    if (!q || !k || !v || !len || !out) return fail(METOK_ERR_INVALID_ARG, "q, the caches, len and out must not be NULL");
    if ((k_new == nullptr) != (v_new == nullptr)) return fail(METOK_ERR_INVALID_ARG, "k_new and v_new go together");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(out))
        return fail(METOK_ERR_INVALID_ARG, "q, the caches, k_new, v_new and out must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(len) | reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(weight)) & 3u)
        return fail(METOK_ERR_INVALID_ARG, "len, lse and weight must be 4-byte aligned");
    // (in fp32 a smaller one could become 0: no cap, or 0 times -inf)
    if (!(scale >= 1e-30 && scale < 1e30)) return fail(METOK_ERR_INVALID_ARG, "scale must be positive and finite, in [1e-30, 1e30)");
    if (logit_cap != 0.0 && !(logit_cap >= 1e-30 && logit_cap < 1e30))
        return fail(METOK_ERR_INVALID_ARG, "logit_cap must be 0 (none) or positive and finite, in [1e-30, 1e30)");
    if (logit_cap != 0.0 && !(scale / logit_cap >= 1e-30 && scale / logit_cap < 1e30))
        return fail(METOK_ERR_INVALID_ARG, "scale / logit_cap must be in [1e-30, 1e30)");
    if (weight && weight_stride < S_cap) return fail(METOK_ERR_INVALID_ARG, "weight_stride must be at least the capacity");
    const size_t esize = dtype_size(dtype), head = static_cast<size_t>(dh) * esize;
    if (plan.bytes && (!workspace || workspace_bytes < plan.bytes || !aligned16(workspace)))
        return fail(METOK_ERR_WORKSPACE, "workspace of %zu bytes needed (16-byte aligned), %zu given", plan.bytes, workspace_bytes);
    const Span spans[] = {
        {"out", out, B * Hq * head}, {"lse", lse, static_cast<size_t>(B) * Hq * 4},
        {"weight", weight, weight ? (static_cast<size_t>(B - 1) * weight_stride + S_cap) * 4 : 0}, {"workspace", workspace, plan.bytes},
        {"the K cache", k, cache_bytes}, {"the V cache", v, cache_bytes},
        {"q", q, B * Hq * head}, {"k_new", k_new, B * Hkv * head}, {"v_new", v_new, B * Hkv * head},
        {"len", len, static_cast<size_t>(B) * 4}, {"page_table", table, static_cast<size_t>(B) * pages_per_seq * 4}};
    constexpr int n_written = 6, k_span = 4, n_spans = sizeof(spans) / sizeof(spans[0]);        // K and V are only read where no row is appended
    for (int i = 0; i < n_written; ++i)
        for (int j = i + 1; j < n_spans; ++j)
            if (overlap(spans[i], spans[j]) && !(i == k_span && j == k_span + 1 && !k_new)) return fail(METOK_ERR_INVALID_ARG, "%s overlaps %s", spans[i].name, spans[j].name);

    DecodeArgs a{};
    a.q = static_cast<const char*>(q); a.k = static_cast<char*>(k); a.v = static_cast<char*>(v);
    a.k_new = static_cast<const char*>(k_new); a.v_new = static_cast<const char*>(v_new);
    a.len = len; a.table = table; a.out = static_cast<char*>(out); a.lse = lse; a.weight = weight;
    char* ws = static_cast<char*>(workspace);
    a.pair_workers = plan.joined || weight ? reinterpret_cast<int2*>(ws + plan.pair_workers) : nullptr;
    a.part_ml = reinterpret_cast<float*>(ws + plan.part_ml); a.part_o = reinterpret_cast<float*>(ws + plan.part_o);
    a.norm = reinterpret_cast<float2*>(ws + plan.lse2); a.logits = reinterpret_cast<float*>(ws + plan.logits);
    a.teams = plan.teams;
    a.weight_stride = weight_stride; a.logit_stride = plan.logit_stride;
    a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.group = Hq / Hkv; a.row_blocks = plan.row_blocks; a.rows = plan.rows; a.block_rows = plan.block_rows;
    a.S_cap = static_cast<int>(S_cap); a.page_size = page_size; a.pages_per_seq = pages_per_seq; a.n_pages = static_cast<int>(n_pages);
    int bits = 0;                // 2^bits >= page_size: ceil(2^(31 + bits) / page_size) is below 2^32 and off by less than 2^bits / page_size
    while ((static_cast<int64_t>(1) << bits) < page_size) ++bits;
    a.page_mul = static_cast<uint32_t>(((static_cast<uint64_t>(1) << (31 + bits)) + page_size - 1) / page_size);
    a.page_shift = 31 + bits;
    constexpr double log2e = 1.4426950408889634074;
    a.scale = static_cast<float>(logit_cap > 0.0 ? scale / logit_cap : scale * log2e);
    a.cap = static_cast<float>(logit_cap * log2e);
    // every workgroup of the weights sums up the heads' shares for itself: enough of them for the chip, not more
    const int64_t most = (S_cap + kWeightRows - 1) / kWeightRows, enough = (1024 + B - 1) / B;
    a.weight_blocks = static_cast<int>(most < enough ? most : enough);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int rc = launch(a, plan, dtype, dh, st)) return rc;
    if (dtype == METOK_BF16) {
        if (dh == 32) return launch_join<bf16_t, 32>(a, plan, st);
        if (dh == 64) return launch_join<bf16_t, 64>(a, plan, st);
        if (dh == 128) return launch_join<bf16_t, 128>(a, plan, st);
        return launch_join<bf16_t, 256>(a, plan, st);
    }
    if (dh == 32) return launch_join<float, 32>(a, plan, st);
    if (dh == 64) return launch_join<float, 64>(a, plan, st);
    return launch_join<float, 128>(a, plan, st);
}

}  // namespace metok

using namespace metok;

extern "C" size_t metok_decode_attention_workspace_bytes(int B, int Hq, int Hkv, int64_t S_cap, int dh, int dtype, int with_weight) {
    if (bad_shape(B, Hq, Hkv, S_cap, dh, dtype)) return 0;
    return plan_attend(B, Hq, Hkv, S_cap, dh, static_cast<int>(dtype_size(dtype)), with_weight != 0).bytes;
}

extern "C" int metok_decode_attention(const void* q, int B, int Hq, int Hkv, int dh, int dtype,
                                      void* k_cache, void* v_cache, int64_t S_cap, const int32_t* len,
                                      const void* k_new, const void* v_new, double scale, double logit_cap,
                                      void* out, float* lse, float* weight, int64_t weight_stride,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    if (const char* why = bad_shape(B, Hq, Hkv, S_cap, dh, dtype)) return fail(METOK_ERR_INVALID_ARG, "%s", why);
    const size_t bytes = static_cast<size_t>(B) * Hkv * S_cap * dh * dtype_size(dtype);
    return attend_call({q, B, Hq, Hkv, dh, dtype, k_cache, v_cache, S_cap, bytes, nullptr, 0, 1, 0, len, k_new, v_new, scale, logit_cap,
                        out, lse, weight, weight_stride, workspace, workspace_bytes, stream},
                       plan_attend(B, Hq, Hkv, S_cap, dh, static_cast<int>(dtype_size(dtype)), weight != nullptr), &launch_decode);
}

extern "C" int metok_decode_attention_paged(const void* q, int B, int Hq, int Hkv, int dh, int dtype,
                                            void* k_pool, void* v_pool, int64_t n_pages_pool, int page_size,
                                            const int32_t* page_table, int pages_per_seq, const int32_t* len,
                                            const void* k_new, const void* v_new, double scale, double logit_cap,
                                            void* out, float* lse, float* weight, int64_t weight_stride,
                                            void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    if (!page_table || (reinterpret_cast<uintptr_t>(page_table) & 3u)) return fail(METOK_ERR_INVALID_ARG, "page_table NULL or misaligned");
    if (page_size < 1 || pages_per_seq < 1 || n_pages_pool < 1) return fail(METOK_ERR_INVALID_ARG, "page_size, pages_per_seq and n_pages_pool must be positive");
    const int64_t S_cap = static_cast<int64_t>(pages_per_seq) * page_size;
    if (const char* why = bad_shape(B, Hq, Hkv, S_cap, dh, dtype)) return fail(METOK_ERR_INVALID_ARG, "%s", why);
    if (n_pages_pool > INT32_MAX / page_size / Hkv) return fail(METOK_ERR_UNSUPPORTED, "n_pages_pool * Hkv * page_size must be below 2^31");
    const size_t bytes = static_cast<size_t>(n_pages_pool) * Hkv * page_size * dh * dtype_size(dtype);
    return attend_call({q, B, Hq, Hkv, dh, dtype, k_pool, v_pool, S_cap, bytes, page_table, n_pages_pool, page_size, pages_per_seq, len, k_new, v_new, scale, logit_cap,
                        out, lse, weight, weight_stride, workspace, workspace_bytes, stream},
                       plan_attend(B, Hq, Hkv, S_cap, dh, static_cast<int>(dtype_size(dtype)), weight != nullptr), &launch_decode);
}
