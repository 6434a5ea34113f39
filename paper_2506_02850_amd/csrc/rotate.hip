// Queries, keys and values of new tokens on their way from the projections to the attention: norm of every query and key head, rotation by the token's
// position (one to four axes: time, height and width for the tokens of a video), queries laid out head by head, keys and values put into the
// dense or paged cache.
//
// One pass: (Hq + 2 Hkv) dh elements of a token are read and as many written.  HBM bounds a prompt (18560 tokens of 36 heads of 128 in bf16, 342 MB: 64 us,
// 5.3 TB/s; a copy in the order of the addresses 53), the launch and its latencies a step.
#include "common.h"
#include "metok_qkv.h"

namespace metok {

constexpr int kRotateThreads = 256;
constexpr int kRotUnit = 16, kMaxPairs = 128;              // rot is a multiple of; pairs of a head at most
constexpr int kAtOnce = 4;                                 // heads whose loads are on their way together
// Heads that a workgroup takes where there are kRotateSpread workgroups of one head or more: enough for the cosines and sines to be a small part of its work, few enough
// for the writes to stay in order (18560 tokens, 36 heads of 128, bf16: 4 heads 66.5 us, 8 64.4, 12 64.2, 20 73; 11000 of 18 of 64, fp32: 4 20.6, 8 22.1, 12 21.6;
// the prompt without norms and products, the kernel's loads, angles and stores alone, 63.4).  A step of 64 tokens, 36 heads: 5.1 us, which is launch, positions, sine and product one behind the other.
constexpr int rotate_heads(int esize) { return 16 / esize; }
constexpr int kRotateSpread = 4096;
// Rows of more bytes than this are read, or written, with the streaming hint: the prompt above 64 us with both, 68 without that on the reads; the fp32 one, whose rows the
// memory-side cache still holds, 24 with it on the writes, 31 without, 33 on both.
constexpr int64_t kStreamIn = 128 << 20, kStreamOut = 32 << 20;

struct RotateArgs {
    const char *q, *k, *v;
    char *q_out, *k_to, *v_to;
    const char *q_weight, *k_weight;
    const int32_t *pos, *count, *start, *table;
    const float* inv_freq;
    int64_t q_stride, k_stride, v_stride;                  // bytes between tokens
    int64_t n, tokens;                                     // of a video, of all
    int B, Hq, Hkv, S_cap, n_axes, rot, per_group;         // per_group: heads that a workgroup takes
    int page_size, pages_per_seq, n_pages;
    float eps;
    uint8_t axis[kMaxPairs];
};

// 16 bytes of neighbouring elements, a run.
template <typename T> struct Run;
template <> struct Run<bf16_t> {
    static constexpr int kElems = 8;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
        x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
        x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
        return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    }
};
template <> struct Run<float> {
    static constexpr int kElems = 4;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

// Sum over LANES neighbouring lanes (4 .. 32); each receives it.
template <int CTRL> __device__ __forceinline__ float dpp_sum(float v) {
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false));
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
    v = dpp_sum<0xb1>(v);                                  // the neighbour
    v = dpp_sum<0x4e>(v);                                  // two further, within four
    if (LANES >= 8) v = dpp_sum<0x141>(v);                 // mirrored within eight: the other four
    if (LANES >= 16) v = dpp_sum<0x140>(v);                // mirrored within sixteen
    return LANES == 32 ? swap16_add(v, v) : v;
}

// Cosine and sine of pos * freq.  In revolutions, in 64 bits, of which the whole ones are taken off: an fp32 product is off by 2^-24 of itself, 0.006
// radians at a position of 100000.
__device__ __forceinline__ void turn_of(int pos, float freq, float& cos, float& sin) {
    constexpr double inv_two_pi = 0.15915494309189533577;
    const double x = static_cast<double>(pos) * static_cast<double>(freq) * inv_two_pi;
    sincospif(2.f * static_cast<float>(x - rint(x)), &sin, &cos);
}

// A lane has a run of a head of a token, the lanes of a wave the rows of neighbouring tokens, and a workgroup so many tokens of a few heads.  Workgroups with
// neighbouring tokens follow each other, those of the next heads come behind all of them: what is written is written in the order of its addresses, 256
// bytes and more at a time, and it is the reads that jump (18560 tokens of 36 heads of 128 in bf16, by kernels that copy and do nothing else: 56 us so, 61 to 71 with the
// reads in order, 66 with a head's halves in two stores, 53 without any change of the order).
//
// The other half of a pair is with another lane.  With c, s the pair's cosine and sine, g and g' the weights of the lane's element x and of the other one x', and
// f = 1 / root mean square, the result is f (x (g c) +- x' (g' s)): two factors to an element, computed once for all heads of a kind.
template <typename T, int DH, bool ADJACENT, bool STREAM_IN, bool STREAM_OUT>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(const RotateArgs a) {
    constexpr int R = Run<T>::kElems, LANES = DH / R, TOKENS = kRotateThreads / LANES, ES = sizeof(T), PAIRS = DH / 2;
    const int x = threadIdx.x % LANES, mine = threadIdx.x / LANES;
    const int64_t token0 = static_cast<int64_t>(blockIdx.x) * TOKENS, at = min(token0 + mine, a.tokens - 1);
    const int b = static_cast<int>(static_cast<uint32_t>(at) / static_cast<uint32_t>(a.n)), i = static_cast<int>(at - static_cast<int64_t>(b) * a.n);
    const bool here = token0 + mine < a.tokens && (!a.count || i < a.count[b]);
    const int turned_heads = a.Hq + a.Hkv, heads = turned_heads + a.Hkv, h0 = blockIdx.y * a.per_group, h1 = min(h0 + a.per_group, heads);

    // the cosines and sines of the workgroup's tokens, pair by pair over its threads
    __shared__ float s_cos[TOKENS * PAIRS], s_sin[TOKENS * PAIRS];
    if (h0 < turned_heads) {
#pragma unroll
        for (int k = 0; k < TOKENS * PAIRS / kRotateThreads; ++k) {
            const int place = threadIdx.x + k * kRotateThreads, pair = place % PAIRS;
            const int64_t of = min(token0 + place / PAIRS, a.tokens - 1);
            if (pair < a.rot / 2) turn_of(a.pos[a.axis[pair] * a.tokens + of], a.inv_freq[pair], s_cos[place], s_sin[place]);
        }
    }
    __syncthreads();

    // where the token's row is in the cache, before the head
    int64_t row = -1;
    if (h1 > a.Hq) {
        const int64_t j = static_cast<int64_t>(i) + (a.start ? max(a.start[b], 0) : 0);
        if (here && j < a.S_cap) {
            if (!a.table) row = static_cast<int64_t>(b) * a.Hkv * a.S_cap + j;
            else {
                const int p = static_cast<int>(j) / a.page_size, page = a.table[static_cast<int64_t>(b) * a.pages_per_seq + p];
                if (page >= 0 && page < a.n_pages) row = static_cast<int64_t>(page) * a.Hkv * a.page_size + (j - static_cast<int64_t>(p) * a.page_size);
            }
        }
    }
    const int64_t head_rows = a.table ? a.page_size : a.S_cap;

    const int half = a.rot / (2 * R);                      // lanes of a half
    const bool turned = x * R < a.rot, first = ADJACENT || x < half;
    const int other = turned && !ADJACENT ? (first ? x + half : x - half) : x;
    const int other_lane = (threadIdx.x & 63) - x + other;
    float own[R], its[R];                                  // the two factors
    auto factors = [&](const char* weight) {
        float g[R], o[R];
#pragma unroll
        for (int e = 0; e < R; ++e) g[e] = o[e] = 1.f;
        if (weight) {
            Run<T>::unpack(*reinterpret_cast<const uint4*>(weight + x * R * ES), g);
            Run<T>::unpack(*reinterpret_cast<const uint4*>(weight + other * R * ES), o);
        }
#pragma unroll
        for (int e = 0; e < R; ++e) {
            const int pair = mine * PAIRS + (ADJACENT ? (x * R + e) / 2 : (first ? x : x - half) * R + e);
            const float c = turned ? s_cos[pair] : 1.f, s = turned ? s_sin[pair] : 0.f;
            own[e] = g[e] * c;
            its[e] = (ADJACENT ? (e & 1 ? o[e ^ 1] : -o[e ^ 1]) : (first ? -o[e] : o[e])) * s;
        }
    };

    auto source = [&](int h) {
        const char* p = h < a.Hq ? a.q + at * a.q_stride : h < turned_heads ? a.k + at * a.k_stride : a.v + at * a.v_stride;
        return p + (static_cast<int64_t>(h - (h < a.Hq ? 0 : h < turned_heads ? a.Hq : turned_heads)) * DH + x * R) * ES;
    };
    for (int h = h0; h < h1; h += kAtOnce) {
        uint4 in[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const uint4* p = reinterpret_cast<const uint4*>(source(min(h + k, h1 - 1)));
            in[k] = uint4{};
            if (here && h + k < h1) in[k] = STREAM_IN ? load_stream(p) : *p;
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int at_head = h + k;
            if (at_head >= h1) break;
            uint4 y = in[k];
            if (at_head == h0 || at_head == a.Hq) factors(at_head < a.Hq ? a.q_weight : a.k_weight);
            if (at_head < turned_heads) {
                float u[R], w[R];
                Run<T>::unpack(y, u);
                if constexpr (ADJACENT) {
#pragma unroll
                    for (int e = 0; e < R; ++e) w[e] = u[e ^ 1];
                } else {
                    const uint4 z = make_uint4(__shfl(y.x, other_lane, 64), __shfl(y.y, other_lane, 64), __shfl(y.z, other_lane, 64), __shfl(y.w, other_lane, 64));
                    Run<T>::unpack(z, w);
                }
                float f = 1.f;
                if (a.q_weight) {
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < R; ++e) sum = fmaf(u[e], u[e], sum);
                    const float mean = fmaf(lanes_sum<LANES>(sum), 1.f / DH, a.eps);
                    f = mean < 0x1p-126f ? 0.f : __builtin_amdgcn_rsqf(mean);
                }
                // behind the rotated elements no product: 0 times an infinity is none, and -0, unlike 0, changes no number that it is added to
#pragma unroll
                for (int e = 0; e < R; ++e) u[e] = fmaf(u[e], own[e], turned ? w[e] * its[e] : -0.f) * f;
                y = Run<T>::pack(u);
            }
            char* to;
            if (at_head < a.Hq) to = a.q_out + ((static_cast<int64_t>(b) * a.Hq + at_head) * a.n + i) * DH * ES;
            else to = (at_head < turned_heads ? a.k_to + (row + (at_head - a.Hq) * head_rows) * DH * ES : a.v_to + (row + (at_head - turned_heads) * head_rows) * DH * ES);
            if (here && (at_head < a.Hq || row >= 0)) {
                if (STREAM_OUT) store_stream(reinterpret_cast<uint4*>(to) + x, y);
                else reinterpret_cast<uint4*>(to)[x] = y;
            }
        }
    }
}

template <typename T, int DH> static int launch_rotate(RotateArgs& a, bool adjacent, hipStream_t st) {
    constexpr int tokens = kRotateThreads * Run<T>::kElems / DH;
    const int64_t groups = (a.tokens + tokens - 1) / tokens, heads = a.Hq + 2 * a.Hkv;
    a.per_group = groups * heads >= kRotateSpread ? rotate_heads(sizeof(T)) : 1;
    const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>((heads + a.per_group - 1) / a.per_group)), threads(kRotateThreads);
    const int64_t bytes = a.tokens * heads * DH * static_cast<int64_t>(sizeof(T));
    const bool in = bytes > kStreamIn, out = bytes > kStreamOut;
    if (adjacent) {
        if (in) hipLaunchKernelGGL((rotate_kernel<T, DH, true, true, true>), grid, threads, 0, st, a);
        else if (out) hipLaunchKernelGGL((rotate_kernel<T, DH, true, false, true>), grid, threads, 0, st, a);
        else hipLaunchKernelGGL((rotate_kernel<T, DH, true, false, false>), grid, threads, 0, st, a);
    } else {
        if (in) hipLaunchKernelGGL((rotate_kernel<T, DH, false, true, true>), grid, threads, 0, st, a);
        else if (out) hipLaunchKernelGGL((rotate_kernel<T, DH, false, false, true>), grid, threads, 0, st, a);
        else hipLaunchKernelGGL((rotate_kernel<T, DH, false, false, false>), grid, threads, 0, st, a);
    }
    return check_launch("rotate");
}

// Tokens of a call at most: a grid has fewer than 2^32 threads.
constexpr int64_t kMostTokens = 1 << 26;

static int rotate_impl(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride, int B, int64_t n, int Hq, int Hkv, int dh, int dtype,
                       const int32_t* count, const void* q_weight, const void* k_weight, double eps, const int32_t* pos, int n_axes, const float* inv_freq,
                       const uint8_t* pair_axis, int rot, int pairs, void* q_out, void* k_to, void* v_to, int64_t S_cap, int64_t slabs, int64_t slab_rows,
                       const int32_t* table, int64_t n_pages, int page_size, int pages_per_seq, const int32_t* start, void* stream) {
    if (dtype != METOK_F32 && dtype != METOK_BF16) return fail(METOK_ERR_INVALID_ARG, "unknown dtype");
    if (dh != 32 && dh != 64 && dh != 128 && !(dh == 256 && dtype == METOK_BF16)) return fail(METOK_ERR_INVALID_ARG, "dh must be 32, 64, 128 or (bf16) 256");
    if (B < 1 || B > METOK_MAX_DECODE_BATCH) return fail(METOK_ERR_INVALID_ARG, "B must be in [1, METOK_MAX_DECODE_BATCH]");
    if (n < 1 || n > kMostTokens / B) return fail(METOK_ERR_INVALID_ARG, "n must be positive and B * n at most 2^26");
    if (Hq < 1 || Hkv < 1 || Hq > 4096 || Hkv > 4096 || Hq + 2 * Hkv > 4096) return fail(METOK_ERR_INVALID_ARG, "Hq and Hkv must be positive, Hq + 2 Hkv at most 4096");
    if (S_cap < 1 || S_cap >= INT32_MAX - 64) return fail(METOK_ERR_INVALID_ARG, "the capacity must be in [1, 2^31 - 64)");
    if (!q || !k || !v || !pos || !inv_freq || !q_out || !k_to || !v_to) return fail(METOK_ERR_INVALID_ARG, "q, k, v, pos, inv_freq, q_out and the caches must not be NULL");
    if ((q_weight == nullptr) != (k_weight == nullptr)) return fail(METOK_ERR_INVALID_ARG, "q_weight and k_weight go together");
    for (const void* p : {q, k, v, q_weight, k_weight, static_cast<const void*>(inv_freq), static_cast<const void*>(q_out), static_cast<const void*>(k_to), static_cast<const void*>(v_to)})
        if (!aligned16(p)) return fail(METOK_ERR_INVALID_ARG, "q, k, v, the weights, inv_freq, q_out and the caches must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(count) | reinterpret_cast<uintptr_t>(start)) & 3u)
        return fail(METOK_ERR_INVALID_ARG, "pos, count and start must be 4-byte aligned");
    if (!(eps >= 0.0 && eps <= 1.0)) return fail(METOK_ERR_INVALID_ARG, "eps must be in [0, 1]");
    if (n_axes < 1 || n_axes > METOK_MAX_POSITION_AXES) return fail(METOK_ERR_INVALID_ARG, "n_axes must be in [1, METOK_MAX_POSITION_AXES]");
    if (rot < kRotUnit || rot > dh || rot % kRotUnit != 0) return fail(METOK_ERR_INVALID_ARG, "rot must be a positive multiple of 16 and at most dh");
    if (pairs != METOK_PAIRS_HALVES && pairs != METOK_PAIRS_ADJACENT) return fail(METOK_ERR_INVALID_ARG, "unknown pairs");
    const int64_t es = static_cast<int64_t>(dtype_size(dtype)), limit = static_cast<int64_t>(1) << 40;
    const struct { const char* name; int64_t stride, heads; } strides[] = {{"q_stride", q_stride, Hq}, {"k_stride", k_stride, Hkv}, {"v_stride", v_stride, Hkv}};
    for (const auto& x : strides)
        if (x.stride < x.heads * dh || x.stride * es % 16 != 0 || x.stride > limit / (static_cast<int64_t>(B) * n))
            return fail(METOK_ERR_INVALID_ARG, "%s must hold the heads' elements, be a multiple of 16 bytes, and B * n of them at most 2^40 elements", x.name);
    RotateArgs a{};
    for (int p = 0; p < rot / 2; ++p) {
        const int axis = pair_axis ? pair_axis[p] : 0;
        if (axis >= n_axes) return fail(METOK_ERR_INVALID_ARG, "pair_axis[%d] is not below n_axes", p);
        a.axis[p] = static_cast<uint8_t>(axis);
    }
    const int64_t tokens = static_cast<int64_t>(B) * n;
    auto rows = [&](int64_t stride, int heads) { return static_cast<size_t>(((tokens - 1) * stride + static_cast<int64_t>(heads) * dh) * es); };
    const size_t cache = static_cast<size_t>(slabs) * Hkv * slab_rows * dh * es, weight = static_cast<size_t>(dh) * es;
    const Span spans[] = {{"q_out", q_out, static_cast<size_t>(tokens) * Hq * dh * es}, {"the K cache", k_to, cache}, {"the V cache", v_to, cache},
                          {"q", q, rows(q_stride, Hq)}, {"k", k, rows(k_stride, Hkv)}, {"v", v, rows(v_stride, Hkv)},
                          {"count", count, static_cast<size_t>(B) * 4}, {"q_weight", q_weight, weight}, {"k_weight", k_weight, weight},
                          {"pos", pos, static_cast<size_t>(n_axes) * tokens * 4}, {"inv_freq", inv_freq, static_cast<size_t>(rot) * 2}, {"start", start, static_cast<size_t>(B) * 4},
                          {"page_table", table, static_cast<size_t>(B) * pages_per_seq * 4}};
    if (int rc = check_spans(spans, 3, sizeof(spans) / sizeof(spans[0]))) return rc;
    a.q = static_cast<const char*>(q); a.k = static_cast<const char*>(k); a.v = static_cast<const char*>(v);
    a.q_out = static_cast<char*>(q_out); a.k_to = static_cast<char*>(k_to); a.v_to = static_cast<char*>(v_to);
    a.q_weight = static_cast<const char*>(q_weight); a.k_weight = static_cast<const char*>(k_weight);
    a.pos = pos; a.count = count; a.start = start; a.table = table; a.inv_freq = inv_freq;
    a.q_stride = q_stride * es; a.k_stride = k_stride * es; a.v_stride = v_stride * es;
    a.n = n; a.tokens = tokens; a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.S_cap = static_cast<int>(S_cap); a.n_axes = n_axes; a.rot = rot;
    a.page_size = page_size; a.pages_per_seq = pages_per_seq; a.n_pages = static_cast<int>(n_pages); a.eps = static_cast<float>(eps);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool adjacent = pairs == METOK_PAIRS_ADJACENT;
    if (dtype == METOK_BF16) {
        if (dh == 32) return launch_rotate<bf16_t, 32>(a, adjacent, st);
        if (dh == 64) return launch_rotate<bf16_t, 64>(a, adjacent, st);
        if (dh == 128) return launch_rotate<bf16_t, 128>(a, adjacent, st);
        return launch_rotate<bf16_t, 256>(a, adjacent, st);
    }
    if (dh == 32) return launch_rotate<float, 32>(a, adjacent, st);
    if (dh == 64) return launch_rotate<float, 64>(a, adjacent, st);
    return launch_rotate<float, 128>(a, adjacent, st);
}

}  // namespace metok

using namespace metok;

extern "C" int metok_rotate_qk(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                               int B, int64_t n, int Hq, int Hkv, int dh, int dtype, const int32_t* count,
                               const void* q_weight, const void* k_weight, double eps,
                               const int32_t* pos, int n_axes, const float* inv_freq, const uint8_t* pair_axis, int rot, int pairs,
                               void* q_out, void* k_cache, void* v_cache, int64_t S_cap, const int32_t* start, void* stream) {
    clear_error();
    return rotate_impl(q, k, v, q_stride, k_stride, v_stride, B, n, Hq, Hkv, dh, dtype, count, q_weight, k_weight, eps, pos, n_axes, inv_freq, pair_axis, rot, pairs,
                       q_out, k_cache, v_cache, S_cap, B, S_cap, nullptr, 0, 1, 0, start, stream);
}

extern "C" int metok_rotate_qk_paged(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                     int B, int64_t n, int Hq, int Hkv, int dh, int dtype, const int32_t* count,
                                     const void* q_weight, const void* k_weight, double eps,
                                     const int32_t* pos, int n_axes, const float* inv_freq, const uint8_t* pair_axis, int rot, int pairs,
                                     void* q_out, void* k_pool, void* v_pool, int64_t n_pages_pool, int page_size,
                                     const int32_t* page_table, int pages_per_seq, const int32_t* start, void* stream) {
    clear_error();
    if (!page_table || (reinterpret_cast<uintptr_t>(page_table) & 3u)) return fail(METOK_ERR_INVALID_ARG, "page_table NULL or misaligned");
    if (page_size < 1 || pages_per_seq < 1 || n_pages_pool < 1) return fail(METOK_ERR_INVALID_ARG, "page_size, pages_per_seq and n_pages_pool must be positive");
    if (Hkv >= 1 && n_pages_pool > INT32_MAX / page_size / Hkv) return fail(METOK_ERR_UNSUPPORTED, "n_pages_pool * Hkv * page_size must be below 2^31");
    return rotate_impl(q, k, v, q_stride, k_stride, v_stride, B, n, Hq, Hkv, dh, dtype, count, q_weight, k_weight, eps, pos, n_axes, inv_freq, pair_axis, rot, pairs,
                       q_out, k_pool, v_pool, static_cast<int64_t>(pages_per_seq) * page_size, n_pages_pool, page_size, page_table, n_pages_pool, page_size, pages_per_seq,
                       start, stream);
}
