// Queries, keys and values of new tokens on their way from the projections to the attention: norm of every query and key head, rotation by the token's
// position (one to four axes: time, height and width for the tokens of a video), queries laid out head by head, keys and values put into the
// dense or paged cache.
//
// One pass: (Hq + 2 Hkv) dh elements of a token are read and as many written.  HBM bounds a prompt, the launch a step.
#include "common.h"
#include "metok_qkv.h"

namespace metok {

constexpr int kRotateThreads = 256, kRotateWaves = kRotateThreads / 64;
constexpr int kLaneElems = 16;                             // elements of a head that a lane has
constexpr int kMaxHead = 256;
// Waves that a call is spread over, at most: where it has fewer (token, head) rows, a wave takes one head of its tokens, and the cosines and
// sines are computed by each of them.
constexpr int kRotateSpread = 8192;

struct RotateArgs {
    const char *q, *k, *v;
    char *q_out, *k_to, *v_to;
    const char *q_weight, *k_weight;
    const int32_t *pos, *count, *start, *table;
    const float* inv_freq;
    int64_t q_stride, k_stride, v_stride;                  // bytes between tokens
    int64_t n, tokens;                                     // of a video, of all
    int B, Hq, Hkv, S_cap, n_axes, rot, per_wave;          // per_wave: heads that a wave takes
    int page_size, pages_per_seq, n_pages;
    float eps;
    uint64_t axis[kMaxHead / kLaneElems];                  // a byte per pair
};

// Eight neighbouring elements.
template <typename T> struct Chunk8;
template <> struct Chunk8<bf16_t> {
    typedef uint4 type;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
        x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
        x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
        return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    }
};
template <> struct Chunk8<float> {
    struct type { float4 a, b; };
    static __device__ __forceinline__ void unpack(const type& v, float (&x)[8]) {
        x[0] = v.a.x; x[1] = v.a.y; x[2] = v.a.z; x[3] = v.a.w; x[4] = v.b.x; x[5] = v.b.y; x[6] = v.b.z; x[7] = v.b.w;
    }
    static __device__ __forceinline__ type pack(const float (&x)[8]) {
        return {make_float4(x[0], x[1], x[2], x[3]), make_float4(x[4], x[5], x[6], x[7])};
    }
};

// Cosine and sine of pos * freq.  In revolutions, in 64 bits, of which the whole ones are taken off: an fp32 product is off by 2^-24 of itself, 0.006
// radians at a position of 100000.
__device__ __forceinline__ void turn_of(int pos, float freq, float& cos, float& sin) {
    constexpr double inv_two_pi = 0.15915494309189533577;
    const double x = static_cast<double>(pos) * static_cast<double>(freq) * inv_two_pi;
    sincospif(2.f * static_cast<float>(x - rint(x)), &sin, &cos);
}

// A lane has 16 elements of a head of a token, as two runs of 8: rotated halves p .. p + 7 and rot / 2 + p .. of 8 pairs (16 neighbouring elements where the
// pairs are adjacent or not rotated).  It keeps its token and its pairs, and with them the cosines and sines, through the heads that the wave takes.
template <typename T, int DH, bool ADJACENT>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(const RotateArgs a) {
    constexpr int LANES = DH / kLaneElems, TOKENS = 64 / LANES, ES = sizeof(T);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), x = lane % LANES;
    const int64_t token = (static_cast<int64_t>(blockIdx.x) * kRotateWaves + wave) * TOKENS + lane / LANES;
    const int64_t at = min(token, a.tokens - 1);
    const int b = static_cast<int>(static_cast<uint32_t>(at) / static_cast<uint32_t>(a.n)), i = static_cast<int>(at - b * a.n);
    const bool here = token < a.tokens && (!a.count || i < a.count[b]);
    const int heads = a.Hq + 2 * a.Hkv, h0 = blockIdx.y * a.per_wave, h1 = min(h0 + a.per_wave, heads);
    if (!__any(here)) return;

    const bool turned = x * kLaneElems < a.rot;
    const int e0 = ADJACENT || !turned ? x * kLaneElems : x * 8, e1 = ADJACENT || !turned ? e0 + 8 : a.rot / 2 + x * 8;
    float cos[8], sin[8];
    if (turned && h0 < a.Hq + a.Hkv) {
        int pos[METOK_MAX_POSITION_AXES];
#pragma unroll
        for (int d = 0; d < METOK_MAX_POSITION_AXES; ++d) pos[d] = d < a.n_axes ? a.pos[d * a.tokens + at] : 0;
        const uint64_t axis = a.axis[x];
        const float4 f0 = *reinterpret_cast<const float4*>(a.inv_freq + 8 * x), f1 = *reinterpret_cast<const float4*>(a.inv_freq + 8 * x + 4);
        const float freq[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const int d = static_cast<int>(axis >> (8 * p)) & 3;
            turn_of(d < 2 ? (d == 0 ? pos[0] : pos[1]) : (d == 2 ? pos[2] : pos[3]), freq[p], cos[p], sin[p]);
        }
    } else {
#pragma unroll
        for (int p = 0; p < 8; ++p) { cos[p] = 1.f; sin[p] = 0.f; }
    }

    // where the token's row is in the cache, before the head
    int64_t row = -1;
    int64_t head_rows = a.S_cap;
    {
        const int64_t j = static_cast<int64_t>(i) + (a.start ? max(a.start[b], 0) : 0);
        if (here && j < a.S_cap) {
            if (!a.table) row = static_cast<int64_t>(b) * a.Hkv * a.S_cap + j;
            else {
                const int p = static_cast<int>(j) / a.page_size, page = a.table[static_cast<int64_t>(b) * a.pages_per_seq + p];
                if (page >= 0 && page < a.n_pages) row = static_cast<int64_t>(page) * a.Hkv * a.page_size + (j - static_cast<int64_t>(p) * a.page_size);
            }
        }
        if (a.table) head_rows = a.page_size;
    }

    typedef typename Chunk8<T>::type chunk_t;
    auto source = [&](int h) {
        if (h < a.Hq) return a.q + at * a.q_stride + static_cast<int64_t>(h) * DH * ES;
        if (h < a.Hq + a.Hkv) return a.k + at * a.k_stride + static_cast<int64_t>(h - a.Hq) * DH * ES;
        return a.v + at * a.v_stride + static_cast<int64_t>(h - a.Hq - a.Hkv) * DH * ES;
    };
    float g0[8], g1[8];                                    // the norm's weights
    chunk_t c0{}, c1{};
    if (here) {
        const char* p = source(h0);
        c0 = *reinterpret_cast<const chunk_t*>(p + e0 * ES);
        c1 = *reinterpret_cast<const chunk_t*>(p + e1 * ES);
    }
    for (int h = h0; h < h1; ++h) {
        chunk_t y0 = c0, y1 = c1;
        if (here && h + 1 < h1) {                          // the next head is on its way meanwhile
            const char* p = source(h + 1);
            c0 = *reinterpret_cast<const chunk_t*>(p + e0 * ES);
            c1 = *reinterpret_cast<const chunk_t*>(p + e1 * ES);
        }
        char* to;
        if (h < a.Hq) to = a.q_out + ((static_cast<int64_t>(b) * a.Hq + h) * a.n + i) * DH * ES;
        else {
            const bool value = h >= a.Hq + a.Hkv;
            to = (value ? a.v_to : a.k_to) + (row + (h - a.Hq - (value ? a.Hkv : 0)) * head_rows) * DH * ES;
        }
        if (h < a.Hq + a.Hkv) {
            float u[8], w[8];
            Chunk8<T>::unpack(y0, u);
            Chunk8<T>::unpack(y1, w);
            if (a.q_weight) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(u[e], u[e], fmaf(w[e], w[e], sum));
#pragma unroll
                for (int off = 1; off < LANES; off <<= 1) sum += __shfl_xor(sum, off, 64);
                const float mean = fmaf(sum, 1.f / DH, a.eps), inv = mean > 0.f ? 1.f / sqrtf(mean) : 0.f;
                if (h == h0 || h == a.Hq) {
                    const char* weight = h < a.Hq ? a.q_weight : a.k_weight;
                    Chunk8<T>::unpack(*reinterpret_cast<const chunk_t*>(weight + e0 * ES), g0);
                    Chunk8<T>::unpack(*reinterpret_cast<const chunk_t*>(weight + e1 * ES), g1);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) { u[e] = u[e] * inv * g0[e]; w[e] = w[e] * inv * g1[e]; }
            }
            float s[8], t[8];
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                if constexpr (ADJACENT) {                  // pairs 0 .. 3 in the first run, 4 .. 7 in the second
                    float(&z)[8] = p < 4 ? u : w;
                    float(&o)[8] = p < 4 ? s : t;
                    const int e = 2 * (p & 3);
                    o[e] = z[e] * cos[p] - z[e + 1] * sin[p];
                    o[e + 1] = z[e + 1] * cos[p] + z[e] * sin[p];
                } else {
                    s[p] = u[p] * cos[p] - w[p] * sin[p];
                    t[p] = w[p] * cos[p] + u[p] * sin[p];
                }
            }
            y0 = Chunk8<T>::pack(s);
            y1 = Chunk8<T>::pack(t);
        }
        if (here && (h < a.Hq || row >= 0)) {
            *reinterpret_cast<chunk_t*>(to + e0 * ES) = y0;
            *reinterpret_cast<chunk_t*>(to + e1 * ES) = y1;
        }
    }
}

template <typename T, int DH> static int launch_rotate(RotateArgs& a, bool adjacent, hipStream_t st) {
    constexpr int per_group = kRotateWaves * 64 / (DH / kLaneElems);
    const int64_t groups = (a.tokens + per_group - 1) / per_group, heads = a.Hq + 2 * a.Hkv;
    const int64_t rows = groups * kRotateWaves * heads, most = (rows + kRotateSpread - 1) / kRotateSpread;
    const int64_t turns = (heads + most - 1) / most;       // alike, so that no wave has much less than the others
    a.per_wave = static_cast<int>((heads + turns - 1) / turns);
    const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>((heads + a.per_wave - 1) / a.per_wave));
    if (adjacent) hipLaunchKernelGGL((rotate_kernel<T, DH, true>), grid, dim3(kRotateThreads), 0, st, a);
    else hipLaunchKernelGGL((rotate_kernel<T, DH, false>), grid, dim3(kRotateThreads), 0, st, a);
    return check_launch("rotate");
}

// Tokens of a call at most: a grid has fewer than 2^32 threads.
constexpr int64_t kMostTokens = 1 << 27;

static int rotate_impl(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride, int B, int64_t n, int Hq, int Hkv, int dh, int dtype,
                       const int32_t* count, const void* q_weight, const void* k_weight, double eps, const int32_t* pos, int n_axes, const float* inv_freq,
                       const uint8_t* pair_axis, int rot, int pairs, void* q_out, void* k_to, void* v_to, int64_t S_cap, int64_t slabs, int64_t slab_rows,
                       const int32_t* table, int64_t n_pages, int page_size, int pages_per_seq, const int32_t* start, void* stream) {
    if (dtype != METOK_F32 && dtype != METOK_BF16) return fail(METOK_ERR_INVALID_ARG, "unknown dtype");
    if (dh != 32 && dh != 64 && dh != 128 && !(dh == 256 && dtype == METOK_BF16)) return fail(METOK_ERR_INVALID_ARG, "dh must be 32, 64, 128 or (bf16) 256");
    if (B < 1 || B > METOK_MAX_DECODE_BATCH) return fail(METOK_ERR_INVALID_ARG, "B must be in [1, METOK_MAX_DECODE_BATCH]");
    if (n < 1 || n > kMostTokens / B) return fail(METOK_ERR_INVALID_ARG, "n must be positive and B * n at most 2^27");
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
    if (rot < kLaneElems || rot > dh || rot % kLaneElems != 0) return fail(METOK_ERR_INVALID_ARG, "rot must be a positive multiple of 16 and at most dh");
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
        a.axis[p / 8] |= static_cast<uint64_t>(axis) << (8 * (p % 8));
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
