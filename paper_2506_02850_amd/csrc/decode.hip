// Attention of one new token per video over the dense or paged KV cache that stage 3 leaves (Sec. 3.3), with the token's own row
// appended and, if asked, the attention weight of every cached row accumulated (what metok_kv_evict ranks the rows by).
//
//   decode_attention_kernel  a workgroup's share of the rows of one (video, kv head, block of 16 query heads): scores, running
//                            maximum and sum of the softmax, weighted sum of the values, in one pass over K and V
//   decode_join_kernel       joins the shares of a (video, query head); and, with weights, turns the scores that the first kernel kept
//                            into probabilities and adds their mean over the heads to the rows' weights
//
// What bounds it is the stream of K and V: 4 Hq dh operations a row on 2 Hkv dh elements, 7 operations a byte with seven query
// heads to a kv head in bf16.  The query heads of a kv head are the columns of one MFMA, so a row is read once for all of them.
#include "common.h"
#include "decode_plan.h"
#include "metok_decode.h"

namespace metok {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;

struct DecodeArgs {
    const char* q;
    char* k;                     // cache [B, Hkv, S_cap, dh], or pool [n_pages, Hkv, page_size, dh]
    char* v;
    const char* k_new;           // [B, Hkv, dh] or NULL
    const char* v_new;
    const int32_t* len;          // [B]
    const int32_t* table;        // [B, pages_per_seq], NULL: dense
    char* out;
    float* lse;                  // [B, Hq] or NULL
    float* weight;               // [B, weight_stride] or NULL
    float* part_ml;              // [grid][rows][2]: maximum and sum of a share, log2 domain
    float* part_o;               // [grid][rows][dh]
    float* lse2;                 // [B, Hq]: log2 of the sum, where one workgroup had all rows
    float* logits;               // [B, Hq, logit_stride], log2 domain
    int64_t weight_stride, logit_stride;
    int B, Hq, Hkv, group, row_blocks, rows;
    int S_cap;                   // capacity
    int page_size, pages_per_seq, n_pages;
    uint32_t page_mul, page_shift;       // j / page_size = j * page_mul >> page_shift for 0 <= j < 2^31
    float scale;                 // without cap: of the logits in the log2 domain; with cap: scale / cap
    float cap;                   // cap in the log2 domain, 0: none
    int join_blocks, weight_blocks;      // of decode_join_kernel
};

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }

__device__ __forceinline__ int rows_before(const DecodeArgs& a, int b) {
    const int n = a.len[b];
    return n < 0 ? 0 : (n > a.S_cap ? a.S_cap : n);
}

// The rows of a video and its workgroups.
struct VideoShare { int b, n_cache, tiles, splits, first; };     // first: its first workgroup

// Goes through the videos, 64 a step, one to a lane.  WANT_VIDEO: the share of video `want`; else of the video that has workgroup
// `want`, b = -1 if there is none.  Uniform over the wave.
template <int TILE, bool WANT_VIDEO>
__device__ __forceinline__ VideoShare find_share(const DecodeArgs& a, int want) {
    const int lane = threadIdx.x & 63, fresh = a.k_new != nullptr, heads = a.Hkv * a.row_blocks;
    int n = 0, tiles = 0;
    int64_t total = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const bool in = b0 + lane < a.B;
        n = in ? rows_before(a, b0 + lane) : 0;
        tiles = in ? (n + fresh + TILE - 1) / TILE : 0;
        total += __builtin_amdgcn_readlane(wave_inclusive_scan(tiles), 63);
    }
    const int64_t per64 = attend_tiles_per_group(total * heads);
    const uint32_t per = per64 > 0x7fffffff ? 0x7fffffffu : static_cast<uint32_t>(per64);
    int first = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const bool in = b0 + lane < a.B;
        if (a.B > 64) {
            n = in ? rows_before(a, b0 + lane) : 0;
            tiles = in ? (n + fresh + TILE - 1) / TILE : 0;
        }
        int splits = in ? static_cast<int>((static_cast<uint32_t>(tiles) + per - 1) / per) : 0;
        if (in && splits < 1) splits = 1;
        const int groups = splits * heads;
        const int incl = wave_inclusive_scan(groups);
        const unsigned long long hit = __ballot(in && (WANT_VIDEO ? b0 + lane == want : first + incl > want));
        if (hit) {
            const int l = __ffsll(static_cast<long long>(hit)) - 1;
            return {b0 + __builtin_amdgcn_readfirstlane(l), __builtin_amdgcn_readlane(n, l), __builtin_amdgcn_readlane(tiles, l), __builtin_amdgcn_readlane(splits, l),
                    first + __builtin_amdgcn_readlane(incl - groups, l)};
        }
        first += __builtin_amdgcn_readlane(incl, 63);
    }
    return {-1, 0, 0, 0, 0};
}

// Largest of the four lanes r, r + 16, r + 32, r + 48; each receives it.
__device__ __forceinline__ float rows_max(float v) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// tanh to about 2 units of the last place: the odd series where 1 - exp would cancel (its first missing term is 9e-9 of the result
// at 0.25).
__device__ __forceinline__ float tanh_of(float x) {
    const float y = fabsf(x), x2 = x * x;
    const float e = exp2_of(y * -2.8853900817779268f);               // exp(-2 |x|)
    const float far = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), x);
    const float near = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 0.021869488536155203f, -0.053968253968253968f), 0.13333333333333333f), -0.33333333333333333f), 1.f);
    return y < 0.25f ? near : far;
}

// Read by scalar loads: written by nobody during the kernel.
typedef const __attribute__((address_space(4))) int32_t* scalar_ints;

#ifndef NTL
#define NTL 0
#endif
__device__ __forceinline__ u32x4_t load_piece(const char* p) {
    if (NTL) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
    return *reinterpret_cast<const u32x4_t*>(p);
}
template <int WORDS> __device__ __forceinline__ void load_words(uint32_t (&w)[WORDS], const char* p) {
    if constexpr (WORDS == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
    else if constexpr (WORDS == 2) { const uint2 x = *reinterpret_cast<const uint2*>(p); w[0] = x.x; w[1] = x.y; }
    else {
#pragma unroll
        for (int i = 0; i < WORDS; i += 4) {
            const u32x4_t x = load_piece(p + 4 * i);
            w[i] = x.x; w[i + 1] = x.y; w[i + 2] = x.z; w[i + 3] = x.w;
        }
    }
}

template <typename T, int DH> struct AttendShape {
    static constexpr int kRowBytes = DH * static_cast<int>(sizeof(T));
    static constexpr int kTile = attend_tile(sizeof(T), DH);
    static constexpr int kSub = kTile / 16;              // MFMA row blocks of a tile
    static constexpr int kPieces = kRowBytes / 64;       // 16-byte pieces of a K row that a lane holds (every fourth one)
    static constexpr int kKeys = kSub * 4;               // rows of V that a lane holds a part of
    static constexpr int kElems = DH / 16;               // elements of that part
    static constexpr int kWords = kElems * static_cast<int>(sizeof(T)) / 4;
};

// Rows of a cache as seen by a lane: >= 0 a row of the slab or pool, or one of these.
constexpr int kNoRow = -1, kNewRow = -2;
__device__ __forceinline__ const char* row_address(const char* base, const char* fresh, int row, int row_bytes) {
    const char* p = base + static_cast<uint64_t>(static_cast<uint32_t>(row < 0 ? 0 : row)) * static_cast<uint32_t>(row_bytes);
    return row == kNewRow ? fresh : p;
}

// A lane's place: r = lane % 16, c = lane / 16.  K Q^T is taken with the rows of K as rows of the product: the lane has query
// head r of the scores of rows 4 c .. 4 c + 3 of every 16.  That is already the operand layout of the second product, V^T P^T with
// the cache rows as contraction index, in the order 16 t + 4 c + i, so no value changes lanes between the two; a lane loads
// kElems neighbouring elements r * kElems ... of its kKeys rows of V, whole rows of 16 lanes, and picks the rows' elements together
// in registers.  The softmax state of a query head is one (maximum, sum) per lane, the sum over the lane's own rows only.
template <typename T, int DH, bool PAGED, bool WEIGHTS>
__global__ __launch_bounds__(kAttendThreads, 2) void decode_attention_kernel(const DecodeArgs a) {
    using S = AttendShape<T, DH>;
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int TILE = S::kTile, NT = S::kSub, KS = S::kPieces, NV = S::kKeys, E = S::kElems, VW = S::kWords, RB = S::kRowBytes;
    __shared__ float s_o[kAttendWaves][kAttendRows][DH + 4];
    __shared__ float s_ml[kAttendWaves][kAttendRows][2];

    const VideoShare sh = find_share<TILE, false>(a, blockIdx.x);
    if (sh.b < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
    const int b = sh.b, local = static_cast<int>(blockIdx.x) - sh.first;
    const int hr = __builtin_amdgcn_readfirstlane(local / sh.splits), split = local - hr * sh.splits;
    const int kvh = __builtin_amdgcn_readfirstlane(hr / a.row_blocks), rb = hr - kvh * a.row_blocks;
    const int t0 = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<int64_t>(sh.tiles) * split / sh.splits));
    const int t1 = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<int64_t>(sh.tiles) * (split + 1) / sh.splits));
    const bool fresh = a.k_new != nullptr;
    const int n_cache = sh.n_cache;
    const int64_t slab = static_cast<int64_t>(b) * a.Hkv + kvh;
    const char* k_base = PAGED ? a.k : a.k + slab * a.S_cap * RB;
    const char* v_base = PAGED ? a.v : a.v + slab * a.S_cap * RB;
    const char* k_fresh = fresh ? a.k_new + slab * RB : nullptr;
    const char* v_fresh = fresh ? a.v_new + slab * RB : nullptr;
    const int32_t* table = PAGED ? a.table + static_cast<int64_t>(b) * a.pages_per_seq : nullptr;
    const int head0 = kvh * a.group + rb * kAttendRows, heads = min(a.group - rb * kAttendRows, kAttendRows);

    // the query heads as the second operand of K Q^T, columns beyond them zero
    u32x4_t qf[KS];
    {
        const char* p = a.q + (static_cast<int64_t>(b) * a.Hq + head0 + min(r, heads - 1)) * RB + c * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            qf[s] = *reinterpret_cast<const u32x4_t*>(p + s * 64);
            if (r >= heads) qf[s] = u32x4_t{0, 0, 0, 0};
        }
    }

    const bool by_blocks = !PAGED || a.page_size % 16 == 0;
    const int last = max(n_cache - 1, 0);
    auto page_index = [&](int j) { return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(j)) * a.page_mul) >> a.page_shift); };

    u32x4_t kf[NT][KS];
    uint32_t vf[NV][VW];
    f32x4_t acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    float* logits = WEIGHTS ? a.logits + (static_cast<int64_t>(b) * a.Hq + head0 + min(r, heads - 1)) * a.logit_stride + 4 * c : nullptr;

    struct Scores { f32x4_t x[NT]; };
    auto scores = [&] {
        Scores s;
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            s.x[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < KS; ++p) {
                if constexpr (BF16) {
                    s.x[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[x][p]), __builtin_bit_cast(bf16x8_t, qf[p]), s.x[x], 0, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s.x[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[x][p][i]), __uint_as_float(qf[p][i]), s.x[x], 0, 0, 0);
                }
            }
        }
        return s;
    };
    // Takes in the rows of tile t, those whose bit is set in `mask`.  (all: every bit is, in every lane)
    auto take = [&](int t, Scores& s, bool all, uint32_t mask) {
        if (a.cap > 0.f) {
#pragma unroll
            for (int i = 0; i < NV; ++i) s.x[i >> 2][i & 3] = a.cap * tanh_of(s.x[i >> 2][i & 3] * a.scale);
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) s.x[i >> 2][i & 3] *= a.scale;
        }
        if (!all) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (!((mask >> i) & 1u)) {
                    s.x[i >> 2][i & 3] = -INFINITY;
#pragma unroll
                    for (int w = 0; w < VW; ++w) vf[i][w] = 0u;      // nothing times whatever is there must be nothing
                }
        }
        if (WEIGHTS && r < heads) {
#pragma unroll
            for (int x = 0; x < NT; ++x) *reinterpret_cast<f32x4_t*>(logits + t * TILE + 16 * x) = s.x[x];
        }
        float top = s.x[0][0];
#pragma unroll
        for (int i = 1; i < NV; ++i) top = fmaxf(top, s.x[i >> 2][i & 3]);
        top = rows_max(top);
        if (__any(top > m)) {
            const float to = fmaxf(m, top), f = exp2_of(m - (to == -INFINITY ? 0.f : to));
            m = to;
            l *= f;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float p[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) { p[i] = exp2_of(s.x[i >> 2][i & 3] - ref); l += p[i]; }
        if constexpr (BF16) {
            // a probability is the sum of two bf16 numbers, 16 of its bits: with one, the result would be as far from the exact one
            // as its own rounding is once more; the second product hides in the wait for memory
            typedef short operand_t __attribute__((ext_vector_type(4)));
            uint32_t hi[NV / 2], lo[NV / 2];
#pragma unroll
            for (int i = 0; i < NV / 2; ++i) {
                hi[i] = pack_bf16x2(p[2 * i], p[2 * i + 1]);
                lo[i] = pack_bf16x2(p[2 * i] - bf16_lo(hi[i]), p[2 * i + 1] - bf16_hi(hi[i]));
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                uint32_t f[NV / 2];
#pragma unroll
                for (int i = 0; i < NV / 2; ++i) f[i] = __builtin_amdgcn_perm(vf[2 * i + 1][e >> 1], vf[2 * i][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
                if constexpr (NT == 2) {
                    const bf16x8_t v8 = __builtin_bit_cast(bf16x8_t, u32x4_t{f[0], f[1], f[2], f[3]});
                    acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8_t, u32x4_t{hi[0], hi[1], hi[2], hi[3]}), acc[e], 0, 0, 0);
                    acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8_t, u32x4_t{lo[0], lo[1], lo[2], lo[3]}), acc[e], 0, 0, 0);
                } else {
                    const operand_t v4 = __builtin_bit_cast(operand_t, make_uint2(f[0], f[1]));
                    acc[e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v4, __builtin_bit_cast(operand_t, make_uint2(hi[0], hi[1])), acc[e], 0, 0, 0);
                    acc[e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v4, __builtin_bit_cast(operand_t, make_uint2(lo[0], lo[1])), acc[e], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[i][e]), p[i], acc[e], 0, 0, 0);
        }
    };

    // Tiles in which every row of the cache is there are loaded by blocks of 16 neighbouring rows: one address for the wave, from scalar
    // loads of the table, and constant offsets per lane.  A page that is none counts as row 0, and its rows are masked.
    struct Blocks {
        int row[NT];
        bool ok;
        uint32_t mask;
    };
    typedef int Pages __attribute__((ext_vector_type(2)));
    const scalar_ints table_s = reinterpret_cast<scalar_ints>(reinterpret_cast<uintptr_t>(table));
    auto pages_of = [&](int t) {
        Pages p = {0, 0};
        if constexpr (PAGED) {
            p.x = table_s[page_index(min(t * TILE, last))];
            if (NT == 2) p.y = table_s[page_index(min(t * TILE + 16, last))];
        }
        return p;
    };
    auto blocks_of = [&](int t, Pages p) {
        Blocks f{};
        f.ok = true;
        f.mask = (1u << NV) - 1;
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const int j = t * TILE + 16 * x;
            f.row[x] = j;
            if constexpr (PAGED) {
                const int page = x ? p.y : p.x;
                const bool ok = page >= 0 && page < a.n_pages;
                f.row[x] = ok ? (page * a.Hkv + kvh) * a.page_size + (j - page_index(j) * a.page_size) : 0;
                f.ok = f.ok && ok;
                if (!ok) f.mask &= ~(0xfu << (4 * x));
            }
        }
        return f;
    };
    const uint32_t k_lane = r * RB + c * 16, v_lane = 4 * c * RB + r * VW * 4;
    auto load_k_blocks = [&](const Blocks& f) {
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const char* block = k_base + static_cast<uint64_t>(static_cast<uint32_t>(f.row[x])) * RB;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[x][s] = load_piece(block + s * 64 + k_lane);
        }
    };
    auto load_v_blocks = [&](const Blocks& f) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const char* block = v_base + static_cast<uint64_t>(static_cast<uint32_t>(f.row[i >> 2])) * RB;
            load_words<VW>(vf[i], block + (i & 3) * RB + v_lane);
        }
    };
    // The other tiles -- the one with the last row or the new one, all of them where pages are no multiples of 16 rows -- row by row.
    auto row_in = [&](int t) {                             // the row that lane % TILE stands for: of the slab or pool, kNoRow or kNewRow
        const int j = t * TILE + (lane & (TILE - 1));
        if (j >= n_cache) return fresh && j == n_cache ? kNewRow : kNoRow;
        if constexpr (!PAGED) return j;
        const int index = page_index(j), page = table[index];
        return page >= 0 && page < a.n_pages ? (page * a.Hkv + kvh) * a.page_size + (j - index * a.page_size) : kNoRow;
    };
    auto load_k_rows = [&](int mine) {
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const char* row = row_address(k_base, k_fresh, __shfl(mine, 16 * x + r, 64), RB) + c * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[x][s] = load_piece(row + s * 64);
        }
    };
    auto load_v_rows = [&](int mine) {
        uint32_t mask = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int row = __shfl(mine, 16 * (i >> 2) + 4 * c + (i & 3), 64);
            load_words<VW>(vf[i], row_address(v_base, v_fresh, row, RB) + r * VW * 4);
            mask |= (row != kNoRow ? 1u : 0u) << i;
        }
        return mask;
    };

    // Both loops have K and V of a tile on their way at their top, ask for the next K as soon as the scores are taken and for
    // the next V as soon as the sums are; nothing about these loads is conditional, so that the waits count them exactly (with the
    // two kinds of tiles in one loop every product waited for all loads: 8 x 36992 rows 102 us).
    const int t_whole = by_blocks ? min(t1, n_cache / TILE) : t0;      // tiles from here on go row by row
    int t = t0 + wave;
    if (t < t_whole) {
        Blocks f = blocks_of(t, pages_of(t));
        load_k_blocks(f);
        load_v_blocks(f);
        Pages pages = pages_of(t + kAttendWaves);
        for (; t + kAttendWaves < t_whole; t += kAttendWaves) {
            Scores s = scores();
            const Blocks g = blocks_of(t + kAttendWaves, pages);
            load_k_blocks(g);
            pages = pages_of(t + 2 * kAttendWaves);
            take(t, s, f.ok, f.mask);
            load_v_blocks(g);
            f = g;
        }
        Scores s = scores();
        take(t, s, f.ok, f.mask);
        t += kAttendWaves;
    }
    if (t < t1) {
        int mine = row_in(t);
        load_k_rows(mine);
        uint32_t mask = load_v_rows(mine);
        int mine_next = row_in(min(t + kAttendWaves, t1 - 1));
        for (; t + kAttendWaves < t1; t += kAttendWaves) {
            Scores s = scores();
            mine = mine_next;
            load_k_rows(mine);
            mine_next = row_in(min(t + 2 * kAttendWaves, t1 - 1));
            take(t, s, false, mask);
            mask = load_v_rows(mine);
        }
        Scores s = scores();
        take(t, s, false, mask);
    }
    l = swap16_add(l, l);
    l = swap32_add(l, l);

    // the new row joins the cache: nobody reads that row of the cache in this call
    if (fresh && rb == 0 && split == sh.splits - 1 && n_cache < a.S_cap) {
        const int to = PAGED ? table[n_cache / a.page_size] : 0;
        if (!PAGED || (to >= 0 && to < a.n_pages)) {
            const int64_t at = PAGED ? (static_cast<int64_t>(to) * a.Hkv + kvh) * a.page_size + n_cache % a.page_size : slab * a.S_cap + n_cache;
            const bool value = threadIdx.x >= RB / 16;
            const int piece = (value ? threadIdx.x - RB / 16 : threadIdx.x) * 16;
            if (threadIdx.x < 2 * (RB / 16))
                *reinterpret_cast<uint4*>((value ? a.v : a.k) + at * RB + piece) = *reinterpret_cast<const uint4*>((value ? v_fresh : k_fresh) + piece);
        }
    }
    // the waves' results are joined: accumulator i of element e is dimension E (4 c + i) + e of query row r
    if (c == 0) { s_ml[wave][r][0] = m; s_ml[wave][r][1] = l; }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) s_o[wave][r][E * (4 * c + i) + e] = acc[e][i];
    __syncthreads();
    // (No divergent branch lies inside another from here on: with one there, and the registers short, the compiler restored a
    // value of all lanes where only some were enabled.)
    const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * E;
    auto joined = [&](int of, float& top, float (&f)[kAttendWaves]) {
        top = -INFINITY;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) top = fmaxf(top, s_ml[w][of][0]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) {
            f[w] = exp2_of(s_ml[w][of][0] - ref);
            sum = fmaf(s_ml[w][of][1], f[w], sum);
        }
        return sum;
    };
    float top, f[kAttendWaves], o[E];
    const float sum = joined(row, top, f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        o[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) o[e] = fmaf(s_o[w][row][d0 + e], f[w], o[e]);
    }
    const int64_t first = static_cast<int64_t>(b) * a.Hq + head0;
    const bool whole = sh.splits == 1;
    if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        char* to = a.out + (first + row) * RB + d0 * sizeof(T);
        if (row < heads) {
            if constexpr (BF16) {
#pragma unroll
                for (int e = 0; e < E; e += 2) reinterpret_cast<uint32_t*>(to)[e / 2] = pack_bf16x2(o[e] * inv, o[e + 1] * inv);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) reinterpret_cast<float*>(to)[e] = o[e] * inv;
            }
        }
    } else if (row < heads) {
        float* to = a.part_o + (static_cast<int64_t>(blockIdx.x) * a.rows + row) * DH + d0;
#pragma unroll
        for (int e = 0; e < E; ++e) to[e] = o[e];
    }
    if (static_cast<int>(threadIdx.x) < heads) {
        const float l_row = joined(threadIdx.x, top, f);
        if (whole) {
            const float lse2 = l_row == 0.f ? -INFINITY : top + log2_of(l_row);
            if (a.lse) a.lse[first + threadIdx.x] = lse2 * 0.693147180559945309f;
            if (WEIGHTS) a.lse2[first + threadIdx.x] = lse2;
        } else {
            reinterpret_cast<float2*>(a.part_ml)[static_cast<int64_t>(blockIdx.x) * a.rows + threadIdx.x] = make_float2(top, l_row);
        }
    }
}

constexpr int kJoinThreads = 256;
constexpr int kWeightRows = 256;       // cache rows a workgroup adds up at a time: four to a lane

// log2 of the sum of a query head's shares, +inf where no row counts; all lanes of the wave.
__device__ __forceinline__ float wave_lse2(const DecodeArgs& a, const VideoShare& sh, int head) {
    const int kvh = head / a.group, qi = head - kvh * a.group, rb = qi / kAttendRows;
    float lse2;
    if (sh.splits == 1) lse2 = a.lse2[static_cast<int64_t>(sh.b) * a.Hq + head];
    else {
        const int64_t slot0 = static_cast<int64_t>(sh.first + (kvh * a.row_blocks + rb) * sh.splits) * a.rows + (qi - rb * kAttendRows);
        float m = -INFINITY, l = 0.f;
        for (int p = threadIdx.x & 63; p < sh.splits; p += 64) {
            const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * (slot0 + static_cast<int64_t>(p) * a.rows));
            const float to = fmaxf(m, ml.x), ref = to == -INFINITY ? 0.f : to;
            l = l * exp2_of(m - ref) + ml.y * exp2_of(ml.x - ref);
            m = to;
        }
#pragma unroll
        for (int off = 32; off; off >>= 1) {
            const float m2 = __shfl_xor(m, off, 64), l2 = __shfl_xor(l, off, 64), to = fmaxf(m, m2), ref = to == -INFINITY ? 0.f : to;
            l = l * exp2_of(m - ref) + l2 * exp2_of(m2 - ref);
            m = to;
        }
        lse2 = l == 0.f ? -INFINITY : m + log2_of(l);
    }
    return lse2 == -INFINITY ? INFINITY : lse2;
}

template <typename T, int DH>
__global__ __launch_bounds__(kJoinThreads) void decode_join_kernel(const DecodeArgs a) {
    constexpr int TILE = attend_tile(sizeof(T), DH);
    constexpr int LANES = DH / 4, GROUPS = kJoinThreads / LANES;       // lanes of a row, rows at a time
    __shared__ float s_x[1024];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (static_cast<int>(blockIdx.x) < a.join_blocks) {
        // one (video, query head)
        __shared__ float4 s_part[kJoinThreads];
        const int b = blockIdx.x / a.Hq, head = blockIdx.x - b * a.Hq;
        const VideoShare sh = find_share<TILE, true>(a, b);
        if (sh.splits == 1) return;
        const int kvh = head / a.group, qi = head - kvh * a.group, rb = qi / kAttendRows;
        const int64_t slot0 = static_cast<int64_t>(sh.first + (kvh * a.row_blocks + rb) * sh.splits) * a.rows + (qi - rb * kAttendRows);
        const float lse2 = wave_lse2(a, sh, head);                      // +inf: the factors below are 0
        const int g = threadIdx.x / LANES, x = threadIdx.x % LANES;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p = g; p < sh.splits; p += GROUPS) {
            const int64_t slot = slot0 + static_cast<int64_t>(p) * a.rows;
            const float f = exp2_of(a.part_ml[2 * slot] - lse2);
            const float4 v = *reinterpret_cast<const float4*>(a.part_o + slot * DH + x * 4);
            o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
        }
        s_part[threadIdx.x] = o;
        __syncthreads();
        if (g == 0) {
            for (int k = 1; k < GROUPS; ++k) {
                const float4 v = s_part[k * LANES + x];
                o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
            }
            const int64_t at = static_cast<int64_t>(b) * a.Hq + head;
            if constexpr (sizeof(T) == 2)
                *reinterpret_cast<uint2*>(a.out + (at * DH + x * 4) * 2) = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
            else *reinterpret_cast<float4*>(a.out + (at * DH + x * 4) * 4) = o;
            if (x == 0 && a.lse) a.lse[at] = lse2 == INFINITY ? -INFINITY : lse2 * 0.693147180559945309f;
        }
        return;
    }
    // rows of one video: every lane has four neighbouring rows, the waves share the heads
    __shared__ float4 s_sum[kJoinThreads];
    const int w = static_cast<int>(blockIdx.x) - a.join_blocks, b = w / a.weight_blocks, first = w - b * a.weight_blocks;
    const VideoShare sh = find_share<TILE, true>(a, b);
    const int fresh = a.k_new != nullptr, n = min(sh.n_cache + fresh, a.S_cap);       // rows that have a place
    if (static_cast<int64_t>(first) * kWeightRows >= n) return;
    for (int h = wave; h < a.Hq; h += kJoinThreads / 64) {
        const float v = wave_lse2(a, sh, h);
        if (lane == 0) s_x[h] = v;
    }
    __syncthreads();
    const float inv = 1.f / static_cast<float>(a.Hq);
    for (int64_t j0 = static_cast<int64_t>(first) * kWeightRows; j0 < n; j0 += static_cast<int64_t>(a.weight_blocks) * kWeightRows) {
        const int64_t j = j0 + 4 * lane;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j < n) {
            const float* p = a.logits + static_cast<int64_t>(b) * a.Hq * a.logit_stride + j;
            for (int h = wave; h < a.Hq; h += kJoinThreads / 64) {
                const float4 x = *reinterpret_cast<const float4*>(p + h * a.logit_stride);
                const float z = s_x[h];
                sum.x += exp2_of(x.x - z); sum.y += exp2_of(x.y - z); sum.z += exp2_of(x.z - z); sum.w += exp2_of(x.w - z);
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
            *out = (mine < sh.n_cache ? *out : 0.f) + total * inv;
        }
        __syncthreads();
    }
}

template <typename T, int DH>
static int launch_attend(const DecodeArgs& a, const AttendPlan& plan, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(plan.grid)), block(kAttendThreads);
    if (a.table) {
        if (a.weight) hipLaunchKernelGGL((decode_attention_kernel<T, DH, true, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((decode_attention_kernel<T, DH, true, false>), grid, block, 0, st, a);
    } else {
        if (a.weight) hipLaunchKernelGGL((decode_attention_kernel<T, DH, false, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((decode_attention_kernel<T, DH, false, false>), grid, block, 0, st, a);
    }
    int rc = check_launch("decode attention");
    if (rc) return rc;
    const int64_t blocks = a.join_blocks + static_cast<int64_t>(a.weight ? a.B : 0) * a.weight_blocks;
    if (blocks == 0) return METOK_OK;
    hipLaunchKernelGGL((decode_join_kernel<T, DH>), dim3(static_cast<unsigned>(blocks)), dim3(kJoinThreads), 0, st, a);
    return check_launch("decode join");
}

// The shapes that the calls and the workspace query take, NULL or the reason why not.
static const char* bad_shape(int B, int Hq, int Hkv, int64_t S_cap, int dh, int dtype) {
    if (dtype != METOK_F32 && dtype != METOK_BF16) return "unknown dtype";
    if (B < 1 || B > METOK_MAX_DECODE_BATCH) return "B must be in [1, METOK_MAX_DECODE_BATCH]";
    if (Hkv < 1 || Hq < 1 || Hq > 1024 || Hq % Hkv != 0) return "Hq must be a multiple of Hkv and at most 1024";
    if (dh != 32 && dh != 64 && dh != 128 && !(dh == 256 && dtype == METOK_BF16)) return "dh must be 32, 64, 128 or (bf16) 256";
    if (S_cap < 1 || S_cap >= INT32_MAX - 64) return "the capacity must be in [1, 2^31 - 64)";
    const int64_t pairs = static_cast<int64_t>(B) * Hkv * ((Hq / Hkv + kAttendRows - 1) / kAttendRows);
    if (pairs + kAttendTarget > INT32_MAX || static_cast<int64_t>(B) * (S_cap / 16 + 2) > INT32_MAX) return "too many rows";
    return nullptr;
}

struct Span { const char* name; const void* p; size_t bytes; };
static bool overlap(const Span& x, const Span& y) {
    if (!x.p || !y.p || !x.bytes || !y.bytes) return false;
    const char *a = static_cast<const char*>(x.p), *b = static_cast<const char*>(y.p);
    return a < b + y.bytes && b < a + x.bytes;
}

static int attend_impl(const void* q, int B, int Hq, int Hkv, int dh, int dtype, void* k, void* v, int64_t S_cap, size_t cache_bytes,
                       const int32_t* table, int64_t n_pages, int page_size, int pages_per_seq, const int32_t* len,
                       const void* k_new, const void* v_new, double scale, double logit_cap,
                       void* out, float* lse, float* weight, int64_t weight_stride, void* workspace, size_t workspace_bytes, void* stream) {
    if (!q || !k || !v || !len || !out) return fail(METOK_ERR_INVALID_ARG, "q, the caches, len and out must not be NULL");
    if ((k_new == nullptr) != (v_new == nullptr)) return fail(METOK_ERR_INVALID_ARG, "k_new and v_new go together");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(out))
        return fail(METOK_ERR_INVALID_ARG, "q, the caches, k_new, v_new and out must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(len) | reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(weight)) & 3u)
        return fail(METOK_ERR_INVALID_ARG, "len, lse and weight must be 4-byte aligned");
    if (!(scale > 0.0 && scale < 1e30)) return fail(METOK_ERR_INVALID_ARG, "scale must be positive and finite");
    if (!(logit_cap >= 0.0 && logit_cap < 1e30)) return fail(METOK_ERR_INVALID_ARG, "logit_cap must be 0 (none) or positive and finite");
    if (weight && weight_stride < S_cap) return fail(METOK_ERR_INVALID_ARG, "weight_stride must be at least the capacity");
    const size_t esize = dtype_size(dtype), head = static_cast<size_t>(dh) * esize;
    const AttendPlan plan = plan_attend(B, Hq, Hkv, S_cap, dh, static_cast<int>(esize), weight != nullptr);
    if (plan.bytes && (!workspace || workspace_bytes < plan.bytes || !aligned16(workspace)))
        return fail(METOK_ERR_WORKSPACE, "workspace of %zu bytes needed (16-byte aligned), %zu given", plan.bytes, workspace_bytes);
    const Span spans[] = {
        {"out", out, B * Hq * head}, {"lse", lse, static_cast<size_t>(B) * Hq * 4},
        {"weight", weight, weight ? (static_cast<size_t>(B - 1) * weight_stride + S_cap) * 4 : 0}, {"workspace", workspace, plan.bytes},
        {"the K cache", k, cache_bytes}, {"the V cache", v, cache_bytes},
        {"q", q, B * Hq * head}, {"k_new", k_new, B * Hkv * head}, {"v_new", v_new, B * Hkv * head},
        {"len", len, static_cast<size_t>(B) * 4}, {"page_table", table, static_cast<size_t>(B) * pages_per_seq * 4}};
    constexpr int n_written = 6, n_spans = sizeof(spans) / sizeof(spans[0]);
    for (int i = 0; i < n_written; ++i)
        for (int j = i + 1; j < n_spans; ++j)
            if (overlap(spans[i], spans[j])) return fail(METOK_ERR_INVALID_ARG, "%s overlaps %s", spans[i].name, spans[j].name);

    DecodeArgs a{};
    a.q = static_cast<const char*>(q); a.k = static_cast<char*>(k); a.v = static_cast<char*>(v);
    a.k_new = static_cast<const char*>(k_new); a.v_new = static_cast<const char*>(v_new);
    a.len = len; a.table = table; a.out = static_cast<char*>(out); a.lse = lse; a.weight = weight;
    char* ws = static_cast<char*>(workspace);
    a.part_ml = reinterpret_cast<float*>(ws + plan.part_ml); a.part_o = reinterpret_cast<float*>(ws + plan.part_o);
    a.lse2 = reinterpret_cast<float*>(ws + plan.lse2); a.logits = reinterpret_cast<float*>(ws + plan.logits);
    a.weight_stride = weight_stride; a.logit_stride = plan.logit_stride;
    a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.group = Hq / Hkv; a.row_blocks = plan.row_blocks; a.rows = plan.rows;
    a.S_cap = static_cast<int>(S_cap); a.page_size = page_size; a.pages_per_seq = pages_per_seq; a.n_pages = static_cast<int>(n_pages);
    int bits = 0;                // 2^bits >= page_size: ceil(2^(31 + bits) / page_size) is below 2^32 and off by less than 2^bits / page_size
    while ((static_cast<int64_t>(1) << bits) < page_size) ++bits;
    a.page_mul = static_cast<uint32_t>(((static_cast<uint64_t>(1) << (31 + bits)) + page_size - 1) / page_size);
    a.page_shift = 31 + bits;
    constexpr double log2e = 1.4426950408889634074;
    a.scale = static_cast<float>(logit_cap > 0.0 ? scale / logit_cap : scale * log2e);
    a.cap = static_cast<float>(logit_cap * log2e);
    a.join_blocks = plan.joined ? B * Hq : 0;
    // every workgroup of the weights sums up the heads' shares for itself: enough of them for the chip, not more
    const int64_t most = (S_cap + kWeightRows - 1) / kWeightRows, enough = (1024 + B - 1) / B;
    a.weight_blocks = static_cast<int>(most < enough ? most : enough);
    hipStream_t st = static_cast<hipStream_t>(stream);
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
    return attend_impl(q, B, Hq, Hkv, dh, dtype, k_cache, v_cache, S_cap, bytes, nullptr, 0, 1, 0, len, k_new, v_new, scale, logit_cap,
                       out, lse, weight, weight_stride, workspace, workspace_bytes, stream);
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
    return attend_impl(q, B, Hq, Hkv, dh, dtype, k_pool, v_pool, S_cap, bytes, page_table, n_pages_pool, page_size, pages_per_seq, len,
                       k_new, v_new, scale, logit_cap, out, lse, weight, weight_stride, workspace, workspace_bytes, stream);
}
