// The kernel that reads the cache for the attention of one new token: for one block of 16 query heads to a kv head at a time (decode.hip),
// for several (decode_wide.hip), and for short caches in one launch (decode_short.hip).
//
// For changes: no instantiation may spill vector registers (the build refuses it), and no branch that some lanes take may hold another one.
// With both, the compiler has restored a value that all lanes need behind the inner branch, where only some of them are on.
#pragma once

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
    int2* pair_workers;          // [pairs]: first and last worker of a (video, kv head, row block)
    float* part_ml;              // [slots][rows][2]: maximum (before score_scale) and sum of a partial result
    float* part_o;               // [slots][rows][dh]
    float2* norm;                // [B, Hq]: maximum (before score_scale) and 1 / sum, 0 and 0 without rows, where one worker had all of them
    float* logits;               // [B, Hq, logit_stride], before score_scale
    int64_t weight_stride, logit_stride;
    int B, Hq, Hkv, group, row_blocks, block_rows, rows;
    int S_cap;                   // capacity
    int page_size, pages_per_seq, n_pages;
    uint32_t page_mul, page_shift;       // j / page_size = j * page_mul >> page_shift for 0 <= j < 2^31
    float scale;                 // without cap: of the logits in the log2 domain; with cap: scale / cap
    float cap;                   // cap in the log2 domain, 0: none
    int join_blocks, join_lanes, weight_blocks, head_lanes;      // of decode_join_kernel
};

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }

// What takes scores to the log2 domain (capped ones are there), and 2^(score - reference).  The difference is taken before the scale: it is 0 for the
// reference itself, so that probabilities are relative to the largest one whatever the size of the scores.  (With the scale and the
// difference in one rounding, to a reference that was rounded at its full size, scores from 2e9 on became 0 or infinite.)
__device__ __forceinline__ float score_scale(const DecodeArgs& a) { return a.cap > 0.f ? 1.f : a.scale; }
__device__ __forceinline__ float exp2_from(float score, float reference, float scale) { return exp2_of((score - reference) * scale); }

__device__ __forceinline__ int rows_before(const DecodeArgs& a, int b) {
    const int n = a.len[b];
    return n < 0 ? 0 : (n > a.S_cap ? a.S_cap : n);
}

// Where a worker begins: video, its tiles and rows, unit of all its pairs; and how many units it has.
struct Place { int b, n, tiles, at, left; };

// Goes through the videos, 64 a step, one to a lane.  An empty video has a tile, too, without rows.  Uniform over the wave.  left = 0: there is
// no such worker.
template <int TILE, typename DEAL>
__device__ __forceinline__ Place find_place(const DecodeArgs& a, int worker) {
    const int lane = threadIdx.x & 63, fresh = a.k_new != nullptr, heads = a.Hkv * a.row_blocks;
    int n = 0, tiles = 0, before = 0;                      // units of a head of the videos before, within the 64
    int total = 0;
    auto look = [&](int b0) {
        const bool in = b0 + lane < a.B;
        n = in ? rows_before(a, b0 + lane) : 0;
        tiles = max(static_cast<int>(static_cast<uint32_t>(n + fresh + TILE - 1) / TILE), 1);
        const int units = in ? tiles + kAttendPairCost : 0;
        const int incl = wave_inclusive_scan(units);
        before = incl - units;
        return __builtin_amdgcn_readlane(incl, 63);
    };
    for (int b0 = 0; b0 < a.B; b0 += 64) total += look(b0);
    const int64_t all = static_cast<int64_t>(total) * heads, first = DEAL::first(worker, all);
    Place p{0, 0, 0, 0, static_cast<int>(DEAL::first(worker + 1, all) - first)};
    if (worker >= DEAL::workers(all)) p.left = 0;
    if (p.left <= 0) return p;
    int base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        int sum = total;
        if (a.B > 64) sum = look(b0);
        const unsigned long long hit = __ballot(b0 + lane < a.B && static_cast<int64_t>(base + before + tiles + kAttendPairCost) * heads > first);
        if (hit) {
            const int l = __builtin_amdgcn_readfirstlane(__ffsll(static_cast<long long>(hit)) - 1);
            p.b = b0 + l;
            p.n = __builtin_amdgcn_readlane(n, l);
            p.tiles = __builtin_amdgcn_readlane(tiles, l);
            p.at = static_cast<int>(first - static_cast<int64_t>(base + __builtin_amdgcn_readlane(before, l)) * heads);
            break;
        }
        base += sum;
    }
    return p;
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

template <bool STREAM> __device__ __forceinline__ u32x4_t load_piece(const char* p) {
    if (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
    return *reinterpret_cast<const u32x4_t*>(p);
}
template <int WORDS, bool STREAM> __device__ __forceinline__ void load_words(uint32_t (&w)[WORDS], const char* p) {
    if constexpr (WORDS == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
    else if constexpr (WORDS == 2) { const uint2 x = *reinterpret_cast<const uint2*>(p); w[0] = x.x; w[1] = x.y; }
    else {
#pragma unroll
        for (int i = 0; i < WORDS; i += 4) {
            const u32x4_t x = load_piece<STREAM>(p + 4 * i);
            w[i] = x.x; w[i + 1] = x.y; w[i + 2] = x.z; w[i + 3] = x.w;
        }
    }
}

// A lane's part of a row of V: RUNS runs of neighbouring words, the runs of 16 lanes one behind the other.
template <int RUNS, int WORDS, bool STREAM> __device__ __forceinline__ void load_part(uint32_t (&w)[WORDS], const char* row, uint32_t off) {
    constexpr int N = WORDS / RUNS;
#pragma unroll
    for (int g = 0; g < RUNS; ++g) {
        uint32_t x[N];
        load_words<N, STREAM>(x, row + g * 16 * N * 4 + off);
#pragma unroll
        for (int i = 0; i < N; ++i) w[g * N + i] = x[i];
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
    // a part is one run of neighbouring elements, or of two runs half a row apart where it is longer than a 16-byte load
    static constexpr int kRuns = kWords > 4 ? kWords / 4 : 1, kRun = kElems / kRuns;
};

enum { kDense = 0, kBlocks = 1, kRows = 2 };              // the cache; pages of a multiple of 16 rows; other pages

// A lane's place: r = lane % 16, c = lane / 16.  K Q^T is taken with the rows of K as rows of the product: the lane has query
// head r of the scores of rows 4 c .. 4 c + 3 of every 16.  That is already the operand layout of the second product, V^T P^T with
// the cache rows as contraction index, in the order 16 t + 4 c + i, so no value changes lanes between the two; a lane loads
// its part of kKeys rows of V, 16 lanes whole rows, and picks the rows' elements together in registers.  The softmax
// state of a query head is one (maximum, sum) per lane, the sum over the lane's own rows only.  No LDS, no barrier.
//
// Every wave is a worker of its own, with as many tiles as any other (one more or less), whatever videos and heads they belong to: equal bytes per
// CU are what counts.  (Workgroups that shared the rows of one pair each, sized alike: with one to a CU as fast where they came
// out equal, 131072 rows of 28 / 4 heads 46.7 us, 20 to 40 % slower where a third of the CUs had one more.)  K of the next tile is on
// its way as soon as the scores are taken, V as soon as the sums are, across the end of a pair too; no load is conditional but
// those of a new pair's queries and of the new row, so that the waits count the others exactly.
//
// WHOLE: a workgroup has a pair to itself, its waves the pair's tiles, neighbouring ones each, and joins their results in LDS.
template <typename T, int DH, int FORM, bool WEIGHTS, bool STREAM, int NB, bool WHOLE = false>
__global__ __launch_bounds__(64 * (WHOLE ? kAttendWholeWaves : kAttendWaves), NB == 1 ? 2 : 1) void decode_attention_kernel(const DecodeArgs a) {
    static_assert(!WHOLE || (NB == 1 && !WEIGHTS), "a pair is all query heads of a kv head");
    using S = AttendShape<T, DH>;
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int TILE = S::kTile, NT = S::kSub, KS = S::kPieces, NV = S::kKeys, E = S::kElems, VW = S::kWords, RB = S::kRowBytes;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
    // neighbouring workers on different CUs, so that few tiles are spread over all of them
    const int worker = wave * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x);
    const bool fresh = a.k_new != nullptr;
    const scalar_ints lens = reinterpret_cast<scalar_ints>(reinterpret_cast<uintptr_t>(a.len));

    // A tile of a pair, its kv head and block of query heads: uniform over the wave.
    struct Cursor { int b, kvh, rb, t, tiles, n; };
    Cursor at;
    int left;                                              // units that the worker still has (WHOLE: tiles)
    if constexpr (WHOLE) {
        at.b = static_cast<int>(blockIdx.x) / a.Hkv;
        at.kvh = static_cast<int>(blockIdx.x) - at.b * a.Hkv;
        at.rb = 0;
        at.n = min(max(lens[at.b], 0), a.S_cap);
        at.tiles = max(static_cast<int>(static_cast<uint32_t>(at.n + static_cast<int>(fresh) + TILE - 1) / TILE), 1);
        at.t = wave * at.tiles / kAttendWholeWaves;
        left = (wave + 1) * at.tiles / kAttendWholeWaves - at.t;
    } else {
        const Place place = find_place<TILE, Deal<attend_groups(sizeof(T), DH)>>(a, worker);
        if (place.left <= 0) return;
        at.b = __builtin_amdgcn_readfirstlane(place.b);
        at.tiles = __builtin_amdgcn_readfirstlane(place.tiles);
        at.n = __builtin_amdgcn_readfirstlane(place.n);
        const int units = at.tiles + kAttendPairCost;
        const int hr = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<uint32_t>(place.at) / static_cast<uint32_t>(units)));
        at.kvh = a.row_blocks == 1 ? hr : __builtin_amdgcn_readfirstlane(hr / a.row_blocks);
        at.rb = hr - at.kvh * a.row_blocks;
        at.t = __builtin_amdgcn_readfirstlane(place.at) - hr * units;
        left = __builtin_amdgcn_readfirstlane(place.left);
    }
    int n_ahead = WHOLE ? 0 : lens[min(at.b + 1, a.B - 1)];
    auto advance = [&](Cursor x) {
        if (++x.t == x.tiles && !WHOLE) {
            x.t = 0;
            if (++x.rb == a.row_blocks) {
                x.rb = 0;
                if (++x.kvh == a.Hkv) {
                    x.kvh = 0;
                    ++x.b;
                    x.n = min(max(n_ahead, 0), a.S_cap);
                    x.tiles = max(static_cast<int>(static_cast<uint32_t>(x.n + static_cast<int>(fresh) + TILE - 1) / TILE), 1);
                    n_ahead = lens[min(x.b + 1, a.B - 1)];
                }
            }
        }
        return x;
    };
    auto first_head = [&](const Cursor& x) { return x.kvh * a.group + x.rb * (NB * kAttendRows); };
    auto n_heads = [&](const Cursor& x) { return min(a.group - x.rb * (NB * kAttendRows), NB * kAttendRows); };

    // ---- loads ----
    auto page_index = [&](int j) { return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(j)) * a.page_mul) >> a.page_shift); };
    typedef int Pages __attribute__((ext_vector_type(2)));         // table entries of a tile's blocks, or .x of the lane's row
    auto pages_of = [&](const Cursor& x) {
        Pages p = {0, 0};
        const int j0 = x.t * TILE, last = max(x.n - 1, 0);
        if constexpr (FORM == kBlocks) {
            const scalar_ints table = reinterpret_cast<scalar_ints>(reinterpret_cast<uintptr_t>(a.table + static_cast<int64_t>(x.b) * a.pages_per_seq));
            p.x = table[page_index(min(j0, last))];
            if (NT == 2) p.y = table[page_index(min(j0 + 16, last))];
        }
        if constexpr (FORM == kRows) p.x = a.table[static_cast<int64_t>(x.b) * a.pages_per_seq + page_index(min(j0 + (lane & (TILE - 1)), last))];
        return p;
    };
    // Where a tile's rows are: by blocks of 16, the first row of each in the slab or pool and how many of it count (rows behind them are loaded as
    // the last one), or the lane's own row; and which rows are there.
    struct Rows { int first[NT], own; bool here, all; uint32_t pages_ok; };        // here: the tile ends before the last row; all: its pages are ones, too
    auto rows_of = [&](const Cursor& x, Pages p) {
        Rows f{};
        const int j0 = x.t * TILE, last = max(x.n - 1, 0), kvh = x.kvh;
        f.here = f.all = j0 + TILE <= x.n;
        f.pages_ok = (1u << NT) - 1;
        if constexpr (FORM == kRows) {
            const int j = min(j0 + (lane & (TILE - 1)), last);
            const bool ok = j0 + (lane & (TILE - 1)) < x.n && p.x >= 0 && p.x < a.n_pages;
            f.own = ok ? (p.x * a.Hkv + kvh) * a.page_size + (j - page_index(j) * a.page_size) : -1;
            f.all = f.all && __all(ok);
        } else {
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const int j = min(j0 + 16 * b, last);
                f.first[b] = j;
                if constexpr (FORM == kBlocks) {
                    const int page = b ? p.y : p.x;
                    const bool ok = page >= 0 && page < a.n_pages;
                    f.first[b] = ok ? (page * a.Hkv + kvh) * a.page_size + (j - page_index(j) * a.page_size) : 0;
                    if (!ok) { f.pages_ok &= ~(1u << b); f.all = false; }
                }
            }
        }
        return f;
    };
    auto slab_of = [&](const Cursor& x) { return (static_cast<int64_t>(x.b) * a.Hkv + x.kvh); };
    auto base_of = [&](const Cursor& x, const char* cache) { return FORM == kDense ? cache + slab_of(x) * a.S_cap * RB : cache; };
    // a row of tile x as a lane finds it: the new one, where it is that
    auto lane_row = [&](const Cursor& x, int row, const char* cached, const char* news) {
        return fresh && x.t * TILE + row == x.n ? news + slab_of(x) * RB : cached;
    };
    u32x4_t kf[NT][KS];
    uint32_t vf[NV][VW];
    auto load_k = [&](const Cursor& x, const Rows& f) {
        const char* base = base_of(x, a.k);
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            if constexpr (FORM == kRows) {
                const char* row = lane_row(x, 16 * b + r, base + static_cast<uint64_t>(static_cast<uint32_t>(max(__shfl(f.own, 16 * b + r, 64), 0))) * RB, a.k_new) + c * 16;
#pragma unroll
                for (int s = 0; s < KS; ++s) kf[b][s] = load_piece<STREAM>(row + s * 64);
            } else {
                const char* block = base + static_cast<uint64_t>(static_cast<uint32_t>(f.first[b])) * RB;
                if (f.here) {
                    const uint32_t off = r * RB + c * 16;
#pragma unroll
                    for (int s = 0; s < KS; ++s) kf[b][s] = load_piece<STREAM>(block + s * 64 + off);
                } else {
                    const char* row = lane_row(x, 16 * b + r, block + static_cast<uint32_t>(min(r, max(x.n - 1 - x.t * TILE - 16 * b, 0))) * RB, a.k_new) + c * 16;
#pragma unroll
                    for (int s = 0; s < KS; ++s) kf[b][s] = load_piece<STREAM>(row + s * 64);
                }
            }
        }
    };
    auto load_v = [&](const Cursor& x, const Rows& f) {
        const char* base = base_of(x, a.v);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (FORM == kRows) {
                const int at_row = 16 * (i >> 2) + 4 * c + (i & 3);
                const char* row = lane_row(x, at_row, base + static_cast<uint64_t>(static_cast<uint32_t>(max(__shfl(f.own, at_row, 64), 0))) * RB, a.v_new);
                load_part<S::kRuns, VW, STREAM>(vf[i], row, r * (VW / S::kRuns * 4));
            } else {
                const char* block = base + static_cast<uint64_t>(static_cast<uint32_t>(f.first[i >> 2])) * RB;
                if (f.here) load_part<S::kRuns, VW, STREAM>(vf[i], block + (i & 3) * RB, 4 * c * RB + r * (VW / S::kRuns * 4));
                else {
                    const int rows = max(x.n - 1 - x.t * TILE - 16 * (i >> 2), 0), row = 4 * c + (i & 3);
                    load_part<S::kRuns, VW, STREAM>(vf[i], lane_row(x, 16 * (i >> 2) + row, block + static_cast<uint32_t>(min(row, rows)) * RB, a.v_new),
                                                    r * (VW / S::kRuns * 4));
                }
            }
        }
    };
    auto load_q = [&](const Cursor& x, u32x4_t (&q)[NB][KS]) {
        const int heads = n_heads(x);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const char* p = a.q + (static_cast<int64_t>(x.b) * a.Hq + first_head(x) + min(16 * nb + r, heads - 1)) * RB + c * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s) q[nb][s] = *reinterpret_cast<const u32x4_t*>(p + s * 64);
        }
    };

    // ---- one tile ----
    u32x4_t qf[NB][KS];
    f32x4_t acc[NB][E];
    float m[NB], l[NB];
    auto clear = [&] {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb] = -INFINITY; l[nb] = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[nb][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    };
    // row n of the cache is the new one where there is one, and is not read from the cache
    auto new_row = [&](const Cursor& x) { return fresh && static_cast<int>(static_cast<uint32_t>(x.n) / TILE) == x.t; };
    auto scores = [&](f32x4_t (&s)[NB][NT]) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                s[nb][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int p = 0; p < KS; ++p) {
                    if constexpr (BF16) {
                        s[nb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[b][p]), __builtin_bit_cast(bf16x8_t, qf[nb][p]), s[nb][b], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            s[nb][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[b][p][i]), __uint_as_float(qf[nb][p][i]), s[nb][b], 0, 0, 0);
                    }
                }
            }
    };
    auto take = [&](const Cursor& x, const Rows& f, f32x4_t (&s)[NB][NT]) {
        if (a.cap > 0.f) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < NV; ++i) s[nb][i >> 2][i & 3] = a.cap * tanh_of(s[nb][i >> 2][i & 3] * a.scale);
        }
        const float scale = score_scale(a);
        if (!f.all) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int row = 16 * (i >> 2) + 4 * c + (i & 3), j = x.t * TILE + row;
                bool there = FORM == kRows ? __shfl(f.own, row, 64) >= 0 : j < x.n && ((f.pages_ok >> (i >> 2)) & 1u);
                there = there || (fresh && j == x.n);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    if (!there) s[nb][i >> 2][i & 3] = -INFINITY;
#pragma unroll
                for (int w = 0; w < VW; ++w) vf[i][w] = there ? vf[i][w] : 0u;       // nothing times whatever is there must be nothing
            }
        }
        if constexpr (WEIGHTS) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                if (16 * nb + r < n_heads(x)) {
                    float* to = a.logits + (static_cast<int64_t>(x.b) * a.Hq + first_head(x) + 16 * nb + r) * a.logit_stride + x.t * TILE + 4 * c;
#pragma unroll
                    for (int b = 0; b < NT; ++b) *reinterpret_cast<f32x4_t*>(to + 16 * b) = s[nb][b];
                }
        }
        float p[NB][NV];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float top = s[nb][0][0];
#pragma unroll
            for (int i = 1; i < NV; ++i) top = fmaxf(top, s[nb][i >> 2][i & 3]);
            top = rows_max(top);
            if (__any(top > m[nb])) {
                const float to = fmaxf(m[nb], top), g = exp2_from(m[nb], to == -INFINITY ? 0.f : to, scale);
                m[nb] = to;
                l[nb] *= g;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[nb][e] *= g;
            }
            const float ref = m[nb] == -INFINITY ? 0.f : m[nb];
#pragma unroll
            for (int i = 0; i < NV; ++i) { p[nb][i] = exp2_from(s[nb][i >> 2][i & 3], ref, scale); l[nb] += p[nb][i]; }
        }
        if constexpr (BF16) {
            // a probability is the sum of two bf16 numbers, 16 of its bits: with one, the result would be as far from the exact one
            // as its own rounding is once more; the second product hides in the wait for memory
            typedef short operand_t __attribute__((ext_vector_type(4)));
            uint32_t hi[NB][NV / 2], lo[NB][NV / 2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < NV / 2; ++i) {
                    hi[nb][i] = pack_bf16x2(p[nb][2 * i], p[nb][2 * i + 1]);
                    lo[nb][i] = pack_bf16x2(p[nb][2 * i] - bf16_lo(hi[nb][i]), p[nb][2 * i + 1] - bf16_hi(hi[nb][i]));
                }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                uint32_t g[NV / 2];
#pragma unroll
                for (int i = 0; i < NV / 2; ++i) g[i] = __builtin_amdgcn_perm(vf[2 * i + 1][e >> 1], vf[2 * i][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const uint32_t (&h)[NV / 2] = hi[nb], (&o)[NV / 2] = lo[nb];
                    if constexpr (NT == 2) {
                        const bf16x8_t v8 = __builtin_bit_cast(bf16x8_t, u32x4_t{g[0], g[1], g[2], g[3]});
                        acc[nb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8_t, u32x4_t{h[0], h[1], h[2], h[3]}), acc[nb][e], 0, 0, 0);
                        acc[nb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8_t, u32x4_t{o[0], o[1], o[2], o[3]}), acc[nb][e], 0, 0, 0);
                    } else {
                        const operand_t v4 = __builtin_bit_cast(operand_t, make_uint2(g[0], g[1]));
                        acc[nb][e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v4, __builtin_bit_cast(operand_t, make_uint2(h[0], h[1])), acc[nb][e], 0, 0, 0);
                        acc[nb][e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v4, __builtin_bit_cast(operand_t, make_uint2(o[0], o[1])), acc[nb][e], 0, 0, 0);
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) acc[nb][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[i][e]), p[nb][i], acc[nb][e], 0, 0, 0);
        }
    };

    // ---- the end of a pair, or of the worker's tiles: the result, or a part of it for the join ----
    auto finish = [&](const Cursor& x, int begun) {         // begun: the first tile of the pair that the worker had
        const bool ends = x.t == x.tiles - 1, whole = begun == 0 && ends;
        if (a.pair_workers && lane == 0) {
            int* to = reinterpret_cast<int*>(a.pair_workers + slab_of(x) * a.row_blocks + x.rb);
            if (begun == 0) to[0] = worker;
            if (ends) to[1] = worker;
        }
        // accumulator i of element e: element kRun (4 c + i) + e % kRun of run e / kRun
        constexpr int N = S::kRun;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int heads = n_heads(x) - 16 * nb;        // of this block
            const float sum = swap32_add(swap16_add(l[nb], l[nb]), swap16_add(l[nb], l[nb]));
            const int64_t head = static_cast<int64_t>(x.b) * a.Hq + first_head(x) + 16 * nb + r;
            const int64_t slot = (2 * static_cast<int64_t>(worker) + (begun == 0 ? 1 : 0)) * a.rows + 16 * nb + r;
            const float lse2 = sum == 0.f ? -INFINITY : fmaf(m[nb], score_scale(a), log2_of(sum)), inv = sum == 0.f ? 0.f : 1.f / sum;
            if (whole) {
                if (r < heads) {
#pragma unroll
                    for (int g = 0; g < S::kRuns; ++g)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            char* to = a.out + head * RB + (g * 16 * N + N * (4 * c + i)) * static_cast<int>(sizeof(T));
#pragma unroll
                            for (int e = 0; e < N; e += BF16 ? 2 : 1) {
                                if constexpr (BF16) reinterpret_cast<uint32_t*>(to)[e / 2] = pack_bf16x2(acc[nb][g * N + e][i] * inv, acc[nb][g * N + e + 1][i] * inv);
                                else reinterpret_cast<float*>(to)[e] = acc[nb][g * N + e][i] * inv;
                            }
                        }
                }
                if (c == 0 && r < heads && a.lse) a.lse[head] = lse2 * 0.693147180559945309f;
                if (WEIGHTS && c == 0 && r < heads) a.norm[head] = make_float2(sum == 0.f ? 0.f : m[nb], inv);
            } else {
                if (r < heads) {
                    float* to = a.part_o + slot * DH;
#pragma unroll
                    for (int g = 0; g < S::kRuns; ++g)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int e = 0; e < N; ++e) to[g * 16 * N + N * (4 * c + i) + e] = acc[nb][g * N + e][i];
                }
                if (c == 0 && r < heads) reinterpret_cast<float2*>(a.part_ml)[slot] = make_float2(m[nb], sum);
            }
        }
    };
    // the new row joins the cache: nobody reads that row of the cache in this call
    auto append = [&](const Cursor& x) {
        if (!new_row(x) || x.rb != 0 || x.n >= a.S_cap) return;
        int64_t to = slab_of(x) * a.S_cap + x.n;
        if constexpr (FORM != kDense) {
            const int index = page_index(x.n), page = a.table[static_cast<int64_t>(x.b) * a.pages_per_seq + index];
            if (page < 0 || page >= a.n_pages) return;
            to = (static_cast<int64_t>(page) * a.Hkv + x.kvh) * a.page_size + (x.n - index * a.page_size);
        }
        constexpr int P = RB / 16;
        if (lane < 2 * P) {
            const bool value = lane >= P;
            const int piece = (value ? lane - P : lane) * 16;
            *reinterpret_cast<uint4*>((value ? a.v : a.k) + to * RB + piece) = *reinterpret_cast<const uint4*>((value ? a.v_new : a.k_new) + slab_of(x) * RB + piece);
        }
    };

    if (!WHOLE && at.t >= at.tiles) {                                // behind a pair: on to the next one, if there is one
        left -= at.tiles + kAttendPairCost - at.t;
        if (left <= 0) return;
        at.t = at.tiles - 1;
        at = advance(at);
    }
    clear();
    if (!WHOLE || left > 0) {
    int begun = at.t;                                      // first tile of the pair that the worker has
    load_q(at, qf);
    Rows rows = rows_of(at, pages_of(at));
    load_k(at, rows);
    load_v(at, rows);
    // one block: the queries of the next pair are on their way with its first tile; several: the registers are needed
    u32x4_t q_next[NB == 1 ? NB : 1][KS];
    for (;;) {
        const bool ends = !WHOLE && at.t == at.tiles - 1;
        left -= ends ? 1 + kAttendPairCost : 1;
        if (left <= 0) break;
        const Cursor next = advance(at);
        const Pages pages = pages_of(next);
        f32x4_t s[NB][NT];
        scores(s);
        const Rows rows_next = rows_of(next, pages);
        load_k(next, rows_next);
        if constexpr (NB == 1) {
            if (ends) load_q(next, q_next);
        }
        take(at, rows, s);
        if (ends) {
            finish(at, begun);
            append(at);
            begun = 0;
            clear();
            if constexpr (NB == 1) {
#pragma unroll
                for (int p = 0; p < KS; ++p) qf[0][p] = q_next[0][p];
            } else load_q(next, qf);
        }
        load_v(next, rows_next);
        at = next;
        rows = rows_next;
    }
    f32x4_t s[NB][NT];
    scores(s);
    take(at, rows, s);
    if constexpr (!WHOLE) finish(at, begun);
    append(at);
    }
    if constexpr (WHOLE) {
        constexpr int W = kAttendWholeWaves, N = S::kRun, PITCH = DH + 4, LPR = DH / 4;       // 4 more: rows 16 bytes apart in the banks
        __shared__ float4 s_o[W * kAttendRows * PITCH / 4];
        __shared__ float2 s_ml[W][kAttendRows];
        const float sum = swap32_add(swap16_add(l[0], l[0]), swap16_add(l[0], l[0]));
        if (c == 0) s_ml[wave][r] = make_float2(m[0], sum);
        float* to = reinterpret_cast<float*>(s_o) + (wave * kAttendRows + r) * PITCH;
#pragma unroll
        for (int g = 0; g < S::kRuns; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) to[g * 16 * N + N * (4 * c + i) + e] = acc[0][g * N + e][i];
        __syncthreads();
        const int x = threadIdx.x % LPR, heads = n_heads(at);
        for (int row = threadIdx.x / LPR; row < heads; row += 64 * W / LPR) {
            float top = -INFINITY, total = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, s_ml[w][row].x);
            const float ref = top == -INFINITY ? 0.f : top, scale = score_scale(a);
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float2 part = s_ml[w][row];
                const float f = exp2_from(part.x, ref, scale);
                const float4 v = s_o[((w * kAttendRows + row) * PITCH + 4 * x) / 4];
                total = fmaf(part.y, f, total);
                o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
            }
            const float inv = total == 0.f ? 0.f : 1.f / total;
            const int64_t head = static_cast<int64_t>(at.b) * a.Hq + first_head(at) + row;
            char* out = a.out + head * RB + 4 * x * static_cast<int>(sizeof(T));
            if constexpr (BF16) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
            else *reinterpret_cast<float4*>(out) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
            if (x == 0 && a.lse) a.lse[head] = total == 0.f ? -INFINITY : fmaf(ref, scale, log2_of(total)) * 0.693147180559945309f;
        }
    }
}

template <typename T, int DH, int FORM, bool STREAM, int NB>
void launch_attention(const DecodeArgs& a, unsigned groups, hipStream_t st) {
    if (a.weight) hipLaunchKernelGGL((decode_attention_kernel<T, DH, FORM, true, STREAM, NB>), dim3(groups), dim3(kAttendThreads), 0, st, a);
    else hipLaunchKernelGGL((decode_attention_kernel<T, DH, FORM, false, STREAM, NB>), dim3(groups), dim3(kAttendThreads), 0, st, a);
}
// The same with several blocks of query heads to a kv head at a time (decode_wide.hip).
void launch_wide_attention(const DecodeArgs& a, int dtype, int dh, bool stream, unsigned groups, hipStream_t st);
// Short caches, a workgroup to a pair, in one launch (decode_short.hip).
void launch_short_attention(const DecodeArgs& a, int dtype, int dh, unsigned pairs, hipStream_t st);

}  // namespace metok
