// Attention of one new token per video over the dense or paged KV cache that stage 3 leaves (Sec. 3.3), with the token's own row
// appended and, if asked, the attention weight of every cached row accumulated (what metok_kv_evict ranks the rows by).
//
//   decode_attention_kernel  every wave's tiles of the rows of all (video, kv head, block of 16 query heads): scores, running maximum and
//                            sum of the softmax, weighted sum of the values, in one pass over K and V
//   decode_join_kernel       joins the parts of a (video, query head) whose rows several waves had; and, with weights, turns the
//                            scores that the first kernel kept into probabilities and adds their mean over the heads to the rows' weights
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
    int2* pair_workers;          // [pairs]: first and last worker of a (video, kv head, row block)
    float* part_ml;              // [slots][rows][2]: maximum and sum of a partial result, log2 domain
    float* part_o;               // [slots][rows][dh]
    float* lse2;                 // [B, Hq]: log2 of the sum, where one worker had all rows
    float* logits;               // [B, Hq, logit_stride], log2 domain
    int64_t weight_stride, logit_stride;
    int B, Hq, Hkv, group, row_blocks, rows;
    int S_cap;                   // capacity
    int page_size, pages_per_seq, n_pages;
    uint32_t page_mul, page_shift;       // j / page_size = j * page_mul >> page_shift for 0 <= j < 2^31
    float scale;                 // without cap: of the logits in the log2 domain; with cap: scale / cap
    float cap;                   // cap in the log2 domain, 0: none
    int join_blocks, join_lanes, weight_blocks, head_lanes;      // of decode_join_kernel
};

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }

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
template <typename T, int DH, int FORM, bool WEIGHTS, bool STREAM>
__global__ __launch_bounds__(kAttendThreads, 2) void decode_attention_kernel(const DecodeArgs a) {
    using S = AttendShape<T, DH>;
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int TILE = S::kTile, NT = S::kSub, KS = S::kPieces, NV = S::kKeys, E = S::kElems, VW = S::kWords, RB = S::kRowBytes;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
    // neighbouring workers on different CUs, so that few tiles are spread over all of them
    const int worker = wave * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x);
    const Place place = find_place<TILE, Deal<attend_groups(sizeof(T), DH)>>(a, worker);
    if (place.left <= 0) return;
    const bool fresh = a.k_new != nullptr;
    const scalar_ints lens = reinterpret_cast<scalar_ints>(reinterpret_cast<uintptr_t>(a.len));

    // A tile of a pair, its kv head and block of query heads: uniform over the wave.
    struct Cursor { int b, kvh, rb, t, tiles, n; };
    Cursor at;
    at.b = __builtin_amdgcn_readfirstlane(place.b);
    at.tiles = __builtin_amdgcn_readfirstlane(place.tiles);
    at.n = __builtin_amdgcn_readfirstlane(place.n);
    const int units = at.tiles + kAttendPairCost;
    const int hr = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<uint32_t>(place.at) / static_cast<uint32_t>(units)));
    at.kvh = a.row_blocks == 1 ? hr : __builtin_amdgcn_readfirstlane(hr / a.row_blocks);
    at.rb = hr - at.kvh * a.row_blocks;
    at.t = __builtin_amdgcn_readfirstlane(place.at) - hr * units;
    int left = __builtin_amdgcn_readfirstlane(place.left);
    int n_ahead = lens[min(at.b + 1, a.B - 1)];
    auto advance = [&](Cursor x) {
        if (++x.t == x.tiles) {
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
    auto first_head = [&](const Cursor& x) { return x.kvh * a.group + x.rb * kAttendRows; };
    auto n_heads = [&](const Cursor& x) { return min(a.group - x.rb * kAttendRows, kAttendRows); };

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
    auto load_q = [&](const Cursor& x, u32x4_t (&q)[KS]) {
        const int heads = n_heads(x);
        const char* p = a.q + (static_cast<int64_t>(x.b) * a.Hq + first_head(x) + min(r, heads - 1)) * RB + c * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const u32x4_t*>(p + s * 64);
    };

    // ---- one tile ----
    u32x4_t qf[KS];
    f32x4_t acc[E];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // row n of the cache is the new one where there is one, and is not read from the cache
    auto new_row = [&](const Cursor& x) { return fresh && static_cast<int>(static_cast<uint32_t>(x.n) / TILE) == x.t; };
    auto scores = [&](f32x4_t (&s)[NT]) {
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            s[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < KS; ++p) {
                if constexpr (BF16) {
                    s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[b][p]), __builtin_bit_cast(bf16x8_t, qf[p]), s[b], 0, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[b][p][i]), __uint_as_float(qf[p][i]), s[b], 0, 0, 0);
                }
            }
        }
    };
    auto take = [&](const Cursor& x, const Rows& f, f32x4_t (&s)[NT]) {
        if (a.cap > 0.f) {
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i >> 2][i & 3] = a.cap * tanh_of(s[i >> 2][i & 3] * a.scale);
        }
        const float scale = a.cap > 0.f ? 1.f : a.scale;       // to the log2 domain, rounded once with the difference to the maximum
        if (!f.all) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int row = 16 * (i >> 2) + 4 * c + (i & 3), j = x.t * TILE + row;
                bool there = FORM == kRows ? __shfl(f.own, row, 64) >= 0 : j < x.n && ((f.pages_ok >> (i >> 2)) & 1u);
                there = there || (fresh && j == x.n);
                if (!there) s[i >> 2][i & 3] = -INFINITY;
#pragma unroll
                for (int w = 0; w < VW; ++w) vf[i][w] = there ? vf[i][w] : 0u;       // nothing times whatever is there must be nothing
            }
        }
        if (WEIGHTS && r < n_heads(x)) {
            float* to = a.logits + (static_cast<int64_t>(x.b) * a.Hq + first_head(x) + r) * a.logit_stride + x.t * TILE + 4 * c;
#pragma unroll
            for (int b = 0; b < NT; ++b) *reinterpret_cast<f32x4_t*>(to + 16 * b) = s[b] * scale;
        }
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < NV; ++i) top = fmaxf(top, s[i >> 2][i & 3]);
        top = rows_max(top) * scale;
        if (__any(top > m)) {
            const float to = fmaxf(m, top), g = exp2_of(m - (to == -INFINITY ? 0.f : to));
            m = to;
            l *= g;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] *= g;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float p[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) { p[i] = exp2_of(fmaf(s[i >> 2][i & 3], scale, -ref)); l += p[i]; }
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
                uint32_t g[NV / 2];
#pragma unroll
                for (int i = 0; i < NV / 2; ++i) g[i] = __builtin_amdgcn_perm(vf[2 * i + 1][e >> 1], vf[2 * i][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
                if constexpr (NT == 2) {
                    const bf16x8_t v8 = __builtin_bit_cast(bf16x8_t, u32x4_t{g[0], g[1], g[2], g[3]});
                    acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8_t, u32x4_t{hi[0], hi[1], hi[2], hi[3]}), acc[e], 0, 0, 0);
                    acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8_t, u32x4_t{lo[0], lo[1], lo[2], lo[3]}), acc[e], 0, 0, 0);
                } else {
                    const operand_t v4 = __builtin_bit_cast(operand_t, make_uint2(g[0], g[1]));
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

    // ---- the end of a pair, or of the worker's tiles: the result, or a part of it for the join ----
    auto finish = [&](const Cursor& x, int begun) {         // begun: the first tile of the pair that the worker had
        l = swap16_add(l, l);
        l = swap32_add(l, l);
        const int heads = n_heads(x);
        const bool ends = x.t == x.tiles - 1, whole = begun == 0 && ends;
        if (a.pair_workers && lane == 0) {
            int* to = reinterpret_cast<int*>(a.pair_workers + slab_of(x) * a.row_blocks + x.rb);
            if (begun == 0) to[0] = worker;
            if (ends) to[1] = worker;
        }
        const int64_t head = static_cast<int64_t>(x.b) * a.Hq + first_head(x) + r;
        const int64_t slot = (2 * static_cast<int64_t>(worker) + (begun == 0 ? 1 : 0)) * a.rows + r;
        const float lse2 = l == 0.f ? -INFINITY : m + log2_of(l), inv = l == 0.f ? 0.f : 1.f / l;
        // accumulator i of element e: element kRun (4 c + i) + e % kRun of run e / kRun
        constexpr int N = S::kRun;
        if (whole) {
            if (r < heads) {
#pragma unroll
                for (int g = 0; g < S::kRuns; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        char* to = a.out + head * RB + (g * 16 * N + N * (4 * c + i)) * static_cast<int>(sizeof(T));
#pragma unroll
                        for (int e = 0; e < N; e += BF16 ? 2 : 1) {
                            if constexpr (BF16) reinterpret_cast<uint32_t*>(to)[e / 2] = pack_bf16x2(acc[g * N + e][i] * inv, acc[g * N + e + 1][i] * inv);
                            else reinterpret_cast<float*>(to)[e] = acc[g * N + e][i] * inv;
                        }
                    }
            }
            if (lane < heads && a.lse) a.lse[head] = lse2 * 0.693147180559945309f;
            if (WEIGHTS && lane < heads) a.lse2[head] = lse2;
        } else {
            if (r < heads) {
                float* to = a.part_o + slot * DH;
#pragma unroll
                for (int g = 0; g < S::kRuns; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < N; ++e) to[g * 16 * N + N * (4 * c + i) + e] = acc[g * N + e][i];
            }
            if (lane < heads) reinterpret_cast<float2*>(a.part_ml)[slot] = make_float2(m, l);
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

    if (at.t >= at.tiles) {                                // behind a pair: on to the next one, if there is one
        left -= at.tiles + kAttendPairCost - at.t;
        if (left <= 0) return;
        at.t = at.tiles - 1;
        at = advance(at);
    }
    int begun = at.t;                                      // first tile of the pair that the worker has
    load_q(at, qf);
    Rows rows = rows_of(at, pages_of(at));
    load_k(at, rows);
    load_v(at, rows);
    u32x4_t q_next[KS];
    for (;;) {
        const bool ends = at.t == at.tiles - 1;
        left -= ends ? 1 + kAttendPairCost : 1;
        if (left <= 0) break;
        const Cursor next = advance(at);
        const Pages pages = pages_of(next);
        f32x4_t s[NT];
        scores(s);
        const Rows rows_next = rows_of(next, pages);
        load_k(next, rows_next);
        if (ends) load_q(next, q_next);
        take(at, rows, s);
        if (ends) {
            finish(at, begun);
            append(at);
            begun = 0;
            m = -INFINITY; l = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < KS; ++p) qf[p] = q_next[p];
        }
        load_v(next, rows_next);
        at = next;
        rows = rows_next;
    }
    f32x4_t s[NT];
    scores(s);
    take(at, rows, s);
    finish(at, begun);
    append(at);
}

constexpr int kJoinThreads = 256;
constexpr int kWeightRows = kJoinThreads;       // cache rows a workgroup adds up at a time: four to a lane
// Up to so many workgroups a head's elements are spread over several of them, 32 each: with few heads every one has many parts (one
// video of 2307 rows, 28 heads: 10.1 us a call with one workgroup a head, 9.0 with four).
constexpr int kJoinSpread = 512;
// (m, l) stands for the sum l 2^m.
__device__ __forceinline__ void add_sum(float& m, float& l, float m2, float l2) {
    const float to = fmaxf(m, m2), ref = to == -INFINITY ? 0.f : to;
    l = l * exp2_of(m - ref) + l2 * exp2_of(m2 - ref);
    m = to;
}

// The workers of a query head's pair, and the place of their partial results.
struct HeadParts {
    int first, n, rows, row;
    __device__ __forceinline__ int64_t slot(int p) const { return static_cast<int64_t>(2 * (first + p) + (p == 0)) * rows + row; }
};
__device__ __forceinline__ HeadParts parts_of(const DecodeArgs& a, int b, int head) {
    const int kvh = head / a.group, qi = head - kvh * a.group, rb = qi / kAttendRows;
    const int2 w = a.pair_workers[(static_cast<int64_t>(b) * a.Hkv + kvh) * a.row_blocks + rb];
    return {w.x, w.y - w.x + 1, a.rows, qi - rb * kAttendRows};
}

template <typename T, int DH>
__global__ __launch_bounds__(kJoinThreads) void decode_join_kernel(const DecodeArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
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
            add_sum(m, l, v.x, v.y);
        }
        const float top = score_of_key(wave_extreme<true>(ordered_key(m))), ref = top == -INFINITY ? 0.f : top;
        l = wave_sum(l * exp2_of(m - ref));
        const float lse2 = l == 0.f ? INFINITY : ref + log2_of(l);            // +inf, no row counts: the factors below are 0
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](const float4& v, float f) { o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w); };
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (g + k * groups < parts.n) add(ahead[k], exp2_of(ahead_m[k] - lse2));
#pragma unroll 4
        for (int p = g + kAhead * groups; p < parts.n; p += groups) {
            const int64_t slot = parts.slot(p);
            add(*reinterpret_cast<const float4*>(part + slot * DH), exp2_of(ml[slot].x - lse2));
        }
        s_part[threadIdx.x] = o;
        __syncthreads();
        if (g == 0) {
#pragma unroll 8
            for (int k = 1; k < groups; ++k) {
                const float4 v = s_part[k * lanes + x];
                o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
            }
            const int64_t at = static_cast<int64_t>(b) * a.Hq + head, to = at * DH + (piece * lanes + x) * 4;
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(a.out + to * 2) = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
            else *reinterpret_cast<float4*>(a.out + to * 4) = o;
        }
        if (threadIdx.x == 0 && piece == 0) {
            const int64_t at = static_cast<int64_t>(b) * a.Hq + head;
            if (a.lse) a.lse[at] = lse2 == INFINITY ? -INFINITY : lse2 * 0.693147180559945309f;
        }
        return;
    }
    // Rows of one video: every lane has four neighbouring rows, the waves share the heads.
    __shared__ float s_lse2[1024];
    __shared__ float4 s_sum[kJoinThreads];
    const int w = static_cast<int>(blockIdx.x) - a.join_blocks, b = w / a.weight_blocks, first = w - b * a.weight_blocks;
    const int fresh = a.k_new != nullptr, n_cache = rows_before(a, b), n = min(n_cache + fresh, a.S_cap);       // rows that have a place
    if (static_cast<int64_t>(first) * kWeightRows >= n) return;
    // log2 of the heads' sums, +inf where no row counts: a.head_lanes neighbouring lanes to a head
    for (int h0 = 0; h0 < a.Hq; h0 += kJoinThreads / a.head_lanes) {
        const int h = min(h0 + static_cast<int>(threadIdx.x) / a.head_lanes, a.Hq - 1), part = threadIdx.x % a.head_lanes;
        const HeadParts parts = parts_of(a, b, h);
        float m = -INFINITY, l = 0.f;
#pragma unroll 8
        for (int p = part; p < (parts.n > 1 ? parts.n : 0); p += a.head_lanes) {
            const float2 v = ml[parts.slot(p)];
            add_sum(m, l, v.x, v.y);
        }
        for (int off = a.head_lanes / 2; off; off >>= 1) add_sum(m, l, __shfl_xor(m, off, 64), __shfl_xor(l, off, 64));
        const float lse2 = parts.n == 1 ? a.lse2[static_cast<int64_t>(b) * a.Hq + h] : m + log2_of(l);
        if (part == 0) s_lse2[h] = lse2 > -INFINITY ? lse2 : INFINITY;       // log2(0) is -inf
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
                const float z = s_lse2[h];
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
            *out = (mine < n_cache ? *out : 0.f) + total * inv;
        }
        __syncthreads();
    }
}

template <typename T, int DH, int FORM, bool STREAM>
static void launch_attention(const DecodeArgs& a, unsigned groups, hipStream_t st) {
    if (a.weight) hipLaunchKernelGGL((decode_attention_kernel<T, DH, FORM, true, STREAM>), dim3(groups), dim3(kAttendThreads), 0, st, a);
    else hipLaunchKernelGGL((decode_attention_kernel<T, DH, FORM, false, STREAM>), dim3(groups), dim3(kAttendThreads), 0, st, a);
}

// Caches of more than this many bytes are read with the streaming hint: 375 MB (4 x 4571 rows, 40 heads of 128) 91 us without, 81 with; 606 MB
// 109 and 98; a tenth of them, that the memory-side cache still holds from the call before, 16.5 and 18.1 (67 MB).
constexpr int64_t kStreamBytes = 128 << 20;

template <typename T, int DH>
static int launch_attend(DecodeArgs& a, const AttendPlan& plan, hipStream_t st) {
    const int64_t bytes = static_cast<int64_t>(a.B) * a.Hkv * a.S_cap * DH * static_cast<int64_t>(sizeof(T)) * 2;
    const unsigned groups = static_cast<unsigned>(plan.grid);
    const bool stream = bytes > kStreamBytes;
    if (!a.table) stream ? launch_attention<T, DH, kDense, true>(a, groups, st) : launch_attention<T, DH, kDense, false>(a, groups, st);
    else if (a.page_size % 16 != 0) launch_attention<T, DH, kRows, false>(a, groups, st);
    else stream ? launch_attention<T, DH, kBlocks, true>(a, groups, st) : launch_attention<T, DH, kBlocks, false>(a, groups, st);
    int rc = check_launch("decode attention");
    if (rc) return rc;
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

// The shapes that the calls and the workspace query take, NULL or the reason why not.
static const char* bad_shape(int B, int Hq, int Hkv, int64_t S_cap, int dh, int dtype) {
    if (dtype != METOK_F32 && dtype != METOK_BF16) return "unknown dtype";
    if (B < 1 || B > METOK_MAX_DECODE_BATCH) return "B must be in [1, METOK_MAX_DECODE_BATCH]";
    if (Hkv < 1 || Hq < 1 || Hq > 1024 || Hq % Hkv != 0) return "Hq must be a multiple of Hkv and at most 1024";
    if (dh != 32 && dh != 64 && dh != 128 && !(dh == 256 && dtype == METOK_BF16)) return "dh must be 32, 64, 128 or (bf16) 256";
    if (S_cap < 1 || S_cap >= INT32_MAX - 64) return "the capacity must be in [1, 2^31 - 64)";
    const int64_t pairs = static_cast<int64_t>(B) * Hkv * ((Hq / Hkv + kAttendRows - 1) / kAttendRows);
    if (pairs * (S_cap / 16 + 4) > INT32_MAX) return "too many rows";
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
    a.pair_workers = plan.joined || weight ? reinterpret_cast<int2*>(ws + plan.pair_workers) : nullptr;
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
