// Eviction by accumulated attention weight (the decoding-time counterpart of stages 2 and 3): which rows of every (layer, video)
// stay, their index list in the form of stage 3, and their weights moved along; the rows of the caches themselves are moved by stage 3's
// row mover.
//
// One workgroup selects for one (layer, video).  It reads the weights once, into registers (up to 40960 rows; longer caches are read
// again from the L2), finds the smallest weight that stays by a histogram of the leading bits of (key - smallest key), key being the
// order-preserving integer of a weight, and by ranking the few keys in the deciding bucket against each other.  Wave w holds the w-th
// sixteenth of the rows, 64 neighbouring rows an instruction, so that the place of a kept row is a population count of lane
// masks away from the number of rows that earlier waves keep: one exchange between the waves, no scan per tile.
// What bounds it is latency: a video of 4224 rows is 17 KB, and some ten barriers and round trips to LDS come one behind the other.  Kernel
// times: 28 x 1 of 4224 rows 8.8 us, 28 x 8 of up to 4096 rows 9.1, 28 x 4 of 18560 rows 21.5, two of 777 rows 6.0.
#include <algorithm>

#include "common.h"
#include "metok_decode.h"

namespace metok {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;
// Weights a thread holds: the fewest that the capacity fits.  4 x 28 selections of 18560 rows 20 and not 40: 7 us less; 28 of 4224 rows 8 and not 20:
// 2 us, 40: 10 us.
constexpr int kEvictCache = 40, kEvictMiddle = 20, kEvictFew = 8;
constexpr int kEvictBins = 2048, kEvictDigit = 11;
constexpr int kEvictList = 512;                                // keys that are ranked against each other

struct EvictArgs {
    const float* weight[METOK_MAX_LAYERS];                     // NULL: the layer is left alone
    float* weight_out[METOK_MAX_LAYERS];
    int32_t* idx[METOK_MAX_LAYERS];
    int32_t budget[METOK_MAX_LAYERS];
    const int32_t* len;                                        // [L, B]
    int32_t* new_len;                                          // [L, B]
    int64_t weight_stride;
    int B, select_blocks, S_cap, n_first, n_last;
    int2* moved;                                               // [L, B] or NULL: the row mover's tiles (see RowMoveStart)
    int rows_per_tile;
    uint32_t* clear;                                           // words that the workgroups behind the selecting ones clear
    uint64_t n_clear;
};
static_assert(sizeof(EvictArgs) <= 4096, "a kernel's arguments");

struct EvictShared {
    int hist[kEvictBins];
    uint32_t list[kEvictList];
    int scan[17];
    uint32_t low[kEvictWaves], high[kEvictWaves];
    int above[kEvictWaves], equal[kEvictWaves];
    int bucket, need, count, n_list, first_moved;
    uint32_t tau;
};

// CACHE: weights a thread holds, 0: none.
template <int CACHE>
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(const EvictArgs a) {
    __shared__ EvictShared s;
    if (static_cast<int>(blockIdx.x) >= a.select_blocks) {
        const uint64_t stride = static_cast<uint64_t>(gridDim.x - a.select_blocks) * kEvictThreads;
        for (uint64_t i = static_cast<uint64_t>(blockIdx.x - a.select_blocks) * kEvictThreads + threadIdx.x; i < a.n_clear; i += stride) a.clear[i] = 0u;
        return;
    }
    const int layer = blockIdx.x / a.B, b = blockIdx.x - layer * a.B;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float* weight = a.weight[layer];                     // may be weight_out
    const int held = a.len[blockIdx.x], n = held < 0 ? 0 : (held > a.S_cap ? a.S_cap : held);
    const int budget = a.budget[layer];
    // new_len may be len: what replaces a larger number waits until all waves have read it (below)
    if (tid == 0 && (!weight || n <= budget)) {
        a.new_len[blockIdx.x] = n;
        if (a.moved) a.moved[blockIdx.x] = make_int2(0, 0);
    }
    if (!weight) return;
    weight += static_cast<int64_t>(b) * a.weight_stride;
    float* weight_out = a.weight_out[layer] + static_cast<int64_t>(b) * a.weight_stride;
    int32_t* idx = a.idx[layer] + static_cast<int64_t>(b) * budget;
    if (n <= budget) {
        for (int i = tid; i < budget; i += kEvictThreads) idx[i] = i;
        if (weight_out != weight)
            for (int i = tid; i < n; i += kEvictThreads) weight_out[i] = weight[i];
        return;
    }

    const int lo = a.n_first, hi = n - a.n_last;               // the rows between are ranked; lo < hi since budget < n
    const int per_wave = ((n + kEvictWaves - 1) / kEvictWaves + 63) & ~63;
    const int base = wave * per_wave + lane, steps = per_wave >> 6;        // the lane's rows are base, base + 64, ...
    float own[CACHE ? CACHE : 1];
    if constexpr (CACHE != 0) {
#pragma unroll
        for (int i = 0; i < CACHE; ++i) own[i] = weight[min(base + (i < steps ? i : 0) * 64, n - 1)];
    }
    // visit(key) for the rows that are ranked
    auto for_each = [&](auto visit) {
        if constexpr (CACHE != 0) {
#pragma unroll
            for (int i = 0; i < CACHE; ++i) {
                const int j = base + i * 64;
                if (i < steps && j >= lo && j < hi) visit(ordered_key(own[i]));
            }
        } else {
            for (int i = 0; i < steps; ++i) {
                const int j = base + i * 64;
                if (j >= lo && j < hi) visit(ordered_key(weight[j]));
            }
        }
    };

    // tau: the smallest key that stays, and how many rows equal to it do
    int need = budget - a.n_first - a.n_last;                  // 0 <= need < hi - lo
    uint32_t tau = 0xffffffffu;
    int equal_kept = 0;
    const bool ranked_stay = need > 0;
    if (ranked_stay) {
        uint32_t kmin = 0xffffffffu, kmax = 0u;
        for_each([&](uint32_t k) { kmin = min(kmin, k); kmax = max(kmax, k); });
        kmin = wave_extreme<false>(kmin);
        kmax = wave_extreme<true>(kmax);
        if (lane == 0) { s.low[wave] = kmin; s.high[wave] = kmax; }
        s.hist[tid] = 0; s.hist[tid + kEvictThreads] = 0;
        if (tid == 0) s.n_list = 0;
        lds_barrier();
        kmin = wave_extreme<false>(s.low[lane & (kEvictWaves - 1)]);
        kmax = wave_extreme<true>(s.high[lane & (kEvictWaves - 1)]);
        const uint32_t range = kmax - kmin;
        int top = range ? 32 - __clz(static_cast<int>(range)) : 0;         // bits of a distance
        uint32_t prefix = 0;                                               // leading bits of the deciding distance, above bit `top`
        int count = hi - lo;                                               // rows that share them
        while (top > 0 && count > kEvictList) {
            const int bits = min(top, kEvictDigit), shift = top - bits;
            // a run of equal digits costs a thread one addition: weights that were never raised are all the same
            int digit = -1, run = 0;
            for_each([&](uint32_t k) {
                const uint32_t d = k - kmin;
                if (top >= 32 || (d >> top) == prefix) {
                    const int x = static_cast<int>((d >> shift) & ((1u << bits) - 1));
                    if (x != digit) {
                        if (run) atomicAdd(&s.hist[digit], run);
                        digit = x; run = 0;
                    }
                    ++run;
                }
            });
            if (run) atomicAdd(&s.hist[digit], run);
            lds_barrier();
            // from the top: thread t has bins 2047 - 2 t and 2046 - 2 t, and leaves them empty
            const int b0 = kEvictBins - 1 - 2 * tid, v0 = s.hist[b0], v1 = s.hist[b0 - 1];
            s.hist[b0] = 0; s.hist[b0 - 1] = 0;
            int all;
            const int before = block_exclusive_scan_lds(v0 + v1, s.scan, &all);
            if (before < need && before + v0 >= need) { s.bucket = b0; s.need = need - before; s.count = v0; }
            else if (before + v0 < need && before + v0 + v1 >= need) { s.bucket = b0 - 1; s.need = need - before - v0; s.count = v1; }
            lds_barrier();
            prefix = (top >= 32 ? 0u : prefix << bits) | static_cast<uint32_t>(s.bucket);
            need = s.need; count = s.count;
            top = shift;
        }
        if (top == 0) {                                                    // every bit is decided: the rows left are equal
            tau = kmin + prefix;
            equal_kept = need;
        } else {
            for_each([&](uint32_t k) {
                if (top >= 32 || ((k - kmin) >> top) == prefix) s.list[atomicAdd(&s.n_list, 1)] = k;      // count of them, at most kEvictList
            });
            lds_barrier();
            if (tid < count) {
                const uint32_t k = s.list[tid];
                int above = 0, equal = 0;
#pragma unroll 8
                for (int i = 0; i < count; ++i) {
                    const uint32_t o = s.list[i];
                    above += o > k;
                    equal += o == k;
                }
                if (above < need && above + equal >= need) { s.tau = k; s.need = need - above; }       // equal keys write the same
            }
            lds_barrier();
            tau = s.tau;
            equal_kept = s.need;
        }
    }
    if (tid == 0) s.first_moved = 0x7fffffff;                  // behind a barrier below

    // Places.  A row stays if it is not ranked, above tau, or among the first equal_kept rows equal to tau.
    auto kind = [&](int j, float w, bool& above, bool& equal) {
        const bool in = j < n, ranked = j >= lo && j < hi;
        const uint32_t k = ordered_key(w);
        above = in && (!ranked || (ranked_stay && k > tau));
        equal = in && ranked && k == tau;
    };
    const unsigned long long below = (1ull << lane) - 1;
    int moved = 0x7fffffff;                                    // first place of this wave that takes a row from behind it
    if constexpr (CACHE != 0) {
        // the kinds of the lane's rows as bits: asked for twice
        unsigned long long is_above = 0, is_equal = 0;
        int above_here = 0, equal_here = 0;
#pragma unroll
        for (int i = 0; i < CACHE; ++i)
            if (i < steps) {
                bool above, equal;
                kind(base + i * 64, own[i], above, equal);
                is_above |= static_cast<unsigned long long>(above) << i;
                is_equal |= static_cast<unsigned long long>(equal) << i;
                above_here += __popcll(__ballot(above));
                equal_here += __popcll(__ballot(equal));
            }
        if (lane == 0) { s.above[wave] = above_here; s.equal[wave] = equal_here; }
        __syncthreads();                                                   // all weights are in registers: weight_out may be weight
        const int sums_above = row16_inclusive_scan(s.above[lane & 15]), sums_equal = row16_inclusive_scan(s.equal[lane & 15]);
        int equals = __builtin_amdgcn_readlane(sums_equal, wave) - equal_here;
        int place = __builtin_amdgcn_readlane(sums_above, wave) - above_here + min(equals, equal_kept);
#pragma unroll
        for (int i = 0; i < CACHE; ++i)
            if (i < steps) {
                const int j = base + i * 64;
                const bool equal = (is_equal >> i) & 1ull;
                const unsigned long long eq = __ballot(equal);
                const bool stays = ((is_above >> i) & 1ull) || (equal && equals + __popcll(eq & below) < equal_kept);
                const unsigned long long st = __ballot(stays);
                const int at = place + __popcll(st & below);
                if (stays) {
                    idx[at] = j;
                    weight_out[at] = own[i];
                    if (at != j) moved = min(moved, at);
                }
                place += __popcll(st);
                equals += __popcll(eq);
            }
    } else {
        // 1024 rows a step, in order: a row's weight moves to its own place or before it, never onto one that is still to be read
        int place = 0, equals = 0;
        for (int j0 = 0; j0 < n; j0 += kEvictThreads) {
            const int j = j0 + tid;
            const float w = weight[min(j, n - 1)];
            bool above, equal;
            kind(j, w, above, equal);
            const unsigned long long eq = __ballot(equal), ab = __ballot(above);
            __syncthreads();
            if (lane == 0) { s.above[wave] = __popcll(ab); s.equal[wave] = __popcll(eq); }
            __syncthreads();
            int above_before = 0, equal_before = 0, above_all = 0, equal_all = 0;
            for (int x = 0; x < kEvictWaves; ++x) {
                if (x == wave) { above_before = above_all; equal_before = equal_all; }
                above_all += s.above[x]; equal_all += s.equal[x];
            }
            const int equal_rank = equals + equal_before + __popcll(eq & below);
            if (above || (equal && equal_rank < equal_kept)) {
                const int at = place + above_before + __popcll(ab & below) + (min(equal_rank, equal_kept) - min(equals, equal_kept));
                idx[at] = j;
                weight_out[at] = w;
                if (at != j) moved = min(moved, at);
            }
            place += above_all + (min(equals + equal_all, equal_kept) - min(equals, equal_kept));
            equals += equal_all;
        }
        __syncthreads();
    }
    if (tid == 0) a.new_len[blockIdx.x] = budget;             // behind a barrier that every wave reaches with n in use
    if (a.moved) {
        const int first = static_cast<int>(wave_extreme<false>(static_cast<uint32_t>(moved)));
        if (lane == 0 && first != 0x7fffffff) atomicMin(&s.first_moved, first);
        lds_barrier();
        if (tid == 0) {
            const int tile = s.first_moved == 0x7fffffff ? 0 : s.first_moved / a.rows_per_tile;
            const int tiles = s.first_moved == 0x7fffffff ? 0 : (budget + a.rows_per_tile - 1) / a.rows_per_tile - tile;
            a.moved[blockIdx.x] = make_int2(tile, tiles);
        }
    }
}

static int launch_select(EvictArgs& a, int L, uint32_t* clear, size_t n_clear, hipStream_t st) {
    a.clear = clear; a.n_clear = n_clear;
    a.select_blocks = L * a.B;
    const size_t blocks = (n_clear + kEvictThreads * 4 - 1) / (kEvictThreads * 4);
    const dim3 grid(static_cast<unsigned>(a.select_blocks + (blocks < 256 ? blocks : 256)));
    if (a.S_cap <= kEvictFew * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<kEvictFew>, grid, dim3(kEvictThreads), 0, st, a);
    else if (a.S_cap <= kEvictMiddle * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<kEvictMiddle>, grid, dim3(kEvictThreads), 0, st, a);
    else if (a.S_cap <= kEvictCache * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<kEvictCache>, grid, dim3(kEvictThreads), 0, st, a);
    else hipLaunchKernelGGL(evict_select_kernel<0>, grid, dim3(kEvictThreads), 0, st, a);
    return check_launch("evict select");
}

// Checks what the selection takes and fills in its arguments.
static int select_args(EvictArgs* a, const float* const* weight, float* const* weight_out, int64_t weight_stride, int L, int B, int64_t S_cap,
                       const int32_t* len, const int32_t* budget, int n_first, int n_last, int32_t* const* idx, int32_t* new_len) {
    if (L < 1 || L > METOK_MAX_LAYERS) return fail(METOK_ERR_INVALID_ARG, "L must be in [1, %d], got %d", METOK_MAX_LAYERS, L);
    if (B < 1 || B > METOK_MAX_DECODE_BATCH) return fail(METOK_ERR_INVALID_ARG, "B must be in [1, %d], got %d", METOK_MAX_DECODE_BATCH, B);
    if (S_cap < 1 || S_cap > INT32_MAX - 4096) return fail(METOK_ERR_INVALID_ARG, "the capacity must be in [1, 2^31 - 4096)");
    if (!weight || !weight_out || !len || !budget || !idx || !new_len) return fail(METOK_ERR_INVALID_ARG, "weight, weight_out, len, budget, idx and new_len must not be NULL");
    if ((reinterpret_cast<uintptr_t>(len) | reinterpret_cast<uintptr_t>(new_len)) & 3u) return fail(METOK_ERR_INVALID_ARG, "len and new_len must be 4-byte aligned");
    if (n_first < 0 || n_last < 0) return fail(METOK_ERR_INVALID_ARG, "n_first and n_last must not be negative");
    if (weight_stride < S_cap) return fail(METOK_ERR_INVALID_ARG, "weight_stride must be at least the capacity");
    const size_t lens = static_cast<size_t>(L) * B;
    // what is read and written, by address: nothing written may overlap anything else
    struct Span { uintptr_t from, to; bool written; } spans[3 * METOK_MAX_LAYERS + 2];
    int n_spans = 0;
    auto uses = [&](const void* p, size_t words, bool written) {
        const uintptr_t from = reinterpret_cast<uintptr_t>(p);
        spans[n_spans++] = {from, from + 4 * words, written};
    };
    uses(new_len, lens, true);
    if (len != new_len) uses(len, lens, false);
    const size_t span = static_cast<size_t>(B - 1) * weight_stride + S_cap;
    for (int l = 0; l < METOK_MAX_LAYERS; ++l) {
        a->weight[l] = l < L ? weight[l] : nullptr;
        a->weight_out[l] = nullptr; a->idx[l] = nullptr; a->budget[l] = 0;
        if (!a->weight[l]) continue;
        const float* w = weight[l];
        float* o = weight_out[l];
        if (!o || !idx[l] || ((reinterpret_cast<uintptr_t>(w) | reinterpret_cast<uintptr_t>(o) | reinterpret_cast<uintptr_t>(idx[l])) & 3u))
            return fail(METOK_ERR_INVALID_ARG, "layer %d: NULL or misaligned weight, weight_out or idx", l);
        if (budget[l] < 1 || budget[l] > S_cap) return fail(METOK_ERR_INVALID_ARG, "budget[%d] = %d outside [1, capacity]", l, budget[l]);
        if (static_cast<int64_t>(n_first) + n_last > budget[l])
            return fail(METOK_ERR_INVALID_ARG, "n_first + n_last = %lld is more than budget[%d] = %d", static_cast<long long>(n_first) + n_last, l, budget[l]);
        a->weight_out[l] = o; a->idx[l] = idx[l]; a->budget[l] = budget[l];
        uses(o, span, true);
        if (o != w) uses(w, span, false);
        uses(idx[l], static_cast<size_t>(B) * budget[l], true);
    }
    std::sort(spans, spans + n_spans, [](const Span& x, const Span& y) { return x.from < y.from; });
    uintptr_t used = 0, written = 0;                           // ends of what lies before
    for (int i = 0; i < n_spans; ++i) {
        if (spans[i].from < (spans[i].written ? used : written))
            return fail(METOK_ERR_INVALID_ARG, "one of weight_out, idx and new_len overlaps another of them, a weight that is not its own, or len");
        used = std::max(used, spans[i].to);
        if (spans[i].written) written = std::max(written, spans[i].to);
    }
    a->len = len; a->new_len = new_len; a->weight_stride = weight_stride;
    a->moved = nullptr; a->rows_per_tile = 1;
    a->B = B; a->S_cap = static_cast<int>(S_cap); a->n_first = n_first; a->n_last = n_last;
    return METOK_OK;
}

static size_t moved_bytes(int L, int B) { return round_up(static_cast<size_t>(L) * B * sizeof(int2), 256); }

// What the row mover runs in place of its own start, all other arguments checked: the selection clears the mover's words, too.
struct SelectStart { EvictArgs* args; int L; size_t workspace_bytes, need; };
static int start_with_selection(void* context, uint32_t* words, size_t n_words, hipStream_t st) {
    const SelectStart* s = static_cast<const SelectStart*>(context);
    if (s->workspace_bytes < s->need) return fail(METOK_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", s->need, s->workspace_bytes);
    return launch_select(*s->args, s->L, words, n_words, st);
}

static int evict_impl(void* const* k, void* const* v, int L, int B, int Hkv, int64_t S_cap, int dh, int dtype,
                      const int32_t* page_table, int page_size, int pages_per_seq, int64_t n_pages,
                      const float* const* weight, float* const* weight_out, int64_t weight_stride, const int32_t* len, const int32_t* budget,
                      int n_first, int n_last, int32_t* const* idx, int32_t* new_len, void* workspace, size_t workspace_bytes, void* stream) {
    EvictArgs a;
    int rc = select_args(&a, weight, weight_out, weight_stride, L, B, S_cap, len, budget, n_first, n_last, idx, new_len);
    if (rc) return rc;
    const size_t mover = metok_kv_compact_workspace_bytes(L, B, Hkv, S_cap, dh, dtype);        // 0: the mover refuses the shape below
    if (mover) {
        a.moved = reinterpret_cast<int2*>(static_cast<char*>(workspace) + mover);
        a.rows_per_tile = row_move_geom(static_cast<int64_t>(dh) * static_cast<int64_t>(dtype_size(dtype))).rows_per_tile;
    }
    SelectStart context{&a, L, workspace_bytes, mover + moved_bytes(L, B)};
    const RowMoveStart start{start_with_selection, &context, a.moved};
    return compact_layers(k, v, L, B, Hkv, S_cap, dh, dtype, a.idx, a.budget, nullptr, page_table, page_size, pages_per_seq, n_pages,
                          workspace, workspace_bytes, stream, &start);
}

}  // namespace metok

using namespace metok;

extern "C" size_t metok_kv_evict_workspace_bytes(int L, int B, int Hkv, int64_t S_cap, int dh, int dtype) {
    if (B > METOK_MAX_DECODE_BATCH || S_cap > INT32_MAX - 4096) return 0;
    const size_t mover = metok_kv_compact_workspace_bytes(L, B, Hkv, S_cap, dh, dtype);
    return mover ? mover + moved_bytes(L, B) : 0;
}

extern "C" int metok_kv_evict(void* const* k_layers, void* const* v_layers, int L, int B, int Hkv, int64_t S_cap, int dh, int dtype,
                              const float* const* weight, float* const* weight_out, int64_t weight_stride,
                              const int32_t* len, const int32_t* budget, int n_first, int n_last,
                              int32_t* const* idx, int32_t* new_len,
                              void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    return evict_impl(k_layers, v_layers, L, B, Hkv, S_cap, dh, dtype, nullptr, 0, 0, 0, weight, weight_out, weight_stride, len, budget,
                      n_first, n_last, idx, new_len, workspace, workspace_bytes, stream);
}

extern "C" int metok_kv_evict_paged(void* const* k_pools, void* const* v_pools, int L, int B, int Hkv,
                                    int64_t n_pages_pool, int page_size, int dh, int dtype,
                                    const int32_t* page_table, int pages_per_seq,
                                    const float* const* weight, float* const* weight_out, int64_t weight_stride,
                                    const int32_t* len, const int32_t* budget, int n_first, int n_last,
                                    int32_t* const* idx, int32_t* new_len,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    if (!page_table || (reinterpret_cast<uintptr_t>(page_table) & 3u)) return fail(METOK_ERR_INVALID_ARG, "page_table NULL or misaligned");
    if (page_size < 1 || pages_per_seq < 1 || n_pages_pool < 1 || n_pages_pool > INT32_MAX)
        return fail(METOK_ERR_INVALID_ARG, "page_size, pages_per_seq and n_pages_pool must be positive");
    return evict_impl(k_pools, v_pools, L, B, Hkv, static_cast<int64_t>(pages_per_seq) * page_size, dh, dtype, page_table, page_size, pages_per_seq,
                      n_pages_pool, weight, weight_out, weight_stride, len, budget, n_first, n_last, idx, new_len, workspace, workspace_bytes, stream);
}

extern "C" int metok_kv_evict_select(const float* const* weight, float* const* weight_out, int64_t weight_stride,
                                     int L, int B, int64_t S_cap, const int32_t* len, const int32_t* budget, int n_first, int n_last,
                                     int32_t* const* idx, int32_t* new_len, void* stream) {
    clear_error();
    EvictArgs a;
    const int rc = select_args(&a, weight, weight_out, weight_stride, L, B, S_cap, len, budget, n_first, n_last, idx, new_len);
    return rc ? rc : launch_select(a, L, nullptr, 0, static_cast<hipStream_t>(stream));
}
