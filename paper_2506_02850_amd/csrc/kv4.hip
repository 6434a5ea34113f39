// Rows into a KV cache of 4 bits and back (include/metok_qkv.h): the compacted rows of stage 3 (Sec. 3.3) or the rows of a chunk, gathered, put into 4 bits and
// stored in one pass; and rows of such a cache as the values they stand for.
//
// Both move bytes and compute little: a row of 128 elements of K and V in bf16 is 512 bytes on one side and 136 on the other.  8 x 36992 rows of 4 heads: 131 us
// into 4 bits, 5.9 TB/s; a few thousand rows 5 to 8 us, which are the launch and the loads that wait for each other (count and start, index, row).
#include "kv4.h"

namespace metok {

struct Rows4Args {
    const char *k, *v;           // pack: the source; unpack: the 4-bit cache
    char *k_to, *v_to;           // pack: the 4-bit cache; unpack: the outputs
    const int32_t *idx, *count, *start, *table;      // count: of unpack the lengths; start: of unpack the first rows
    int64_t n, S_rows;           // rows asked for at most; rows of a slab of the side that is not in 4 bits
    int Hkv, S_cap;              // capacity of the 4-bit side
    int page_size, pages_per_seq, n_pages;
};

// Rows of more bytes than this are read by a pack, written by an unpack, with the streaming hint: 8 x 36992 rows of 4 heads of 128 in bf16, 606 MB, 131 us with it and 163
// without into 4 bits, 108 to 137 and 126 to 139 back; 9333 rows, 19 MB, 9.0 and 7.9 (the memory-side cache has them still), 5.5 and 6.6.
constexpr int64_t kStreamPack = 128 << 20, kStreamUnpack = 16 << 20;
constexpr int kRows4Threads = 256, kRows4Waves = kRows4Threads / 64;

// The block of 16 rows of the 4-bit cache that logical row j of a video lies in; -1: no such page.  0 <= j < S_cap.
__device__ __forceinline__ int64_t block_of(const Rows4Args& a, int b, int h, int j) {
    if (!a.table) return (static_cast<int64_t>(b) * a.Hkv + h) * (a.S_cap / kBlockRows) + j / kBlockRows;
    const int at = j / a.page_size, page = a.table[static_cast<int64_t>(b) * a.pages_per_seq + at];
    if (page < 0 || page >= a.n_pages) return -1;
    return (static_cast<int64_t>(page) * a.Hkv + h) * (a.page_size / kBlockRows) + (j - at * a.page_size) / kBlockRows;
}

// N neighbouring words, with the streaming hint or without.
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
template <int N, bool STREAM, typename V> __device__ __forceinline__ void load_run(uint32_t (&w)[N], const V* p) {
    V v;
    if constexpr (STREAM) v = __builtin_nontemporal_load(p);
    else v = *p;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if constexpr (N == 1) w[j] = v; else w[j] = v[j];
    }
}
template <int N, bool STREAM> __device__ __forceinline__ void load_run(uint32_t (&w)[N], const char* p) {
    if constexpr (N == 4) load_run<N, STREAM>(w, reinterpret_cast<const u32x4_t*>(p));
    else if constexpr (N == 2) load_run<N, STREAM>(w, reinterpret_cast<const u32x2_t*>(p));
    else load_run<N, STREAM>(w, reinterpret_cast<const uint32_t*>(p));
}
template <bool STREAM, typename V> __device__ __forceinline__ void store_run(V* p, V v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// E elements (2, 4, 8) of type T at p, as floats.
template <typename T, int E, bool STREAM> __device__ __forceinline__ void load_elements(float (&x)[E], const char* p) {
    constexpr int WORDS = E * static_cast<int>(sizeof(T)) / 4, N = WORDS < 4 ? WORDS : 4;
#pragma unroll
    for (int k = 0; k < WORDS; k += N) {
        uint32_t w[N];
        load_run<N, STREAM>(w, p + 4 * k);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (sizeof(T) == 2) { x[2 * (k + j)] = bf16_lo(w[j]); x[2 * (k + j) + 1] = bf16_hi(w[j]); }
            else x[k + j] = __uint_as_float(w[j]);
        }
    }
}

template <int BYTES> __device__ __forceinline__ void store_bytes(char* p, uint32_t v) {
    if constexpr (BYTES == 4) *reinterpret_cast<uint32_t*>(p) = v;
    else if constexpr (BYTES == 2) *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(v);
    else *reinterpret_cast<uint8_t*>(p) = static_cast<uint8_t>(v);
}
template <int BYTES> __device__ __forceinline__ uint32_t load_bytes(const char* p) {
    if constexpr (BYTES == 4) return *reinterpret_cast<const uint32_t*>(p);
    else if constexpr (BYTES == 2) return *reinterpret_cast<const uint16_t*>(p);
    else return *reinterpret_cast<const uint8_t*>(p);
}

// A wave per block of the cache, video, kv head and K or V.  Lane (c, r): elements r w / 16 .. of rows 4 c .. 4 c + 3, so that 16 lanes have whole rows
// and a lane's codes of the four rows are what V keeps beside each other.  A block has one writer; where some of its rows are not to be
// written, the others are stored byte by byte as far as they mix.
template <typename T, int DH, bool STREAM>
__global__ __launch_bounds__(kRows4Threads) void pack4_kernel(const Rows4Args a) {
    using F = Block4<DH>;
    constexpr int E = F::kWidth / 16, EB = F::kRunBytes;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
    const int h = blockIdx.y % a.Hkv, which = blockIdx.y / a.Hkv, b = blockIdx.z;
    const int count = static_cast<int>(min(static_cast<int64_t>(a.count ? max(a.count[b], 0) : INT32_MAX), a.n));
    const int start = a.start ? max(a.start[b], 0) : 0;
    const int64_t first = (static_cast<int64_t>(start / kBlockRows) + blockIdx.x * kRows4Waves + wave) * kBlockRows;       // row of the cache
    if (first >= min(static_cast<int64_t>(start) + count, static_cast<int64_t>(a.S_cap))) return;
    const int64_t block = block_of(a, b, h, static_cast<int>(first));
    if (block < 0) return;
    const char* from = (which ? a.v : a.k) + (static_cast<int64_t>(b) * a.Hkv + h) * a.S_rows * DH * static_cast<int64_t>(sizeof(T));
    char* to = (which ? a.v_to : a.k_to) + block * F::kBytes;

    int64_t src[4];
    bool there[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t at = first + 4 * c + i - start;
        there[i] = at >= 0 && at < count;
        src[i] = there[i] ? (a.idx ? a.idx[static_cast<int64_t>(b) * a.n + at] : at) : 0;
        there[i] = there[i] && src[i] >= 0 && src[i] < a.S_rows;
        if (!there[i]) src[i] = 0;
    }
    const bool all = there[0] && there[1] && there[2] && there[3];
#pragma unroll
    for (int p = 0; p < F::kPieces; ++p) {
        float x[4][E];
#pragma unroll
        for (int i = 0; i < 4; ++i) load_elements<T, E, STREAM>(x[i], from + (src[i] * DH + p * F::kWidth + r * E) * static_cast<int64_t>(sizeof(T)));
        uint32_t codes[4], scales = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float m = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) m = fmaxf(m, fabsf(x[i][e]));
            const float s = scale_of(lanes_max<32 / E>(m));
            codes[i] = put_codes<0>(0u, x[i][0], x[i][1], s);
            if constexpr (E >= 4) codes[i] = put_codes<1>(codes[i], x[i][2], x[i][3], s);
            if constexpr (E >= 8) { codes[i] = put_codes<2>(codes[i], x[i][4], x[i][5], s); codes[i] = put_codes<3>(codes[i], x[i][6], x[i][7], s); }
            scales |= scale_byte(s) << (8 * i);
        }
        char* piece = to + p * F::kPieceBytes;
        if (which == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (there[i]) store_bytes<EB>(piece + (4 * c + i) * F::kRowBytes + r * EB, codes[i]);
        } else {
            char* run = piece + c * 2 * F::kWidth + r * 4 * EB;
            if (all) {
                if constexpr (EB == 4) *reinterpret_cast<uint4*>(run) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
                else if constexpr (EB == 2) *reinterpret_cast<uint2*>(run) = make_uint2((codes[0] & 0xffffu) | codes[1] << 16, (codes[2] & 0xffffu) | codes[3] << 16);
                else *reinterpret_cast<uint32_t*>(run) = (codes[0] & 0xffu) | (codes[1] & 0xffu) << 8 | (codes[2] & 0xffu) << 16 | codes[3] << 24;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (there[i]) store_bytes<EB>(run + i * EB, codes[i]);
            }
        }
        if ((r * E) % 32 == 0) {
            char* at = to + F::kScales + p * 16 * F::kGroups + c * 4 * F::kGroups + r * E / 32 * 4;
            if (all) *reinterpret_cast<uint32_t*>(at) = scales;
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (there[i]) at[i] = static_cast<char>(scales >> (8 * i));
            }
        }
    }
}

// A wave per 16 rows of the output, lanes as above.
template <typename T, int DH, bool STREAM>
__global__ __launch_bounds__(kRows4Threads) void unpack4_kernel(const Rows4Args a) {
    using F = Block4<DH>;
    constexpr int E = F::kWidth / 16, EB = F::kRunBytes;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
    const int h = blockIdx.y % a.Hkv, which = blockIdx.y / a.Hkv, b = blockIdx.z;
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * kRows4Waves + wave) * 16;
    if (first >= a.n) return;
    const int len = min(max(a.count[b], 0), a.S_cap), start = a.start ? max(a.start[b], 0) : 0;
    const char* from = which ? a.v : a.k;
    char* to = (which ? a.v_to : a.k_to) + (static_cast<int64_t>(b) * a.Hkv + h) * a.S_rows * DH * static_cast<int64_t>(sizeof(T));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t at = first + 4 * c + i;
        if (at >= a.n) continue;
        const int64_t row = a.idx ? a.idx[static_cast<int64_t>(b) * a.n + at] : start + at;
        if (row < 0 || row >= len) continue;
        const int64_t block = block_of(a, b, h, static_cast<int>(row));
        if (block < 0) continue;
        const int in = static_cast<int>(row) % kBlockRows;
        const char* src = from + block * F::kBytes;
#pragma unroll
        for (int p = 0; p < F::kPieces; ++p) {
            const char* piece = src + p * F::kPieceBytes;
            const uint32_t w = load_bytes<EB>(which ? piece + (in >> 2) * 2 * F::kWidth + r * 4 * EB + (in & 3) * EB : piece + in * F::kRowBytes + r * EB);
            const float s = scale_from(load_bytes<1>(src + F::kScales + p * 16 * F::kGroups + (in >> 2) * 4 * F::kGroups + r * E / 32 * 4 + (in & 3)));
            uint32_t y[E / 2];
            y[0] = take_codes<0>(w, s);
            if constexpr (E >= 4) y[1] = take_codes<1>(w, s);
            if constexpr (E >= 8) { y[2] = take_codes<2>(w, s); y[3] = take_codes<3>(w, s); }
            char* out = to + (at * DH + p * F::kWidth + r * E) * static_cast<int64_t>(sizeof(T));
            auto lo = [](uint32_t two) { return two << 16; };
            auto hi = [](uint32_t two) { return two & 0xffff0000u; };
            if constexpr (sizeof(T) == 2) {
                if constexpr (E == 8) store_run<STREAM>(reinterpret_cast<u32x4_t*>(out), u32x4_t{y[0], y[1], y[2], y[3]});
                else if constexpr (E == 4) store_run<STREAM>(reinterpret_cast<u32x2_t*>(out), u32x2_t{y[0], y[1]});
                else store_run<STREAM>(reinterpret_cast<uint32_t*>(out), y[0]);
            } else if constexpr (E == 2) store_run<STREAM>(reinterpret_cast<u32x2_t*>(out), u32x2_t{lo(y[0]), hi(y[0])});
            else {
                store_run<STREAM>(reinterpret_cast<u32x4_t*>(out), u32x4_t{lo(y[0]), hi(y[0]), lo(y[1]), hi(y[1])});
                if constexpr (E == 8) store_run<STREAM>(reinterpret_cast<u32x4_t*>(out) + 1, u32x4_t{lo(y[2]), hi(y[2]), lo(y[3]), hi(y[3])});
            }
        }
    }
}

template <typename T, int DH> static int launch_rows4(bool pack, const Rows4Args& a, int B, hipStream_t st) {
    // the rows may begin inside a block of the cache
    const int64_t waves = pack ? (a.n + kBlockRows - 1 + kBlockRows - 1) / kBlockRows : (a.n + 15) / 16;
    const dim3 grid(static_cast<unsigned>((waves + kRows4Waves - 1) / kRows4Waves), static_cast<unsigned>(2 * a.Hkv), static_cast<unsigned>(B));
    const int64_t bytes = 2 * static_cast<int64_t>(B) * a.Hkv * a.n * DH * static_cast<int64_t>(sizeof(T));       // of the rows that are not in 4 bits
    const bool stream = bytes > (pack ? kStreamPack : kStreamUnpack);
    const dim3 threads(kRows4Threads);
    if (pack && stream) hipLaunchKernelGGL((pack4_kernel<T, DH, true>), grid, threads, 0, st, a);
    else if (pack) hipLaunchKernelGGL((pack4_kernel<T, DH, false>), grid, threads, 0, st, a);
    else if (stream) hipLaunchKernelGGL((unpack4_kernel<T, DH, true>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((unpack4_kernel<T, DH, false>), grid, threads, 0, st, a);
    return check_launch(pack ? "pack rows" : "unpack rows");
}

static int dispatch_rows4(bool pack, const Rows4Args& a, int B, int dh, int dtype, void* stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == METOK_BF16) {
        if (dh == 32) return launch_rows4<bf16_t, 32>(pack, a, B, st);
        if (dh == 64) return launch_rows4<bf16_t, 64>(pack, a, B, st);
        if (dh == 128) return launch_rows4<bf16_t, 128>(pack, a, B, st);
        return launch_rows4<bf16_t, 256>(pack, a, B, st);
    }
    if (dh == 32) return launch_rows4<float, 32>(pack, a, B, st);
    if (dh == 64) return launch_rows4<float, 64>(pack, a, B, st);
    if (dh == 128) return launch_rows4<float, 128>(pack, a, B, st);
    return launch_rows4<float, 256>(pack, a, B, st);
}

constexpr int64_t kMostRows4 = INT32_MAX - 64, kMostAsked4 = 1 << 29;        // rows of a video are below; rows of a call (a grid has fewer than 2^32 threads)

// What the four calls share.  rows: of a slab of the side that is not in 4 bits.
static const char* bad_rows4(int B, int Hkv, int64_t rows, int64_t n, int64_t S_cap, int dh, int dtype) {
    if (dtype != METOK_F32 && dtype != METOK_BF16) return "unknown dtype";
    if (B < 1 || B > METOK_MAX_DECODE_BATCH) return "B must be in [1, METOK_MAX_DECODE_BATCH]";
    if (Hkv < 1 || Hkv > 1024) return "Hkv must be in [1, 1024]";
    if (dh != 32 && dh != 64 && dh != 128 && dh != 256) return "dh must be 32, 64, 128 or 256";
    if (S_cap < kBlockRows || S_cap % kBlockRows != 0 || S_cap >= kMostRows4) return "the capacity must be a multiple of 16 in [16, 2^31 - 64)";
    if (rows < 1 || rows >= kMostRows4) return "the rows of a video must be in [1, 2^31 - 64)";
    if (n < 1 || n > kMostAsked4) return "n must be in [1, 2^29]";
    return nullptr;
}
static int pack_impl(const void* k, const void* v, int B, int Hkv, int64_t S_src, int dh, int dtype, const int32_t* idx, int64_t n, const int32_t* count,
                     void* k_cache, void* v_cache, int64_t S_cap, size_t cache_bytes, const int32_t* table, int64_t n_pages, int page_size, int pages_per_seq,
                     const int32_t* start, void* stream) {
    if (const char* why = bad_rows4(B, Hkv, S_src, n, S_cap, dh, dtype)) return fail(METOK_ERR_INVALID_ARG, "%s", why);
    if (!k || !v || !k_cache || !v_cache) return fail(METOK_ERR_INVALID_ARG, "k, v and the caches must not be NULL");
    if (!aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache)) return fail(METOK_ERR_INVALID_ARG, "k, v and the caches must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(idx) | reinterpret_cast<uintptr_t>(count) | reinterpret_cast<uintptr_t>(start)) & 3u)
        return fail(METOK_ERR_INVALID_ARG, "idx, count and start must be 4-byte aligned");
    if (!idx && n > S_src) return fail(METOK_ERR_INVALID_ARG, "n must be at most S_src where no idx is given");
    const size_t source = static_cast<size_t>(B) * Hkv * S_src * dh * dtype_size(dtype);
    const Span spans[] = {{"the K cache", k_cache, cache_bytes}, {"the V cache", v_cache, cache_bytes}, {"k", k, source}, {"v", v, source},
                          {"idx", idx, static_cast<size_t>(B) * n * 4}, {"count", count, static_cast<size_t>(B) * 4}, {"start", start, static_cast<size_t>(B) * 4},
                          {"page_table", table, static_cast<size_t>(B) * pages_per_seq * 4}};
    if (int rc = check_spans(spans, 2, sizeof(spans) / sizeof(spans[0]))) return rc;
    Rows4Args a{static_cast<const char*>(k), static_cast<const char*>(v), static_cast<char*>(k_cache), static_cast<char*>(v_cache), idx, count, start, table,
                n, S_src, Hkv, static_cast<int>(S_cap), page_size, pages_per_seq, static_cast<int>(n_pages)};
    return dispatch_rows4(true, a, B, dh, dtype, stream);
}

static int unpack_impl(const void* k_cache, const void* v_cache, int B, int Hkv, int64_t S_cap, size_t cache_bytes, int dh,
                       const int32_t* table, int64_t n_pages, int page_size, int pages_per_seq, const int32_t* len, const int32_t* first, const int32_t* idx, int64_t n,
                       void* k_out, void* v_out, int64_t S_out, int dtype, void* stream) {
    if (const char* why = bad_rows4(B, Hkv, S_out, n, S_cap, dh, dtype)) return fail(METOK_ERR_INVALID_ARG, "%s", why);
    if (!k_cache || !v_cache || !k_out || !v_out || !len) return fail(METOK_ERR_INVALID_ARG, "the caches, len and the outputs must not be NULL");
    if (!aligned16(k_out) || !aligned16(v_out) || !aligned16(k_cache) || !aligned16(v_cache))
        return fail(METOK_ERR_INVALID_ARG, "the caches and the outputs must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(idx) | reinterpret_cast<uintptr_t>(len) | reinterpret_cast<uintptr_t>(first)) & 3u)
        return fail(METOK_ERR_INVALID_ARG, "idx, len and first must be 4-byte aligned");
    if (first && idx) return fail(METOK_ERR_INVALID_ARG, "first and idx do not go together");
    if (n > S_out) return fail(METOK_ERR_CAPACITY, "n must be at most S_out");
    const size_t out = static_cast<size_t>(B) * Hkv * S_out * dh * dtype_size(dtype);
    const Span spans[] = {{"k_out", k_out, out}, {"v_out", v_out, out}, {"the K cache", k_cache, cache_bytes}, {"the V cache", v_cache, cache_bytes},
                          {"idx", idx, static_cast<size_t>(B) * n * 4}, {"len", len, static_cast<size_t>(B) * 4}, {"first", first, static_cast<size_t>(B) * 4},
                          {"page_table", table, static_cast<size_t>(B) * pages_per_seq * 4}};
    if (int rc = check_spans(spans, 2, sizeof(spans) / sizeof(spans[0]))) return rc;
    Rows4Args a{static_cast<const char*>(k_cache), static_cast<const char*>(v_cache), static_cast<char*>(k_out), static_cast<char*>(v_out), idx, len, first, table,
                n, S_out, Hkv, static_cast<int>(S_cap), page_size, pages_per_seq, static_cast<int>(n_pages)};
    return dispatch_rows4(false, a, B, dh, dtype, stream);
}

}  // namespace metok

using namespace metok;

extern "C" size_t metok_kv4_cache_bytes(int64_t B, int Hkv, int64_t S_cap, int dh) {
    if (B < 1 || B > INT32_MAX || bad_rows4(1, Hkv, 1, 1, S_cap, dh, METOK_BF16)) return 0;
    return static_cast<size_t>(B) * Hkv * (S_cap / kBlockRows) * block4_bytes(dh);
}

extern "C" int metok_kv4_pack(const void* k, const void* v, int B, int Hkv, int64_t S_src, int dh, int dtype, const int32_t* idx, int64_t n, const int32_t* count,
                              void* k_cache, void* v_cache, int64_t S_cap, const int32_t* start, void* stream) {
    clear_error();
    return pack_impl(k, v, B, Hkv, S_src, dh, dtype, idx, n, count, k_cache, v_cache, S_cap, metok_kv4_cache_bytes(B, Hkv, S_cap, dh), nullptr, 0, kBlockRows, 0, start, stream);
}

extern "C" int metok_kv4_pack_paged(const void* k, const void* v, int B, int Hkv, int64_t S_src, int dh, int dtype, const int32_t* idx, int64_t n, const int32_t* count,
                                    void* k_pool, void* v_pool, int64_t n_pages_pool, int page_size, const int32_t* page_table, int pages_per_seq,
                                    const int32_t* start, void* stream) {
    clear_error();
    if (int rc = check_pages4(page_table, n_pages_pool, page_size, pages_per_seq, Hkv)) return rc;
    return pack_impl(k, v, B, Hkv, S_src, dh, dtype, idx, n, count, k_pool, v_pool, static_cast<int64_t>(pages_per_seq) * page_size,
                     metok_kv4_cache_bytes(n_pages_pool, Hkv, page_size, dh), page_table, n_pages_pool, page_size, pages_per_seq, start, stream);
}

extern "C" int metok_kv4_unpack(const void* k_cache, const void* v_cache, int B, int Hkv, int64_t S_cap, int dh, const int32_t* len, const int32_t* first, const int32_t* idx,
                                int64_t n, void* k_out, void* v_out, int64_t S_out, int dtype, void* stream) {
    clear_error();
    return unpack_impl(k_cache, v_cache, B, Hkv, S_cap, metok_kv4_cache_bytes(B, Hkv, S_cap, dh), dh, nullptr, 0, kBlockRows, 0, len, first, idx, n, k_out, v_out, S_out, dtype, stream);
}

extern "C" int metok_kv4_unpack_paged(const void* k_pool, const void* v_pool, int B, int Hkv, int64_t n_pages_pool, int page_size, int dh, const int32_t* page_table,
                                      int pages_per_seq, const int32_t* len, const int32_t* first, const int32_t* idx, int64_t n,
                                      void* k_out, void* v_out, int64_t S_out, int dtype, void* stream) {
    clear_error();
    if (int rc = check_pages4(page_table, n_pages_pool, page_size, pages_per_seq, Hkv)) return rc;
    return unpack_impl(k_pool, v_pool, B, Hkv, static_cast<int64_t>(pages_per_seq) * page_size, metok_kv4_cache_bytes(n_pages_pool, Hkv, page_size, dh), dh, page_table,
                       n_pages_pool, page_size, pages_per_seq, len, first, idx, n, k_out, v_out, S_out, dtype, stream);
}
