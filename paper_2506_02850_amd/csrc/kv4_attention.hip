// Attention of one new token per video over a KV cache held in 4 bits (include/metok_qkv.h): the counterpart of decode_attention.h, split over the
// chip and joined as there.
//
// The codes become bf16 numbers in registers, two an instruction and exactly (two bits of mantissa, scales that are powers of two), and go into the same
// MFMA products.  The floor is the stream of K and V, 17 / 32 byte an element, a quarter of the bytes of bf16 rows.  What bounds the largest calls is the
// issue of vector and matrix instructions beside it: an element of K costs half an instruction, one of V a whole one, since the values of two rows have to be brought beside
// each other.  8 x 36992 rows, 28 query heads on 4 of 128, 161 MB: 31.0 us, 5.2 TB/s, as long as from rows that the caches hold, and 4.6 for the join; 16 of them 59.4 us,
// 5.4 TB/s.  Narrower heads and fp32 queries are further from it: a tile of 32 rows costs a wave some 0.9 us at 32 elements, 1.3 at 64, 1.8 at 128, with one tile ahead at any width
// (40 MB: 8 x 36992 rows of 4 heads of 32 18.9 us, of 2 of 64 14.6; 80 MB: 4 x 36992 of 4 of 128 18.5, 8 x 18496 in fp32, with three parts of every factor, 21.4).
#include "decode_attention.h"
#include "kv4.h"

namespace metok {

// The scale in byte I of a word.
template <int I> __device__ __forceinline__ float scale_in(uint32_t w) {
    uint32_t x;
    if constexpr (I == 0) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(x) : "v"(23), "v"(w));
    else if constexpr (I == 1) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(x) : "v"(23), "v"(w));
    else if constexpr (I == 2) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(x) : "v"(23), "v"(w));
    else asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(x) : "v"(23), "v"(w));
    return __uint_as_float(x);
}

// x as the sum of PARTS bf16 numbers, 8 bits each: all of a bf16 number's bits in one, of an fp32 number's in three.
template <int PARTS> __device__ __forceinline__ void split_pair(uint32_t (&part)[PARTS], float a, float b) {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        part[i] = pack_bf16x2(a, b);
        if (i + 1 < PARTS) { a -= bf16_lo(part[i]); b -= bf16_hi(part[i]); }
    }
}

// A lane's place: r = lane % 16, c = lane / 16, as in decode_attention.h.  It has, of every block of 16 rows, a quarter of each piece of row r of K, and of V the
// r-th run of rows 4 c .. 4 c + 3, both as they lie in the block: one load each, and one for the scales.
//
// A new row is put into 4 bits by the wave that has the tile it belongs to, in LDS, and takes its place among the tile's rows from there: what is
// attended to is what is stored.
template <typename T, int DH, bool PAGED, bool WEIGHTS, bool STREAM, bool WHOLE>
__global__ __launch_bounds__(64 * (WHOLE ? kAttendWholeWaves : kAttendWaves), 2) void kv4_attention_kernel(const DecodeArgs a) {
    static_assert(!WHOLE || !WEIGHTS, "the second launch adds the weights up");
    using F = Block4<DH>;
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int TILE = kAttend4Tile, NT = TILE / 16, NV = NT * 4, P = F::kPieces, KW = F::kWidth / 32, EB = F::kRunBytes, E = DH / 16, RB = DH * static_cast<int>(sizeof(T));
    constexpr int QP = BF16 ? 1 : 3, PP = BF16 ? 2 : 3;    // parts of a query, of a probability
    static_assert(NT % 2 == 0 && KW == EB, "32 rows to a product; a lane has as much of K as of V");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
    // Neighbouring workers on different CUs where the capacity holds few tiles, so that these are spread over all of them; in one workgroup where it holds many, so
    // that they can join what they leave of a pair that none of them begins or ends: the parts of 131072 rows are joined in 10.0 us then, not in 15.5.  A short video in a
    // large cache has neighbours in one workgroup, too, and is not slower (2306 rows, 28 heads on 4 of 128: 4.8 us in a cache of 2560 rows, 4.9 in one of 131072).
    const int worker = a.teams ? static_cast<int>(blockIdx.x) * kAttendWaves + wave : wave * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x);
    bool team = false;                                     // the workgroup is in the middle of a pair
    const bool fresh = a.k_new != nullptr;
    const scalar_ints lens = reinterpret_cast<scalar_ints>(reinterpret_cast<uintptr_t>(a.len));
    // of the new row: K's and V's codes in the order of the elements, then the scales
    constexpr int NEW = DH / 2 + DH / 32 + 15 & ~15;
    __shared__ alignas(16) uint8_t s_new[(WHOLE ? kAttendWholeWaves : kAttendWaves)][2][NEW];

    struct Cursor { int b, kvh, rb, t, tiles, n; };        // a tile of a pair, its kv head and block of query heads: uniform over the wave
    Cursor at;
    int left;                                              // units that the worker still has (WHOLE: tiles)
    auto tiles_of = [&](int n) { return max(static_cast<int>(static_cast<uint32_t>(n + static_cast<int>(fresh) + TILE - 1) / TILE), 1); };
    if constexpr (WHOLE) {
        at.b = static_cast<int>(blockIdx.x) / a.Hkv;
        at.kvh = static_cast<int>(blockIdx.x) - at.b * a.Hkv;
        at.rb = 0;
        at.n = min(max(lens[at.b], 0), a.S_cap);
        at.tiles = tiles_of(at.n);
        at.t = wave * at.tiles / kAttendWholeWaves;
        left = (wave + 1) * at.tiles / kAttendWholeWaves - at.t;
    } else {
        typedef Deal4 D;
        const Place place = find_place<TILE, D>(a, worker);
        if (place.left <= 0) return;
        at.b = __builtin_amdgcn_readfirstlane(place.b);
        at.tiles = __builtin_amdgcn_readfirstlane(place.tiles);
        at.n = __builtin_amdgcn_readfirstlane(place.n);
        const int units = at.tiles + kAttend4PairCost;
        const int hr = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<uint32_t>(place.at) / static_cast<uint32_t>(units)));
        at.kvh = a.row_blocks == 1 ? hr : __builtin_amdgcn_readfirstlane(hr / a.row_blocks);
        at.rb = hr - at.kvh * a.row_blocks;
        at.t = __builtin_amdgcn_readfirstlane(place.at) - hr * units;
        left = __builtin_amdgcn_readfirstlane(place.left);
        if (a.teams) team = __builtin_amdgcn_readfirstlane(D::in_the_middle(worker, place.all, at.t, at.tiles));
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
                    x.tiles = tiles_of(x.n);
                    n_ahead = lens[min(x.b + 1, a.B - 1)];
                }
            }
        }
        return x;
    };
    auto first_head = [&](const Cursor& x) { return x.kvh * a.group + x.rb * kAttendRows; };
    auto n_heads = [&](const Cursor& x) { return min(a.group - x.rb * kAttendRows, kAttendRows); };
    auto slab_of = [&](const Cursor& x) { return static_cast<int64_t>(x.b) * a.Hkv + x.kvh; };

    // What depends on the lane is kept from the compiler's sight where it is used.  In the loads it stays the 32-bit offset beside a block's address in scalar
    // registers; elsewhere it is computed when it is needed.  Hoisted out of the loop, as addresses of 64 bits, all that takes 40 registers and an
    // addition a load.
    auto hidden = [](uint32_t x) { asm("" : "+v"(x)); return x; };
    struct Lane { int lane, r, c; };
    auto lane_here = [&] { const int x = static_cast<int>(hidden(lane)); return Lane{x, x & 15, x >> 4}; };

    // ---- loads ----
    auto page_index = [&](int j) { return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(j)) * a.page_mul) >> a.page_shift); };
    struct Pages { int p[PAGED ? NT : 1]; };               // table entries of a tile's blocks
    auto pages_of = [&](const Cursor& x) {
        Pages p{};
        if constexpr (PAGED) {
            const scalar_ints table = reinterpret_cast<scalar_ints>(reinterpret_cast<uintptr_t>(a.table + static_cast<int64_t>(x.b) * a.pages_per_seq));
            const int last = max(x.n - 1, 0);
#pragma unroll
            for (int b = 0; b < NT; ++b) p.p[b] = table[page_index(min(x.t * TILE + 16 * b, last))];
        }
        return p;
    };
    // The tile's blocks in the slab or pool (behind the last row: the block with the last row, where there is none the first one), and which of them are there.
    struct Rows { int block[NT], all; uint32_t pages_ok; };            // all: the tile ends before the last row, and its pages are ones
    auto rows_of = [&](const Cursor& x, const Pages& p) {
        Rows f{};
        const int j0 = x.t * TILE, last = max(x.n - 1, 0);
        f.all = j0 + TILE <= x.n;
        f.pages_ok = (1u << NT) - 1;
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const int j = min(j0 + 16 * b, last);
            f.block[b] = j / kBlockRows;
            if constexpr (PAGED) {
                const bool ok = p.p[b] >= 0 && p.p[b] < a.n_pages;
                f.block[b] = ok ? (p.p[b] * a.Hkv + x.kvh) * (a.page_size / kBlockRows) + (j - page_index(j) * a.page_size) / kBlockRows : 0;
                if (!ok) { f.pages_ok &= ~(1u << b); f.all = 0; }
            }
        }
        return f;
    };
    uint32_t kf[NT][P][KW], vf[NT][P][KW], ks[NT][P], vs[NT][P];
    const uint32_t k_code = r * F::kRowBytes + c * (4 * KW), k_scale = F::kScales + (r >> 2) * 4 * F::kGroups + c * F::kWidth / 128 * 4, k_byte = 8 * (r & 3);
    const uint32_t v_code = c * 2 * F::kWidth + r * 4 * EB, v_scale = F::kScales + c * 4 * F::kGroups + r * F::kWidth / 512 * 4;
    auto base_of = [&](const Cursor& x, const char* cache, int block) {
        return cache + ((PAGED ? 0 : slab_of(x) * (a.S_cap / kBlockRows)) + block) * F::kBytes;
    };
    auto load_k = [&](const Cursor& x, const Rows& f) {
        const uint32_t code = hidden(k_code), scale = hidden(k_scale);
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const char* block = base_of(x, a.k, f.block[b]);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                load_words<KW, STREAM>(kf[b][p], block + p * F::kPieceBytes + code);
                ks[b][p] = *reinterpret_cast<const uint32_t*>(block + p * 16 * F::kGroups + scale);        // of four rows, the lane's own in byte r % 4
            }
        }
    };
    auto load_v = [&](const Cursor& x, const Rows& f) {
        const uint32_t code = hidden(v_code), scale = hidden(v_scale);
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const char* block = base_of(x, a.v, f.block[b]);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                load_words<KW, STREAM>(vf[b][p], block + p * F::kPieceBytes + code);
                vs[b][p] = *reinterpret_cast<const uint32_t*>(block + p * 16 * F::kGroups + scale);
            }
        }
    };
    // queries in the order of the codes: word i of piece p of the lane's part of a row of K is elements p w + c w / 4 + 8 i ..
    u32x4_t qf[P * KW][QP];
    auto load_q = [&](const Cursor& x) {
        const auto [lane, r, c] = lane_here();
        const char* head = a.q + (static_cast<int64_t>(x.b) * a.Hq + first_head(x) + min(r, n_heads(x) - 1)) * RB;
#pragma unroll
        for (int i = 0; i < P * KW; ++i) {
            const char* p = head + (i / KW * F::kWidth + c * (F::kWidth / 4) + i % KW * 8) * static_cast<int>(sizeof(T));
            if constexpr (BF16) qf[i][0] = *reinterpret_cast<const u32x4_t*>(p);
            else {
                const float4 x0 = *reinterpret_cast<const float4*>(p), x1 = *reinterpret_cast<const float4*>(p + 16);
                const float v[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t part[QP];
                    split_pair(part, v[2 * j], v[2 * j + 1]);
#pragma unroll
                    for (int k = 0; k < QP; ++k) qf[i][k][j] = part[k];
                }
            }
        }
    };

    // ---- the new row ----
    auto new_row = [&](const Cursor& x) { return fresh && static_cast<int>(static_cast<uint32_t>(x.n) / TILE) == x.t; };
    // two elements to a lane, 128 at a time; heads of fewer have lanes that do the same
    auto pack_new = [&](const Cursor& x) {
        const auto [lane, r, c] = lane_here();
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int e0 = 0; e0 < DH; e0 += 128) {
                const int e = e0 + (2 * lane) % DH;
                const char* p = (which ? a.v_new : a.k_new) + slab_of(x) * RB + e * static_cast<int>(sizeof(T));
                float u, w;
                if constexpr (BF16) { const uint32_t v = *reinterpret_cast<const uint32_t*>(p); u = bf16_lo(v); w = bf16_hi(v); }
                else { const float2 v = *reinterpret_cast<const float2*>(p); u = v.x; w = v.y; }
                const float s = scale_of(lanes_max<16>(fmaxf(fabsf(u), fabsf(w))));
                s_new[wave][which][e / 2] = static_cast<uint8_t>(put_codes<0>(0u, u, w, s));
                s_new[wave][which][DH / 2 + e / 32] = static_cast<uint8_t>(scale_byte(s));
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");           // written and read by this wave alone
        __builtin_amdgcn_wave_barrier();
    };
    auto place_new = [&](const Cursor& x) {
        const auto [lane, r, c] = lane_here();
        const int in = x.n - x.t * TILE;                   // the new row's place in the tile
        const uint8_t *nk = s_new[wave][0], *nv = s_new[wave][1];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            uint32_t w[KW];
            load_words<KW, false>(w, reinterpret_cast<const char*>(nk + p * F::kRowBytes + c * 4 * KW));
            const uint32_t scale = nk[DH / 2 + p * F::kGroups + c * F::kWidth / 128];
            uint32_t run = 0;                              // the lane's run of V, from the first byte of a word
#pragma unroll
            for (int z = 0; z < EB; ++z) run |= static_cast<uint32_t>(nv[p * F::kRowBytes + r * EB + z]) << (8 * z);
            const uint32_t scale_v = nv[DH / 2 + p * F::kGroups + r * F::kWidth / 512];
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const bool mine = in == 16 * b + r;
#pragma unroll
                for (int i = 0; i < KW; ++i) kf[b][p][i] = mine ? w[i] : kf[b][p][i];
                ks[b][p] = mine ? scale << (8 * (r & 3)) : ks[b][p];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool own = in == 16 * b + 4 * c + i;
                    constexpr uint32_t ones = EB == 4 ? 0xffffffffu : (1u << (8 * EB % 32)) - 1u;
                    const int word = i * EB / 4, shift = i * EB % 4 * 8;
                    const uint32_t mask = own ? ones << shift : 0u, byte = own ? 0xffu << (8 * i) : 0u;
                    vf[b][p][word] = (vf[b][p][word] & ~mask) | (run << shift & mask);
                    vs[b][p] = (vs[b][p] & ~byte) | (scale_v << (8 * i) & byte);
                }
            }
        }
    };
    // it joins the cache: nobody uses what the cache has in that row in this call
    auto append = [&](const Cursor& x) {
        if (!new_row(x) || x.rb != 0 || x.n >= a.S_cap) return;
        const auto [lane, r, c] = lane_here();
        int64_t block = slab_of(x) * (a.S_cap / kBlockRows) + x.n / kBlockRows;
        if constexpr (PAGED) {
            const int index = page_index(x.n), page = a.table[static_cast<int64_t>(x.b) * a.pages_per_seq + index];
            if (page < 0 || page >= a.n_pages) return;
            block = (static_cast<int64_t>(page) * a.Hkv + x.kvh) * (a.page_size / kBlockRows) + (x.n - index * a.page_size) / kBlockRows;
        }
        char *k = a.k + block * F::kBytes, *v = a.v + block * F::kBytes;
        const uint8_t *nk = s_new[wave][0], *nv = s_new[wave][1];
        const int in = x.n % kBlockRows, ci = in >> 2, ii = in & 3;
        if (lane < DH / 8) {                               // four bytes of K
            const int p = lane * 4 / F::kRowBytes, at_byte = lane * 4 % F::kRowBytes;
            *reinterpret_cast<uint32_t*>(k + p * F::kPieceBytes + in * F::kRowBytes + at_byte) = *reinterpret_cast<const uint32_t*>(nk + lane * 4);
        }
        if (lane < 16 * P) {                               // a run of V
            char* to = v + (lane >> 4) * F::kPieceBytes + ci * 2 * F::kWidth + (lane & 15) * 4 * EB + ii * EB;
            const uint8_t* from = nv + lane * EB;
            if constexpr (EB == 4) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
            else if constexpr (EB == 2) *reinterpret_cast<uint16_t*>(to) = *reinterpret_cast<const uint16_t*>(from);
            else *to = static_cast<char>(*from);
        }
        if (lane < DH / 32) {
            const int to = F::kScales + lane / F::kGroups * 16 * F::kGroups + ci * 4 * F::kGroups + lane % F::kGroups * 4 + ii;
            k[to] = static_cast<char>(nk[DH / 2 + lane]);
            v[to] = static_cast<char>(nv[DH / 2 + lane]);
        }
    };

    // ---- one tile ----
    f32x4_t acc[E];
    float m, l;
    auto clear = [&] {
        m = -INFINITY; l = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    };
    auto scores = [&](f32x4_t (&s)[NT]) {
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            s[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const float scale = scale_from((ks[b][p] >> k_byte) & 0xffu);
#pragma unroll
                for (int i = 0; i < KW; ++i) {
                    const uint32_t w = kf[b][p][i];
                    const u32x4_t k = {take_codes<0>(w, scale), take_codes<1>(w, scale), take_codes<2>(w, scale), take_codes<3>(w, scale)};
#pragma unroll
                    for (int q = 0; q < QP; ++q)
                        s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, qf[p * KW + i][q]), s[b], 0, 0, 0);
                }
            }
        }
    };
    auto take = [&](const Cursor& x, const Rows& f, f32x4_t (&s)[NT]) {
        if (a.cap > 0.f) {
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i >> 2][i & 3] = a.cap * tanh_of(s[i >> 2][i & 3] * a.scale);
        }
        const float scale = score_scale(a);
        if (!f.all) {
            const auto [lane, r, c] = lane_here();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = x.t * TILE + 16 * (i >> 2) + 4 * c + (i & 3);
                const bool there = (j < x.n && ((f.pages_ok >> (i >> 2)) & 1u)) || (fresh && j == x.n);
                s[i >> 2][i & 3] = there ? s[i >> 2][i & 3] : -INFINITY;
                const uint32_t byte = 0xffu << (8 * (i & 3)), one = 127u << (8 * (i & 3));
#pragma unroll
                for (int p = 0; p < P; ++p) vs[i >> 2][p] = there ? vs[i >> 2][p] : (vs[i >> 2][p] & ~byte) | one;       // finite: nothing times it is nothing
            }
        }
        if constexpr (WEIGHTS) {
            const auto [lane, r, c] = lane_here();
            if (r < n_heads(x)) {
                float* to = a.logits + (static_cast<int64_t>(x.b) * a.Hq + first_head(x) + r) * a.logit_stride + x.t * TILE + 4 * c;
#pragma unroll
                for (int b = 0; b < NT; ++b) *reinterpret_cast<f32x4_t*>(to + 16 * b) = s[b];
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < NV; ++i) top = fmaxf(top, s[i >> 2][i & 3]);
        // What probabilities are relative to follows the maximum only where that is more than 2^kLag times it: with several heads some maximum grows in most
        // tiles of a short run, and fp32 sums have room for probabilities of up to 2^kLag (as long as that many times the values' magnitudes add up to an fp32 number).
        constexpr float kLag = 8.f;
        if (__any((top - m) * scale > kLag)) {
            const float to = fmaxf(m, rows_max(top)), g = exp2_from(m, to == -INFINITY ? 0.f : to, scale);
            m = to;
            l *= g;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] *= g;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int h = 0; h < NT / 2; ++h) {                 // 32 rows to a product: rows 4 c .. 4 c + 3 of the one block, then of the other
            u32x4_t part[PP];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int b = 2 * h + (i >> 1), at0 = 2 * (i & 1);
                const float p0 = exp2_from(s[b][at0], ref, scale), p1 = exp2_from(s[b][at0 + 1], ref, scale);
                l += p0;
                l += p1;
                uint32_t w[PP];
                split_pair(w, p0, p1);
#pragma unroll
                for (int k = 0; k < PP; ++k) part[k][i] = w[k];
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float vscale[8];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t w = vs[2 * h + b][p];
                    vscale[4 * b] = scale_in<0>(w); vscale[4 * b + 1] = scale_in<1>(w); vscale[4 * b + 2] = scale_in<2>(w); vscale[4 * b + 3] = scale_in<3>(w);
                }
#pragma unroll
                for (int z = 0; z < EB; ++z) {
                    uint32_t two[8];                       // elements 2 z, 2 z + 1 of the run, of each of the lane's rows
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int byte = (i & 3) * EB + z;
                        const uint32_t w = vf[2 * h + (i >> 2)][p][byte >> 2];
                        switch (byte & 3) {
                            case 0: two[i] = take_codes<0>(w, vscale[i]); break;
                            case 1: two[i] = take_codes<1>(w, vscale[i]); break;
                            case 2: two[i] = take_codes<2>(w, vscale[i]); break;
                            default: two[i] = take_codes<3>(w, vscale[i]);
                        }
                    }
#pragma unroll
                    for (int odd = 0; odd < 2; ++odd) {
                        u32x4_t v;
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_perm(two[2 * i + 1], two[2 * i], odd ? 0x07060302u : 0x05040100u);
                        f32x4_t& sum = acc[p * 2 * EB + 2 * z + odd];
#pragma unroll
                        for (int k = 0; k < PP; ++k)
                            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, part[k]), sum, 0, 0, 0);
                    }
                }
            }
        }
    };
    // ---- the end of a pair, or of the worker's tiles: the result, or a part of it for the join ----
    constexpr int N = 2 * EB;                              // accumulator i of element e: element (e / N) * w + N (4 c + i) + e % N
    auto finish = [&](const Cursor& x, int begun) {        // begun: the first tile of the pair that the worker had
        const auto [lane, r, c] = lane_here();
        const bool ends = x.t == x.tiles - 1, whole = begun == 0 && ends;
        if (a.pair_workers && lane == 0) {
            int* to = reinterpret_cast<int*>(a.pair_workers + slab_of(x) * a.row_blocks + x.rb);
            if (begun == 0) to[0] = worker;
            if (ends) to[1] = worker;
        }
        const int heads = n_heads(x);
        const float sum = swap32_add(swap16_add(l, l), swap16_add(l, l));
        const int64_t head = static_cast<int64_t>(x.b) * a.Hq + first_head(x) + r;
        const int64_t slot = (2 * static_cast<int64_t>(worker) + (begun == 0 ? 1 : 0)) * a.rows + r;
        const float lse2 = sum == 0.f ? -INFINITY : fmaf(m, score_scale(a), log2_of(sum)), inv = sum == 0.f ? 0.f : 1.f / sum;
        if (whole) {
            if (r < heads) {
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        char* to = a.out + head * RB + (p * F::kWidth + N * (4 * c + i)) * static_cast<int>(sizeof(T));
#pragma unroll
                        for (int e = 0; e < N; e += 2) {
                            const float x0 = acc[p * N + e][i] * inv, x1 = acc[p * N + e + 1][i] * inv;
                            if constexpr (BF16) reinterpret_cast<uint32_t*>(to)[e / 2] = pack_bf16x2(x0, x1);
                            else reinterpret_cast<float2*>(to)[e / 2] = make_float2(x0, x1);
                        }
                    }
            }
            if (c == 0 && r < heads && a.lse) a.lse[head] = lse2 * 0.693147180559945309f;
            if (WEIGHTS && c == 0 && r < heads) a.norm[head] = make_float2(sum == 0.f ? 0.f : m, inv);
        } else {
            if (r < heads) {
                float* to = a.part_o + slot * DH;
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < N; ++e) to[p * F::kWidth + N * (4 * c + i) + e] = acc[p * N + e][i];
            }
            if (c == 0 && r < heads) reinterpret_cast<float2*>(a.part_ml)[slot] = make_float2(m, sum);
        }
    };

    if (!WHOLE && at.t >= at.tiles) {                      // behind a pair: on to the next one, if there is one
        left -= at.tiles + kAttend4PairCost - at.t;
        if (left <= 0) return;
        at.t = at.tiles - 1;
        at = advance(at);
    }
    clear();
    if (!WHOLE || left > 0) {
        int begun = at.t;                                  // first tile of the pair that the worker has
        load_q(at);
        Rows rows = rows_of(at, pages_of(at));
        __builtin_amdgcn_sched_barrier(0);                 // in the loop's order, or its waits would allow for both
        load_k(at, rows);
        __builtin_amdgcn_sched_barrier(0);
        load_v(at, rows);
        for (;;) {
            const bool ends = !WHOLE && at.t == at.tiles - 1;
            left -= ends ? 1 + kAttend4PairCost : 1;
            const bool last = left <= 0;
            // Behind the last tile the first one of all is loaded, for nobody: with loads that may not be there the waits for those before them would wait for
            // everything (8 x 36992 rows, 28 heads on 4 of 128: 47 us).
            const Cursor next = last ? Cursor{0, 0, 0, 0, 1, 0} : advance(at);
            const Pages pages = pages_of(next);
            if (new_row(at)) {
                pack_new(at);
                place_new(at);
            }
            f32x4_t s[NT];
            scores(s);
            const Rows rows_next = rows_of(next, pages);
            load_k(next, rows_next);
            take(at, rows, s);
            if (ends || (!WHOLE && last && !team)) finish(at, begun);
            append(at);
            if (ends && !last) {
                begun = 0;
                clear();
                load_q(next);
            }
            load_v(next, rows_next);
            if (last) break;
            at = next;
            rows = rows_next;
        }
    }
    if (WHOLE || team) {                                   // the waves' sums become one
        constexpr int W = WHOLE ? kAttendWholeWaves : kAttendWaves, PITCH = DH + 4, LPR = DH / 4;       // 4 more: rows 16 bytes apart in the banks
        __shared__ float4 s_o[W * kAttendRows * PITCH / 4];
        __shared__ float2 s_ml[W][kAttendRows];
        const float sum = swap32_add(swap16_add(l, l), swap16_add(l, l));
        if (c == 0) s_ml[wave][r] = make_float2(m, sum);
        float* to = reinterpret_cast<float*>(s_o) + (wave * kAttendRows + r) * PITCH;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) to[p * F::kWidth + N * (4 * c + i) + e] = acc[p * N + e][i];
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
            if constexpr (WHOLE) {
                const float inv = total == 0.f ? 0.f : 1.f / total;
                const int64_t head = static_cast<int64_t>(at.b) * a.Hq + first_head(at) + row;
                char* out = a.out + head * RB + 4 * x * static_cast<int>(sizeof(T));
                if constexpr (BF16) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
                else *reinterpret_cast<float4*>(out) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
                if (x == 0 && a.lse) a.lse[head] = total == 0.f ? -INFINITY : fmaf(ref, scale, log2_of(total)) * 0.693147180559945309f;
            } else {
                const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) * kAttendWaves * a.rows + row;
                *reinterpret_cast<float4*>(a.part_o + slot * DH + 4 * x) = o;
                if (x == 0) reinterpret_cast<float2*>(a.part_ml)[slot] = make_float2(top, total);
            }
        }
    }
}

// Caches of more than this many bytes are read with the streaming hint: they pass through the 256 MB before memory without staying there (8 x 36992 rows of 4 heads of
// 128, 161 MB: 31.3 us with, 33.3 without; 16 of them 59.4 and 62.2; 4 of them, 80 MB, which stay there from one call to the next, are read without).  A lane's load of
// 4 or 8 bytes, of heads of 32 and 64, has no such hint.
constexpr int64_t kStream4Bytes = 128 << 20;

template <typename T, int DH, bool PAGED>
static int launch_form(const DecodeArgs& a, const AttendPlan& plan, hipStream_t st) {
    const int64_t bytes = static_cast<int64_t>(a.B) * a.Hkv * a.S_cap * DH * 17 / 16;
    const dim3 groups(static_cast<unsigned>(plan.whole ? plan.pairs : plan.grid)), threads(kAttendThreads);
    constexpr bool HINT = DH >= 128;
    const bool stream = HINT && bytes > kStream4Bytes;
    if (plan.whole) hipLaunchKernelGGL((kv4_attention_kernel<T, DH, PAGED, false, false, true>), groups, dim3(64 * kAttendWholeWaves), 0, st, a);
    else if (a.weight && stream) hipLaunchKernelGGL((kv4_attention_kernel<T, DH, PAGED, true, HINT, false>), groups, threads, 0, st, a);
    else if (a.weight) hipLaunchKernelGGL((kv4_attention_kernel<T, DH, PAGED, true, false, false>), groups, threads, 0, st, a);
    else if (stream) hipLaunchKernelGGL((kv4_attention_kernel<T, DH, PAGED, false, HINT, false>), groups, threads, 0, st, a);
    else hipLaunchKernelGGL((kv4_attention_kernel<T, DH, PAGED, false, false, false>), groups, threads, 0, st, a);
    return check_launch("attention over 4 bits");
}
template <typename T, int DH> static int launch_kv4(const DecodeArgs& a, const AttendPlan& plan, hipStream_t st) {
    return a.table ? launch_form<T, DH, true>(a, plan, st) : launch_form<T, DH, false>(a, plan, st);
}
static int launch_attention4(const DecodeArgs& a, const AttendPlan& plan, int dtype, int dh, hipStream_t st) {
    if (dtype == METOK_BF16) {
        if (dh == 32) return launch_kv4<bf16_t, 32>(a, plan, st);
        if (dh == 64) return launch_kv4<bf16_t, 64>(a, plan, st);
        if (dh == 128) return launch_kv4<bf16_t, 128>(a, plan, st);
        return launch_kv4<bf16_t, 256>(a, plan, st);
    }
    if (dh == 32) return launch_kv4<float, 32>(a, plan, st);
    if (dh == 64) return launch_kv4<float, 64>(a, plan, st);
    return launch_kv4<float, 128>(a, plan, st);
}

// The shapes that the calls and the workspace query take, NULL or the reason why not.
static const char* bad_shape4(int B, int Hq, int Hkv, int64_t S_cap, int dh, int dtype) {
    if (const char* why = bad_attend_heads(B, Hq, Hkv, dh, dtype)) return why;
    if (S_cap < kBlockRows || S_cap % kBlockRows != 0 || S_cap >= INT32_MAX - 64) return "the capacity must be a multiple of 16 in [16, 2^31 - 64)";
    const int64_t pairs = static_cast<int64_t>(B) * Hkv * ((Hq / Hkv + kAttendRows - 1) / kAttendRows);
    if (pairs * (S_cap / 16 + 4) > INT32_MAX) return "too many rows";
    return nullptr;
}

}  // namespace metok

using namespace metok;

extern "C" size_t metok_kv4_attention_workspace_bytes(int B, int Hq, int Hkv, int64_t S_cap, int dh, int dtype, int with_weight) {
    if (bad_shape4(B, Hq, Hkv, S_cap, dh, dtype)) return 0;
    return plan_attend4(B, Hq, Hkv, S_cap, dh, with_weight != 0).bytes;
}

extern "C" int metok_kv4_attention(const void* q, int B, int Hq, int Hkv, int dh, int dtype,
                                   void* k_cache, void* v_cache, int64_t S_cap, const int32_t* len,
                                   const void* k_new, const void* v_new, double scale, double logit_cap,
                                   void* out, float* lse, float* weight, int64_t weight_stride,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    if (const char* why = bad_shape4(B, Hq, Hkv, S_cap, dh, dtype)) return fail(METOK_ERR_INVALID_ARG, "%s", why);
    return attend_call({q, B, Hq, Hkv, dh, dtype, k_cache, v_cache, S_cap, metok_kv4_cache_bytes(B, Hkv, S_cap, dh), nullptr, 0, kBlockRows, 0, len, k_new, v_new,
                        scale, logit_cap, out, lse, weight, weight_stride, workspace, workspace_bytes, stream},
                       plan_attend4(B, Hq, Hkv, S_cap, dh, weight != nullptr), &launch_attention4);
}

extern "C" int metok_kv4_attention_paged(const void* q, int B, int Hq, int Hkv, int dh, int dtype,
                                         void* k_pool, void* v_pool, int64_t n_pages_pool, int page_size,
                                         const int32_t* page_table, int pages_per_seq, const int32_t* len,
                                         const void* k_new, const void* v_new, double scale, double logit_cap,
                                         void* out, float* lse, float* weight, int64_t weight_stride,
                                         void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    if (int rc = check_pages4(page_table, n_pages_pool, page_size, pages_per_seq, Hkv)) return rc;
    const int64_t S_cap = static_cast<int64_t>(pages_per_seq) * page_size;
    if (const char* why = bad_shape4(B, Hq, Hkv, S_cap, dh, dtype)) return fail(METOK_ERR_INVALID_ARG, "%s", why);
    return attend_call({q, B, Hq, Hkv, dh, dtype, k_pool, v_pool, S_cap, metok_kv4_cache_bytes(n_pages_pool, Hkv, page_size, dh), page_table, n_pages_pool, page_size,
                        pages_per_seq, len, k_new, v_new, scale, logit_cap, out, lse, weight, weight_stride, workspace, workspace_bytes, stream},
                       plan_attend4(B, Hq, Hkv, S_cap, dh, weight != nullptr), &launch_attention4);
}
