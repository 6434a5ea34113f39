// Rows of K and V in 4 bits: where the codes and scales of a block of 16 rows lie (include/metok_qkv.h), and the step into 4 bits.
#pragma once

#include "common.h"
#include "metok_qkv.h"

namespace metok {

constexpr int kBlockRows = 16;
constexpr float kLeastScale = 0x1p-100f, kMostScale = 0x1p100f;

// The codes are e2m1 numbers and the scales powers of two, which gfx950 converts two of at a time, scale included: a value of K or V costs half an
// instruction.  A piece is a row's part that 16 lanes of the attention hold, 16 bytes of each four rows of V, or of one row of K, to a lane with heads of
// 128 elements or more.
template <int DH> struct Block4 {
    static constexpr int kWidth = DH < 128 ? DH : 128;           // elements of a piece
    static constexpr int kPieces = DH / kWidth, kGroups = kWidth / 32;       // pieces of a row, scales of a piece
    static constexpr int kPieceBytes = 8 * kWidth;               // codes of 16 rows
    static constexpr int kRowBytes = kWidth / 2;                 // K: codes of a row
    static constexpr int kRunBytes = kWidth / 32;                // V: codes of a row in the lane's run of kWidth / 16 elements
    static constexpr int kScales = 8 * DH;                       // the scales begin here
    static constexpr int kBytes = 17 * DH / 2;
    static_assert(kScales + 16 * kPieces * kGroups == kBytes, "codes and scales are the block");
};
// The pages of a 4-bit pool.
inline int check_pages4(const int32_t* table, int64_t n_pages, int page_size, int pages_per_seq, int Hkv) {
    if (!table || (reinterpret_cast<uintptr_t>(table) & 3u)) return fail(METOK_ERR_INVALID_ARG, "page_table NULL or misaligned");
    if (page_size < 1 || pages_per_seq < 1 || n_pages < 1) return fail(METOK_ERR_INVALID_ARG, "page_size, pages_per_seq and n_pages_pool must be positive");
    if (page_size % kBlockRows != 0) return fail(METOK_ERR_INVALID_ARG, "page_size must be a multiple of 16");
    if (Hkv >= 1 && n_pages > INT32_MAX / page_size / Hkv) return fail(METOK_ERR_UNSUPPORTED, "n_pages_pool * Hkv * page_size must be below 2^31");
    return METOK_OK;
}
constexpr size_t block4_bytes(int dh) { return static_cast<size_t>(17) * dh / 2; }

// The scale of a group whose largest magnitude is m: the smallest power of two with m <= 7 s.  7 is 1.75 * 4, so two less than m's exponent, or one less
// where m's mantissa is above 1.75.
__device__ __forceinline__ float scale_of(float m) {
    const uint32_t e = (__float_as_uint(m) + 0x1fffffu) >> 23;
    return fminf(fmaxf(__uint_as_float((e < 2 ? 0u : e - 2) << 23), kLeastScale), kMostScale);
}
__device__ __forceinline__ uint32_t scale_byte(float s) { return __float_as_uint(s) >> 23; }
__device__ __forceinline__ float scale_from(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two elements -> byte SEL of w.
template <int SEL> __device__ __forceinline__ uint32_t put_codes(uint32_t w, float a, float b, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, s, SEL);
}
// Byte SEL of w -> two elements, as a bf16 pair (exact: two bits of mantissa).
template <int SEL> __device__ __forceinline__ uint32_t take_codes(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL));
}

// Largest of G neighbouring lanes (G = 4, 8, 16); each receives it.
template <int CTRL> __device__ __forceinline__ float dpp_max(float v) {
    return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false)));
}
template <int G> __device__ __forceinline__ float lanes_max(float v) {
    v = dpp_max<0xb1>(v);                       // the neighbour
    v = dpp_max<0x4e>(v);                       // two further, within four
    if (G >= 8) v = dpp_max<0x141>(v);          // mirrored within eight: the other four
    if (G >= 16) v = dpp_max<0x140>(v);         // mirrored within sixteen
    return v;
}

}  // namespace metok
