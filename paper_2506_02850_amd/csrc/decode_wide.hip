// Attention of one new token where a kv head serves more than 16 query heads: a wave takes two or four blocks of 16 at a time, so that a row
// of the cache is read once for 64 heads (32 where they have more than 64 elements), not once for every 16.  The sums of a block are up
// to 64 registers and its queries up to 32, so that one wave per SIMD is what fits; it is what the launch has, too.  The streaming hint only
// where rows are read once: 8 x 73980 rows, 64 heads on 2 of 128, 107 us with it, 122 without; with rows that are read twice, which should
// stay in the caches (18490 rows, 40 heads of 128 on one), 33.4 and 28.8.
//
// Measured against a block per wave (the blocks of a pair in different workers), bf16: 8 videos of 36990 rows with 71 heads of 64 on one
// kv head 48.9 us against 59.7; 18490 rows with 40 heads of 128 on one 29.3 against 41.8; with 64 on two, in pages, 40.5 against 50.8.
// Passing over the blocks that have no heads (3 of 8 with 71) costs the loop its schedule: 56.1 us, so they are computed like the others.
#include "decode_attention.h"

namespace metok {

template <typename T, int DH, bool STREAM, int NB>
static void launch_form(const DecodeArgs& a, unsigned groups, hipStream_t st) {
    if (!a.table) launch_attention<T, DH, kDense, STREAM, NB>(a, groups, st);
    else if (a.page_size % 16 != 0) launch_attention<T, DH, kRows, STREAM, NB>(a, groups, st);
    else launch_attention<T, DH, kBlocks, STREAM, NB>(a, groups, st);
}

template <typename T, int DH>
static void launch_blocks(const DecodeArgs& a, bool stream, unsigned groups, hipStream_t st) {
    if constexpr (attend_blocks(DH, 64) == 4) {
        if (a.block_rows == 64) return stream ? launch_form<T, DH, true, 4>(a, groups, st) : launch_form<T, DH, false, 4>(a, groups, st);
    }
    stream ? launch_form<T, DH, true, 2>(a, groups, st) : launch_form<T, DH, false, 2>(a, groups, st);
}

void launch_wide_attention(const DecodeArgs& a, int dtype, int dh, bool stream, unsigned groups, hipStream_t st) {
    stream = stream && a.row_blocks == 1;
    if (dtype == METOK_BF16) {
        if (dh == 32) launch_blocks<bf16_t, 32>(a, stream, groups, st);
        else if (dh == 64) launch_blocks<bf16_t, 64>(a, stream, groups, st);
        else if (dh == 128) launch_blocks<bf16_t, 128>(a, stream, groups, st);
        else launch_blocks<bf16_t, 256>(a, stream, groups, st);
    } else {
        if (dh == 32) launch_blocks<float, 32>(a, stream, groups, st);
        else if (dh == 64) launch_blocks<float, 64>(a, stream, groups, st);
        else launch_blocks<float, 128>(a, stream, groups, st);
    }
}

}  // namespace metok
