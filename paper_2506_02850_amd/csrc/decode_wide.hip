// Attention of one new token where a kv head serves more than 16 query heads: a wave takes several blocks of 16 at a time, so that a row
// of the cache is read once for 64 heads (32 where they have more than 64 elements), not once for every 16.  The sums of a block are up
// to 64 registers and its queries up to 32, so that one wave per SIMD is what fits; it is what the launch has, too.  No streaming hint:
// rows that are read more than once should stay in the caches.
//
// Measured against a block per wave (the blocks of a pair in different workers), bf16: 8 videos of 36990 rows with 71 heads of 64 on one
// kv head 48.9 us against 59.7; 18490 rows with 40 heads of 128 on one 29.3 against 41.8; with 64 on two, in pages, 45.0 against 50.8.
// Passing over the blocks that have no heads (3 of 8 with 71) costs the loop its schedule: 56.1 us, so they are computed like the others.
#include "decode_attention.h"

namespace metok {

template <typename T, int DH>
static void launch_form(const DecodeArgs& a, unsigned groups, hipStream_t st) {
    constexpr int NB = attend_blocks(DH);
    if (!a.table) launch_attention<T, DH, kDense, false, NB>(a, groups, st);
    else if (a.page_size % 16 != 0) launch_attention<T, DH, kRows, false, NB>(a, groups, st);
    else launch_attention<T, DH, kBlocks, false, NB>(a, groups, st);
}

void launch_wide_attention(const DecodeArgs& a, int dtype, int dh, unsigned groups, hipStream_t st) {
    if (dtype == METOK_BF16) {
        if (dh == 32) launch_form<bf16_t, 32>(a, groups, st);
        else if (dh == 64) launch_form<bf16_t, 64>(a, groups, st);
        else if (dh == 128) launch_form<bf16_t, 128>(a, groups, st);
        else launch_form<bf16_t, 256>(a, groups, st);
    } else {
        if (dh == 32) launch_form<float, 32>(a, groups, st);
        else if (dh == 64) launch_form<float, 64>(a, groups, st);
        else launch_form<float, 128>(a, groups, st);
    }
}

}  // namespace metok
