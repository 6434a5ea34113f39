// Attention of one new token over short caches: a workgroup to every (video, kv head), its waves the pair's tiles, their results joined in
// LDS.  One launch, no workspace.
#include "decode_attention.h"

namespace metok {

template <typename T, int DH>
static void launch_form(const DecodeArgs& a, unsigned pairs, hipStream_t st) {
    constexpr dim3 threads(64 * kAttendWholeWaves);
    if (!a.table) hipLaunchKernelGGL((decode_attention_kernel<T, DH, kDense, false, false, 1, true>), dim3(pairs), threads, 0, st, a);
    else if (a.page_size % 16 != 0) hipLaunchKernelGGL((decode_attention_kernel<T, DH, kRows, false, false, 1, true>), dim3(pairs), threads, 0, st, a);
    else hipLaunchKernelGGL((decode_attention_kernel<T, DH, kBlocks, false, false, 1, true>), dim3(pairs), threads, 0, st, a);
}

void launch_short_attention(const DecodeArgs& a, int dtype, int dh, unsigned pairs, hipStream_t st) {
    if (dtype == METOK_BF16) {
        if (dh == 32) launch_form<bf16_t, 32>(a, pairs, st);
        else if (dh == 64) launch_form<bf16_t, 64>(a, pairs, st);
        else if (dh == 128) launch_form<bf16_t, 128>(a, pairs, st);
        else launch_form<bf16_t, 256>(a, pairs, st);
    } else {
        if (dh == 32) launch_form<float, 32>(a, pairs, st);
        else if (dh == 64) launch_form<float, 64>(a, pairs, st);
        else launch_form<float, 128>(a, pairs, st);
    }
}

}  // namespace metok
