// Attention over bf16 caches.
#include "wg_attend.h"

int32_t attend_bf16(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st) {
    return launch_attend<__nv_bfloat16>(c, a, most_tiles, st);
}
