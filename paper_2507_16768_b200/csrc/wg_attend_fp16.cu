// Attention over fp16 caches.
#include "wg_attend.h"

int32_t attend_fp16(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st) {
    return launch_attend<__half>(c, a, most_tiles, st);
}
