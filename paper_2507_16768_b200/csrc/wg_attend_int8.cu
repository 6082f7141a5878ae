// Attention over int8 caches.
#include "wg_attend.h"

int32_t attend_int8(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st) {
    return launch_attend<Int8>(c, a, most_tiles, st);
}
