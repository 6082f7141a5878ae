// Attention over caches of 8-bit floats.
#include "wg_attend.h"

int32_t attend_e4m3(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st) {
    return launch_attend<E4m3>(c, a, most_tiles, st);
}
