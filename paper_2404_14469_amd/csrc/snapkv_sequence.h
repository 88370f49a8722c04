// Which sequence of a packed batch a token belongs to (snapkv_append.hip, snapkv_mx.hip, snapkv_shared.hip).
#ifndef SNAPKV_SEQUENCE_H_
#define SNAPKV_SEQUENCE_H_

#include <hip/hip_runtime.h>

namespace snapkv {
namespace {

// Sequences whose end lies at or before token t (cu ascending): t's sequence, or B behind the last.  All lanes look at once, each at
// the last end of a 64th of those in question, and go on within the first 64th whose end lies behind t: one trip to memory for
// up to 64 sequences, four for 2^24.  (2^18 sequences of one token each 21 ms with all ends counted, 0.14 so.)
__device__ __forceinline__ int sequence_of(const int32_t* cu, int B, int t, int lane) {
    int lo = 0;
    for (int width = B; width > 0;) {                 // the ends before lo are at or before t, those from lo + width on are not
        const int w = (width + 63) / 64, last = min((lane + 1) * w, width) - 1;
        const int k = __popcll(__ballot(lane * w < width && cu[lo + last + 1] <= t));
        lo += min(k * w, width);
        width = min(w, width - k * w) - 1;            // (its last end lies behind t)
    }
    return lo;
}

}  // namespace
}  // namespace snapkv
#endif
