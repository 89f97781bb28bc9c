// Which part of which product a wave of dw_of_few (few_tokens.hpp) takes.  Plain integer arithmetic without HIP: a CPU test compiles this header.
#pragma once
#include <stdint.h>

#ifndef FG_HOST_DEVICE
#ifdef __HIP__
#define FG_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define FG_HOST_DEVICE inline
#endif
#endif

namespace fg {

// A product of words x dim results is cut into items of `each` words and 128 columns (a strip).
constexpr int64_t kFewStrip = 128;
FG_HOST_DEVICE int64_t few_items(int64_t words, int64_t dim, int64_t each) { return (words + each - 1) / each * ((dim + kFewStrip - 1) / kFewStrip); }

// Wave `wave` of a launch for two products, either of which may be empty: their items one after the other, then the spare waves of the last workgroup, which have
// nothing to do (false; an empty product has no strips to divide by).
struct FewItem { bool second; int64_t word; int strip; };
FG_HOST_DEVICE bool few_item(int64_t wave, int64_t items0, int64_t dim0, int64_t items1, int64_t dim1, int64_t each, FewItem &out) {
    out.second = wave >= items0;
    const int64_t item = out.second ? wave - items0 : wave;
    if (item >= (out.second ? items1 : items0)) return false;
    const int strips = (int)(((out.second ? dim1 : dim0) + kFewStrip - 1) / kFewStrip);
    out.word = item / strips * each;
    out.strip = (int)(item % strips);
    return true;
}

}  // namespace fg
