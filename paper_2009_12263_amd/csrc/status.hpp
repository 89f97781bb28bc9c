// What the host files of the library share: the message of a failing call and checks of pointers.
#pragma once
#include <stdint.h>

#include "../../include/flexgemm.h"

namespace fg {

// Notes the message that fg_last_error() returns and gives the status back.
fg_status fail(fg_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// fg_gemm where an operand that is not K-contiguous stores its first k_rows k's only (0: all of them); the others count as zero, and K can be
// rounded up to what the tiled kernels take.  For operands that meet their alignment (aligned16 pointers, leading dimensions of 8).  Partial products of a split of
// K go to `scratch` (16-byte aligned); one that does not fit its scratch_bytes is computed in one pass.  Nothing is allocated.
fg_status gemm_stored(int64_t M, int64_t N, int64_t K, int64_t k_rows, float alpha, const fg_matrix *A, const fg_matrix *B, float beta,
                      const fg_matrix *C, const fg_matrix *D, float *scratch, int64_t scratch_bytes, void *hip_stream);
// The scratch that gemm_stored has a use for, where A, B and D are row-major.
int64_t gemm_stored_scratch(int64_t M, int64_t N, int64_t K);

// Leading dimensions that the tiled kernels take stay below these: of A and B where they are K-contiguous (a lane's offsets within a tile's rows fit 31 bits),
// and of C and D.
constexpr int64_t kKContiguousLd = 1ll << 22, kResultLd = 1ll << 21;

inline bool aligned_to(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace fg
