// The vocabulary loss of a few rows; see lm_loss_rows.cu.
#pragma once
#include <stddef.h>

#include "../../include/slim_lm.h"

namespace slim {
namespace lm {

// Whether these sizes take this path.
bool rows_fit(long long N, int D, slim_dtype dtype);
size_t rows_workspace(int N, int D, int V, bool bwd);
// Arguments as in slim_vocab_loss_fwd / slim_vocab_loss_bwd, already checked.
slim_status rows_fwd(const void* x, const void* w, const void* targets, slim_index it, int N, int D,
                     int V, slim_dtype dtype, long long ignore, float* loss, float* lse,
                     float* total, void* workspace, cudaStream_t s);
slim_status rows_bwd(const void* x, const void* w, const void* targets, slim_index it,
                     const float* lse, const float* dloss, int dstride, const float* count, int N,
                     int D, int V, slim_dtype dtype, long long ignore, void* dx, void* dw,
                     void* workspace, cudaStream_t s);

}  // namespace lm
}  // namespace slim
