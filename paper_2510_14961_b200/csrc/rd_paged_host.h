// Host side of the paged cache, as rd_paged.cu offers it to the C ABI and to a session's layers.
#pragma once
#include <cuda_runtime.h>

#include "../../include/rd.h"
#include "rd_paged.cuh"

namespace rd {
// Records the text rd_last_cuda_error returns; RD_E_OOM or RD_E_CUDA.
int cuda_fail_at(cudaError_t e, const char* what, const char* file, int line);

// A row source other than three arrays: the sums of a layer's QKV GEMM.
int paged_append_sums(rd_paged* c, const PgBatch& b, int layer, const RowSource& sums, void* q_out, cudaStream_t st, bool chained);
int paged_attend(rd_paged* c, const PgBatch& b, int max_group_rows, int layer, const void* q, long long ldq, void* out, long long ldo,
                 float* lse, int window, int sinks, float scale, cudaStream_t st, bool chained, int* launches);
// Device word the kernels of this cache raise.
int* paged_status(rd_paged* c);
}  // namespace rd
