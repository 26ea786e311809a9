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
// The kernels of this cache raise `status` (a device word) instead of the cache's own.
void paged_set_status(rd_paged* c, int* status);
// K (which 0) or V of positions pos0 .. pos0 + n - 1 of the sequence with this table row, as float32 [n, n_kv_heads * head_dim];
// positions without a page read as zeros.
int paged_gather(rd_paged* c, const int* table_row, int table_stride, int layer, int which, int pos0, int n, float* dst, cudaStream_t st);
}  // namespace rd
