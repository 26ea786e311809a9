// Host side of the paged K/V cache: checks of arguments, choice of kernels, launches.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>

#include <algorithm>
#include <mutex>
#include <new>

#include "rd_paged_host.h"
#include "rd_paged_mma.cuh"
#include "rd_paged_simt.cuh"
#include "rd_paged_tc.cuh"

using namespace rd;
typedef __nv_bfloat16 bf16;

#define PCU(expr)                                                                    \
    do {                                                                             \
        cudaError_t e_ = (expr);                                                     \
        if (e_ != cudaSuccess) return cuda_fail_at(e_, #expr, "rd_paged.cu", __LINE__); \
    } while (0)
#define PTRY(expr)                    \
    do {                              \
        int rc_ = (expr);             \
        if (rc_ != RD_OK) return rc_; \
    } while (0)

struct rd_paged {
    rd_paged_config cfg;
    int device = 0, n_sms = 148, page_shift = 0;
    size_t es = 2;
    bool own_pages = false, tensor = false;
    void *k = nullptr, *v = nullptr;
    float2* cs = nullptr;
    char* work = nullptr;              // one allocation: everything below
    PgWork wa = {}, wb = {};           // launches that handle few / many rows per group
    int cap_a = 0, cap_b = 0;
    int* status = nullptr;
    PgMaps maps_few = {}, maps_many = {};  // boxes of at most 32 / 128 positions
    ~rd_paged() {
        if (own_pages) { cudaFree(k); cudaFree(v); }
        cudaFree(cs);
        cudaFree(work);
    }
};

// Packed rows (rows x query heads per K/V head) up to which a group goes to the kernel for few rows.
constexpr int PG_FEW_TENSOR = 64;
constexpr int PG_MAX_DEVICES = 64;

template <typename F> static cudaError_t opt_in(F* kern, int smem) {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
}
template <int D> static cudaError_t opt_in_tensor() {
    cudaError_t e = opt_in(pg_attend_mma_kernel<D, 1>, PgmCfg<D, 1>::SMEM);
    if (e == cudaSuccess) e = opt_in(pg_attend_mma_kernel<D, 2>, PgmCfg<D, 2>::SMEM);
    if (e == cudaSuccess) e = opt_in(pg_attend_mma_kernel<D, 4>, PgmCfg<D, 4>::SMEM);
    if (e == cudaSuccess) e = opt_in(pg_attend_tc_kernel<D>, PgtCfg<D>::SMEM);
    return e;
}
template <typename T, int DP> static cudaError_t opt_in_simt() {
    cudaError_t e = opt_in(pg_attend_few_kernel<T, DP>, PgsFew<T, DP>::SMEM);
    if (e == cudaSuccess) e = opt_in(pg_attend_many_kernel<T, DP>, PgsMany<T, DP>::SMEM);
    return e;
}
static int configure_device(int device) {
    static bool done[PG_MAX_DEVICES];
    static std::mutex mu;
    if (device < 0 || device >= PG_MAX_DEVICES) return RD_E_INVALID_ARG;
    std::lock_guard<std::mutex> lock(mu);
    if (done[device]) return RD_OK;
    PCU(opt_in_tensor<64>());
    PCU(opt_in_tensor<96>());
    PCU(opt_in_tensor<128>());
    PCU((opt_in_simt<float, 32>())); PCU((opt_in_simt<float, 64>())); PCU((opt_in_simt<float, 96>())); PCU((opt_in_simt<float, 128>()));
    PCU((opt_in_simt<bf16, 32>())); PCU((opt_in_simt<bf16, 64>())); PCU((opt_in_simt<bf16, 96>())); PCU((opt_in_simt<bf16, 128>()));
    done[device] = true;
    return RD_OK;
}

// 2-D view [rows, D] of the pages in boxes of `box_rows` positions x `cols` columns (128-byte swizzle for 64 columns,
// 64-byte swizzle for 32); boxes beyond the pages read as zeros.
static int encode(CUtensorMap* map, const void* ptr, unsigned long long rows, int D, int cols, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)D * 2};
    const cuuint32_t box[2] = {(cuuint32_t)cols, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = g_encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr,
                                      CU_TENSOR_MAP_INTERLEAVE_NONE, cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? RD_OK : RD_E_CUDA;
}
static int encode_set(PgMaps* m, const void* k, const void* v, unsigned long long rows, int D, int box_rows) {
    PTRY(encode(&m->k64, k, rows, D, 64, box_rows));
    PTRY(encode(&m->v64, v, rows, D, 64, box_rows));
    PTRY(encode(&m->k32, k, rows, D, 32, box_rows));
    return encode(&m->v32, v, rows, D, 32, box_rows);
}

static int create_impl(rd_paged* c, void* k, void* v) {
    const rd_paged_config& g = c->cfg;
    const unsigned long long pool_rows = (unsigned long long)g.n_layers * g.n_pages * g.n_kv_heads * g.page_size;
    PTRY(configure_device(c->device));
    if (k) {
        c->k = k; c->v = v;
    } else {
        c->own_pages = true;
        const size_t bytes = pool_rows * g.head_dim * c->es;
        PCU(cudaMalloc(&c->k, bytes));
        PCU(cudaMalloc(&c->v, bytes));
        PCU(cudaMemset(c->k, 0, bytes));
        PCU(cudaMemset(c->v, 0, bytes));
    }
    if (g.rope_base > 0.f) {
        const long long n = (long long)g.max_context * (g.head_dim / 2);
        PCU(cudaMalloc((void**)&c->cs, n * sizeof(float2)));
        pg_rope_table_kernel<<<(unsigned)std::min<long long>(2048, (n + 255) / 256), 256>>>(c->cs, g.max_context, g.head_dim / 2, log2((double)g.rope_base));
        PCU(cudaGetLastError());
    }
    c->tensor = g.dtype == RD_BF16 && (g.head_dim == 64 || g.head_dim == 96 || g.head_dim == 128);
    if (c->tensor) {
        PTRY(tc_init_driver());
        PTRY(encode_set(&c->maps_few, c->k, c->v, pool_rows, g.head_dim, std::min(g.page_size, PGM_KT)));
        PTRY(encode_set(&c->maps_many, c->k, c->v, pool_rows, g.head_dim, std::min(g.page_size, PGT_KT)));
    }
    // workspace: status | counters a | counters b | n_rec a, b | records a | records b | partial results a | b
    const int nb = 2 * c->n_sms, grp = g.n_heads / g.n_kv_heads, mb = c->tensor ? PGT_M : PGS_MANY;
    const long long packed = (long long)g.max_rows * grp;
    c->cap_a = (int)std::min<long long>(PG_MAX_GROUPS + packed / 16 + 1, 1 << 28);
    c->cap_b = (int)std::min<long long>(PG_MAX_GROUPS + packed / 64 + 1, 1 << 28);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    const size_t o_st = take(256), o_ca = take((size_t)nb * 4), o_cb = take((size_t)nb * 4), o_cut = take((size_t)nb * sizeof(PgPiece));     // (at most two blocks per SM)
    const size_t o_ra = take((size_t)c->cap_a * sizeof(PgRecord)), o_rb = take((size_t)c->cap_b * sizeof(PgRecord));
    // the kernels on tensor cores run one block per SM, the others up to two
    const size_t slots = 2 * (size_t)(c->tensor ? c->n_sms : nb);
    const size_t o_pa = take(slots * 64 * (g.head_dim + 2) * 4), o_pb = take(slots * mb * (g.head_dim + 2) * 4);
    PCU(cudaMalloc((void**)&c->work, at));
    PCU(cudaMemset(c->work, 0, o_ra));
    c->status = (int*)(c->work + o_st);
    c->wa = PgWork{(PgRecord*)(c->work + o_ra), c->status + 1, (int*)(c->work + o_ca), (float*)(c->work + o_pa), nullptr, c->status};
    c->wb = PgWork{(PgRecord*)(c->work + o_rb), c->status + 2, (int*)(c->work + o_cb), (float*)(c->work + o_pb), (PgPiece*)(c->work + o_cut), c->status};
    PCU(cudaDeviceSynchronize());
    return RD_OK;
}

extern "C" int rd_paged_create(const rd_paged_config* cfg, void* k_pages, void* v_pages, rd_paged** out) {
    if (!cfg || !out || (k_pages == nullptr) != (v_pages == nullptr)) return RD_E_INVALID_ARG;
    rd_paged_config g = *cfg;
    if (g.n_heads < 1 || g.n_kv_heads < 1 || g.n_heads % g.n_kv_heads) return RD_E_INVALID_ARG;
    if (g.head_dim < 2 || g.head_dim > 128 || g.head_dim % 2) return RD_E_INVALID_ARG;
    if (g.dtype != RD_F32 && g.dtype != RD_BF16) return RD_E_INVALID_ARG;
    if (g.page_size < 16 || g.page_size > 256 || (g.page_size & (g.page_size - 1))) return RD_E_INVALID_ARG;
    if (g.n_pages < 1 || g.n_layers < 1 || g.max_context < 1 || g.max_rows < 0 || !(g.rope_base >= 0.f) || !isfinite(g.rope_base)) return RD_E_INVALID_ARG;
    if (g.n_heads > 65536 || g.n_kv_heads > 65536 || ((uintptr_t)k_pages & 15) || ((uintptr_t)v_pages & 15)) return RD_E_INVALID_ARG;
    if (g.max_context > (1 << 30)) return RD_E_CAPACITY;
    // TMA names pool rows by 32-bit coordinates
    const double rows = (double)g.n_layers * g.n_pages * g.n_kv_heads * g.page_size;
    if (rows > 2147483647.0 - 512.0) return RD_E_CAPACITY;
    const size_t pool = (size_t)rows * g.head_dim * (g.dtype == RD_BF16 ? 2 : 4);
    if (k_pages && (uintptr_t)k_pages < (uintptr_t)v_pages + pool && (uintptr_t)v_pages < (uintptr_t)k_pages + pool) return RD_E_INVALID_ARG;
    if (g.max_rows == 0) g.max_rows = 65536;
    // packed rows (rows x query heads per K/V head) are counted in 31 bits
    if (g.max_rows > (1 << 24) || (double)g.max_rows * (g.n_heads / g.n_kv_heads) > 1e9) return RD_E_CAPACITY;
    rd_paged* c = new (std::nothrow) rd_paged();
    if (!c) return RD_E_OOM;
    c->cfg = g;
    c->es = g.dtype == RD_BF16 ? 2 : 4;
    while ((1 << c->page_shift) < g.page_size) c->page_shift++;
    cudaError_t e = cudaGetDevice(&c->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->n_sms, cudaDevAttrMultiProcessorCount, c->device);
    const int rc = e == cudaSuccess ? create_impl(c, k_pages, v_pages) : cuda_fail_at(e, "cudaGetDevice", "rd_paged.cu", __LINE__);
    if (rc) { delete c; return rc; }
    *out = c;
    return RD_OK;
}
extern "C" void rd_paged_destroy(rd_paged* c) {
    if (!c) return;
    int dev = -1;
    if (cudaGetDevice(&dev) == cudaSuccess && dev != c->device) cudaSetDevice(c->device);
    cudaDeviceSynchronize();
    const int own = c->device;
    delete c;
    if (dev >= 0 && dev != own) cudaSetDevice(dev);
}
extern "C" int rd_paged_pages(const rd_paged* c, void** k_pages, void** v_pages) {
    if (!c || !k_pages || !v_pages) return RD_E_INVALID_ARG;
    *k_pages = c->k;
    *v_pages = c->v;
    return RD_OK;
}

// ---- launches ---------------------------------------------------------------------------------------------------
static PgGeom geometry(const rd_paged* c, int layer) {
    const rd_paged_config& g = c->cfg;
    return PgGeom{g.n_heads, g.n_kv_heads, g.n_heads / g.n_kv_heads, g.head_dim, c->page_shift, g.n_pages, layer, g.max_context};
}
void rd::paged_set_status(rd_paged* c, int* status) { c->status = c->wa.status = c->wb.status = status; }

template <typename T>
__global__ void __launch_bounds__(256) pg_gather_kernel(const T* __restrict__ pages, PgGeom ge, const int* __restrict__ table, int table_stride,
                                                        int pos0, int n, float* __restrict__ dst) {
    const int width = ge.n_kv * ge.D;
    const long long total = (long long)n * width;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
        const int pos = pos0 + (int)(i / width), m = (int)(i % width), pi = pos >> ge.page_shift;
        const int pg = pi < table_stride ? table[pi] : -1;
        float x = 0.f;
        if (pg >= 0 && pg < ge.n_pages)
            x = pg_to_f(pages[((((((size_t)ge.layer * ge.n_pages + pg) * ge.n_kv + m / ge.D) << ge.page_shift) + (pos & ((1 << ge.page_shift) - 1))) * ge.D) + m % ge.D]);
        dst[i] = x;
    }
}
int rd::paged_gather(rd_paged* c, const int* table_row, int table_stride, int layer, int which, int pos0, int n, float* dst, cudaStream_t st) {
    const PgGeom ge = geometry(c, layer);
    const void* pages = which ? c->v : c->k;
    if (c->cfg.dtype == RD_BF16) pg_gather_kernel<bf16><<<256, 256, 0, st>>>((const bf16*)pages, ge, table_row, table_stride, pos0, n, dst);
    else pg_gather_kernel<float><<<256, 256, 0, st>>>((const float*)pages, ge, table_row, table_stride, pos0, n, dst);
    PCU(cudaGetLastError());
    return RD_OK;
}

template <typename T, int VEC, typename Src>
static int append_launch(rd_paged* c, const PgAppend& a, const Src& src, cudaStream_t st, bool chained) {
    const int per_head = a.ge.D / VEC, items = (a.ge.n_heads + 2 * a.ge.n_kv) * per_head;
    const int parts = (items + 32 * PG_APPEND_U - 1) / (32 * PG_APPEND_U), warps = std::min(parts, PG_APPEND_WARPS);       // warps of a row, of a block
    PgAppend b = a;
    b.head_magic = (unsigned)((0x100000000ull + per_head - 1) / per_head);
    PCU(launch_chained(pg_append_kernel<T, VEC, Src>, dim3(a.b.n_rows, (parts + warps - 1) / warps), dim3(32 * warps), 0, st, chained, b, src));
    return RD_OK;
}
// Features a thread moves at once: 16 bytes where head_dim is made of them, else four or two elements.
static int append_vec(const rd_paged* c) {
    const int d = c->cfg.head_dim, full = 16 / (int)c->es;
    return d % full == 0 ? full : d % 4 == 0 ? 4 : 2;
}
int rd::paged_append_sums(rd_paged* c, const PgBatch& b, int layer, const RowSource& sums, void* q_out, cudaStream_t st, bool chained) {
    const rd_paged_config& g = c->cfg;
    const PgAppend a{b, geometry(c, layer), c->status, c->cs, q_out, (long long)g.n_heads * g.head_dim, c->k, c->v};
    const PgSums src{sums, g.n_heads * g.head_dim, g.n_kv_heads * g.head_dim};
    if (g.dtype == RD_BF16) return g.head_dim % 4 == 0 ? append_launch<bf16, 4>(c, a, src, st, chained) : append_launch<bf16, 2>(c, a, src, st, chained);
    return g.head_dim % 4 == 0 ? append_launch<float, 4>(c, a, src, st, chained) : append_launch<float, 2>(c, a, src, st, chained);
}

// One attention launch: the plan (inside the kernel while it is small, else a kernel in front), then the kernel.
struct AttendShape { int M, threads, per_sm; };
template <int KT, typename Kern, typename... Extra>
static int attend_launch(rd_paged* c, PgAttend a, bool part_b, const AttendShape& s, bool can_inline, Kern kern, int smem, cudaStream_t st,
                         bool chained, int* launches, const Extra&... extra) {
    a.w = part_b ? c->wb : c->wa;
    a.rec_cap = part_b ? c->cap_b : c->cap_a;
    const long long packed = (long long)a.b.n_rows * a.ge.g;
    const long long tiles = std::min<long long>(a.b.n_groups + packed / s.M, a.rec_cap);       // most row tiles there can be
    const int lanes = pg_lanes(s.M, a.ge.g);
    a.inline_plan = can_inline && a.b.n_groups <= PG_INLINE_REC && tiles <= PG_INLINE_REC && tiles * lanes <= 4ll * s.threads;
    if (a.inline_plan) {
        a.rec_cap = PG_INLINE_REC;
    } else {
        const int blocks = (int)std::max<long long>(1, std::min<long long>(c->n_sms, (tiles * lanes + PG_PLAN_THREADS - 1) / PG_PLAN_THREADS));
        PCU(launch_chained(pg_plan_kernel<KT>, dim3(blocks), dim3(PG_PLAN_THREADS), (size_t)a.b.n_groups * sizeof(int), st, chained, a, s.M));
        if (launches) ++*launches;
    }
    PCU(launch_chained(kern, dim3(c->n_sms * s.per_sm), dim3(s.threads), (size_t)smem, st, chained, a, extra...));
    if (launches) ++*launches;
    return RD_OK;
}
template <int D> static int attend_few_tensor(rd_paged* c, const PgAttend& a, int m, cudaStream_t st, bool chained, int* launches) {
    if (m <= 16) return attend_launch<PGM_KT>(c, a, false, {16, PGM_THREADS, 1}, true, pg_attend_mma_kernel<D, 1>, PgmCfg<D, 1>::SMEM, st, chained, launches, c->maps_few);
    if (m <= 32) return attend_launch<PGM_KT>(c, a, false, {32, PGM_THREADS, 1}, true, pg_attend_mma_kernel<D, 2>, PgmCfg<D, 2>::SMEM, st, chained, launches, c->maps_few);
    return attend_launch<PGM_KT>(c, a, false, {64, PGM_THREADS, 1}, true, pg_attend_mma_kernel<D, 4>, PgmCfg<D, 4>::SMEM, st, chained, launches, c->maps_few);
}
template <int D> static int attend_many_tensor(rd_paged* c, const PgAttend& a, cudaStream_t st, bool chained, int* launches) {
    PTRY(attend_launch<PGT_KT>(c, a, true, {PGT_M, PGT_THREADS, 1}, false, pg_attend_tc_kernel<D>, PgtCfg<D>::SMEM, st, chained, launches, c->maps_many));
    PgAttend j = a;
    j.w = c->wb;
    PCU(launch_chained(pg_join_tc_kernel<D>, dim3(c->n_sms, PGT_M / 32), dim3(256), 0, st, chained, j));
    if (launches) ++*launches;
    return RD_OK;
}
template <typename T, int DP> static int attend_simt(rd_paged* c, const PgAttend& a, bool many, cudaStream_t st, bool chained, int* launches) {
    if (!many) return attend_launch<PGS_KT>(c, a, false, {PGS_FEW, PGS_THREADS, 1}, true, pg_attend_few_kernel<T, DP>, PgsFew<T, DP>::SMEM, st, chained, launches);
    return attend_launch<PGS_KT>(c, a, true, {PGS_MANY, PGS_THREADS, PgsMany<T, DP>::PER_SM}, true, pg_attend_many_kernel<T, DP>, PgsMany<T, DP>::SMEM, st, chained, launches);
}
template <typename T> static int attend_simt_d(rd_paged* c, const PgAttend& a, bool many, cudaStream_t st, bool chained, int* launches) {
    if (a.ge.D <= 32) return attend_simt<T, 32>(c, a, many, st, chained, launches);
    if (a.ge.D <= 64) return attend_simt<T, 64>(c, a, many, st, chained, launches);
    if (a.ge.D <= 96) return attend_simt<T, 96>(c, a, many, st, chained, launches);
    return attend_simt<T, 128>(c, a, many, st, chained, launches);
}
static int attend_part(rd_paged* c, PgAttend a, bool many, int m, cudaStream_t st, bool chained, int* launches) {
    // The division's three numbers (rd_paged.cuh), in key tiles of the kernel, as measured:
    // few rows, tiles of 32 keys: an item's query, output and pipeline refill cost as much as 12 tiles (64 ragged tokens: 171 us
    // counted as 2, 130 as 6, 118 as 12); up to 40 tiles an item is faster alone than cut and joined (one token behind 543
    // positions, 55 heads: 17.5 us cut, 12.4 whole; one behind 1,000 on 8 heads: 13.3 cut, 17.1 whole).
    // many rows, tiles of 128 keys: 4 tiles (8,192-token prompt: 606 us counted as 2, 491 as 4 or 6), whole up to 8 (128 rows
    // behind 300 positions x 8: 35.6 cut, 25.7 whole).
    if (c->tensor) {
        a.min_share = many ? 1 : 8;
        a.item_cost = many ? 4 : 12;
        a.whole_units = many ? 8 : 40;
        if (many) return a.ge.D == 64 ? attend_many_tensor<64>(c, a, st, chained, launches) : a.ge.D == 96 ? attend_many_tensor<96>(c, a, st, chained, launches)
                                                                                                : attend_many_tensor<128>(c, a, st, chained, launches);
        return a.ge.D == 64 ? attend_few_tensor<64>(c, a, m, st, chained, launches) : a.ge.D == 96 ? attend_few_tensor<96>(c, a, m, st, chained, launches)
                                                                                       : attend_few_tensor<128>(c, a, m, st, chained, launches);
    }
    // CUDA cores, tiles of 64 keys: a tile takes longer than joining, so items are cut down to single tiles (24 rows behind 1,000
    // positions x 4: 50 us; with at least 4 tiles a share 68, whole up to 20 tiles 154)
    a.min_share = 1;
    a.item_cost = 2;
    a.whole_units = 2;
    return c->cfg.dtype == RD_BF16 ? attend_simt_d<bf16>(c, a, many, st, chained, launches) : attend_simt_d<float>(c, a, many, st, chained, launches);
}

int rd::paged_attend(rd_paged* c, const PgBatch& b, int max_group_rows, int layer, const void* q, long long ldq, void* out, long long ldo,
                     float* lse, int window, int sinks, float scale, cudaStream_t st, bool chained, int* launches) {
    PgAttend a = {};
    a.b = b;
    a.ge = geometry(c, layer);
    a.q = q; a.out = out; a.lse = lse; a.ldq = ldq; a.ldo = ldo; a.k = c->k; a.v = c->v;
    a.window = window;
    a.sinks = window > 0 ? sinks : 0;
    a.scale_log2 = (float)((scale > 0.f ? (double)scale : 1.0 / sqrt((double)c->cfg.head_dim)) * 1.4426950408889634);
    a.packed_lo = 0;
    a.packed_hi = 0x7fffffff;
    const int g = a.ge.g, few = c->tensor ? PG_FEW_TENSOR : PGS_FEW;
    const long long most = (long long)(max_group_rows > 0 ? std::min(max_group_rows, b.n_rows) : b.n_rows) * g;
    // Every group has few packed rows, or as many as the largest: one kernel takes them all.  Otherwise two
    // launches share the groups between them by their size.
    if (most <= few) return attend_part(c, a, false, (int)most, st, chained, launches);
    if (b.n_groups == 1 || !b.group_start || (long long)b.n_groups * most <= (long long)b.n_rows * g)
        return attend_part(c, a, true, 0, st, chained, launches);
    PgAttend small = a;
    small.packed_hi = few;
    a.packed_lo = few;
    PTRY(attend_part(c, a, true, 0, st, chained, launches));
    return attend_part(c, small, false, std::min(g, few), st, chained, launches);
}

// ---- C ABI --------------------------------------------------------------------------------------------------------
static int check_rows(const rd_paged* c, const rd_paged_rows* r, int layer, PgBatch* b) {
    if (!c || !r || layer < 0 || layer >= c->cfg.n_layers) return RD_E_INVALID_ARG;
    if (r->n_rows < 0 || r->n_groups < 1 || r->n_groups > PG_MAX_GROUPS || r->max_group_rows < 0 || r->table_stride < 1) return RD_E_INVALID_ARG;
    if ((!r->row_pos && r->n_rows) || !r->table || (!r->group_start && r->max_group_rows < 1)) return RD_E_INVALID_ARG;
    if (((uintptr_t)r->row_pos | (uintptr_t)r->table | (uintptr_t)r->group_start) & 3) return RD_E_INVALID_ARG;
    if (r->n_rows > c->cfg.max_rows) return RD_E_CAPACITY;
    int dev = -1;
    PCU(cudaGetDevice(&dev));
    if (dev != c->device) return RD_E_STATE;
    *b = PgBatch{r->n_rows, r->n_groups, r->max_group_rows, r->group_start, r->row_pos, r->table, r->table_stride};
    return RD_OK;
}
// An array of n_rows rows of `width` elements, `ld` apart: aligned to the vectors the kernels move.
static bool array_ok(const rd_paged* c, const void* p, int64_t ld, int64_t width) {
    const size_t vec = append_vec(c) * c->es;
    return p && ld >= width && ld < (1ll << 40) && (uintptr_t)p % vec == 0 && (size_t)ld * c->es % vec == 0;
}
struct Extent { uintptr_t lo, hi; };
static Extent extent(const rd_paged* c, const void* p, int64_t ld, int64_t width, int n_rows) {
    return {(uintptr_t)p, (uintptr_t)p + ((size_t)(n_rows - 1) * ld + width) * c->es};
}
static bool overlap(const Extent& a, const Extent& b) { return a.lo < b.hi && b.lo < a.hi; }

extern "C" int rd_paged_append(rd_paged* c, const rd_paged_rows* rows, int32_t layer, const void* q, int64_t ldq, const void* k, int64_t ldk,
                               const void* v, int64_t ldv, void* q_out, int64_t ldqo, void* cuda_stream) {
    PgBatch b;
    PTRY(check_rows(c, rows, layer, &b));
    const rd_paged_config& g = c->cfg;
    const int64_t wq = (int64_t)g.n_heads * g.head_dim, wk = (int64_t)g.n_kv_heads * g.head_dim;
    if (b.n_rows == 0) return RD_OK;
    if (!array_ok(c, q, ldq, wq) || !array_ok(c, k, ldk, wk) || !array_ok(c, v, ldv, wk) || !array_ok(c, q_out, ldqo, wq)) return RD_E_INVALID_ARG;
    const bool in_place = q_out == q && ldqo == ldq;
    const Extent eo = extent(c, q_out, ldqo, wq, b.n_rows);
    // (q, k and v are only read and may share one array; written are q_out and the pages)
    if (!in_place && overlap(eo, extent(c, q, ldq, wq, b.n_rows))) return RD_E_INVALID_ARG;
    const Extent ek = extent(c, k, ldk, wk, b.n_rows), ev = extent(c, v, ldv, wk, b.n_rows);
    if (!in_place && (overlap(eo, ek) || overlap(eo, ev))) return RD_E_INVALID_ARG;
    const size_t pool = (size_t)g.n_layers * g.n_pages * g.n_kv_heads * g.page_size * g.head_dim * c->es;
    for (const void* pages : {(const void*)c->k, (const void*)c->v}) {
        const Extent ep{(uintptr_t)pages, (uintptr_t)pages + pool};
        if (overlap(ep, eo) || overlap(ep, ek) || overlap(ep, ev) || overlap(ep, extent(c, q, ldq, wq, b.n_rows))) return RD_E_INVALID_ARG;
    }
    const PgAppend a{b, geometry(c, layer), c->status, c->cs, q_out, ldqo, c->k, c->v};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int vec = append_vec(c);
    if (g.dtype == RD_BF16) {
        const PgArrays<bf16> src{(const bf16*)q, (const bf16*)k, (const bf16*)v, ldq, ldk, ldv};
        return vec == 8 ? append_launch<bf16, 8>(c, a, src, st, true) : vec == 4 ? append_launch<bf16, 4>(c, a, src, st, true) : append_launch<bf16, 2>(c, a, src, st, true);
    }
    const PgArrays<float> src{(const float*)q, (const float*)k, (const float*)v, ldq, ldk, ldv};
    return vec == 4 ? append_launch<float, 4>(c, a, src, st, true) : append_launch<float, 2>(c, a, src, st, true);
}

extern "C" int rd_paged_attend(rd_paged* c, const rd_paged_rows* rows, int32_t layer, const void* q, int64_t ldq, void* out, int64_t ldo,
                               float* lse, int32_t window, int32_t sinks, float scale, void* cuda_stream) {
    PgBatch b;
    PTRY(check_rows(c, rows, layer, &b));
    const rd_paged_config& g = c->cfg;
    const int64_t wq = (int64_t)g.n_heads * g.head_dim;
    if (window < 0 || sinks < 0 || !(scale >= 0.f) || !isfinite(scale)) return RD_E_INVALID_ARG;
    if (b.n_rows == 0) return RD_OK;
    if (!array_ok(c, q, ldq, wq) || !array_ok(c, out, ldo, wq) || ((uintptr_t)lse & 3)) return RD_E_INVALID_ARG;
    const Extent eo = extent(c, out, ldo, wq, b.n_rows), eq = extent(c, q, ldq, wq, b.n_rows);
    const size_t pool = (size_t)g.n_layers * g.n_pages * g.n_kv_heads * g.page_size * g.head_dim * c->es;
    const Extent pk{(uintptr_t)c->k, (uintptr_t)c->k + pool}, pv{(uintptr_t)c->v, (uintptr_t)c->v + pool};
    if (overlap(eo, eq) || overlap(eo, pk) || overlap(eo, pv)) return RD_E_INVALID_ARG;
    if (lse) {
        const Extent el{(uintptr_t)lse, (uintptr_t)lse + (size_t)b.n_rows * g.n_heads * 4};
        if (overlap(el, eo) || overlap(el, eq) || overlap(el, pk) || overlap(el, pv)) return RD_E_INVALID_ARG;
    }
    return paged_attend(c, b, rows->max_group_rows, layer, q, ldq, out, ldo, lse, window, sinks, scale, (cudaStream_t)cuda_stream, true, nullptr);
}

extern "C" int rd_paged_sync(rd_paged* c, void* cuda_stream) {
    if (!c) return RD_E_INVALID_ARG;
    int dev = -1, st = 0;
    PCU(cudaGetDevice(&dev));
    if (dev != c->device) return RD_E_STATE;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    PCU(cudaMemcpyAsync(&st, c->status, sizeof st, cudaMemcpyDeviceToHost, s));
    PCU(cudaStreamSynchronize(s));
    if (st & PG_ST_TIMEOUT) return RD_E_TIMEOUT;
    if (st == 0) return RD_OK;
    PCU(cudaMemsetAsync(c->status, 0, sizeof(int), s));
    PCU(cudaStreamSynchronize(s));
    return RD_E_INVALID_ARG;
}
