// Attention over a paged cache on the CUDA cores: float32 (whose products the tensor cores would round), and
// bf16 with head sizes the tensor-core kernels do not take.  Any even head_dim up to DP = 32, 64, 96 or 128
// (shared-memory rows are padded with zeros).  Arguments, row tiles and the division of the work: rd_paged.cuh.
//
// pg_attend_few_kernel (row tiles of 16): bound by the K/V stream.  A 64-key tile is eight runs of 8 keys, one
//   per warp; a warp brings its run in by itself (16-byte cp.async, three stages of its own) and keeps its own
//   maximum, sum and output, so no warp waits for another before the end of an item.  Four lanes share a key's
//   dot product, a lane owns DP / 32 output features.
// pg_attend_many_kernel (row tiles of 64): bound by the FMA rate.  Eight warps own 8 rows each; a lane takes
//   keys `lane` and `lane + 32` of the tile for 8 rows (16 FMAs per two K and eight Q reads of 4 floats, the Q
//   reads being broadcasts), then DP / 32 output features for 8 rows.  K(t + 1) is requested behind Q K^T of
//   tile t and V(t + 1) behind P V, so one buffer each suffices.
//
// Measured: 16 tokens behind 8,000 positions, 16/4 heads of 64, float32: 103 us = 2.5 TB/s; 4 x 24 rows behind 1,000: 50 us, about
// 6 us per 64-key tile of a block, barriers and shared-memory reads beside 1,024 FMAs per warp.  (mma.sync on sums of two tf32
// numbers took 44 us and lost precision: 1e-6 to 6e-6 against 64 bits where float32 sums have 4e-7.)
// Keys no row of a tile sees are not read; a tile with a key that some row does not see goes key by key where V is not
// finite (0 times an infinity would be a NaN), so what lies in unwritten places of a page does not matter.
#pragma once
#include "rd_paged.cuh"

namespace rd {

constexpr int PGS_THREADS = 256;
constexpr int PGS_KT = 64;
constexpr int PGS_FEW = 16, PGS_MANY = 64;

__device__ __forceinline__ void pgs_cp16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void pgs_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void pgs_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void pgs_f4(const float* p, float* x) { const float4 v = *reinterpret_cast<const float4*>(p); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
__device__ __forceinline__ void pgs_f4(const __nv_bfloat16* p, float* x) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
    x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
}
// One cache row into shared memory (columns from D on stay zero): whole 16-byte chunks, or element by element
// when the row is not made of them.  Chunks c0, c0 + step, ...
template <typename T>
__device__ __forceinline__ void pgs_row_in(T* dst, const T* src, int D, int c0, int step) {
    constexpr int V = 16 / sizeof(T);
    if (D % V == 0) {
        for (int c = c0; c < D / V; c += step) pgs_cp16(dst + c * V, src + c * V);
    } else {
        for (int c = c0; c < D; c += step) dst[c] = src[c];
    }
}
// Where a thread's key of successive tiles lies: the table entry is asked for a tile ahead of its use, so that no
// copy waits for one.  row < 0: a key no row sees (it is not read: it may lie beyond the sequence's pages).
struct PgsKey {
    int next_key, entry;                                   // key of the next tile (-1: none), its table entry
    bool bad;
    __device__ __forceinline__ void ask(const PgAttend& p, const PgPiece& pc, const PgSpan& span, int lo_key, int i, int offset) {
        next_key = -1;
        if (i < pc.i1) {
            const int key = pg_tile_key(span, i, 64) + offset;
            if (key <= pc.pmax && (key >= lo_key || key < p.sinks)) next_key = key;
        }
        const int pi = next_key >> p.ge.page_shift;
        entry = next_key >= 0 && pi < p.b.table_stride ? p.b.table[(size_t)pc.grp * p.b.table_stride + pi] : -1;
    }
    __device__ __forceinline__ long long row(const PgAttend& p, const PgPiece& pc) {
        if (next_key < 0) return -1;
        if (entry < 0 || entry >= p.ge.n_pages) { bad = true; return -1; }      // (results of such rows are undefined)
        return ((((long long)p.ge.layer * p.ge.n_pages + entry) * p.ge.n_kv + pc.head) << p.ge.page_shift) + (next_key & ((1 << p.ge.page_shift) - 1));
    }
};
__device__ __forceinline__ int pgs_row_position(const PgAttend& p, const PgPiece& pc, int M, int r, int limit) {
    const long long pk = (long long)pc.rt * M + r;
    if (r >= M || pk >= (long long)pc.n * p.ge.g) return -1;
    const int pos = p.b.row_pos[pc.a + (int)(pk / p.ge.g)];
    return pos < limit ? pos : -1;
}

template <typename T, int DP> struct PgsFew {
    static constexpr int LD = DP + 16 / (int)sizeof(T);          // padded row: 16 bytes
    static constexpr int KEYS = 8;
    static constexpr int RUN = KEYS * LD * (int)sizeof(T);       // 8 rows of K or V
    static constexpr int STAGES = 204800 / (16 * RUN) < 8 ? 204800 / (16 * RUN) : 8;      // as many as fit: bytes in flight are the stream's rate
    static constexpr int RING = 8 * STAGES * 2 * RUN;            // every warp's own
    static constexpr int QLD = DP + 4;
    static constexpr int Q_BYTES = PGS_FEW * QLD * 4;
    static constexpr int O_BYTES = 8 * PGS_FEW * (DP + 2) * 4;   // the warps' results at the end of an item (ring space)
    static constexpr int SMEM = (RING > O_BYTES ? RING : O_BYTES) + Q_BYTES;
};

template <typename T, int DP>
__global__ void __launch_bounds__(PGS_THREADS, 1) pg_attend_few_kernel(const __grid_constant__ PgAttend p) {
    using C = PgsFew<T, DP>;
    constexpr int M = PGS_FEW, LD = C::LD, QLD = C::QLD, S = C::STAGES, E = DP / 32;
    extern __shared__ __align__(16) uint8_t pgs_raw[];
    float* Qs = reinterpret_cast<float*>(pgs_raw);
    uint8_t* ring = pgs_raw + C::Q_BYTES;
    __shared__ PgPlanSmem<PG_INLINE_REC> plan;
    __shared__ int flag;
    __shared__ float4 Ps[8][C::KEYS];                              // per warp: probabilities of 8 keys for four rows
    pdl_enter();
    pg_plan_share<PGS_THREADS, PGS_KT>(p, M, plan);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, D = p.ge.D;
    const int limit = pg_pos_limit(p.b, p.ge);
    T* mine = reinterpret_cast<T*>(ring + warp * S * 2 * C::RUN);
    const int key_l = lane >> 2, quarter = lane & 3;
    PgsKey key;
    key.bad = false;
    auto sync = [] { __syncthreads(); };
    PgWalk walk;
    walk.start(p, plan);
    PgPiece pc;
    while (walk.next(p.ge.n_kv, &pc)) {
        const PgSpan span = pg_span<PGS_KT>(pc.pmin, pc.pmax, p.window, p.sinks);
        const int rows = (int)min((long long)M, (long long)pc.n * p.ge.g - (long long)pc.rt * M);
        const int lo_key = p.window > 0 ? max(0, pc.pmin - p.window + 1) : 0;
        // the ring is zero where a row is padded (and where rows are not loaded): it held the last item's results
        for (int i = tid; i < C::RING / 16; i += PGS_THREADS) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
        for (int i = tid; i < M * DP; i += PGS_THREADS) {
            const int r = i / DP, e = i % DP;
            float x = 0.f;
            if (r < rows && e < D) {
                const long long pk = (long long)pc.rt * M + r;
                x = pg_to_f(((const T*)p.q)[(size_t)(pc.a + pk / p.ge.g) * p.ldq + (size_t)(pc.head * p.ge.g + pk % p.ge.g) * D + e]) * p.scale_log2;
            }
            Qs[r * QLD + e] = x;
        }
        __syncthreads();
        key.ask(p, pc, span, lo_key, pc.i0, warp * C::KEYS + key_l);
        auto issue = [&](int i) {                                  // tile i's run of this warp into stage (i - i0) % S
            T* kd = mine + (size_t)((i - pc.i0) % S) * 2 * C::KEYS * LD;
            const long long row = key.row(p, pc);
            if (row >= 0) {
                pgs_row_in(kd + key_l * LD, (const T*)p.k + (size_t)row * D, D, quarter, 4);
                pgs_row_in(kd + (C::KEYS + key_l) * LD, (const T*)p.v + (size_t)row * D, D, quarter, 4);
            }
            pgs_commit();
            key.ask(p, pc, span, lo_key, i + 1, warp * C::KEYS + key_l);
        };
        int pos[M];
#pragma unroll
        for (int r = 0; r < M; r++) pos[r] = pgs_row_position(p, pc, M, r, limit);
        float m[M], l[M], o[M][E];
#pragma unroll
        for (int r = 0; r < M; r++) {
            m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
            for (int e = 0; e < E; e++) o[r][e] = 0.f;
        }
        for (int i = 0; i < S - 1; i++) issue(pc.i0 + i);
        for (int i = pc.i0; i < pc.i1; i++) {
            issue(i + S - 1);
            pgs_wait<S - 1>();
            __syncwarp();
            const T* Kt = mine + (size_t)((i - pc.i0) % S) * 2 * C::KEYS * LD;
            const T* Vt = Kt + C::KEYS * LD;
            const int key0 = pg_tile_key(span, i, PGS_KT) + warp * C::KEYS;
            float kk[DP / 4];
#pragma unroll
            for (int c = 0; c < DP / 16; c++) pgs_f4(Kt + key_l * LD + c * 16 + quarter * 4, kk + c * 4);
            float v[C::KEYS][E];
#pragma unroll
            for (int j = 0; j < C::KEYS; j++)
#pragma unroll
                for (int e = 0; e < E; e++) v[j][e] = pg_to_f(Vt[j * LD + lane + 32 * e]);
            const bool partial = pg_partial<PGS_KT>(key0 - warp * C::KEYS, pc.pmin, pc.pmax, p.window, p.sinks);
            bool exact = false;                                    // an unseen key with a V that is not finite: 0 times it would be a NaN
            if (partial) {
                float probe = 0.f;
#pragma unroll
                for (int j = 0; j < C::KEYS; j++)
#pragma unroll
                    for (int e = 0; e < E; e++) probe = fmaf(v[j][e], 0.f, probe);
                exact = __any_sync(0xffffffffu, probe != 0.f);
            }
            // four rows at a time: their reductions run next to each other, their probabilities go through shared memory once
#pragma unroll
            for (int r0 = 0; r0 < M; r0 += 4) {
                if (r0 >= rows) break;
                float s[4] = {0.f, 0.f, 0.f, 0.f}, mx[4];
#pragma unroll
                for (int c = 0; c < DP / 16; c++)
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        const float4 x = *reinterpret_cast<const float4*>(Qs + (r0 + q) * QLD + c * 16 + quarter * 4);
                        s[q] = fmaf(x.x, kk[c * 4], s[q]); s[q] = fmaf(x.y, kk[c * 4 + 1], s[q]);
                        s[q] = fmaf(x.z, kk[c * 4 + 2], s[q]); s[q] = fmaf(x.w, kk[c * 4 + 3], s[q]);
                    }
#pragma unroll
                for (int w = 1; w < 4; w *= 2)
#pragma unroll
                    for (int q = 0; q < 4; q++) s[q] += __shfl_xor_sync(0xffffffffu, s[q], w);
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    if (partial && !(pos[r0 + q] >= 0 && pg_sees(pos[r0 + q], key0 + key_l, p.window, p.sinks))) s[q] = -INFINITY;
                    mx[q] = s[q];
                }
#pragma unroll
                for (int w = 4; w < 32; w *= 2)
#pragma unroll
                    for (int q = 0; q < 4; q++) mx[q] = fmaxf(mx[q], __shfl_xor_sync(0xffffffffu, mx[q], w));
                float4 pj;
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const float mn = fmaxf(m[r0 + q], mx[q]), u = mn == -INFINITY ? 0.f : mn, f = exp2f(m[r0 + q] - u);      // (0 while nothing was seen)
                    m[r0 + q] = mn;
                    const float x = exp2f(s[q] - u);
                    l[r0 + q] = l[r0 + q] * f + (quarter == 0 ? x : 0.f);
#pragma unroll
                    for (int e = 0; e < E; e++) o[r0 + q][e] *= f;
                    if (q == 0) pj.x = x; else if (q == 1) pj.y = x; else if (q == 2) pj.z = x; else pj.w = x;
                }
                if (quarter == 0) Ps[warp][key_l] = pj;
                __syncwarp();
#pragma unroll
                for (int j = 0; j < C::KEYS; j++) {
                    const float4 w = Ps[warp][j];
                    if (!exact) {
#pragma unroll
                        for (int e = 0; e < E; e++) {
                            o[r0][e] = fmaf(w.x, v[j][e], o[r0][e]); o[r0 + 1][e] = fmaf(w.y, v[j][e], o[r0 + 1][e]);
                            o[r0 + 2][e] = fmaf(w.z, v[j][e], o[r0 + 2][e]); o[r0 + 3][e] = fmaf(w.w, v[j][e], o[r0 + 3][e]);
                        }
                    } else {
                        const int jj = key0 + j;
#pragma unroll
                        for (int q = 0; q < 4; q++) {
                            if (pos[r0 + q] < 0 || !pg_sees(pos[r0 + q], jj, p.window, p.sinks)) continue;
                            const float wq = q == 0 ? w.x : q == 1 ? w.y : q == 2 ? w.z : w.w;
#pragma unroll
                            for (int e = 0; e < E; e++) o[r0 + q][e] = fmaf(wq, v[j][e], o[r0 + q][e]);
                        }
                    }
                }
                __syncwarp();
            }
            __syncwarp();                                          // the run is free for the next copy
        }
        pgs_wait<0>();
        __syncthreads();
        // the eight warps' results meet in shared memory: [warp][row][DP + 2]
        float* Os = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int r = 0; r < M; r++) {
            float ls = l[r];
#pragma unroll
            for (int w = 1; w < 32; w *= 2) ls += __shfl_xor_sync(0xffffffffu, ls, w);
            float* d = Os + (size_t)(warp * M + r) * (DP + 2);
#pragma unroll
            for (int e = 0; e < E; e++) d[lane + 32 * e] = o[r][e];
            if (lane == 0) { d[DP] = m[r]; d[DP + 1] = ls; }
        }
        __syncthreads();
        const bool whole = pc.c_first == pc.c_last;
        float* slot = whole ? nullptr : pg_slot(p.w, blockIdx.x, pc.c_first, M, D);
        for (int it = tid; it < rows * D; it += PGS_THREADS) {
            const int r = it / D, e = it % D;
            float mx = -INFINITY;
            for (int w = 0; w < 8; w++) mx = fmaxf(mx, Os[(size_t)(w * M + r) * (DP + 2) + DP]);
            float acc = 0.f, den = 0.f;
            for (int w = 0; w < 8; w++) {
                const float* d = Os + (size_t)(w * M + r) * (DP + 2);
                const float f = d[DP] == -INFINITY ? 0.f : exp2f(d[DP] - mx);
                acc = fmaf(d[e], f, acc);
                den = fmaf(d[DP + 1], f, den);
            }
            const long long pk = (long long)pc.rt * M + r;
            const int row = pc.a + (int)(pk / p.ge.g), hd = pc.head * p.ge.g + (int)(pk % p.ge.g);
            if (whole) {
                const int rp = p.b.row_pos[row];
                if (rp < 0 || rp >= limit) continue;
                ((T*)p.out)[(size_t)row * p.ldo + (size_t)hd * D + e] = pg_from_f<T>(acc / den);
                if (p.lse && e == 0) p.lse[(size_t)row * p.ge.n_heads + hd] = (mx + log2f(den)) * 0.6931471805599453f;
            } else {
                slot[(size_t)r * D + e] = acc;
                if (e == 0) { slot[(size_t)M * D + 2 * r] = mx; slot[(size_t)M * D + 2 * r + 1] = den; }
            }
        }
        if (!whole && pg_arrive_last(p.w, pc, tid == 0, &flag, sync)) pg_join_any<T>(p, pc, M, D, tid, PGS_THREADS);
        __syncthreads();
    }
    if (key.bad) atomicOr(p.w.status, PG_ST_BAD_PAGE);
}

template <typename T, int DP> struct PgsMany {
    static constexpr int LD = DP + 16 / (int)sizeof(T);
    static constexpr int TILE = PGS_KT * LD * (int)sizeof(T);
    static constexpr int QLD = DP + 4, PLD = PGS_KT + 4;
    static constexpr int SMEM = 2 * TILE + PGS_MANY * QLD * 4 + PGS_MANY * PLD * 4;
    static constexpr int PER_SM = DP <= 64 ? 2 : 1;
};

// Two blocks share an SM where their tiles fit (head_dim up to 64): one block's barriers hide behind the other's work.
template <typename T, int DP>
__global__ void __launch_bounds__(PGS_THREADS, PgsMany<T, DP>::PER_SM) pg_attend_many_kernel(const __grid_constant__ PgAttend p) {
    using C = PgsMany<T, DP>;
    constexpr int M = PGS_MANY, LD = C::LD, QLD = C::QLD, PLD = C::PLD, E = DP / 32, RW = 8;
    extern __shared__ __align__(16) uint8_t pgs_raw[];
    T* Ks = reinterpret_cast<T*>(pgs_raw);
    T* Vs = reinterpret_cast<T*>(pgs_raw + C::TILE);
    float* Qs = reinterpret_cast<float*>(pgs_raw + 2 * C::TILE);
    float* Ps = Qs + M * QLD;
    __shared__ PgPlanSmem<PG_INLINE_REC> plan;
    __shared__ int flag;
    pdl_enter();
    pg_plan_share<PGS_THREADS, PGS_KT>(p, M, plan);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, D = p.ge.D;
    const int limit = pg_pos_limit(p.b, p.ge), r_w = warp * RW, kl = tid >> 2;
    PgsKey key;
    key.bad = false;
    auto sync = [] { __syncthreads(); };
    for (int i = tid; i < 2 * C::TILE / 16; i += PGS_THREADS) reinterpret_cast<uint4*>(pgs_raw)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    PgWalk walk;
    walk.start(p, plan);
    PgPiece pc;
    while (walk.next(p.ge.n_kv, &pc)) {
        const PgSpan span = pg_span<PGS_KT>(pc.pmin, pc.pmax, p.window, p.sinks);
        const int rows = (int)min((long long)M, (long long)pc.n * p.ge.g - (long long)pc.rt * M);
        const int lo_key = p.window > 0 ? max(0, pc.pmin - p.window + 1) : 0;
        // four threads bring one key's row in; `row` is where the tile whose K was asked for last lies
        key.ask(p, pc, span, lo_key, pc.i0, kl);
        long long row_k = -1;
        auto load_k = [&](int i) {
            row_k = key.row(p, pc);
            if (row_k >= 0) pgs_row_in(Ks + kl * LD, (const T*)p.k + (size_t)row_k * D, D, tid & 3, 4);
            pgs_commit();
            key.ask(p, pc, span, lo_key, i + 1, kl);
        };
        auto load_v = [&]() {
            if (row_k >= 0) pgs_row_in(Vs + kl * LD, (const T*)p.v + (size_t)row_k * D, D, tid & 3, 4);
            pgs_commit();
        };
        load_k(pc.i0);
        load_v();
        for (int i = tid; i < M * DP; i += PGS_THREADS) {
            const int r = i / DP, e = i % DP;
            float x = 0.f;
            if (r < rows && e < D) {
                const long long pk = (long long)pc.rt * M + r;
                x = pg_to_f(((const T*)p.q)[(size_t)(pc.a + pk / p.ge.g) * p.ldq + (size_t)(pc.head * p.ge.g + pk % p.ge.g) * D + e]) * p.scale_log2;
            }
            Qs[r * QLD + e] = x;
        }
        int pos[RW];
        float m[RW], l[RW], o[RW][E];
#pragma unroll
        for (int r = 0; r < RW; r++) {
            pos[r] = pgs_row_position(p, pc, M, r_w + r, limit);
            m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
            for (int e = 0; e < E; e++) o[r][e] = 0.f;
        }
        const bool work = r_w < rows;                              // warps whose rows are all padding only help loading
        for (int i = pc.i0; i < pc.i1; i++) {
            const int key0 = pg_tile_key(span, i, PGS_KT);
            pgs_wait<1>();
            __syncthreads();                                       // K(i) and Q are there
            float s[RW][2];
            if (work) {
#pragma unroll
                for (int r = 0; r < RW; r++) s[r][0] = s[r][1] = 0.f;
#pragma unroll 4
                for (int c = 0; c < DP / 4; c++) {
                    float k0[4], k1[4];
                    pgs_f4(Ks + lane * LD + c * 4, k0);
                    pgs_f4(Ks + (lane + 32) * LD + c * 4, k1);
#pragma unroll
                    for (int r = 0; r < RW; r++) {
                        const float4 q = *reinterpret_cast<const float4*>(Qs + (r_w + r) * QLD + c * 4);
                        s[r][0] = fmaf(q.x, k0[0], s[r][0]); s[r][0] = fmaf(q.y, k0[1], s[r][0]);
                        s[r][0] = fmaf(q.z, k0[2], s[r][0]); s[r][0] = fmaf(q.w, k0[3], s[r][0]);
                        s[r][1] = fmaf(q.x, k1[0], s[r][1]); s[r][1] = fmaf(q.y, k1[1], s[r][1]);
                        s[r][1] = fmaf(q.z, k1[2], s[r][1]); s[r][1] = fmaf(q.w, k1[3], s[r][1]);
                    }
                }
            }
            __syncthreads();                                       // K(i) has been read
            load_k(i + 1);
            if (work) {
#pragma unroll
                for (int r = 0; r < RW; r++) {
                    const bool v0 = pos[r] >= 0 && pg_sees(pos[r], key0 + lane, p.window, p.sinks);
                    const bool v1 = pos[r] >= 0 && pg_sees(pos[r], key0 + lane + 32, p.window, p.sinks);
                    float mx = fmaxf(v0 ? s[r][0] : -INFINITY, v1 ? s[r][1] : -INFINITY);
#pragma unroll
                    for (int w = 1; w < 32; w *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                    if (mx > m[r]) {
                        const float f = exp2f(m[r] - mx);
                        l[r] *= f;
#pragma unroll
                        for (int e = 0; e < E; e++) o[r][e] *= f;
                        m[r] = mx;
                    }
                    const float p0 = v0 ? exp2f(s[r][0] - m[r]) : 0.f, p1 = v1 ? exp2f(s[r][1] - m[r]) : 0.f;
                    l[r] += p0 + p1;
                    Ps[(r_w + r) * PLD + lane] = p0;
                    Ps[(r_w + r) * PLD + lane + 32] = p1;
                }
            }
            pgs_wait<1>();
            __syncthreads();                                       // V(i) is there (and the warp's own P)
            if (work) {
                // four keys at a time; a tile with a key that some row does not see goes key by key when V is not finite all
                // over it (0 times an infinity would be a NaN)
                bool fast = true;
                if (pg_partial<PGS_KT>(key0, pc.pmin, pc.pmax, p.window, p.sinks)) {
                    float probe = 0.f;
#pragma unroll 4
                    for (int j = 0; j < PGS_KT; j++)
#pragma unroll
                        for (int e = 0; e < E; e++) probe = fmaf(pg_to_f(Vs[j * LD + lane + 32 * e]), 0.f, probe);
                    fast = __all_sync(0xffffffffu, probe == 0.f);
                }
                if (fast) {
#pragma unroll 2
                    for (int j = 0; j < PGS_KT; j += 4) {
                        float v[4][E];
#pragma unroll
                        for (int t = 0; t < 4; t++)
#pragma unroll
                            for (int e = 0; e < E; e++) v[t][e] = pg_to_f(Vs[(j + t) * LD + lane + 32 * e]);
#pragma unroll
                        for (int r = 0; r < RW; r++) {
                            const float4 w = *reinterpret_cast<const float4*>(Ps + (r_w + r) * PLD + j);
#pragma unroll
                            for (int e = 0; e < E; e++) {
                                o[r][e] = fmaf(w.x, v[0][e], o[r][e]); o[r][e] = fmaf(w.y, v[1][e], o[r][e]);
                                o[r][e] = fmaf(w.z, v[2][e], o[r][e]); o[r][e] = fmaf(w.w, v[3][e], o[r][e]);
                            }
                        }
                    }
                } else {
                    for (int j = 0; j < PGS_KT; j++) {
                        const int key = key0 + j;
#pragma unroll
                        for (int r = 0; r < RW; r++) {
                            if (pos[r] < 0 || !pg_sees(pos[r], key, p.window, p.sinks)) continue;
                            const float w = Ps[(r_w + r) * PLD + j];
#pragma unroll
                            for (int e = 0; e < E; e++) o[r][e] = fmaf(w, pg_to_f(Vs[j * LD + lane + 32 * e]), o[r][e]);
                        }
                    }
                }
            }
            __syncthreads();                                       // V(i) has been read
            load_v();
        }
        pgs_wait<0>();
        const bool whole = pc.c_first == pc.c_last;
        float* slot = whole ? nullptr : pg_slot(p.w, blockIdx.x, pc.c_first, M, D);
#pragma unroll
        for (int r = 0; r < RW; r++) {
            float ls = l[r];
#pragma unroll
            for (int w = 1; w < 32; w *= 2) ls += __shfl_xor_sync(0xffffffffu, ls, w);
            const int rr = r_w + r;
            if (rr >= rows) continue;
            const long long pk = (long long)pc.rt * M + rr;
            const int row = pc.a + (int)(pk / p.ge.g), hd = pc.head * p.ge.g + (int)(pk % p.ge.g);
            if (whole) {
                if (pos[r] < 0) continue;
#pragma unroll
                for (int e = 0; e < E; e++)
                    if (lane + 32 * e < D) ((T*)p.out)[(size_t)row * p.ldo + (size_t)hd * D + lane + 32 * e] = pg_from_f<T>(o[r][e] / ls);
                if (p.lse && lane == 0) p.lse[(size_t)row * p.ge.n_heads + hd] = (m[r] + log2f(ls)) * 0.6931471805599453f;
            } else {
#pragma unroll
                for (int e = 0; e < E; e++)
                    if (lane + 32 * e < D) slot[(size_t)rr * D + lane + 32 * e] = o[r][e];
                if (lane == 0) { slot[(size_t)M * D + 2 * rr] = m[r]; slot[(size_t)M * D + 2 * rr + 1] = ls; }
            }
        }
        if (!whole && pg_arrive_last(p.w, pc, tid == 0, &flag, sync)) pg_join_any<T>(p, pc, M, D, tid, PGS_THREADS);
        __syncthreads();
    }
    if (key.bad) atomicOr(p.w.status, PG_ST_BAD_PAGE);
}

}  // namespace rd
