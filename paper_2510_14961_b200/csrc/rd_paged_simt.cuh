// Attention over a paged cache in float32, and in bf16 with head sizes the kernels on tcgen05 and bf16 mma.sync do not
// take.  Any even head_dim up to DP = 32, 64, 96 or 128 (shared-memory rows are padded with zeros).  Arguments, row tiles
// and the division of the work: rd_paged.cuh.
//
// pg_attend_few_kernel (row tiles of 16): CUDA cores, bound by the K/V stream.  A 64-key tile is eight runs of 8 keys, one
//   per warp; a warp brings its run in by itself (16-byte cp.async, three stages of its own) and keeps its own
//   maximum, sum and output, so no warp waits for another before the end of an item.  Four lanes share a key's
//   dot product, a lane owns DP / 32 output features.
// pg_attend_many_kernel (row tiles of 64): mma.sync m16n8k8 in tf32 with every float32 operand as a sum of two tf32
//   numbers (x = hi + lo up to 2^-22 |x|): hi hi + hi lo + lo hi, accumulated in float32, errs by about 2^-21 of a
//   product, next to the 2^-24 of an FMA chain's every step; bf16 operands are tf32 numbers already.  (The same tile on FMAs
//   took 7 us: 1,024 FMAs and 160 shared-memory reads per warp for the scores alone.)  Four blocks of 16 rows x two halves of
//   a 64-key tile; the halves keep (m, l, O) of their own and meet at the end of a piece.  P goes from the
//   accumulators of S into the A operand of P V as it lies: an 8-key step of that product takes the keys in the
//   order 0 2 4 6 1 3 5 7, for P and V alike.  K(t + 1) is requested behind Q K^T of tile t and V(t + 1) behind P V, so
//   one buffer each suffices.
//
// Keys that some row of a tile does not see: the first kernel never multiplies by them; the second takes non-finite
// elements of V out of such tiles and gives them to the rows that see them at the end (pg_nonfinite).
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
    static constexpr int STAGES = 3, KEYS = 8;
    static constexpr int RUN = KEYS * LD * (int)sizeof(T);       // 8 rows of K or V
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
#pragma unroll
            for (int r = 0; r < M; r++) {
                if (r >= rows) break;
                float s = 0.f;
#pragma unroll
                for (int c = 0; c < DP / 16; c++) {
                    const float4 q = *reinterpret_cast<const float4*>(Qs + r * QLD + c * 16 + quarter * 4);
                    s = fmaf(q.x, kk[c * 4], s); s = fmaf(q.y, kk[c * 4 + 1], s); s = fmaf(q.z, kk[c * 4 + 2], s); s = fmaf(q.w, kk[c * 4 + 3], s);
                }
                s += __shfl_xor_sync(0xffffffffu, s, 1);
                s += __shfl_xor_sync(0xffffffffu, s, 2);
                const bool see = pos[r] >= 0 && pg_sees(pos[r], key0 + key_l, p.window, p.sinks);
                float mx = see ? s : -INFINITY;
#pragma unroll
                for (int w = 4; w < 32; w *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                if (mx > m[r]) {
                    const float f = exp2f(m[r] - mx);              // m = -inf: 0, nothing accumulated yet
                    l[r] *= f;
#pragma unroll
                    for (int e = 0; e < E; e++) o[r][e] *= f;
                    m[r] = mx;
                }
                const float pj = see ? exp2f(s - m[r]) : 0.f;
                l[r] += quarter == 0 ? pj : 0.f;
                const unsigned any = __ballot_sync(0xffffffffu, see);
                for (int j = 0; j < C::KEYS; j++) {
                    const float w = __shfl_sync(0xffffffffu, pj, j * 4);
                    if (!(any >> (j * 4) & 1)) continue;           // V of an unseen key is not touched
#pragma unroll
                    for (int e = 0; e < E; e++) o[r][e] = fmaf(w, pg_to_f(Vt[j * LD + lane + 32 * e]), o[r][e]);
                }
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
    static constexpr int QLD = DP + 4;
    static constexpr int SMEM = 2 * TILE + 2 * PGS_MANY * QLD * 4 + PGS_MANY * 8;      // K, V, Q, the second halves' O and (m, l)
    static constexpr int PER_SM = DP <= 64 ? 2 : 1;
};

__device__ __forceinline__ uint32_t pgs_tf32(float x) { uint32_t r; asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x)); return r; }
__device__ __forceinline__ void pgs_split(float x, uint32_t* hi, uint32_t* lo) {
    *hi = pgs_tf32(x);
    *lo = pgs_tf32(x - __uint_as_float(*hi));
}
__device__ __forceinline__ void pgs_mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two blocks share an SM where their tiles fit (head_dim up to 64): one block's barriers hide behind the other's work.
template <typename T, int DP>
__global__ void __launch_bounds__(PGS_THREADS, PgsMany<T, DP>::PER_SM) pg_attend_many_kernel(const __grid_constant__ PgAttend p) {
    using C = PgsMany<T, DP>;
    constexpr int M = PGS_MANY, LD = C::LD, QLD = C::QLD, NO = DP / 8, KH = PGS_KT / 2, NS = KH / 8;
    constexpr bool EXACT = sizeof(T) == 2;                     // bf16 operands need no second part
    extern __shared__ __align__(16) uint8_t pgs_raw[];
    T* Ks = reinterpret_cast<T*>(pgs_raw);
    T* Vs = reinterpret_cast<T*>(pgs_raw + C::TILE);
    float* Qs = reinterpret_cast<float*>(pgs_raw + 2 * C::TILE);
    float* Os = Qs + M * QLD;
    float* MLs = Os + M * QLD;
    __shared__ PgPlanSmem<PG_INLINE_REC> plan;
    __shared__ int flag, found_s;
    pdl_enter();
    if (threadIdx.x == 0) found_s = 0;
    pg_plan_share<PGS_THREADS, PGS_KT>(p, M, plan);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, D = p.ge.D, g = lane >> 2, tq = lane & 3;
    const int limit = pg_pos_limit(p.b, p.ge), qb = warp & 3, kh = warp >> 2, kl = tid >> 2;
    const float c2 = p.scale_log2;
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
        // four threads bring one key's row in; `row_k` is where the tile whose K was asked for last lies
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
                const unsigned pk = (unsigned)pc.rt * M + r, of = pk / (unsigned)p.ge.g;
                x = pg_to_f(((const T*)p.q)[(size_t)(pc.a + (int)of) * p.ldq + (size_t)(pc.head * p.ge.g + (int)(pk - of * p.ge.g)) * D + e]);
            }
            Qs[r * QLD + e] = x;
        }
        // this thread's rows: qb * 16 + g and 8 further on
        const int pos_a = pgs_row_position(p, pc, M, qb * 16 + g, limit), pos_b = pgs_row_position(p, pc, M, qb * 16 + g + 8, limit);
        const int low_a = pg_window_lo(pos_a, p.window), low_b = pg_window_lo(pos_b, p.window);
        float m_a = -INFINITY, m_b = -INFINITY, l_a = 0.f, l_b = 0.f, o[NO][4];
#pragma unroll
        for (int j = 0; j < NO; j++) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
        bool found = false;
        const bool work = qb * 16 < rows;                      // warps whose rows are all padding only help loading
        for (int i = pc.i0; i < pc.i1; i++) {
            const int key0 = pg_tile_key(span, i, PGS_KT) + kh * KH;
            pgs_wait<1>();
            __syncthreads();                                   // K(i) and Q are there
            float s[NS][4];
            if (work) {
#pragma unroll
                for (int j = 0; j < NS; j++) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
                const float* qr = Qs + (qb * 16 + g) * QLD + tq;
                const T* kr = Ks + (kh * KH + g) * LD + tq;
#pragma unroll 4
                for (int k = 0; k < DP; k += 8) {
                    uint32_t ah[4], al[4];
                    const float x[4] = {qr[k], qr[8 * QLD + k], qr[k + 4], qr[8 * QLD + k + 4]};
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        if constexpr (EXACT) ah[q] = __float_as_uint(x[q]);
                        else pgs_split(x[q], &ah[q], &al[q]);
                    }
uint32_t h[NS][2], w[NS][2];                       // one product of every column block after the other: no MMA waits for the last
#pragma unroll
                    for (int j = 0; j < NS; j++) {
#pragma unroll
                        for (int q = 0; q < 2; q++) {
                            const float b = pg_to_f(kr[j * 8 * LD + k + 4 * q]);
                            if constexpr (EXACT) h[j][q] = __float_as_uint(b);
                            else pgs_split(b, &h[j][q], &w[j][q]);
                        }
                    }
                    if constexpr (!EXACT) {
#pragma unroll
                        for (int j = 0; j < NS; j++) pgs_mma(s[j], al, h[j][0], h[j][1]);
#pragma unroll
                        for (int j = 0; j < NS; j++) pgs_mma(s[j], ah, w[j][0], w[j][1]);
                    }
#pragma unroll
                    for (int j = 0; j < NS; j++) pgs_mma(s[j], ah, h[j][0], h[j][1]);
                }
            }
            __syncthreads();                                   // K(i) has been read
            load_k(i + 1);
            const bool partial = pg_partial<PGS_KT>(key0 - kh * KH, pc.pmin, pc.pmax, p.window, p.sinks);
            if (work) {
                if (partial) {
                    const uint32_t see_a = pg_see_bits(key0, pos_a, low_a, p.sinks), see_b = pg_see_bits(key0, pos_b, low_b, p.sinks);
#pragma unroll
                    for (int j = 0; j < NS; j++) {
                        const int k0 = j * 8 + 2 * tq;
                        s[j][0] = (see_a >> k0 & 1) ? s[j][0] : -INFINITY;
                        s[j][1] = (see_a >> k0 & 2) ? s[j][1] : -INFINITY;
                        s[j][2] = (see_b >> k0 & 1) ? s[j][2] : -INFINITY;
                        s[j][3] = (see_b >> k0 & 2) ? s[j][3] : -INFINITY;
                    }
                }
                float mx_a = -INFINITY, mx_b = -INFINITY;
#pragma unroll
                for (int j = 0; j < NS; j++) {
                    mx_a = fmaxf(mx_a, fmaxf(s[j][0], s[j][1]));
                    mx_b = fmaxf(mx_b, fmaxf(s[j][2], s[j][3]));
                }
#pragma unroll
                for (int w = 1; w < 4; w *= 2) {
                    mx_a = fmaxf(mx_a, __shfl_xor_sync(0xffffffffu, mx_a, w));
                    mx_b = fmaxf(mx_b, __shfl_xor_sync(0xffffffffu, mx_b, w));
                }
                const float mn_a = fmaxf(m_a, mx_a * c2), mn_b = fmaxf(m_b, mx_b * c2);
                const float ua = mn_a == -INFINITY ? 0.f : mn_a, ub = mn_b == -INFINITY ? 0.f : mn_b;
                const float ca = exp2f(m_a - ua), cb = exp2f(m_b - ub);
                m_a = mn_a; m_b = mn_b;
                float sa = 0.f, sb = 0.f;
#pragma unroll
                for (int j = 0; j < NS; j++) {
                    s[j][0] = exp2f(fmaf(s[j][0], c2, -ua)); s[j][1] = exp2f(fmaf(s[j][1], c2, -ua));
                    s[j][2] = exp2f(fmaf(s[j][2], c2, -ub)); s[j][3] = exp2f(fmaf(s[j][3], c2, -ub));
                    sa += s[j][0] + s[j][1];
                    sb += s[j][2] + s[j][3];
                }
                l_a = l_a * ca + sa;
                l_b = l_b * cb + sb;
#pragma unroll
                for (int j = 0; j < NO; j++) { o[j][0] *= ca; o[j][1] *= ca; o[j][2] *= cb; o[j][3] *= cb; }
            }
            pgs_wait<1>();
            __syncthreads();                                   // V(i) is there
            if (work) {
#pragma unroll
                for (int j = 0; j < NS; j++) {
                    uint32_t ah[4], al[4];
                    pgs_split(s[j][0], &ah[0], &al[0]); pgs_split(s[j][2], &ah[1], &al[1]);
                    pgs_split(s[j][1], &ah[2], &al[2]); pgs_split(s[j][3], &ah[3], &al[3]);
                    const T* vr = Vs + (kh * KH + j * 8 + 2 * tq) * LD + g;
#pragma unroll
                    for (int n0 = 0; n0 < NO; n0 += 4) {
                        uint32_t h[4][2], w[4][2];
#pragma unroll
                        for (int n = 0; n < 4; n++)
#pragma unroll
                            for (int q = 0; q < 2; q++) {
                                float b = pg_to_f(vr[q * LD + (n0 + n) * 8]);
                                if (partial && !isfinite(b)) { b = 0.f; found = true; }
                                if constexpr (EXACT) h[n][q] = __float_as_uint(b);
                                else pgs_split(b, &h[n][q], &w[n][q]);
                            }
#pragma unroll
                        for (int n = 0; n < 4; n++) pgs_mma(o[n0 + n], al, h[n][0], h[n][1]);
                        if constexpr (!EXACT) {
#pragma unroll
                            for (int n = 0; n < 4; n++) pgs_mma(o[n0 + n], ah, w[n][0], w[n][1]);
                        }
#pragma unroll
                        for (int n = 0; n < 4; n++) pgs_mma(o[n0 + n], ah, h[n][0], h[n][1]);
                    }
                }
            }
            __syncthreads();                                   // V(i) has been read
            load_v();
        }
        pgs_wait<0>();
        if (found) found_s = 1;
        // the two halves of the keys meet: the second's results through shared memory
#pragma unroll
        for (int w = 1; w < 4; w *= 2) {
            l_a += __shfl_xor_sync(0xffffffffu, l_a, w);
            l_b += __shfl_xor_sync(0xffffffffu, l_b, w);
        }
        const int ra = qb * 16 + g;
        if (kh == 1 && work) {
#pragma unroll
            for (int n = 0; n < NO; n++) {
                *reinterpret_cast<float2*>(Os + ra * QLD + n * 8 + 2 * tq) = make_float2(o[n][0], o[n][1]);
                *reinterpret_cast<float2*>(Os + (ra + 8) * QLD + n * 8 + 2 * tq) = make_float2(o[n][2], o[n][3]);
            }
            if (tq == 0) {
                *reinterpret_cast<float2*>(MLs + 2 * ra) = make_float2(m_a, l_a);
                *reinterpret_cast<float2*>(MLs + 2 * (ra + 8)) = make_float2(m_b, l_b);
            }
        }
        __syncthreads();
        const bool whole = pc.c_first == pc.c_last, fix = found_s != 0;
        float* slot = whole ? nullptr : pg_slot(p.w, blockIdx.x, pc.c_first, M, D);
        if (kh == 0 && work) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int r = ra + 8 * h, pos = h ? pos_b : pos_a;
                if (pos < 0) continue;
                const unsigned pk = (unsigned)pc.rt * M + r, of = pk / (unsigned)p.ge.g;
                const int row = pc.a + (int)of, hd = pc.head * p.ge.g + (int)(pk - of * p.ge.g);
                const float2 ml = *reinterpret_cast<const float2*>(MLs + 2 * r);
                const float m = h ? m_b : m_a, mx = fmaxf(m, ml.x), u = mx == -INFINITY ? 0.f : mx;
                const float f0 = exp2f(m - u), f1 = exp2f(ml.x - u), den = (h ? l_b : l_a) * f0 + ml.y * f1, inv = whole ? 1.0f / den : 1.0f;
#pragma unroll
                for (int n = 0; n < NO; n++) {
                    const int e = n * 8 + 2 * tq;
                    if (e >= D) continue;                       // (D is even)
                    const float2 x = *reinterpret_cast<const float2*>(Os + r * QLD + e);
                    float y0 = o[n][2 * h] * f0 + x.x * f1, y1 = o[n][2 * h + 1] * f0 + x.y * f1;
                    if (fix) { y0 += pg_nonfinite<T, PGS_KT>(p, pc, pos, e); y1 += pg_nonfinite<T, PGS_KT>(p, pc, pos, e + 1); }
                    if (whole) pg_set_pair((T*)p.out + (size_t)row * p.ldo + (size_t)hd * D + e, y0 * inv, y1 * inv);
                    else *reinterpret_cast<float2*>(slot + (size_t)r * D + e) = make_float2(y0, y1);
                }
                if (tq == 0) {
                    if (!whole) *reinterpret_cast<float2*>(slot + (size_t)M * D + 2 * r) = make_float2(mx, den);
                    else if (p.lse) p.lse[(size_t)row * p.ge.n_heads + hd] = (mx + log2f(den)) * 0.6931471805599453f;
                }
            }
        }
        if (!whole && pg_arrive_last(p.w, pc, tid == 0, &flag, sync)) pg_join_any<T>(p, pc, M, D, tid, PGS_THREADS);
        __syncthreads();
        if (tid == 0) found_s = 0;
    }
    if (key.bad) atomicOr(p.w.status, PG_ST_BAD_PAGE);
}

}  // namespace rd
