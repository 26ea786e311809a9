// Attention over a paged cache for few rows per sequence (decode tokens, wavefronts, short slices), bf16.
//
// Up to 64 packed rows share a key tile, so the K/V stream is the bound: 4 FLOP per byte and row, far below
// the tensor cores.  One block per SM lives for the whole call:
//   warp 8      walks the block's share (rd_paged.cuh), looks the pages up and keeps a ring of 32-key tiles (K and V,
//               16 KB at head_dim 128, 128 KB of ring) filled by TMA: one box per page piece, written with the
//               128-byte (64 columns) and 64-byte (32 columns) swizzle.  It runs ahead across items, so the
//               stream does not stop while an item is finished.
//   warps 0-7   WQ blocks of 16 packed rows x WK = 8 / WQ key groups; the block's tile number c belongs to key group
//               c % WK, whose warps do S = Q K^T, the online softmax (float32) and O += P V on mma.sync m16n8k16
//               with P rounded to bf16 (the operand type; its rounding averages out over the keys).  A key group
//               keeps its own (m, l, O) and has stages of its own (the number of stages is a multiple of WK), so no
//               warp waits for another inside a piece and nobody waits on a barrier two phases ahead.
// At the end of a piece the key groups meet in shared memory (in key-group order), and the piece either
// becomes rows of the output or a slot of the workspace.
// Measured (copy peak 6.57 TB/s): one token behind 131,071 positions, 32/8 heads of 128: 97 us = 5.56 TB/s; 64 tokens behind
// 16 to 16,384, pages of 16: 120 us = 5.2 TB/s; 4 x 32 rows behind 8,200, 55 heads of 96: 152 us = 4.6 TB/s, where the softmax
// and products of 32 rows take as long as the stream; one token behind 543, 55 heads: 13 us, latency.  Two producers
// instead of one: 98 against 106 us; tiles of 32 keys with a stage per key group instead of 64 with half as many: no warp idles.
// mma.sync, not tcgen05: at M <= 64 rows the tensor pipe is far from the bound, and S and O stay in registers.
//
// Keys that some row of the tile does not see get P = 0; so that an infinity or NaN in V there does not
// become a NaN in that row, tiles with such keys are multiplied with the non-finite elements of V as zeros, and
// the rows that do see them get them at the end (pg_add_nonfinite).
#pragma once
#include "rd_paged.cuh"
#include "rd_attn.cuh"
#include "rd_gemm_tc.cuh"

namespace rd {

constexpr int PGM_KT = 32;
constexpr int PGM_THREADS = 384;           // two warpgroups of consumers, one for the producer (register split)
constexpr int PGM_QUEUE = 8;               // pieces known in advance

struct PgMaps { CUtensorMap k64, k32, v64, v32; };   // boxes of min(page_size, KT) positions x 64 / 32 columns

// One K or V tile: D / 64 sub-tiles of 64 columns, then one of 32 when D is no multiple of 64.
template <int D> struct PgmTile {
    static constexpr int NA = D / 64, NB = (D % 64) / 32;
    static constexpr int A_BYTES = PGM_KT * 128, B_BYTES = PGM_KT * 64;
    static constexpr int BYTES = NA * A_BYTES + NB * B_BYTES;
    // byte offset of the 16-byte chunk holding (row, col), col a multiple of 8, as the swizzles place it
    __device__ static __forceinline__ uint32_t off(int row, int col) {
        if (col < 64 * NA) {
            const uint32_t o = (uint32_t)(row * 128 + (col & 63) * 2);
            return (uint32_t)(col >> 6) * A_BYTES + (o ^ (((o >> 7) & 7u) << 4));
        }
        const uint32_t o = (uint32_t)(row * 64 + (col - 64 * NA) * 2);
        return (uint32_t)NA * A_BYTES + (o ^ (((o >> 7) & 3u) << 4));
    }
};
template <int D, int WQ> struct PgmCfg {
    using T = PgmTile<D>;
    static constexpr int M = 16 * WQ, WK = 8 / WQ;
    static constexpr int STAGES = D == 64 ? 16 : 8;
    static_assert(STAGES % WK == 0, "a stage belongs to one key group");
    static constexpr int STAGE_BYTES = 2 * T::BYTES;
    static constexpr int RING = STAGES * STAGE_BYTES;
    static constexpr int OLD = D + 4;
    static constexpr int O_BYTES = 128 * OLD * 4, ML_BYTES = 128 * 8;
    static constexpr int SMEM = 1024 + RING + O_BYTES + ML_BYTES;
};

// bf16 pairs with infinities and NaNs as zeros; *found is raised when there was one.
__device__ __forceinline__ uint32_t pgm_finite(uint32_t x, bool* found) {
    const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
    if (lo) x &= 0xffff0000u;
    if (hi) x &= 0x0000ffffu;
    *found |= lo || hi;
    return x;
}
// mbar_wait in few instructions: these kernels wait in many places, and their code competes for the instruction caches.
__device__ __forceinline__ bool pg_wait(uint64_t* bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t i = 0; i < TC_SPIN_LIMIT; i++) {
        if (mbar_test(bar, parity)) return true;
        if (i > 64) __nanosleep(64);
    }
    return false;
}
// One lane of a converged warp, the same every time.
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}

// A producer warp's view of a share: it walks the pieces into a queue in shared memory, one ahead of the piece it
// loads, and turns key tiles into pool rows.  The table is read 32 boxes at a time, one per lane, a chunk ahead of its use
// (the first chunk of a piece while the piece before it is being loaded), and a table entry is not looked at before it
// is needed, so that no copy waits for one.
template <int KT, int DEPTH> struct PgProducer {
    PgPiece* queue;                    // [DEPTH]; i1 < 0: no more pieces
    uint64_t *full, *empty;            // [DEPTH], or null: a queue nobody else reads
    int* found;                        // [DEPTH], cleared with every piece, or null
    int box_shift, lg_box;             // log2 of a box's positions, of a tile's boxes
    int cur;                           // pool row of this lane's box of the current chunk
    int ahead, first;                  // table entries: next chunk, first chunk of the next piece
    int at;                            // lane of the next tile's first box
    int qn;                            // pieces pushed
    bool bad;
    PgWalk walk;
    __device__ __forceinline__ int key_of(const PgAttend& p, const PgPiece& q, int i) const {      // of this lane's box, -1: none
        const int lane = threadIdx.x & 31;
        i += lane >> lg_box;
        if (i >= q.i1) return -1;
        const int key = pg_tile_key(pg_span<KT>(q.pmin, q.pmax, p.window, p.sinks), i, KT) + ((lane & ((1 << lg_box) - 1)) << box_shift);
        return key <= q.pmax ? key : -1;
    }
    __device__ __forceinline__ int entry(const PgAttend& p, const PgPiece& q, int i) const {
        const int key = key_of(p, q, i), pi = key >> p.ge.page_shift;
        return key >= 0 && pi < p.b.table_stride ? p.b.table[(size_t)q.grp * p.b.table_stride + pi] : -1;
    }
    __device__ __forceinline__ int resolve(const PgAttend& p, const PgPiece& q, int i, int pg) {
        const int key = key_of(p, q, i);
        if (key < 0) return 0x7fffff00;            // beyond the pages: the box reads as zeros
        if (pg < 0 || pg >= p.ge.n_pages) {
            if (p.window <= 0 || key < p.sinks || key + (1 << box_shift) > q.pmin - p.window + 1) bad = true;      // a page some row needs
            return 0x7fffff00;
        }
        return ((((p.ge.layer * p.ge.n_pages + pg) * p.ge.n_kv) + q.head) << p.ge.page_shift) + (key & ((1 << p.ge.page_shift) - 1));
    }
    // the next piece (or the end) into the queue, the table entries of its first boxes on their way; false: a wait ran out
    __device__ __forceinline__ bool push(const PgAttend& p) {
        PgPiece pc;
        const bool more = walk.next(p.ge.n_kv, &pc);
        const int s = qn % DEPTH;
        if (empty && qn >= DEPTH && !pg_wait(&empty[s], ((qn / DEPTH) - 1) & 1)) return false;
        if ((threadIdx.x & 31) == 0) {
            if (!more) pc.i1 = -1;
            queue[s] = pc;
            if (found) found[s] = 0;
            if (full) mbar_arrive(&full[s]);
        }
        __syncwarp();
        qn++;
        if (more) first = entry(p, queue[s], queue[s].i0);
        return true;
    }
    template <typename Plan> __device__ __forceinline__ bool start(const PgAttend& p, const Plan& plan) {
        box_shift = min(p.ge.page_shift, KT == 32 ? 5 : 7);
        static_assert(KT == 32 || KT == 128, "tile heights of the two kernels");
        lg_box = (KT == 32 ? 5 : 7) - box_shift;
        bad = false;
        qn = 0;
        walk.start(p, plan);
        return push(p);
    }
    // begins the piece pushed last (null: the end); push() the next one once the first tile has been asked for
    __device__ __forceinline__ const PgPiece* begin(const PgAttend& p) {
        const PgPiece* q = &queue[(qn - 1) % DEPTH];
        if (q->i1 < 0) return nullptr;
        cur = resolve(p, *q, q->i0, first);
        ahead = entry(p, *q, q->i0 + (32 >> lg_box));
        at = 0;
        return q;
    }
    // lane that holds the row of tile i's first box; tiles are asked for in order, from the piece's first
    __device__ __forceinline__ int tile_lane(const PgAttend& p, const PgPiece* q, int i) {
        if (at == 32) { cur = resolve(p, *q, i, ahead); ahead = entry(p, *q, i + (32 >> lg_box)); at = 0; }
        const int l = at;
        at += 1 << lg_box;
        return l;
    }
    __device__ __forceinline__ int row(int lane) const { return __shfl_sync(0xffffffffu, cur, lane); }
};

template <int D, int WQ>
__global__ void __launch_bounds__(PGM_THREADS, 1)
pg_attend_mma_kernel(const __grid_constant__ PgAttend p, const __grid_constant__ PgMaps maps) {
    using C = PgmCfg<D, WQ>;
    using T = PgmTile<D>;
    constexpr int M = C::M, WK = C::WK, S = C::STAGES, OLD = C::OLD;
    extern __shared__ uint8_t pgm_raw[];
    uint8_t* ring = (uint8_t*)(((uintptr_t)pgm_raw + 1023) & ~(uintptr_t)1023);
    float* Os = reinterpret_cast<float*>(ring + C::RING);
    float* MLs = reinterpret_cast<float*>(ring + C::RING + C::O_BYTES);
    __shared__ PgPlanSmem<PG_INLINE_REC> plan;
    __shared__ uint64_t full[S], empty[S], q_full[PGM_QUEUE], q_empty[PGM_QUEUE];
    __shared__ PgPiece queue[PGM_QUEUE], queue_v[PGM_QUEUE];          // i1 < 0: no more pieces
    __shared__ int abort_s, stop_s, flag_s, found_s;
    volatile int* abort_flag = &abort_s;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k64) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v64) : "memory");
        for (int s = 0; s < S; s++) { mbar_init(&full[s], 2); mbar_init(&empty[s], WQ); }
        for (int s = 0; s < PGM_QUEUE; s++) { mbar_init(&q_full[s], 1); mbar_init(&q_empty[s], 1); }
        abort_s = 0; stop_s = 0; found_s = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    pdl_enter();
    pg_plan_share<PGM_THREADS, PGM_KT>(p, M, plan);        // (starts and ends with a block barrier)

    if (warp >= 8) {
        pg_regs_less<PG_REGS_LESS>();
        if (warp <= 9) {
        // ---- producers: warp 8 the K tiles (and the queue of pieces), warp 9 the V tiles ----
        const bool is_v = warp == 9;
        PgProducer<PGM_KT, PGM_QUEUE> bx;
        bx.queue = is_v ? queue_v : queue; bx.full = is_v ? nullptr : q_full; bx.empty = is_v ? nullptr : q_empty; bx.found = nullptr;
        bool ok = bx.start(p, plan);
        const bool issuer = elect_one();
        const CUtensorMap *m64 = is_v ? &maps.v64 : &maps.k64, *m32 = is_v ? &maps.v32 : &maps.k32;
        uint8_t* const base = ring + (is_v ? T::BYTES : 0);
        const int nbox = 1 << bx.lg_box;
        int cnt = 0;
        while (ok) {
            const PgPiece* q = bx.begin(p);
            if (!q) break;
            const int i0 = q->i0, i1 = q->i1;
            for (int i = i0; i < i1; i++, cnt++) {
                const int s = cnt % S, l0 = bx.tile_lane(p, q, i);
                if (cnt >= S && !pg_wait(&empty[s], ((cnt / S) - 1) & 1)) { ok = false; break; }
                uint8_t* dst = base + s * C::STAGE_BYTES;
                if (issuer) mbar_expect_tx(&full[s], T::BYTES);
#pragma unroll 1
                for (int b = 0; b < nbox; b++) {
                    const int y = bx.row(l0 + b), at = b << bx.box_shift;
                    if (issuer) {
#pragma unroll
                        for (int a = 0; a < T::NA; a++) tma_load_2d(dst + a * T::A_BYTES + at * 128, m64, a * 64, y, &full[s]);
                        if (T::NB) tma_load_2d(dst + T::NA * T::A_BYTES + at * 64, m32, T::NA * 64, y, &full[s]);
                    }
                }
                if (i == i0 && !bx.push(p)) { cnt++; ok = false; break; }
            }
        }
        if (!ok) *abort_flag = 1;
        if (__any_sync(0xffffffffu, bx.bad) && lane == 0) atomicOr(p.w.status, PG_ST_BAD_PAGE);
        if (*abort_flag)                                   // every copy lands before the block's memory is released
            for (int c = max(0, cnt - S); c < cnt; c++) pg_wait(&full[c % S], (c / S) & 1);
        }
    } else {
        // ---- consumers ----
        pg_regs_more<PG_REGS_MORE>();
        const int qb = warp % WQ, kg = warp / WQ, g = lane >> 2, tq = lane & 3;
        const int limit = pg_pos_limit(p.b, p.ge);
        auto sync = [] { named_bar_sync(1, 256); };
        const float c2 = p.scale_log2;
        int cnt = 0;
        for (int qn = 0; ; qn++) {
            const int qs = qn % PGM_QUEUE;
            if (tid == 0) {
                const bool got = !*abort_flag && pg_wait(&q_full[qs], (qn / PGM_QUEUE) & 1);
                if (!got) *abort_flag = 1;
                stop_s = !got;
            }
            sync();
            if (stop_s) break;
            const PgPiece pc = queue[qs];
            if (pc.i1 < 0) break;
            const PgSpan span = pg_span<PGM_KT>(pc.pmin, pc.pmax, p.window, p.sinks);
            const int rows = (int)min((long long)M, (long long)pc.n * p.ge.g - (long long)pc.rt * M);
            // this thread's two packed rows: their positions and (as MMA fragments) their queries
            int pos[2];
            uint32_t qf[D / 16][4];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int r = qb * 16 + g + 8 * h;
                const long long pk = (long long)pc.rt * M + r;
                const int row = pc.a + (int)(pk / p.ge.g), hd = pc.head * p.ge.g + (int)(pk % p.ge.g);
                pos[h] = r < rows ? p.b.row_pos[row] : -1;
                if (pos[h] >= limit) pos[h] = -1;
                const __nv_bfloat16* qr = (const __nv_bfloat16*)p.q + (r < rows ? (size_t)row * p.ldq + (size_t)hd * D : 0);
#pragma unroll
                for (int kk = 0; kk < D / 16; kk++) {
                    qf[kk][h] = r < rows ? *reinterpret_cast<const uint32_t*>(qr + kk * 16 + 2 * tq) : 0u;
                    qf[kk][2 + h] = r < rows ? *reinterpret_cast<const uint32_t*>(qr + kk * 16 + 8 + 2 * tq) : 0u;
                }
            }
            float m_a = -INFINITY, m_b = -INFINITY, l_a = 0.f, l_b = 0.f;
            float o[D / 8][4];
#pragma unroll
            for (int j = 0; j < D / 8; j++) { o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f; }
            bool found = false, ok = true;
            const int len = pc.i1 - pc.i0;
            for (int t = (kg - cnt % WK + WK) % WK; t < len && ok; t += WK) {
                const int c = cnt + t, s = c % S;
                ok = pg_wait(&full[s], (c / S) & 1) && !*abort_flag;
                if (!ok) break;
                const uint8_t* Kt = ring + s * C::STAGE_BYTES;
                const uint8_t* Vt = Kt + T::BYTES;
                float sc[PGM_KT / 8][4];
#pragma unroll
                for (int j = 0; j < PGM_KT / 8; j++) { sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f; }
#pragma unroll
                for (int kk = 0; kk < D / 16; kk++) {
#pragma unroll
                    for (int jn = 0; jn < PGM_KT / 16; jn++) {
                        uint32_t kb[4];
                        ldsm_x4(kb, Kt + T::off(jn * 16 + (lane & 7) + (lane >> 4) * 8, kk * 16 + ((lane >> 3) & 1) * 8));
                        mma_bf16_16816(sc[2 * jn], qf[kk], kb[0], kb[1]);
                        mma_bf16_16816(sc[2 * jn + 1], qf[kk], kb[2], kb[3]);
                    }
                }
                const int key0 = pg_tile_key(span, pc.i0 + t, PGM_KT);
                const bool partial = pg_partial<PGM_KT>(key0, pc.pmin, pc.pmax, p.window, p.sinks);
                if (partial) {
                    const uint32_t see_a = pg_see_bits(key0, pos[0], pg_window_lo(pos[0], p.window), p.sinks);
                    const uint32_t see_b = pg_see_bits(key0, pos[1], pg_window_lo(pos[1], p.window), p.sinks);
#pragma unroll
                    for (int j = 0; j < PGM_KT / 8; j++) {
                        const int k0 = j * 8 + 2 * tq;
                        sc[j][0] = (see_a >> k0 & 1) ? sc[j][0] : -INFINITY;
                        sc[j][1] = (see_a >> k0 & 2) ? sc[j][1] : -INFINITY;
                        sc[j][2] = (see_b >> k0 & 1) ? sc[j][2] : -INFINITY;
                        sc[j][3] = (see_b >> k0 & 2) ? sc[j][3] : -INFINITY;
                    }
                }
                float mx_a = -INFINITY, mx_b = -INFINITY;
#pragma unroll
                for (int j = 0; j < PGM_KT / 8; j++) {
                    mx_a = fmaxf(mx_a, fmaxf(sc[j][0], sc[j][1]));
                    mx_b = fmaxf(mx_b, fmaxf(sc[j][2], sc[j][3]));
                }
                mx_a = fmaxf(mx_a, __shfl_xor_sync(0xffffffffu, mx_a, 1));
                mx_a = fmaxf(mx_a, __shfl_xor_sync(0xffffffffu, mx_a, 2));
                mx_b = fmaxf(mx_b, __shfl_xor_sync(0xffffffffu, mx_b, 1));
                mx_b = fmaxf(mx_b, __shfl_xor_sync(0xffffffffu, mx_b, 2));
                const float mn_a = fmaxf(m_a, mx_a * c2), mn_b = fmaxf(m_b, mx_b * c2);      // c2 > 0
                const float ua = mn_a == -INFINITY ? 0.f : mn_a, ub = mn_b == -INFINITY ? 0.f : mn_b;
                const float ca = exp2f(m_a - ua), cb = exp2f(m_b - ub);
                m_a = mn_a; m_b = mn_b;
                float sa = 0.f, sb = 0.f;
                uint32_t pf[PGM_KT / 16][4];
#pragma unroll
                for (int j = 0; j < PGM_KT / 8; j++) {
                    const float p0 = exp2f(fmaf(sc[j][0], c2, -ua)), p1 = exp2f(fmaf(sc[j][1], c2, -ua));
                    const float p2 = exp2f(fmaf(sc[j][2], c2, -ub)), p3 = exp2f(fmaf(sc[j][3], c2, -ub));
                    sa += p0 + p1;
                    sb += p2 + p3;
                    pf[j >> 1][(j & 1) * 2] = pack_bf16(p0, p1);
                    pf[j >> 1][(j & 1) * 2 + 1] = pack_bf16(p2, p3);
                }
                l_a = l_a * ca + sa;
                l_b = l_b * cb + sb;
#pragma unroll
                for (int j = 0; j < D / 8; j++) { o[j][0] *= ca; o[j][1] *= ca; o[j][2] *= cb; o[j][3] *= cb; }
#pragma unroll
                for (int kk = 0; kk < PGM_KT / 16; kk++) {
#pragma unroll
                    for (int jn = 0; jn < D / 16; jn++) {
                        uint32_t vb[4];
                        ldsm_x4_t(vb, Vt + T::off(kk * 16 + (lane & 7) + ((lane >> 3) & 1) * 8, jn * 16 + (lane >> 4) * 8));
                        if (partial) {
#pragma unroll
                            for (int x = 0; x < 4; x++) vb[x] = pgm_finite(vb[x], &found);
                        }
                        mma_bf16_16816(o[2 * jn], pf[kk], vb[0], vb[1]);
                        mma_bf16_16816(o[2 * jn + 1], pf[kk], vb[2], vb[3]);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty[s]);
            }
            cnt += len;
            if (!ok) *abort_flag = 1;
            if (found) found_s = 1;
            // ---- the key groups meet ----
            l_a += __shfl_xor_sync(0xffffffffu, l_a, 1);
            l_a += __shfl_xor_sync(0xffffffffu, l_a, 2);
            l_b += __shfl_xor_sync(0xffffffffu, l_b, 1);
            l_b += __shfl_xor_sync(0xffffffffu, l_b, 2);
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int r = kg * M + qb * 16 + g + 8 * h;
                const float m = h ? m_b : m_a;
                if (qb * 16 + g + 8 * h >= rows) continue;
                if (tq == 0) *reinterpret_cast<float2*>(MLs + 2 * r) = make_float2(m, h ? l_b : l_a);
                if (m == -INFINITY) continue;              // nothing seen: its O is not looked at
#pragma unroll
                for (int j = 0; j < D / 8; j++)
                    *reinterpret_cast<float2*>(Os + (size_t)r * OLD + j * 8 + 2 * tq) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
            }
            sync();
            if (tid == 0) mbar_arrive(&q_empty[qs]);       // everyone has copied the piece
            const bool whole = pc.c_first == pc.c_last, fix = found_s != 0;
            float* slot = whole ? nullptr : pg_slot(p.w, blockIdx.x, pc.c_first, M, D);
            for (int it = tid; it < rows * (D / 4); it += 256) {
                const int r = it / (D / 4), e = (it % (D / 4)) * 4;
                float mx = -INFINITY;
#pragma unroll
                for (int w = 0; w < WK; w++) mx = fmaxf(mx, MLs[2 * (w * M + r)]);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                float den = 0.f;
#pragma unroll
                for (int w = 0; w < WK; w++) {
                    const float2 ml = *reinterpret_cast<const float2*>(MLs + 2 * (w * M + r));
                    if (ml.x == -INFINITY) continue;
                    const float f = exp2f(ml.x - mx);
                    const float4 v = *reinterpret_cast<const float4*>(Os + (size_t)(w * M + r) * OLD + e);
                    acc.x = fmaf(v.x, f, acc.x); acc.y = fmaf(v.y, f, acc.y); acc.z = fmaf(v.z, f, acc.z); acc.w = fmaf(v.w, f, acc.w);
                    den = fmaf(ml.y, f, den);
                }
                const long long pk = (long long)pc.rt * M + r;
                const int row = pc.a + (int)(pk / p.ge.g), hd = pc.head * p.ge.g + (int)(pk % p.ge.g);
                const int rp = p.b.row_pos[row];
                if (rp < 0 || rp >= limit) continue;
                if (fix) {
                    acc.x += pg_nonfinite<__nv_bfloat16, PGM_KT>(p, pc, rp, e); acc.y += pg_nonfinite<__nv_bfloat16, PGM_KT>(p, pc, rp, e + 1);
                    acc.z += pg_nonfinite<__nv_bfloat16, PGM_KT>(p, pc, rp, e + 2); acc.w += pg_nonfinite<__nv_bfloat16, PGM_KT>(p, pc, rp, e + 3);
                }
                if (whole) {
                    const float inv = 1.0f / den;
                    pg_store4((__nv_bfloat16*)p.out + (size_t)row * p.ldo + (size_t)hd * D + e, acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
                    if (p.lse && e == 0) p.lse[(size_t)row * p.ge.n_heads + hd] = (mx + log2f(den)) * 0.6931471805599453f;
                } else {
                    *reinterpret_cast<float4*>(slot + (size_t)r * D + e) = acc;
                    if (e == 0) *reinterpret_cast<float2*>(slot + (size_t)M * D + 2 * r) = make_float2(mx, den);
                }
            }
            if (!whole && pg_arrive_last(p.w, pc, tid == 0, &flag_s, sync)) pg_join<__nv_bfloat16, 4>(p, pc, M, D, tid, 256);
            sync();                                        // Os, MLs, found_s and the flags may be written again
            if (tid == 0) found_s = 0;
        }
    }
    __syncthreads();
    if (tid == 0 && abort_s) atomicOr(p.w.status, PG_ST_TIMEOUT);
}

}  // namespace rd
