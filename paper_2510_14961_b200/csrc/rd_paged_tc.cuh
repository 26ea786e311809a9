// Attention over a paged cache for many rows per sequence (prompts, slices of prompts, wide wavefronts of
// grouped heads), bf16, on the 5th-generation tensor cores.
//
// A row tile is 256 packed rows (two blocks A and B of 128), a key tile 128 positions.  Per key tile and block of
// rows the tensor core does S = Q K^T and O += P V (2 x 128 x 128 x D MACs each, about 1,024 cycles at head_dim
// 128) and the softmax 16,384 exponentials (about 1,024 cycles of the SM's 16 per cycle): the two take turns,
// A's softmax under B's products and the other way round.
//   warps 0-3 / 4-7  softmax of A / B: one packed row per thread (TMEM lane = row); S from TMEM to registers, mask,
//                    online softmax in float32, P (bf16) back into the columns S came from
//   warps 8, 10      walk the block's share (rd_paged.cuh) and fill a ring of K and V tiles by TMA, one box per page
//                    piece; they run ahead across items
//   warp 11          looks through the V tiles of which some row does not see every key (see below)
//   warp 9           issues the MMAs: S_A(0) S_B(0), then PV_A(j) S_A(j+1) PV_B(j) S_B(j+1); P is the A operand
//                    from TMEM, V the MN-major B operand as it lies in its page
// TMEM: S/P of A and B (128 columns each), O of A and B (D columns each).  MMAs complete in the order they are
// issued, so the arrival of S(j+1) also says that P V(j) is done: a thread may then move its row's maximum and
// rescale O in place.  The maximum moves only when a tile exceeds it by more than 2^8 (P stays below 256; the
// result does not depend on which maximum was used).
// P is rounded to bf16 (the operand type); sums, maxima and O are float32.
// Measured: a prompt of 8,192 rows, 32/8 heads of 128: 464 to 500 us = 1.10 to 1.19 PFLOP/s (0.66 to 0.71 of the cuBLAS burst).
// A pair of tiles takes about 3,000 cycles, 2,048 of them on the tensor core: what is left is each block's chain softmax
// (1,850) -> P V -> Q K^T -> softmax.  Steps that counted: MMAs issued by an elected lane of a converged warp (8 MMAs 850 -> 250
// cycles), P handed over after 96 of 128 keys, masks in loops of their own, code small enough for the instruction caches.
// Keys some rows do not see: as in rd_paged_mma.cuh (P = 0, non-finite elements of V are taken out of the tile in
// shared memory and given to the rows that see them at the end).
// Every wait is bounded; on time-out the roles leave their loops, the copies in flight land, TMEM is freed and the
// status word raised.  No role ever waits at a block barrier between the first and the last.
#pragma once
#include "rd_attn_tc.cuh"
#include "rd_paged_mma.cuh"

namespace rd {

constexpr int PGT_KT = 128, PGT_M = 256;
constexpr int PGT_THREADS = 384;           // two warpgroups of softmax, one for the other roles (register split)
constexpr int PGT_QUEUE = 4;

template <int D> struct PgtCfg {
    static constexpr int NA = D / 64, NB = (D % 64) / 32;
    static constexpr int A_BYTES = 128 * 128, B_BYTES = 128 * 64;        // 128 rows of 64 / 32 columns
    static constexpr int TILE = NA * A_BYTES + NB * B_BYTES;
    // K and V have stages of their own: whoever waits for one kind only then never waits two phases ahead
    static constexpr int SK = D == 128 ? 2 : D == 96 ? 3 : 5, SV = D == 128 ? 3 : D == 96 ? 4 : 5;
    static constexpr int SMEM = 1024 + (2 + SK + SV) * TILE;
    static constexpr int S_COL = 0, O_COL = 256;                         // + 128 for block B
};

__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
          "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
          "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr) : "memory");
}
// Waits for the loads issued so far; the registers are operands so that no use of them moves in front of it.
__device__ __forceinline__ void tmem_ld32_wait(uint32_t* v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
          "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
          "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
          "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]) :: "memory");
}
__device__ __forceinline__ void tmem_st32_issue(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
          "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]),
          "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]),
          "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
__device__ __forceinline__ void tmem_st16_issue(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
          "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D += A B with A in TMEM (row = lane, two bf16 of k per column), B from shared memory
__device__ __forceinline__ void umma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// MN-major operand of several 64-column blocks, `apart` bytes from one to the next (128-byte swizzle)
__device__ __forceinline__ uint64_t umma_desc_mn128_blocks(uint32_t saddr, uint32_t apart) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(apart >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// Two floats at once (the FMA pipe's packed forms).
typedef unsigned long long pgt_f2;
__device__ __forceinline__ pgt_f2 pgt_pack(float a, float b) { pgt_f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void pgt_unpack(pgt_f2 v, float* a, float* b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(v)); }
__device__ __forceinline__ pgt_f2 pgt_fma(pgt_f2 a, pgt_f2 b, pgt_f2 c) { pgt_f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ pgt_f2 pgt_add(pgt_f2 a, pgt_f2 b) { pgt_f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
// largest of three, NaN if one is (a NaN score has to reach its row)
__device__ __forceinline__ float pgt_max3(float a, float b, float c) { float r; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

template <int D>
__global__ void __launch_bounds__(PGT_THREADS, 1)
pg_attend_tc_kernel(const __grid_constant__ PgAttend p, const __grid_constant__ PgMaps maps) {
    using C = PgtCfg<D>;
    constexpr int SK = C::SK, SV = C::SV, M = PGT_M, KT = PGT_KT;
    extern __shared__ uint8_t pgt_raw[];
    uint8_t* Qs = (uint8_t*)(((uintptr_t)pgt_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* ring_k = Qs + 2 * C::TILE;
    uint8_t* ring_v = ring_k + SK * C::TILE;
    __shared__ PgPlanSmem<1> plan;
    __shared__ uint64_t k_full[SK], k_empty[SK], v_full[SV], v_empty[SV], v_clean[SV], qu_full[PGT_QUEUE], qu_empty[PGT_QUEUE];
    __shared__ uint64_t q_full[2], s_full[2], p_lo[2], p_hi[2], o_full[2];     // P in two parts: 96 keys, 32 keys
    __shared__ PgPiece queue[PGT_QUEUE], queue_v[PGT_QUEUE];
    __shared__ int found[PGT_QUEUE];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_s;
    volatile int* abort_flag = &abort_s;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < SK; s++) { mbar_init(&k_full[s], 1); mbar_init(&k_empty[s], 1); }
        for (int s = 0; s < SV; s++) { mbar_init(&v_full[s], 1); mbar_init(&v_empty[s], 1); mbar_init(&v_clean[s], 1); }
        for (int s = 0; s < PGT_QUEUE; s++) { mbar_init(&qu_full[s], 1); mbar_init(&qu_empty[s], 10); }
        for (int w = 0; w < 2; w++) { mbar_init(&q_full[w], 4); mbar_init(&s_full[w], 1); mbar_init(&p_lo[w], 4); mbar_init(&p_hi[w], 4); mbar_init(&o_full[w], 1); }
        abort_s = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 9) tmem_alloc(&tmem_slot, 512);
    pdl_enter();
    if (tid == 0) p.w.cut[blockIdx.x].i1 = -1;
    tc_fence_before();
    pg_plan_share<PGT_THREADS, PGT_KT>(p, M, plan);
    tc_fence_after();
    const uint32_t tmem = tmem_slot;

    if (warp >= 8) {
        pg_regs_less<PG_REGS_LESS>();
        if (warp == 8 || warp == 10) {
        // ---- producers: warp 8 the K tiles (and the queue), warp 10 the V tiles ----
        const int kv = warp == 10;
        PgProducer<KT, PGT_QUEUE> bx;
        bx.queue = kv ? queue_v : queue; bx.full = kv ? nullptr : qu_full; bx.empty = kv ? nullptr : qu_empty; bx.found = kv ? nullptr : found;
        bool ok = bx.start(p, plan);
        const bool issuer = elect_one();
        const CUtensorMap *m64 = kv ? &maps.v64 : &maps.k64, *m32 = kv ? &maps.v32 : &maps.k32;
        uint8_t* const ring = kv ? ring_v : ring_k;
        uint64_t *const full = kv ? v_full : k_full, *const empty = kv ? v_empty : k_empty;
        const int nbox = 1 << bx.lg_box;
        int cnt = 0, s = 0;                                // tiles asked for, stage of the next one
        uint32_t ph = 1;                                   // parity of the phase that frees it (the first round is free)
        while (ok) {
            const PgPiece* q = bx.begin(p);
            if (!q) break;
            const int i0 = q->i0, i1 = q->i1;
            for (int i = i0; i < i1; i++) {
                const int l0 = bx.tile_lane(p, q, i);
                if (!pg_wait(&empty[s], ph)) { ok = false; break; }
                uint8_t* d = ring + s * C::TILE;
                if (issuer) mbar_expect_tx(&full[s], C::TILE);
#pragma unroll 1
                for (int b = 0; b < nbox; b++) {
                    const int y = bx.row(l0 + b), at = b << bx.box_shift;
                    if (issuer) {
#pragma unroll
                        for (int a = 0; a < C::NA; a++) tma_load_2d(d + a * C::A_BYTES + at * 128, m64, a * 64, y, &full[s]);
                        if (C::NB) tma_load_2d(d + C::NA * C::A_BYTES + at * 64, m32, C::NA * 64, y, &full[s]);
                    }
                }
                cnt++;
                if (++s == (kv ? SV : SK)) { s = 0; ph ^= 1; }
                if (i == i0 && !bx.push(p)) { ok = false; break; }
            }
        }
        if (!ok) *abort_flag = 1;
        if (__any_sync(0xffffffffu, bx.bad) && lane == 0) atomicOr(p.w.status, PG_ST_BAD_PAGE);
        if (*abort_flag)
            for (int c = max(0, cnt - (kv ? SV : SK)); c < cnt; c++) pg_wait(&full[c % (kv ? SV : SK)], (c / (kv ? SV : SK)) & 1);
        } else if (warp == 11) {
        // ---- V tiles that some row does not see all of: non-finite elements out, before anyone multiplies by them ----
        int cnt = 0;
        bool ok = true;
        for (int qn = 0; ok; qn++) {
            const int qs = qn % PGT_QUEUE;
            ok = !*abort_flag && pg_wait(&qu_full[qs], (qn / PGT_QUEUE) & 1);
            if (!ok) break;
            const PgPiece pc = queue[qs];
            if (pc.i1 < 0) break;
            const PgSpan span = pg_span<KT>(pc.pmin, pc.pmax, p.window, p.sinks);
            for (int i = pc.i0; i < pc.i1 && ok; i++, cnt++) {
                const int s = cnt % SV;
                ok = pg_wait(&v_full[s], (cnt / SV) & 1);
                if (ok && pg_partial<KT>(pg_tile_key(span, i, KT), pc.pmin, pc.pmax, p.window, p.sinks)) {
                    uint8_t* vt = ring_v + s * C::TILE;
                    // 16-byte chunks in the order they lie in: D * 128 / 8 of them, the same for every swizzle
                    uint32_t seen = 0;
#pragma unroll 8
                    for (int c = lane; c < C::TILE / 16; c += 32) {
                        const uint4 v = *reinterpret_cast<const uint4*>(vt + c * 16);      // an exponent of all ones carries into bit 15 (31)
                        seen |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) |
                                ((v.z & 0x7f807f80u) + 0x00800080u) | ((v.w & 0x7f807f80u) + 0x00800080u);
                    }
                    if (seen & 0x80008000u) {
                        bool hit = false;
                        for (int c = lane; c < C::TILE / 16; c += 32) {
                            uint4 v = *reinterpret_cast<const uint4*>(vt + c * 16);
                            v.x = pgm_finite(v.x, &hit); v.y = pgm_finite(v.y, &hit); v.z = pgm_finite(v.z, &hit); v.w = pgm_finite(v.w, &hit);
                            *reinterpret_cast<uint4*>(vt + c * 16) = v;
                        }
                        *(volatile int*)&found[qs] = 1;
                        __threadfence_block();
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(&v_clean[s]);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&qu_empty[qs]);
        }
        if (!ok) *abort_flag = 1;
        } else if (warp == 9) {
        // ---- MMA issuer ----
        constexpr uint32_t idesc_s = umma_idesc(KT);
        constexpr uint32_t idesc_o = umma_idesc_bmn(C::NB ? 64 * C::NA : D);
        constexpr uint32_t idesc_o32 = umma_idesc_bmn(32);
        const uint32_t q0 = smem_u32(Qs), rk = smem_u32(ring_k), rv = smem_u32(ring_v);
        int cnt = 0;
        uint32_t np[2] = {0, 0}, nq[2] = {0, 0};           // per block: P tiles consumed, queries multiplied
        bool ok = true;
        for (int qn = 0; ok; qn++) {
            const int qs = qn % PGT_QUEUE;
            ok = !*abort_flag && pg_wait(&qu_full[qs], (qn / PGT_QUEUE) & 1);
            if (!ok) break;
            const PgPiece pc = queue[qs];
            if (pc.i1 < 0) break;
            const int len = pc.i1 - pc.i0;
            const int nb = (unsigned)pc.n * p.ge.g - (unsigned)pc.rt * M > 128u ? 2 : 1;
            auto qk = [&](int w, int c) {                  // S_w = Q_w K^T, K tile number c of the block
                const uint32_t k0 = rk + (c % SK) * C::TILE, qw = q0 + w * C::TILE, d = tmem + C::S_COL + w * 128;
                tc_fence_after();
#pragma unroll
                for (int a = 0; a < C::NA; a++)
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        umma_bf16(d, umma_desc_k128(qw + a * C::A_BYTES) + (uint64_t)(k * 2),
                                  umma_desc_k128(k0 + a * C::A_BYTES) + (uint64_t)(k * 2), idesc_s, (a | k) ? 1u : 0u);
                if (C::NB) {
#pragma unroll
                    for (int k = 0; k < 2; k++)
                        umma_bf16(d, umma_desc_k64(qw + C::NA * C::A_BYTES) + (uint64_t)(k * 2),
                                  umma_desc_k64(k0 + C::NA * C::A_BYTES) + (uint64_t)(k * 2), idesc_s, 1u);
                }
            };
            auto pv = [&](int w, int c, bool first, int k0, int k1) {      // O_w += P_w V over keys 16 k0 .. 16 k1, V tile number c
                const uint32_t v0 = rv + (c % SV) * C::TILE, a0 = tmem + C::S_COL + w * 128, d = tmem + C::O_COL + w * 128;
                tc_fence_after();
#pragma unroll
                for (int k = k0; k < k1; k++)
                    umma_bf16_ts(d, a0 + k * 8, umma_desc_mn128_blocks(v0 + k * 2048, C::A_BYTES), idesc_o, (!first || k) ? 1u : 0u);
                if (C::NB) {
#pragma unroll
                    for (int k = k0; k < k1; k++)
                        umma_bf16_ts(d + C::NA * 64, a0 + k * 8, umma_desc_mn64(v0 + C::NA * C::A_BYTES + k * 1024), idesc_o32, (!first || k) ? 1u : 0u);
                }
            };
            const bool issuer = elect_one();
            ok = pg_wait(&k_full[cnt % SK], (cnt / SK) & 1);
            for (int w = 0; w < nb && ok; w++) {
                ok = !*abort_flag && pg_wait(&q_full[w], nq[w] & 1);
                nq[w]++;
                if (ok && issuer) {
                    qk(w, cnt);
                    umma_commit(&s_full[w]);
                    if (w == nb - 1) umma_commit(&k_empty[cnt % SK]);      // K(0)
                }
            }
            for (int j = 0; j < len && ok; j++) {
                const int cv = cnt + j, ck = cv + 1;
                const bool more = j + 1 < len;
                ok = pg_wait(&v_clean[cv % SV], (cv / SV) & 1) && (!more || pg_wait(&k_full[ck % SK], (ck / SK) & 1));
                for (int w = 0; w < nb && ok; w++) {
                    ok = !*abort_flag && pg_wait(&p_lo[w], np[w] & 1);
                    if (ok && issuer) pv(w, cv, j == 0, 0, 6);
                    __syncwarp();
                    ok = ok && pg_wait(&p_hi[w], np[w] & 1);
                    np[w]++;
                    if (ok && issuer) {
                        pv(w, cv, false, 6, 8);
                        if (w == nb - 1) umma_commit(&v_empty[cv % SV]);
                        if (more) {
                            qk(w, ck);
                            umma_commit(&s_full[w]);
                            if (w == nb - 1) umma_commit(&k_empty[ck % SK]);
                        } else {
                            umma_commit(&o_full[w]);
                        }
                    }
                    __syncwarp();
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) *abort_flag = 1;
            __syncwarp();
            cnt += len;
            if (lane == 0) mbar_arrive(&qu_empty[qs]);
        }
        if (!ok) *abort_flag = 1;
        }
    } else {
        // ---- softmax ----
        pg_regs_more<PG_REGS_MORE>();
        const int w = warp >> 2, quad = warp & 3, rl = quad * 32 + lane;      // row of the block of 128
        const uint32_t t_lane = tmem + ((uint32_t)(quad * 32) << 16);
        const uint32_t t_s = t_lane + C::S_COL + w * 128, t_o = t_lane + C::O_COL + w * 128;
        const int limit = pg_pos_limit(p.b, p.ge);
        const float c2 = p.scale_log2;
        uint32_t n_s = 0, n_o = 0;
        bool ok = true;
        for (int qn = 0; ok; qn++) {
            const int qs = qn % PGT_QUEUE;
            ok = !*abort_flag && pg_wait(&qu_full[qs], (qn / PGT_QUEUE) & 1);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const PgPiece pc = queue[qs];
            if (pc.i1 < 0) break;
            const PgSpan span = pg_span<KT>(pc.pmin, pc.pmax, p.window, p.sinks);
            const int len = pc.i1 - pc.i0;
            const unsigned packed = (unsigned)pc.n * p.ge.g, pk = (unsigned)pc.rt * M + w * 128 + rl;     // (below 2^31: max_rows)
            const bool have = pk < packed;
            const unsigned of = have ? pk / (unsigned)p.ge.g : 0u;
            const int row = have ? pc.a + (int)of : 0, hd = pc.head * p.ge.g + (have ? (int)(pk - of * p.ge.g) : 0);
            int pos = have ? p.b.row_pos[row] : -1;
            if (pos >= limit) pos = -1;
            if (w == 1 && packed - (unsigned)pc.rt * M <= 128u) {             // block B is empty
                __syncwarp();
                if (lane == 0) mbar_arrive(&qu_empty[qs]);
                continue;
            }
            // the warp's 32 queries into the block's operand tile: D / 8 lanes share a row (whole lines from memory)
            uint8_t* qd = Qs + w * C::TILE + quad * 32 * 128;      // (64-column sub-tiles; the 32-column one has rows of 64 bytes)
            constexpr int CH = D / 8, RI = 32 / CH;                // 16-byte chunks of a row, rows per turn
            const int ch = lane % CH, rr = lane / CH;
            const uint32_t c_off = ch < 8 * C::NA ? (uint32_t)((ch >> 3) * C::A_BYTES) : (uint32_t)(C::NA * C::A_BYTES - quad * 32 * 64);
            auto place = [&](int r) {                              // chunk `ch` of the warp's row r
                return ch < 8 * C::NA ? qd + c_off + r * 128 + (((ch & 7) ^ (r & 7)) << 4) : qd + c_off + r * 64 + (((ch & 3) ^ ((r >> 1) & 3)) << 4);
            };
            {
                const unsigned long long my = have ? (unsigned long long)((const __nv_bfloat16*)p.q + (size_t)row * p.ldq + (size_t)hd * D) : 0ull;
uint4 x[(32 + RI - 1) / RI];                   // every load is under way before the first store
#pragma unroll
                for (int i = 0; i < 32; i += RI) {
                    const int r = i + rr;
                    const unsigned long long src = __shfl_sync(0xffffffffu, my, r & 31);
                    x[i / RI] = make_uint4(0, 0, 0, 0);
                    if (rr < RI && r < 32 && src) x[i / RI] = __ldg(reinterpret_cast<const uint4*>(src) + ch);
                }
#pragma unroll
                for (int i = 0; i < 32; i += RI)
                    if (rr < RI && i + rr < 32) *reinterpret_cast<uint4*>(place(i + rr)) = x[i / RI];
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[w]);
            }
            const int lo = pg_window_lo(pos, p.window);
            float m = -INFINITY, l = 0.f;                  // m: the maximum (log2 domain) the row's P and O are scaled by
            for (int j = 0; j < len; j++) {
                ok = !*abort_flag && pg_wait(&s_full[w], n_s & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                n_s++;
                tc_fence_after();
                const int key0 = pg_tile_key(span, pc.i0 + j, KT);
                pgt_f2 sums[2] = {0ull, 0ull};
                // moves the row's maximum to `mx` where the tile asks for it, and O and l with it
                auto settle = [&](float mx) {
                    const bool move = !(mx <= m + 8.0f) || (m == -INFINITY && mx > -INFINITY);      // (a NaN moves it, too)
                    if (__any_sync(0xffffffffu, move && l > 0.f)) {
                        // O is at rest: the commit that announced S(j) covers P V(j - 1)
                        const float corr = move ? ex2_approx(m - mx) : 1.0f;
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t orow[32];
                            tmem_ld32(t_o + c, orow);
#pragma unroll
                            for (int k = 0; k < 32; k++) orow[k] = __float_as_uint(__uint_as_float(orow[k]) * corr);
                            tmem_st32(t_o + c, orow);
                        }
                        l *= corr;
                    }
                    if (move) m = mx;
                };
                const pgt_f2 cc = pgt_pack(c2, c2);
                // P of 32 keys (16 packed words) from their scores.  (Giving a part of the exponentials to the FMA pipe, as a polynomial,
                // costs more issue slots than it frees MUFU slots: 1/2, 1/4, 1/8, 1/16, none of them: 540, 506, 480, 477, 464 us for
                // an 8,192-token prompt.)
                auto exps = [&](const uint32_t* s, uint32_t* pw, pgt_f2 uu) {
#pragma unroll
                    for (int k = 0; k < 16; k++) {
                        const pgt_f2 x = pgt_fma(pgt_pack(__uint_as_float(s[2 * k]), __uint_as_float(s[2 * k + 1])), cc, uu);
                        float e0, e1;
                        pgt_unpack(x, &e0, &e1);
                        e0 = ex2_approx(e0);
                        e1 = ex2_approx(e1);
                        sums[k & 1] = pgt_add(sums[k & 1], pgt_pack(e0, e1));
                        pw[k] = pack_bf16(e0, e1);
                    }
                };
                auto max32 = [&](const uint32_t* s, float* mx4) {
#pragma unroll
                    for (int k = 0; k < 32; k += 8)
#pragma unroll
                        for (int q = 0; q < 4; q++) mx4[q] = pgt_max3(mx4[q], __uint_as_float(s[k + 2 * q]), __uint_as_float(s[k + 2 * q + 1]));
                };
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                if (!pg_partial<KT>(key0, pc.pmin, pc.pmax, p.window, p.sinks)) {
                    // every row sees every key: the whole row of S in registers, read once
                    uint32_t sr[KT], pw[32];
#pragma unroll
                    for (int c = 0; c < KT; c += 32) tmem_ld32_issue(t_s + c, sr + c);
#pragma unroll
                    for (int c = 0; c < KT; c += 32) tmem_ld32_wait(sr + c);
#pragma unroll
                    for (int c = 0; c < KT; c += 32) max32(sr + c, mx4);
                    settle(pgt_max3(pgt_max3(mx4[0], mx4[1], mx4[2]), mx4[3], mx4[3]) * c2);
                    const float u = m == -INFINITY ? 0.f : m;
                    const pgt_f2 uu = pgt_pack(-u, -u);
                    exps(sr, pw, uu);
                    exps(sr + 32, pw + 16, uu);
                    tmem_st32_issue(t_s, pw);
                    exps(sr + 64, pw, uu);
                    tmem_st16_issue(t_s + 32, pw);
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_lo[w]);      // the product may begin with these 96 keys
                    exps(sr + 96, pw, uu);
                    tmem_st16_issue(t_s + 48, pw);
                } else {
                    // a tile with masked keys: 32 keys at a time in loops that stay small (unrolled like the path above, the
                    // masks cost more in instruction fetches than in work), S read twice; P goes where S has been read
                    uint32_t sr[32], pw[16];
#pragma unroll 1
                    for (int c = 0; c < KT; c += 32) {
                        const uint32_t see = pg_see_bits(key0 + c, pos, lo, p.sinks);
                        if (!__any_sync(0xffffffffu, see != 0)) continue;
                        tmem_ld32(t_s + c, sr);
#pragma unroll
                        for (int k = 0; k < 32; k++) sr[k] = (see >> k & 1) ? sr[k] : 0xff800000u;      // -inf
                        max32(sr, mx4);
                    }
                    settle(pgt_max3(pgt_max3(mx4[0], mx4[1], mx4[2]), mx4[3], mx4[3]) * c2);
                    const float u = m == -INFINITY ? 0.f : m;
                    const pgt_f2 uu = pgt_pack(-u, -u);
#pragma unroll 1
                    for (int c = 0; c < KT; c += 32) {
                        const uint32_t see = pg_see_bits(key0 + c, pos, lo, p.sinks);
                        if (__any_sync(0xffffffffu, see != 0)) {
                            tmem_ld32(t_s + c, sr);
#pragma unroll
                            for (int k = 0; k < 32; k++) sr[k] = (see >> k & 1) ? sr[k] : 0xff800000u;
                            exps(sr, pw, uu);
                        } else {
#pragma unroll
                            for (int k = 0; k < 16; k++) pw[k] = 0;
                        }
                        tmem_st16_issue(t_s + c / 2, pw);
                        if (c == 64) {
                            tmem_st_wait();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&p_lo[w]);
                        }
                    }
                }
                float s0, s1, s2, s3;
                pgt_unpack(sums[0], &s0, &s1);
                pgt_unpack(sums[1], &s2, &s3);
                l += (s0 + s1) + (s2 + s3);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_hi[w]);
            }
            if (ok) ok = __all_sync(0xffffffffu, pg_wait(&o_full[w], n_o & 1));
            n_o++;
            if (!ok) { *abort_flag = 1; break; }
            tc_fence_after();
            const bool whole = pc.c_first == pc.c_last, fix = *(volatile int*)&found[qs] != 0;
            const bool real = pos >= 0;
            float* slot = whole ? nullptr : pg_slot(p.w, blockIdx.x, pc.c_first, M, D);
            const int rm = w * 128 + rl;
            const float inv = 1.0f / l;
            __nv_bfloat16* dst = (__nv_bfloat16*)p.out + (size_t)row * p.ldo + (size_t)hd * D;
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                uint32_t orow[32];
                __syncwarp();                              // the load is the whole warp's
                tmem_ld32(t_o + c, orow);
                if (whole) {
                    // the block's queries are no longer needed (every S has been computed): their place takes the outputs
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {
                        uint32_t x[4];
#pragma unroll
                        for (int q = 0; q < 4; q++) x[q] = pack_bf16(__uint_as_float(orow[k + 2 * q]) * inv, __uint_as_float(orow[k + 2 * q + 1]) * inv);
                        const int oc = (c + k) / 8;
                        uint8_t* d = oc < 8 * C::NA ? qd + (oc >> 3) * C::A_BYTES + lane * 128 + (((oc & 7) ^ (lane & 7)) << 4)
                                                    : qd + C::NA * C::A_BYTES - quad * 32 * 64 + lane * 64 + (((oc & 3) ^ ((lane >> 1) & 3)) << 4);
                        *reinterpret_cast<uint4*>(d) = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                } else if (real) {
                    // slot layout of this kernel: [D / 4][256 rows][4], then (m, l) [256][2]
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        *reinterpret_cast<uint4*>(slot + ((size_t)((c + k) / 4) * M + rm) * 4) = make_uint4(orow[k], orow[k + 1], orow[k + 2], orow[k + 3]);
                }
            }
            if (fix && real) {
                // rare: what non-finite elements of V do to this row
#pragma unroll 1
                for (int e = 0; e < D; e++) {
                    const float add = pg_nonfinite<__nv_bfloat16, KT>(p, pc, pos, e);
                    if (add == 0.f) continue;
                    if (whole) {
                        const int oc = e / 8;
                        uint8_t* d = oc < 8 * C::NA ? qd + (oc >> 3) * C::A_BYTES + lane * 128 + (((oc & 7) ^ (lane & 7)) << 4)
                                                    : qd + C::NA * C::A_BYTES - quad * 32 * 64 + lane * 64 + (((oc & 3) ^ ((lane >> 1) & 3)) << 4);
                        __nv_bfloat16* x = reinterpret_cast<__nv_bfloat16*>(d) + e % 8;
                        *x = __float2bfloat16_rn(__bfloat162float(*x) + add);
                    } else {
                        slot[((size_t)(e / 4) * M + rm) * 4 + e % 4] += add;
                    }
                }
            }
            if (whole) {
                __syncwarp();
                const unsigned long long my = real ? (unsigned long long)dst : 0ull;
#pragma unroll
                for (int i = 0; i < 32; i += RI) {
                    const int r = i + rr;
                    const unsigned long long to = __shfl_sync(0xffffffffu, my, r & 31);
                    if (rr < RI && r < 32 && to) *reinterpret_cast<uint4*>(to + ch * 16) = *reinterpret_cast<const uint4*>(place(r));
                }
                if (real && p.lse) p.lse[(size_t)row * p.ge.n_heads + hd] = (m + log2f(l)) * 0.6931471805599453f;
            } else {
                if (real) *reinterpret_cast<float2*>(slot + (size_t)M * D + 2 * rm) = make_float2(m, l);
                if (tid == 0 && pc.c_first == (int)blockIdx.x) p.w.cut[blockIdx.x] = pc;      // for the joining kernel
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&qu_empty[qs]);
        }
        if (!ok) *abort_flag = 1;
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && abort_s) atomicOr(p.w.status, PG_ST_TIMEOUT);
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Joins the items that were cut between blocks, all over the GPU (a block that joined the parts of its item by itself
// read up to 18 parts of 133 KB through one SM: 64 rows behind 8,000 positions took 84 us).  Grid (blocks of the
// attention kernel, 8 runs of 32 rows); a thread takes D / 8 features of a row, parts in key order.
template <int D>
__global__ void __launch_bounds__(256) pg_join_tc_kernel(const __grid_constant__ PgAttend p) {
    constexpr int M = PGT_M, E = D / 8;
    pdl_enter();
    const PgPiece pc = p.w.cut[blockIdx.x];
    const int rows = pc.i1 < 0 ? 0 : (int)min((unsigned)M, (unsigned)pc.n * p.ge.g - (unsigned)pc.rt * M);
    const int r = blockIdx.y * 32 + (threadIdx.x & 31), e0 = (threadIdx.x >> 5) * E;
    if (r >= rows) return;
    const unsigned pk = (unsigned)pc.rt * M + r, of = pk / (unsigned)p.ge.g;
    const int row = pc.a + (int)of, hd = pc.head * p.ge.g + (int)(pk - of * p.ge.g), pos = p.b.row_pos[row];
    if (pos < 0 || pos >= pg_pos_limit(p.b, p.ge)) return;
    const int ns = pc.c_last - pc.c_first + 1;
    float mx = -INFINITY, den = 0.f, acc[E];
#pragma unroll 4
    for (int s = 0; s < ns; s++) mx = fmaxf(mx, __ldcg(pg_slot(p.w, pc.c_first + s, pc.c_first, M, D) + (size_t)M * D + 2 * r));
#pragma unroll
    for (int e = 0; e < E; e++) acc[e] = 0.f;
#pragma unroll 2
    for (int s = 0; s < ns; s++) {
        const float* sl = pg_slot(p.w, pc.c_first + s, pc.c_first, M, D);
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(sl + (size_t)M * D + 2 * r));
        float4 x[E / 4];
#pragma unroll
        for (int e = 0; e < E / 4; e++) x[e] = __ldcg(reinterpret_cast<const float4*>(sl + ((size_t)(e0 / 4 + e) * M + r) * 4));
        const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - mx);
#pragma unroll
        for (int e = 0; e < E / 4; e++) {
            acc[4 * e] = fmaf(x[e].x, f, acc[4 * e]); acc[4 * e + 1] = fmaf(x[e].y, f, acc[4 * e + 1]);
            acc[4 * e + 2] = fmaf(x[e].z, f, acc[4 * e + 2]); acc[4 * e + 3] = fmaf(x[e].w, f, acc[4 * e + 3]);
        }
        den = fmaf(ml.y, f, den);
    }
    const float inv = 1.0f / den;
    __nv_bfloat16* dst = (__nv_bfloat16*)p.out + (size_t)row * p.ldo + (size_t)hd * D + e0;
#pragma unroll
    for (int e = 0; e < E; e += 4) pg_store4(dst + e, acc[e] * inv, acc[e + 1] * inv, acc[e + 2] * inv, acc[e + 3] * inv);
    if (p.lse && e0 == 0) p.lse[(size_t)row * p.ge.n_heads + hd] = (mx + log2f(den)) * 0.6931471805599453f;
}

}  // namespace rd
