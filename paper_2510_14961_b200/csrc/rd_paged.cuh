// Paged K/V cache: what its kernels share (arguments, row spans, the division of the work, the joining of
// partial results), and the kernel that writes new rows into the pages.
//
// Pages: [layer][page][kv head][page_size][head_dim] for K and for V; a sequence's positions
// page_size * i .. page_size * (i + 1) - 1 lie on page table[group][i].  A call names rows (one new token
// each) by groups: the rows of one sequence, every row with its position.  A row at position p sees the keys
// j <= p of its sequence, with a window w > 0 only those with j > p - w or j < sinks.
//
// The g = n_heads / n_kv_heads query heads that share a K/V head are extra rows of the same product:
// "packed" row i of a group is head i % g of its row i / g.  A row tile is M consecutive packed rows, and
// its keys are those at least one of its rows sees, in tiles of KT keys: first the tiles of the sinks, then
// those from the oldest key inside a window to the newest position.
//
// Division of the work.  The units of all (row tile, kv head) items - an item's fixed cost, then its key tiles -
// are numbered in one sequence and cut into one equal contiguous share per block, whatever the batch looks
// like: one sequence of 131,072 positions is split over all SMs, 64 ragged ones are packed onto them.  Items that
// take less time than joining their parts would are left whole (the block in whose share they begin does them).  An item that lies in one share is
// finished there; the shares of an item that is cut leave (maximum, sum, unnormalised output) in a workspace,
// and the block that arrives last joins them in key order, so results do not depend on which block that is.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "rd_common.cuh"
#include "rd_partial.cuh"

namespace rd {

struct PgBatch {
    int n_rows, n_groups;
    int uniform;                 // rows per group when group_start is null
    const int* group_start;      // [n_groups + 1], or null
    const int* row_pos;          // [n_rows]; negative: the row belongs to no sequence
    const int* table;            // [n_groups][table_stride]
    int table_stride;
};
struct PgGeom {
    int n_heads, n_kv, g, D;
    int page_shift, n_pages, layer;
    int max_pos;                 // positions the rotary table covers
};
// Device status word: bits a kernel raises, turned into an error code when the cache is synchronised.
constexpr int PG_ST_TIMEOUT = 1, PG_ST_BAD_ROW = 2, PG_ST_BAD_PAGE = 4;

struct PgRecord {                // one row tile
    int grp, a, n, rt;           // group, its first row, its rows, number of the tile in the group
    int pmin, pmax, nt, pad;     // smallest and largest position of its rows, key tiles
};
// One piece of an item: key tiles [i0, i1) of (row tile, kv head).
struct PgPiece {
    int grp, a, n, rt, head, i0, i1, nt, pmin, pmax;
    int c_first, c_last;         // blocks whose shares hold the item; equal: the piece is the whole item
};
struct PgWork {                  // one launch's share of the workspace
    PgRecord* rec;               // external plan: records, with their number in *n_rec
    int* n_rec;
    int* counter;                // [blocks] shares of the cut item that starts in a block which have arrived; 0 between launches
    float* part;                 // [2 * blocks][M][D + 2]
    PgPiece* cut;                // [blocks] the cut item that starts in a block (i1 < 0: none), for a joining kernel
    int* status;
};
struct PgAttend {
    PgBatch b;
    PgGeom ge;
    PgWork w;
    const void* q; void* out; float* lse;
    long long ldq, ldo;          // elements between rows
    const void *k, *v;           // pages (the kernels without tensor maps)
    int window, sinks;
    float scale_log2;            // scale * log2(e)
    int packed_lo, packed_hi;    // groups with packed_lo < packed rows <= packed_hi are this launch's
    int inline_plan;             // every block makes the plan itself (few row tiles)
    int min_share;               // units a share has at least
    int item_cost;               // units an item counts for besides its key tiles (its query, its output)
    int whole_units;             // items of at most this many units are not cut: the block in whose share they begin does them
    int rec_cap;                 // row tiles the plan's array holds (more only come from a group_start that is not ascending)
};

__device__ __forceinline__ void pg_group_rows(const PgBatch& b, int i, int* a, int* n) {
    int lo, hi;
    if (b.group_start) { lo = b.group_start[i]; hi = b.group_start[i + 1]; }
    else { const long long f = (long long)i * b.uniform; lo = (int)min(f, (long long)b.n_rows); hi = (int)min(f + b.uniform, (long long)b.n_rows); }
    lo = max(0, min(lo, b.n_rows));
    hi = max(lo, min(hi, b.n_rows));
    *a = lo;
    *n = hi - lo;
}
// Positions a call may name: those the table row and the rotary table cover.
__device__ __forceinline__ int pg_pos_limit(const PgBatch& b, const PgGeom& ge) {
    const long long t = (long long)b.table_stride << ge.page_shift;
    return (int)min(t, (long long)ge.max_pos);
}
// Row of the [layers * pages * kv heads * page_size, D] view of the pages that holds position `key` of group
// `grp`, or -1 when its table entry is no page.
__device__ __forceinline__ long long pg_row_of(const PgBatch& b, const PgGeom& ge, int grp, int kvh, int key) {
    const int pi = key >> ge.page_shift;
    if (pi >= b.table_stride) return -1;
    const int pg = b.table[(size_t)grp * b.table_stride + pi];
    if (pg < 0 || pg >= ge.n_pages) return -1;
    return ((((long long)ge.layer * ge.n_pages + pg) * ge.n_kv + kvh) << ge.page_shift) + (key & ((1 << ge.page_shift) - 1));
}

// Key tiles of a row tile.  lo: first tile inside the window; ns: tiles of the sinks in front of it.
struct PgSpan { int nt, ns, lo; };
template <int KT>
__device__ __forceinline__ PgSpan pg_span(int pmin, int pmax, int window, int sinks) {
    PgSpan s = {0, 0, 0};
    if (pmax < 0) return s;
    const int lo_key = window > 0 ? max(0, pmin - window + 1) : 0;
    s.lo = lo_key / KT;
    if (window > 0) s.ns = min((min(sinks, pmax + 1) + KT - 1) / KT, s.lo);
    s.nt = s.ns + pmax / KT + 1 - s.lo;
    return s;
}
__device__ __forceinline__ int pg_tile_key(const PgSpan& s, int i, int kt) { return (i < s.ns ? i : i - s.ns + s.lo) * kt; }
// Whether row position p (>= 0) sees key j.
__device__ __forceinline__ bool pg_sees(int p, int j, int window, int sinks) {
    return j <= p && (window <= 0 || p - j < window || j < sinks);
}
// Whether some row of a row tile does not see some key of the tile that starts at key0.
template <int KT> __device__ __forceinline__ bool pg_partial(int key0, int pmin, int pmax, int window, int sinks) {
    return key0 + KT - 1 > pmin || (window > 0 && pmax - key0 >= window && key0 + KT > sinks);
}
// The keys a row sees in 32 positions from key0 on, as bits: key0 + i <= pos, and i's key inside the window or a sink.
// lo: oldest position inside the row's window (INT_MIN without one).
__device__ __forceinline__ uint32_t pg_upto(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }   // lowest n bits
__device__ __forceinline__ uint32_t pg_see_bits(int key0, int pos, int lo, int sinks) {
    return pg_upto(pos + 1 - key0) & (~pg_upto(max(lo, key0) - key0) | pg_upto(sinks - key0));
}
__device__ __forceinline__ int pg_window_lo(int pos, int window) { return window > 0 ? pos - window + 1 : (int)0x80000000; }

// ---- the plan -----------------------------------------------------------------------------------------------
constexpr int PG_MAX_GROUPS = 4096;       // groups of a call
constexpr int PG_INLINE_REC = 256;        // row tiles a block plans by itself

// Lanes that look at the rows of one row tile together.
__host__ __device__ __forceinline__ int pg_lanes(int M, int g) {
    const int rows = (M + g - 1) / g + 1;
    int l = 1;
    while (l < 32 && l * 4 < rows) l *= 2;
    return l;
}
// Positions of a row tile by `lanes` neighbouring lanes (all 32 lanes of the warp call this).
__device__ __forceinline__ void pg_tile_positions(const PgBatch& b, const PgGeom& ge, int M, int a, int n, int rt, bool valid, int lanes,
                                                  int lane_in, int limit, int* pmin, int* pmax, bool* bad) {
    int lo = 0x7fffffff, hi = -1;
    if (valid) {
        const int r0 = (int)((long long)rt * M / ge.g);
        const int r1 = (int)min((long long)n, ((long long)(rt + 1) * M + ge.g - 1) / ge.g);
#pragma unroll 8
        for (int r = r0 + lane_in; r < r1; r += lanes) {
            const int p = b.row_pos[a + r];
            if (p >= limit) *bad = true;
            else if (p >= 0) { lo = min(lo, p); hi = max(hi, p); }
        }
    }
    for (int s = 1; s < lanes; s *= 2) {
        lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, s));
        hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, s));
    }
    *pmin = hi < 0 ? -1 : lo;
    *pmax = hi;
}
// Exclusive prefix sum over the block's threads (NT threads, NT a multiple of 32); *total: the sum.
template <int NT, typename V> __device__ __forceinline__ V pg_block_scan(V v, V* warp_sums, V* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    V inc = v;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
        const V o = __shfl_up_sync(0xffffffffu, inc, s);
        if (lane >= s) inc += o;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    V base = 0, tot = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; w++) {
        const V x = warp_sums[w];
        if (w < warp) base += x;
        tot += x;
    }
    *total = tot;
    return base + inc - v;
}

// Row tiles of all groups: `first` (shared memory, n_groups entries) receives the number of the first
// row tile of every group; returns how many there are.
template <int NT>
__device__ int pg_count_tiles(const PgAttend& p, int M, int* first, long long* warp_sums) {
    const int ng = p.b.n_groups;
    long long base = 0;                                    // (borders that do not ascend can name rows many times over)
    for (int c0 = 0; c0 < ng; c0 += NT) {
        const int i = c0 + (int)threadIdx.x;
        long long t = 0;
        if (i < ng) {
            int a, n;
            pg_group_rows(p.b, i, &a, &n);
            const long long packed = (long long)n * p.ge.g;
            if (packed > p.packed_lo && packed <= p.packed_hi) t = (packed + M - 1) / M;
        }
        long long tot;
        const long long at = base + pg_block_scan<NT, long long>(t, warp_sums, &tot);
        if (i < ng) first[i] = (int)min(at, 0x7fffffffll);
        base += tot;
    }
    if (base > p.rec_cap) {
        if (threadIdx.x == 0) atomicOr(p.w.status, PG_ST_BAD_ROW);
        base = p.rec_cap;
    }
    __syncthreads();
    return (int)base;
}
// Records r0, r0 + step, ... of the n_rec row tiles (each by `lanes` lanes) into dst.
template <int NT, int KT>
__device__ void pg_make_records(const PgAttend& p, int M, const int* first, int n_rec, PgRecord* dst, int part, int n_parts) {
    const int lanes = pg_lanes(M, p.ge.g), per_block = NT / lanes;
    const int lane_in = (int)threadIdx.x % lanes, slot = (int)threadIdx.x / lanes;
    const int limit = pg_pos_limit(p.b, p.ge);
    bool bad = false;
    for (int r0 = part * per_block; r0 < n_rec; r0 += n_parts * per_block) {
        const int r = r0 + slot;
        const bool valid = r < n_rec;
        PgRecord rec = {};
        if (valid) {
            int lo = 0, hi = p.b.n_groups - 1;             // last group whose first tile is <= r
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (first[mid] <= r) lo = mid; else hi = mid - 1;
            }
            rec.grp = lo;
            pg_group_rows(p.b, lo, &rec.a, &rec.n);
            rec.rt = r - first[lo];
        }
        pg_tile_positions(p.b, p.ge, M, rec.a, rec.n, rec.rt, valid, lanes, lane_in, limit, &rec.pmin, &rec.pmax, &bad);
        rec.nt = pg_span<KT>(rec.pmin, rec.pmax, p.window, p.sinks).nt;
        if (valid && lane_in == 0) dst[r] = rec;
    }
    if (bad) atomicOr(p.w.status, PG_ST_BAD_ROW);
}

// The plan as a kernel of its own, for calls with many row tiles.  Dynamic shared memory: n_groups ints.
constexpr int PG_PLAN_THREADS = 256;
template <int KT>
__global__ void __launch_bounds__(PG_PLAN_THREADS) pg_plan_kernel(const __grid_constant__ PgAttend p, int M) {
    extern __shared__ int first[];
    __shared__ long long warp_sums[PG_PLAN_THREADS / 32];
    pdl_enter();
    const int n_rec = pg_count_tiles<PG_PLAN_THREADS>(p, M, first, warp_sums);
    pg_make_records<PG_PLAN_THREADS, KT>(p, M, first, n_rec, p.w.rec, blockIdx.x, gridDim.x);
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.w.n_rec = n_rec;
}

// A block's share: units [u0, u1), and where u0 lies (unit `at` of the item: the fixed cost comes first).
struct PgShare {
    long long u0, u1, per;
    int rec, head, at, n_rec;
};
__device__ __forceinline__ int pg_units(const PgAttend& p, int nt) { return nt > 0 ? nt + p.item_cost : 0; }
template <int CAP> struct PgPlanSmem {
    PgRecord rec[CAP];           // CAP = PG_INLINE_REC, or 1 for a kernel whose plan is always made before it
    int first[CAP];
    long long warp_sums[32];
    PgShare share;
};
// All NT threads call this; the plan ends in sm.share, records in sm.rec (inline) or p.w.rec.
template <int NT, int KT, int CAP>
__device__ void pg_plan_share(const PgAttend& p, int M, PgPlanSmem<CAP>& sm) {
    int n_rec;
    const PgRecord* rec = p.w.rec;
    if (CAP > 1 && p.inline_plan) {
        n_rec = pg_count_tiles<NT>(p, M, sm.first, sm.warp_sums);
        pg_make_records<NT, KT>(p, M, sm.first, n_rec, sm.rec, 0, 1);
        rec = sm.rec;
        __syncthreads();
    } else {
        n_rec = *p.w.n_rec;
    }
    const int chunk = (n_rec + NT - 1) / NT, r0 = min(n_rec, (int)threadIdx.x * chunk), r1 = min(n_rec, r0 + chunk);
    long long mine = 0;
    for (int r = r0; r < r1; r++) mine += pg_units(p, rec[r].nt);
    mine *= p.ge.n_kv;
    long long total;
    const long long before = pg_block_scan<NT, long long>(mine, sm.warp_sums, &total);
    const long long per = max((total + gridDim.x - 1) / gridDim.x, (long long)p.min_share);
    const long long u0 = min(total, per * blockIdx.x), u1 = min(total, u0 + per);
    if (threadIdx.x == 0) { sm.share.u0 = u0; sm.share.u1 = u1; sm.share.per = per; sm.share.n_rec = n_rec; sm.share.rec = n_rec; }
    __syncthreads();
    if (u0 < u1 && u0 >= before && u0 < before + mine) {
        long long u = before;
        for (int r = r0; r < r1; r++) {
            const int units = pg_units(p, rec[r].nt);
            const long long len = (long long)units * p.ge.n_kv;
            if (u0 < u + len) {
                sm.share.rec = r;
                sm.share.head = (int)((u0 - u) / units);
                sm.share.at = (int)((u0 - u) % units);
                break;
            }
            u += len;
        }
    }
    __syncthreads();
}

// Walks a share piece by piece; every caller that walks (several warps may) sees the same pieces.
struct PgWalk {
    long long u, u1, per;
    int rec, head, at, n_rec, cost, whole;
    const PgRecord* recs;
    template <int CAP> __device__ __forceinline__ void start(const PgAttend& p, const PgPlanSmem<CAP>& sm) {
        u = sm.share.u0; u1 = sm.share.u1; per = sm.share.per;
        rec = sm.share.rec; head = sm.share.head; at = sm.share.at; n_rec = sm.share.n_rec; cost = p.item_cost; whole = p.whole_units;
        recs = CAP > 1 && p.inline_plan ? sm.rec : p.w.rec;
    }
    __device__ __forceinline__ bool next(int n_kv, PgPiece* o) {
        while (u < u1 && rec < n_rec) {
            const PgRecord r = recs[rec];
            if (r.nt == 0) { rec++; continue; }       // a row tile without a row of a sequence
            const int units = r.nt + cost;
            const bool uncut = units <= whole;
            const int len = uncut ? units - at : (int)min((long long)(units - at), u1 - u);
            const bool mine = !uncut || at == 0;      // (an uncut item that began in the share before is done there)
            const int i0 = max(0, at - cost), i1 = at + len - cost;
            const long long first = u - at + cost;    // unit of the item's first key tile
            o->grp = r.grp; o->a = r.a; o->n = r.n; o->rt = r.rt; o->head = head;
            o->i0 = i0; o->i1 = i1; o->nt = r.nt; o->pmin = r.pmin; o->pmax = r.pmax;
            o->c_first = uncut ? 0 : (int)(first / per);
            o->c_last = uncut ? 0 : (int)((first + r.nt - 1) / per);
            u += len;
            at += len;
            if (at == units) {
                at = 0;
                if (++head == n_kv) { head = 0; rec++; }
            }
            if (mine && i1 > i0) return true;                 // (a share may end inside an item's fixed cost)
        }
        return false;
    }
};

// Hands registers from the warps that need few to those that need many.  A block of 384 threads is launched with
// 168 registers a thread (64,512); 2 x 128 threads at 216 and 128 at 72 make the same.
template <int N> __device__ __forceinline__ void pg_regs_more() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void pg_regs_less() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
constexpr int PG_REGS_MORE = 216, PG_REGS_LESS = 72;

// ---- partial results ------------------------------------------------------------------------------------------
// Slot of block c for the item that starts in block c_first: the item is the last of c_first's share and
// the first of every later one.
__device__ __forceinline__ float* pg_slot(const PgWork& w, int c, int c_first, int M, int D) {
    return w.part + (size_t)(2 * c + (c == c_first ? 1 : 0)) * M * (D + 2);
}
// To be called by all `threads` threads of a group (barrier `bar`) that have written their share's slot: true
// in the block that arrives last, which then sees every slot.
template <typename Sync>
__device__ __forceinline__ bool pg_arrive_last(const PgWork& w, const PgPiece& pc, bool leader, int* flag, Sync sync) {
    sync();                                        // (the leader's fence covers what the barrier has ordered before it)
    if (leader) {
        __threadfence();
        const int want = pc.c_last - pc.c_first;
        const int seen = atomicAdd(&w.counter[pc.c_first], 1);
        const bool last = seen == want;
        if (last) atomicExch(&w.counter[pc.c_first], 0);       // for the next launch
        *flag = last;
        __threadfence();
    }
    sync();
    return *flag != 0;
}
__device__ __forceinline__ void pg_store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void pg_store4(__nv_bfloat16* p, float a, float b, float c, float d) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b), y = __floats2bfloat162_rn(c, d);
    uint2 u;
    u.x = *reinterpret_cast<const uint32_t*>(&x); u.y = *reinterpret_cast<const uint32_t*>(&y);
    *reinterpret_cast<uint2*>(p) = u;
}
// Joins the shares of an item and writes its rows.  Slot layout: outputs [M][D] (unnormalised, scaled by
// 2^m), then (m, l) [M][2].  tid counts the `threads` callers, a thread takes V features (4, or 1 when D is not
// a multiple of 4).
template <typename T, int V>
__device__ __forceinline__ void pg_join(const PgAttend& p, const PgPiece& pc, int M, int D, int tid, int threads) {
    const int rows = (int)min((long long)M, (long long)pc.n * p.ge.g - (long long)pc.rt * M);
    const int ns = pc.c_last - pc.c_first + 1, q4 = D / V, limit = pg_pos_limit(p.b, p.ge);
    for (int it = tid; it < rows * q4; it += threads) {
        const int r = it / q4, e = (it % q4) * V;
        const long long pk = (long long)pc.rt * M + r;
        const int row = pc.a + (int)(pk / p.ge.g), hd = pc.head * p.ge.g + (int)(pk % p.ge.g);
        const int pos = p.b.row_pos[row];
        if (pos < 0 || pos >= limit) continue;
        float mx = -INFINITY;
#pragma unroll 4
        for (int s = 0; s < ns; s++) mx = fmaxf(mx, __ldcg(pg_slot(p.w, pc.c_first + s, pc.c_first, M, D) + (size_t)M * D + 2 * r));
        float acc[V], den = 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] = 0.f;
#pragma unroll 4
        for (int s = 0; s < ns; s++) {
            const float* sl = pg_slot(p.w, pc.c_first + s, pc.c_first, M, D);
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(sl + (size_t)M * D + 2 * r));
            const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - mx);
            float v[V];
            if constexpr (V == 4) {
                const float4 u = __ldcg(reinterpret_cast<const float4*>(sl + (size_t)r * D + e));
                v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
            } else {
                v[0] = __ldcg(sl + (size_t)r * D + e);
            }
#pragma unroll
            for (int i = 0; i < V; i++) acc[i] = fmaf(v[i], w, acc[i]);
            den = fmaf(ml.y, w, den);
        }
        const float inv = 1.0f / den;
        T* dst = (T*)p.out + (size_t)row * p.ldo + hd * D + e;
        if constexpr (V == 4) pg_store4(dst, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
        else dst[0] = (T)(acc[0] * inv);
        if (p.lse && e == 0) p.lse[(size_t)row * p.ge.n_heads + hd] = (mx + log2f(den)) * 0.6931471805599453f;
    }
}
template <typename T>
__device__ __forceinline__ void pg_join_any(const PgAttend& p, const PgPiece& pc, int M, int D, int tid, int threads) {
    if (D % 4 == 0) pg_join<T, 4>(p, pc, M, D, tid, threads);
    else pg_join<T, 1>(p, pc, M, D, tid, threads);
}

// What feature e of the row at position `pos` gets from the non-finite elements of V among the keys it sees in
// key tiles [i0, i1) that were multiplied without them (partial tiles).  A weight is positive, so an infinity
// stays one.  Rare, hence slow and simple.
template <typename T, int KT>
__device__ __noinline__ float pg_nonfinite(const PgAttend& p, const PgPiece& pc, int pos, int e) {
    const PgSpan span = pg_span<KT>(pc.pmin, pc.pmax, p.window, p.sinks);
    float add = 0.f;
    for (int i = pc.i0; i < pc.i1; i++) {
        const int key0 = pg_tile_key(span, i, KT);
        if (!pg_partial<KT>(key0, pc.pmin, pc.pmax, p.window, p.sinks)) continue;
        for (int j = key0; j < key0 + KT; j++) {
            if (!pg_sees(pos, j, p.window, p.sinks)) continue;
            const long long row = pg_row_of(p.b, p.ge, pc.grp, pc.head, j);
            if (row < 0) continue;
            const float v = (float)((const T*)p.v)[(size_t)row * p.ge.D + e];
            if (!isfinite(v)) add += v;
        }
    }
    return add;
}

// ---- new rows into the pages ------------------------------------------------------------------------------------
// cos/sin of pos * base^(-2i/d), [max_pos][d/2]: angles in double (far positions keep their fraction), stored as float32.
static __global__ void __launch_bounds__(256) pg_rope_table_kernel(float2* __restrict__ cs, int max_pos, int half, double log2_base) {
    const long long n = (long long)max_pos * half;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const int p = (int)(i / half), j = (int)(i % half);
        double s, c;
        sincos((double)p * exp2(-log2_base * (double)j / (double)half), &s, &c);
        cs[i] = make_float2((float)c, (float)s);
    }
}

template <typename T> __device__ __forceinline__ float pg_to_f(T x) { return (float)x; }
template <typename T> __device__ __forceinline__ T pg_from_f(float x);
template <> __device__ __forceinline__ float pg_from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 pg_from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// VEC features at once, as wide as their bytes allow.
template <typename T, int VEC> struct alignas(sizeof(T) * VEC > 16 ? 16 : sizeof(T) * VEC) PgVec { T x[VEC]; };

// Two neighbouring features of a vector as floats, and back (bf16: one word; its high halves are the floats' own bits).
__device__ __forceinline__ void pg_pair(const float* x, float* a, float* b) { *a = x[0]; *b = x[1]; }
__device__ __forceinline__ void pg_pair(const __nv_bfloat16* x, float* a, float* b) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(x);
    *a = __uint_as_float(w << 16); *b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void pg_set_pair(float* x, float a, float b) { x[0] = a; x[1] = b; }
__device__ __forceinline__ void pg_set_pair(__nv_bfloat16* x, float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    *reinterpret_cast<uint32_t*>(x) = *reinterpret_cast<const uint32_t*>(&v);
}

// Sources of the new rows: q of feature m (0 .. n_heads D - 1), k and v of feature m (0 .. n_kv D - 1).
template <typename T> struct PgArrays {                   // three arrays of the cache's type (rd_paged_append)
    const T *q, *k, *v;
    long long ldq, ldk, ldv;
    template <int VEC> using Raw = PgVec<T, VEC>;         // (stays packed until it is used)
    template <int VEC> __device__ __forceinline__ Raw<VEC> load(int what, int r, int m) const {
        const T* s = what == 0 ? q + (size_t)r * ldq : what == 1 ? k + (size_t)r * ldk : v + (size_t)r * ldv;
        return *reinterpret_cast<const PgVec<T, VEC>*>(s + m);
    }
};
struct PgSums {                                           // sums of a QKV GEMM, [rows][q | k | v] (a session's layer)
    RowSource src;
    int nq, nk;                                           // features of q, of k
    template <int VEC> using Raw = PgVec<float, VEC>;
    template <int VEC> __device__ __forceinline__ Raw<VEC> load(int what, int r, int m) const {
        Raw<VEC> o;
        float* x = o.x;
        const int at = m + (what == 0 ? 0 : what == 1 ? nq : nq + nk);
        if constexpr (VEC % 4 == 0) {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                const float4 u = row_source_load4(src, r, at + i);
                x[i] = u.x; x[i + 1] = u.y; x[i + 2] = u.z; x[i + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i++) x[i] = row_source_load(src, r, at + i);
        }
        return o;
    }
};

struct PgAppend {
    PgBatch b;
    PgGeom ge;
    int* status;
    const float2* cs;            // rotary table, or null: q and k are stored as they come
    void* q_out; long long ldqo;
    void *k, *v;                 // pages
    unsigned head_magic;         // 2^32 / (vectors of a head), rounded up: vector -> head by one multiplication (vectors of a row < 2^26)
};

// Group of row r among ascending group borders, by a whole warp: 32 borders are looked at a time.  -1: behind the last group.
__device__ __forceinline__ int pg_group_of(const PgBatch& b, int r) {
    if (!b.group_start) {
        const int g = r / b.uniform;
        return g < b.n_groups ? g : -1;
    }
    const int lane = threadIdx.x & 31;
    int lo = 0, n = b.n_groups + 1;                        // the last border <= r lies in [lo, lo + n)
    while (n > 128) {
        const int step = (n + 31) / 32, i = lane * step;
        const unsigned le = __ballot_sync(0xffffffffu, i < n && b.group_start[lo + i] <= r);
        if (le == 0) return -1;
        const int k = (31 - __clz(le)) * step;
        lo += k;
        n = min(step, n - k);
    }
    int count = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) count += __popc(__ballot_sync(0xffffffffu, lane + 32 * j < n && b.group_start[lo + min(lane + 32 * j, n - 1)] <= r));
    lo += count - 1;
    return count > 0 && lo < b.n_groups ? lo : -1;
}

// Rotary embedding (adjacent pairs) of q and k at the row's position; q to q_out, k and v to the row's place
// in its page.  Bound by memory: every value is read and written once.  A warp takes U x 32 vectors of VEC features
// (16 bytes of bf16) of one row and asks for them before it looks for the row's group and page, whose loads depend on
// one another; the angles come from L1 for all heads but the first.  8,208 rows of 32/8 heads of 128: 37 us = 5.4 TB/s,
// 0.82 of the copy peak (71 us with a block per row and divisions for the indexes).  Grid (rows, parts of a row), up to PG_APPEND_WARPS warps.
constexpr int PG_APPEND_WARPS = 8, PG_APPEND_U = 4;
template <typename T, int VEC, typename Src>
__global__ void __launch_bounds__(32 * PG_APPEND_WARPS) pg_append_kernel(const __grid_constant__ PgAppend p, const __grid_constant__ Src src) {
    pdl_enter();
    const int lane = threadIdx.x & 31, r = blockIdx.x, part = blockIdx.y * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int D = p.ge.D, per_head = D / VEC, items = (p.ge.n_heads + 2 * p.ge.n_kv) * per_head;
    constexpr int U = PG_APPEND_U;
    typename Src::template Raw<VEC> x[U];
    const int first = part * U * 32 + lane, nq = p.ge.n_heads, nk = p.ge.n_kv;
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int c = first + u * 32;
        if (c < items) {
            const int hd = per_head == 1 ? c : (int)__umulhi((unsigned)c, p.head_magic), what = hd < nq ? 0 : hd < nq + nk ? 1 : 2;
            x[u] = src.template load<VEC>(what, r, (hd - (what == 0 ? 0 : what == 1 ? nq : nq + nk)) * D + (c - hd * per_head) * VEC);
        }
    }
    const int pos = p.b.row_pos[r];
    const int grp = pg_group_of(p.b, r);
    if (pos < 0 || grp < 0) return;
    const bool far = pos >= pg_pos_limit(p.b, p.ge);
    // where a head's vectors are a divisor of a warp every turn of a lane has the same angles
    const float2* cs = p.cs && !far ? p.cs + (size_t)pos * (D / 2) : nullptr;
    const bool same = (per_head & (per_head - 1)) == 0 && per_head <= 32;
    float2 a[VEC / 2];
#pragma unroll
    for (int i = 0; i < VEC / 2; i++) a[i] = cs && same ? cs[(lane & (per_head - 1)) * (VEC / 2) + i] : make_float2(1.f, 0.f);
    const long long row0 = far ? -1 : pg_row_of(p.b, p.ge, grp, 0, pos);
    if (row0 < 0) {
        if (lane == 0) atomicOr(p.status, far ? PG_ST_BAD_ROW : PG_ST_BAD_PAGE);
        return;
    }
    T* kd = (T*)p.k + (size_t)row0 * D;
    T* vd = (T*)p.v + (size_t)row0 * D;
    const size_t head = (size_t)D << p.ge.page_shift;      // elements between a page's heads
    T* qd = (T*)p.q_out + (size_t)r * p.ldqo;
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int c = first + u * 32;
        if (c >= items) break;
        const int hd = per_head == 1 ? c : (int)__umulhi((unsigned)c, p.head_magic), e = (c - hd * per_head) * VEC;
        if (cs && !same) {
#pragma unroll
            for (int i = 0; i < VEC / 2; i++) a[i] = cs[e / 2 + i];
        }
        T* dst = hd < nq ? qd + (size_t)hd * D + e : hd < nq + nk ? kd + (size_t)(hd - nq) * head + e : vd + (size_t)(hd - nq - nk) * head + e;
        const bool turn = cs && hd < nq + nk;
        PgVec<T, VEC> o;
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
            float s, t;
            pg_pair(x[u].x + i, &s, &t);
            pg_set_pair(o.x + i, turn ? s * a[i / 2].x - t * a[i / 2].y : s, turn ? s * a[i / 2].y + t * a[i / 2].x : t);
        }
        *reinterpret_cast<PgVec<T, VEC>*>(dst) = o;
    }
}

}  // namespace rd
