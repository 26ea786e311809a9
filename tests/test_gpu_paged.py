"""GPU tests of the paged K/V cache's operators against their definitions in 64 bits."""
import pytest
import torch

import paper_2510_14961_b200 as rd
from paged_harness import FILL, Case

pytestmark = pytest.mark.gpu
BF, F4 = rd.RD_BF16, rd.RD_F32


# ---- append ---------------------------------------------------------------------------------------------------------
APPEND = [
    # dtype, H, G, D, page, groups, options
    (BF, 4, 2, 128, 16, [(1, 0), (3, 14), (40, 100)], {}),
    (BF, 55, 55, 96, 64, [(32, 500)], dict(uniform=True)),
    (BF, 6, 3, 64, 32, [(1, 5)] * 70, dict(pad=5)),
    (F4, 4, 4, 64, 16, [(17, 0), (2, 31)], dict(ld_extra=8)),
    (F4, 2, 1, 10, 16, [(5, 3)], {}),                     # pairs only
    (BF, 3, 3, 12, 256, [(9, 250)], dict(ld_extra=4)),    # four features at a time
    (BF, 2, 2, 128, 128, [(300, 0), [7, 3, -1, 5]], dict(pad=2, n_layers=3, layer=1)),
    (F4, 8, 2, 32, 64, [(3, 60)], dict(rope_base=0.0)),
    (BF, 5, 5, 8, 16, [(6, 3)], {}), (F4, 3, 1, 4, 16, [(4, 14)], {}), (F4, 3, 3, 2, 16, [(4, 14)], {}),       # a head is one vector
    (BF, 48, 16, 128, 16, [(3, 2)], {}), (BF, 64, 64, 96, 32, [(2, 31)], {}),                                 # several parts of a row
    (BF, 2, 1, 64, 16, [(2, 130000)], {}),                # far positions: the angle keeps its fraction
]


@pytest.mark.parametrize("dtype,H,G,D,page,groups,opt", APPEND)
def test_append_writes_the_rows_into_their_pages(dtype, H, G, D, page, groups, opt):
    c = Case(dtype, H, G, D, page, groups, seed=3, **opt)
    kp, vp = c.kp.clone(), c.vp.clone()
    c.append()
    # a rotation multiplies twice and adds once in float32 with angles rounded to float32 (each factor off by
    # 2^-24 of 1, three roundings of 2^-24): 5 * 2^-24 (|a| + |b|); then half a step of the stored type
    half = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    live = [i for i, p in enumerate(c.row_pos[:c.n].tolist()) if p >= 0]

    def near(got, want, x):
        mag = x.double().abs()
        mag = mag + mag.reshape(*mag.shape[:-1], D // 2, 2).flip(-1).reshape(mag.shape)
        off = (got.double() - want).abs() - (5 * 2.0 ** -24 * mag + half * want.abs() + 1e-30)
        assert off.max() <= 0, f"{(got.double() - want).abs().max():.3e}"

    wq, wk = c.want_rope(c.q, H), c.want_rope(c.k, G)
    near(c.q_out[:c.n].reshape(c.n, H, D)[live], wq[live], c.q[:c.n].reshape(c.n, H, D)[live])
    assert (c.q_out[c.row_pos < 0] == FILL).all()
    # the pages: the new rows, and nothing else changed
    r = 0
    for g, ps in enumerate(c.pos):
        for p in ps:
            if p >= 0:
                pg = int(c.table_np[g, p // page])
                near(c.kp[c.layer, pg, :, p % page], wk[r], c.k[r].reshape(G, D))
                assert torch.equal(c.vp[c.layer, pg, :, p % page], c.v[r].reshape(G, D))
                kp[c.layer, pg, :, p % page] = c.kp[c.layer, pg, :, p % page]
                vp[c.layer, pg, :, p % page] = c.vp[c.layer, pg, :, p % page]
            r += 1
    assert torch.equal(kp, c.kp) and torch.equal(vp, c.vp)


def test_append_in_place_gives_the_same_bits():
    a, b = (Case(BF, 4, 2, 128, 16, [(33, 5), (1, 900)], seed=1) for _ in range(2))
    a.append()
    q = b.q.clone()
    b.q = q
    b.append(q_out=q)
    assert torch.equal(a.q_out, q) and torch.equal(a.kp, b.kp)


# ---- attention ------------------------------------------------------------------------------------------------------
ONE = [
    # the CUDA-core kernels: float32, and head sizes of their own
    (F4, 4, 4, 64, 16, [(1, 0)], {}),
    (F4, 4, 2, 64, 16, [(1, 76), (1, 0), (1, 300)], dict(pad=2)),
    (F4, 8, 1, 128, 32, [(1, 1000)], {}),
    (F4, 6, 2, 96, 64, [(24, 500), (20, 40)], {}),
    (F4, 2, 2, 10, 16, [(70, 3)], {}),
    (F4, 2, 1, 32, 16, [(1, 40), (200, 0), (1, 7)], dict(pad=1)),          # both kernels
    (BF, 2, 2, 80, 16, [(3, 77), (90, 200)], {}),
    (BF, 3, 1, 16, 256, [(1, 513)], {}),
    (F4, 4, 4, 48, 128, [(128, 0)], dict(uniform=True)),
    # few rows per sequence, bf16
    (BF, 4, 4, 64, 64, [(1, 0)], {}),
    (BF, 4, 4, 128, 16, [(1, 15), (1, 16), (1, 63), (1, 64), (1, 65)], {}),
    (BF, 8, 2, 128, 32, [(1, 700), (1, 3), (1, 0), (1, 129)], dict(pad=3)),
    (BF, 55, 55, 96, 64, [(1, 543)], {}),
    (BF, 5, 5, 96, 64, [(32, 511)], dict(uniform=True)),
    (BF, 6, 1, 96, 16, [(7, 100), (10, 3)], {}),
    (BF, 4, 1, 64, 128, [(16, 1000)], {}),
    (BF, 64, 1, 128, 16, [(1, 200)], {}),                                    # 64 query heads on one K/V head
    (BF, 7, 1, 64, 32, [(3, 64), (5, 11)], {}),
    (BF, 2, 2, 128, 256, [(1, 5000)], {}),                                   # split over the blocks
    (BF, 1, 1, 64, 16, [(1, 9999)], {}),
    (BF, 4, 2, 128, 16, [(1, 30 + 7 * i) for i in range(300)], {}),           # a plan of its own
    (BF, 4, 2, 64, 64, [[40, 41, 9, -1, 8], [-1, -1], [3]], dict(pad=1)),   # any order, a group without a row
    # many rows per sequence, bf16
    (BF, 1, 1, 64, 64, [(128, 0)], {}),
    (BF, 1, 1, 128, 64, [(128, 0)], {}),
    (BF, 2, 2, 96, 128, [(256, 0)], {}),
    (BF, 8, 2, 128, 16, [(200, 37)], {}),
    (BF, 4, 1, 64, 32, [(500, 1), (65, 300)], {}),
    (BF, 3, 1, 96, 256, [(333, 100)], dict(ld_extra=16)),
    (BF, 2, 1, 128, 64, [(1024, 0)], {}),
    (BF, 6, 2, 128, 64, [(70, 2000)], {}),
    (BF, 8, 2, 64, 32, [(300, 900), (1, 40), (1, 700), (20, 5), (1, 0)], dict(pad=4)),
    (BF, 16, 2, 128, 16, [(1, 40), (129, 0), (1, 700), (64, 500)], dict(hint=False)),
]


@pytest.mark.parametrize("dtype,H,G,D,page,groups,opt", ONE)
def test_attend(dtype, H, G, D, page, groups, opt):
    c = Case(dtype, H, G, D, page, groups, seed=5, **opt)
    c.attend()
    c.check_attend()


# ---- sliding window and sinks ---------------------------------------------------------------------------------------
WINDOW = [
    # dtype, H, G, D, page, groups, window, sinks
    (F4, 4, 2, 64, 16, [(1, 300), (1, 5), (20, 200)], 33, 4),
    (F4, 2, 2, 128, 32, [(100, 50)], 1, 0),
    (F4, 2, 2, 128, 32, [(100, 50)], 7, 129),
    (BF, 2, 1, 16, 16, [(1, 500), (70, 90)], 64, 64),
    (BF, 8, 2, 128, 16, [(1, 2000), (1, 63), (1, 64), (1, 65)], 64, 0),
    (BF, 8, 2, 128, 16, [(1, 2000), (1, 63), (1, 64), (1, 65)], 64, 4),
    (BF, 4, 4, 96, 64, [(32, 700), (30, 0)], 16, 1),
    (BF, 4, 4, 64, 128, [(1, 4000)], 4096, 33),
    (BF, 4, 4, 64, 128, [(1, 4000)], 1, 0),
    (BF, 4, 4, 64, 128, [(1, 4000)], 1000, 2000),                # many tiles of sinks
    (BF, 4, 1, 128, 32, [(300, 1000)], 128, 4),
    (BF, 4, 1, 64, 16, [(300, 0), (200, 513)], 100, 16),
    (BF, 2, 2, 96, 64, [(400, 300)], 1, 1),
    (BF, 2, 2, 128, 64, [(700, 0)], 1000, 5),                    # a window nobody has reached
    (BF, 4, 2, 128, 256, [(500, 900), (1, 3000), (1, 2)], 130, 300),
    (BF, 4, 2, 128, 64, [(65, 900)], 2 ** 31 - 1, 2 ** 31 - 1),
    (F4, 4, 2, 64, 64, [(65, 100)], 2 ** 31 - 1, 2 ** 31 - 1),
]


@pytest.mark.parametrize("dtype,H,G,D,page,groups,window,sinks", WINDOW)
def test_window_and_sinks(dtype, H, G, D, page, groups, window, sinks):
    c = Case(dtype, H, G, D, page, groups, seed=6, pad=1)
    c.attend(window, sinks)
    c.check_attend(window, sinks)


@pytest.mark.parametrize("dtype,H,G,D,rows", [(F4, 2, 2, 64, 1), (F4, 2, 2, 64, 80), (BF, 4, 2, 80, 40), (BF, 4, 2, 128, 1), (BF, 4, 4, 96, 24),
                                              (BF, 4, 2, 64, 300)])
def test_pages_no_row_sees_may_be_missing(dtype, H, G, D, rows):
    # entries between the sinks and the window hold -1 or the number of a page far outside the pool
    c = Case(dtype, H, G, D, 16, [(rows, 1000), (rows, 400)], seed=7)
    c.attend(100, 20)
    want, lse = c.out.clone(), c.lse.clone()
    for g, before in ((0, 1000), (1, 400)):
        for i in range(2, (before - 100 + 1) // 16):
            c.table[g, i] = -1 if i % 2 else 10 ** 9
    c.out.fill_(FILL)
    c.attend(100, 20)
    assert torch.equal(want, c.out) and torch.equal(lse, c.lse)
    c.check_attend(100, 20)


# ---- what lies in masked places -------------------------------------------------------------------------------------
KINDS = [(F4, 4, 2, 64, 1), (F4, 4, 2, 64, 40), (BF, 4, 2, 80, 1), (BF, 4, 2, 80, 30), (BF, 8, 2, 128, 1), (BF, 4, 4, 96, 24), (BF, 4, 2, 64, 20),
         (BF, 4, 2, 128, 200), (BF, 4, 2, 96, 200), (BF, 2, 2, 64, 300)]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,H,G,D,n", KINDS)
def test_unwritten_places_have_no_influence(dtype, H, G, D, n, bad):
    c = Case(dtype, H, G, D, 32, [(n, 130), (n, 0)], seed=8)
    c.attend(40, 3)
    want, lse = c.out.clone(), c.lse.clone()
    used = set()
    for g in range(2):
        L = c.len[g]
        low = c.pos[g][0] - 40 + 1
        for i in range((L + 31) // 32):
            pg = int(c.table_np[g, i])
            used.add(pg)
            for o in range(32):
                j = i * 32 + o
                if j >= L or 3 <= j < low:                 # behind the newest position, or between sinks and window
                    c.kp[0, pg, :, o] = bad
                    c.vp[0, pg, :, o] = bad
    for pg in range(c.n_pages):
        if pg not in used:
            c.kp[0, pg] = bad
            c.vp[0, pg] = bad
    c.out.fill_(FILL)
    c.attend(40, 3)
    assert torch.equal(want, c.out) and torch.equal(lse, c.lse)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,H,G,D,n", KINDS)
def test_a_key_that_is_not_finite_reaches_the_rows_that_see_it_only(dtype, H, G, D, n, bad):
    # V of one position holds `bad` in two features; rows before it must not notice, rows that see it get it
    c = Case(dtype, H, G, D, 32, [(n, 130)], seed=9)
    at = 130 + n // 2
    c.attend()
    clean = c.out.clone().reshape(n, H, D)
    pg, o = int(c.table_np[0, at // 32]), at % 32
    for f in (1, D - 3):
        c.vp[0, pg, 0, o, f] = bad
    c.out.fill_(FILL)
    c.attend()
    got = c.out.reshape(n, H, D)
    first, rep = n // 2, H // G                              # rows first .. see position `at`
    assert torch.equal(got[:first], clean[:first])
    assert torch.equal(got[:, rep:], clean[:, rep:])         # the other K/V head
    hit = torch.zeros(D, dtype=torch.bool, device="cuda")
    hit[1] = hit[D - 3] = True
    seen = got[first:, :rep]
    assert torch.isfinite(seen[..., ~hit]).all()
    tol = 2.0 ** -8 if dtype == BF else 1e-5
    assert (seen[..., ~hit].double() - clean[first:, :rep][..., ~hit].double()).abs().max() <= 4 * tol   # order of sums may change: |out| < 4
    assert (torch.isnan(seen[..., hit]).all() if bad != bad else (seen[..., hit] == bad).all())


@pytest.mark.parametrize("dtype,H,G,D,n", KINDS)
def test_scores_far_apart(dtype, H, G, D, n):
    # keys with large norms: the softmax is nearly one-hot and the running maximum moves often
    c = Case(dtype, H, G, D, 16, [(n, 200)], seed=10, kscale=12.0)
    c.attend()
    c.check_attend()
    c.attend(scale=0.01)
    c.check_attend(scale=0.01)


# ---- the division of the work ---------------------------------------------------------------------------------------
SPLIT = [(F4, 2, 1, 64, [(1, 20000)]), (F4, 2, 1, 64, [(40, 9000)]), (BF, 2, 1, 128, [(1, 70000)]), (BF, 16, 1, 64, [(4, 30000)]),
         (BF, 8, 1, 96, [(1, 33000), (1, 1), (1, 5000)]), (BF, 2, 1, 128, [(130, 20000)]), (BF, 2, 1, 64, [(300, 17000), (200, 3)]),
         (BF, 2, 2, 96, [(256, 9000)])]


@pytest.mark.parametrize("dtype,H,G,D,groups", SPLIT)
def test_long_contexts_are_split_and_joined(dtype, H, G, D, groups):
    c = Case(dtype, H, G, D, 64, groups, seed=11)
    c.attend()
    c.check_attend()
    first, lse = c.out.clone(), c.lse.clone()
    for _ in range(5):                                       # the order in which blocks arrive has no say
        c.out.fill_(FILL)
        c.attend()
        assert torch.equal(first, c.out) and torch.equal(lse, c.lse)


@pytest.mark.parametrize("dtype,D", [(F4, 64), (BF, 64), (BF, 128)])
def test_many_groups(dtype, D):
    c = Case(dtype, 2, 1, D, 16, [(1 + (i % 3 == 0), (i * 7) % 40) for i in range(4096)], seed=12)
    c.attend()
    c.check_attend()


def test_results_do_not_depend_on_the_hint():
    groups = [(1, 500), (90, 40), (3, 77), (1, 0)]
    outs = []
    for most in (90, 0, 1, 100000):
        c = Case(BF, 8, 2, 128, 32, groups, seed=13)
        c.rows = rd.PagedRows(c.row_pos, c.table, group_start=c.start, max_group_rows=most)
        c.attend()
        c.check_attend()
        outs.append(c.out.clone())


def test_offsets_beyond_32_bits():
    # a pool of more than 2^32 elements whose used pages lie at its end
    H, G, D, page = 8, 8, 128, 128
    n_pages = (1 << 32) // (G * page * D) + 40
    c = Case(BF, H, G, D, page, [(1, 1000), (70, 300)], seed=14)
    kp = torch.zeros(1, n_pages, G, page, D, dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    shift = n_pages - c.n_pages
    kp[0, shift:], vp[0, shift:] = c.kp[0], c.vp[0]
    cache = rd.PagedCache(H, G, D, page, n_pages, max_context=c.cache.cfg.max_context, dtype=BF, k_pages=kp, v_pages=vp)
    rows = rd.PagedRows(c.row_pos, c.table + shift, group_start=c.start, max_group_rows=c.most)
    cache.append(rows, c.q, c.k, c.v, c.q_out)
    cache.attend(rows, c.q_out, c.out, c.lse)
    cache.sync()
    c.append()
    want_q = c.q_out.clone()
    assert torch.equal(kp[0, shift:], c.kp[0]) and torch.equal(vp[0, shift:], c.vp[0])
    got = c.out.clone()
    c.cache.attend(c.rows, want_q, c.out, c.lse)
    c.cache.sync()
    assert torch.equal(got, c.out)


# ---- how it is called -----------------------------------------------------------------------------------------------
def test_append_then_attend_as_a_decode_loop():
    """A prompt in two slices, then single tokens: every step appends and attends; at the end the cache and the
    outputs are those of the whole sequence at once."""
    H, G, D, page, n = 8, 2, 128, 16, 150
    whole = Case(BF, H, G, D, page, [(n, 0)], seed=15)
    whole.append()
    q_all = whole.q_out.clone()
    whole.q.copy_(q_all)
    whole.attend()
    whole.check_attend()
    c = Case(BF, H, G, D, page, [(n, 0)], seed=15)
    done = torch.zeros_like(c.out)
    for a, b in [(0, 70), (70, 130)] + [(i, i + 1) for i in range(130, n)]:
        rows = rd.PagedRows(c.row_pos[a:b].contiguous(), c.table, max_group_rows=b - a)
        qo = torch.empty(b - a, H * D, dtype=torch.bfloat16, device="cuda")
        out = torch.empty_like(qo)
        c.cache.append(rows, c.q[a:b], c.k[a:b], c.v[a:b], qo)
        c.cache.attend(rows, qo, out)
        done[a:b] = out
    c.cache.sync()
    assert torch.equal(c.kp, whole.kp) and torch.equal(c.vp, whole.vp)
    c.q.copy_(q_all)
    c.out.copy_(done)
    c.lse.copy_(whole.lse)
    c.check_attend()


@pytest.mark.parametrize("groups,H,G", [([(1, 9000), (1, 40)], 8, 2), ([(300, 2000), (1, 5)], 4, 2)])
def test_captured_and_replayed_with_other_contents(groups, H, G):
    c = Case(BF, H, G, 128, 16, groups, seed=16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.cache.append(c.rows, c.q, c.k, c.v, c.q_out, stream=side.cuda_stream)
        c.cache.attend(c.rows, c.q_out, c.out, c.lse, stream=side.cuda_stream)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        graph.capture_begin()
        c.cache.append(c.rows, c.q, c.k, c.v, c.q_out, stream=side.cuda_stream)
        c.cache.attend(c.rows, c.q_out, c.out, c.lse, stream=side.cuda_stream)
        graph.capture_end()
    torch.cuda.synchronize()
    for seed in (17, 18):
        d = Case(BF, H, G, 128, 16, groups, seed=seed)
        for name in ("q", "k", "v", "kp", "vp", "table", "row_pos"):
            getattr(c, name).copy_(getattr(d, name))
        c.table_np = d.table_np
        c.out.fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        c.cache.sync()
        d.append()
        d.cache.attend(d.rows, d.q_out, d.out, d.lse)
        d.cache.sync()
        assert torch.equal(c.out, d.out) and torch.equal(c.kp, d.kp)


def test_two_caches_over_the_same_pages_at_the_same_time():
    c = Case(BF, 4, 2, 128, 64, [(1, 20000), (1, 9000)], seed=19)
    c.attend()
    want = c.out.clone()
    other = rd.PagedCache(4, 2, 128, 64, c.n_pages, max_context=c.cache.cfg.max_context, dtype=BF, k_pages=c.kp, v_pages=c.vp)
    outs = [torch.empty_like(c.out) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for cache, out, st in zip((c.cache, other), outs, streams):
            cache.attend(c.rows, c.q, out, stream=st.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_pages_of_the_librarys_own():
    cache = rd.PagedCache(2, 2, 64, 16, 4, max_context=64)
    k, v = cache.pages()
    assert k and v and k != v
    row_pos = torch.arange(5, dtype=torch.int32, device="cuda")
    rows = rd.PagedRows(row_pos, torch.tensor([[2]], dtype=torch.int32, device="cuda"), max_group_rows=5)
    x = torch.randn(5, 128, device="cuda").bfloat16()
    q, out = torch.empty_like(x), torch.empty_like(x)
    cache.append(rows, x, x, x, q)
    cache.attend(rows, q, out)
    cache.sync()
    assert torch.equal(out[0], x[0])                          # one key: its V


# ---- refusals -------------------------------------------------------------------------------------------------------
def _small(dtype=BF):
    return Case(dtype, 4, 2, 64, 16, [(2, 3)], seed=20)


def test_calls_that_are_refused():
    c = _small()

    def refused(code, f, *a, **kw):
        with pytest.raises(rd.RdError) as err:
            f(*a, **kw)
        assert err.value.code == code

    refused(rd.RD_E_INVALID_ARG, c.attend, window=-1)
    refused(rd.RD_E_INVALID_ARG, c.attend, sinks=-1)
    for s in (-1.0, float("nan"), float("inf")):
        refused(rd.RD_E_INVALID_ARG, c.attend, scale=s)
    refused(rd.RD_E_INVALID_ARG, c.cache.attend, c.rows, c.q, c.out, layer=1)
    refused(rd.RD_E_INVALID_ARG, c.cache.attend, c.rows, c.q, c.q)               # in place
    refused(rd.RD_E_INVALID_ARG, c.cache.append, c.rows, c.q, c.k, c.v, c.kp.reshape(-1)[:512].reshape(2, 256))
    odd = torch.zeros(2 * 257 + 8, dtype=torch.bfloat16, device="cuda")
    refused(rd.RD_E_INVALID_ARG, c.cache.attend, c.rows, odd[1:513].reshape(2, 256), c.out)          # address
    refused(rd.RD_E_INVALID_ARG, c.cache.attend, c.rows, odd[:514].reshape(2, 257)[:, :256], c.out)  # stride
    few = rd.PagedCache(4, 2, 64, 16, 4, max_context=16, max_rows=1)
    refused(rd.RD_E_CAPACITY, few.attend, c.rows, c.q, c.out)
    for kw in (dict(n_heads=3), dict(head_dim=130), dict(head_dim=63), dict(page_size=24), dict(page_size=8), dict(page_size=512), dict(n_pages=0),
               dict(n_layers=0), dict(max_context=0), dict(rope_base=-1.0), dict(dtype=2), dict(max_rows=-1)):
        args = dict(n_heads=4, n_kv_heads=2, head_dim=64, page_size=16, n_pages=4, max_context=16) | kw
        refused(rd.RD_E_INVALID_ARG, rd.PagedCache, **args)
    refused(rd.RD_E_CAPACITY, rd.PagedCache, n_heads=128, n_kv_heads=128, head_dim=64, page_size=256, n_pages=70000, max_context=16)
    for wrong in (c.q.float(), c.q.half(), c.q[:, :128], c.q[:1]):
        with pytest.raises(ValueError):
            c.cache.attend(c.rows, wrong, c.out)
    with pytest.raises(ValueError):
        rd.PagedRows(c.row_pos.long(), c.table, max_group_rows=2)
    with pytest.raises(ValueError):
        rd.PagedRows(c.row_pos, c.table, group_start=c.start[:1])
    none = rd.PagedRows(c.row_pos[:0], c.table, max_group_rows=1)               # no rows: nothing happens
    c.cache.attend(none, c.q[:0], c.out[:0])
    c.cache.append(none, c.q[:0], c.k[:0], c.v[:0], c.q_out[:0])
    c.attend()                                                                   # and the cache still works
    c.check_attend()


@pytest.mark.parametrize("dtype,D,n", [(F4, 64, 1), (F4, 64, 80), (BF, 128, 1), (BF, 128, 200)])
def test_rows_the_device_finds_wrong_are_reported(dtype, D, n):
    def case():
        return Case(dtype, 4, 2, D, 16, [(n, 40), (n, 100)], seed=21)

    def reported(c, call):
        call(c)
        with pytest.raises(rd.RdError) as err:
            c.cache.sync()
        assert err.value.code == rd.RD_E_INVALID_ARG
        c.cache.sync()                                                           # reported once

    def attend(c):
        c.cache.attend(c.rows, c.q, c.out, c.lse)

    def append(c):
        c.cache.append(c.rows, c.q, c.k, c.v, c.q_out)

    for value in (-1, 10 ** 9):                                                  # a needed entry that is no page
        for call in (attend, append):
            c = case()
            c.table[0, 2] = value
            reported(c, call)
    for call in (attend, append):                                                # a position beyond table and max_context
        c = case()
        c.row_pos[-1] = 10 ** 6
        kp = c.kp.clone()
        reported(c, call)
        assert (c.out[-1] == FILL).all() and (c.q_out[-1] == FILL).all()
        if call is attend:
            assert torch.equal(kp, c.kp)


@pytest.mark.parametrize("H,G,D,page,window,sinks", [(8, 8, 64, 32, 0, 0), (8, 8, 128, 64, 100, 16), (16, 2, 96, 16, 70, 0)])
def test_blocks_that_walk_over_many_items(H, G, D, page, window, sinks):
    # more items than blocks, row tiles whose second half is empty between full ones, short and long ones next to each
    # other, called again and again: every piece finds its barriers where the one before left them
    c = Case(BF, H, G, D, page, [(257 + 9 * (i % 5) + (100 if i % 3 == 0 else 0), 5 + 37 * (i % 7)) for i in range(26)], seed=22, pad=2)
    c.attend(window, sinks)
    c.check_attend(window, sinks)
    first = c.out.clone()
    for _ in range(20):
        c.attend(window, sinks)
        assert torch.equal(first, c.out)


@pytest.mark.parametrize("dtype,D,n", [(F4, 64, 40), (BF, 128, 1), (BF, 128, 100)])
def test_group_borders_that_do_not_ascend_are_survived(dtype, D, n):
    # overlapping and reversed groups: results are undefined, every access stays inside, the call after it is right
    c = Case(dtype, 4, 2, D, 16, [(n, 40)] * 6, seed=23)
    good = c.start.clone()
    for border in ([0, 6 * n, 0, 6 * n, 0, 6 * n, 0], [6 * n, 5 * n, 4 * n, 3 * n, 2 * n, n, 0], [-5, 10 ** 9, -7, 3, 2 ** 31 - 1, -2 ** 31, 6 * n]):
        c.start.copy_(torch.tensor(border, dtype=torch.int32))
        for call in (lambda: c.cache.attend(c.rows, c.q, c.out, c.lse), lambda: c.cache.append(c.rows, c.q, c.k, c.v, c.q_out)):
            call()
            try:
                c.cache.sync()
            except rd.RdError as err:
                assert err.code == rd.RD_E_INVALID_ARG
    c.start.copy_(good)
    c.out.fill_(FILL)
    c.attend()
    c.check_attend()


def test_rows_of_a_fused_projection():
    # q, k and v as column ranges of one array, q turned in place
    H, G, D, n = 4, 2, 64, 70
    c = Case(BF, H, G, D, 16, [(n, 33)], seed=24)
    buf = torch.cat([c.q, c.k, c.v], dim=1).contiguous()
    q, k, v = buf[:, :H * D], buf[:, H * D:(H + G) * D], buf[:, (H + G) * D:]
    c.append()
    kp = c.kp.clone()
    c.kp.normal_()
    c.cache.append(c.rows, q, k, v, q)
    c.cache.sync()
    used = [int(x) for x in c.table_np[0]]
    assert torch.equal(q, c.q_out)
    for p in range(33, 33 + n):
        assert torch.equal(c.kp[0, used[p // 16], :, p % 16], kp[0, used[p // 16], :, p % 16])
