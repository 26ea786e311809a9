"""GPU tests of paged sessions: the model's layers on the paged operators, in lock step with the oracle and
against sessions with contiguous caches."""
import numpy as np
import pytest

import paper_2510_14961_b200 as rd
import rd_inputs
from oracle import rd_oracle as orc
from gpu_harness import LockStep, Tolerance, gpu_model
from helpers import SMALL, make_oracle

pytestmark = pytest.mark.gpu
F32_TOL, BF16_TOL, TIE_GAP = Tolerance(1e-4), Tolerance(5e-2, 2e-2), 3e-2      # those of the parity tests


def _setup(shape, bf16, batch, W, max_new, page, n_pages, window=0, sinks=0, max_ctx=256, cap=64, temperature=0.0, seed=0, **wkw):
    model, w = make_oracle(shape, seed=seed, bf16=bf16, contract=bf16, gain_jitter=0.0, max_ctx=max_ctx, attn_window=window, attn_sinks=sinks, **wkw)
    gm = gpu_model(shape, w, bf16=bf16)
    sess = rd.Session(gm, batch=batch, max_context=max_ctx, max_window=W, max_iters_per_pos=cap, max_new_tokens=max_new, keep_logits=True,
                      temperature=temperature, seed=seed + 7, page_size=page, n_pages=n_pages, attn_window=window, attn_sinks=sinks)
    sm = orc.Sampler(model, seed=seed + 7, temperature=temperature, max_iters_per_pos=cap)
    return gm, sess, sm


def _prefill(sm, sess, shape, lens, r, max_new, seed=0):
    seqs = []
    for b, L in enumerate(lens):
        prompt = rd_inputs.make_prompt(int(L), shape["vocab"], seed=seed + b)
        seqs.append(sm.prefill(b, prompt, r, max_new))
        sess.prefill(b, prompt, r)
    return seqs


def _run(ls, W, inner, eps):
    for _ in range(500):
        if ls.all_done():
            break
        ls.df(W, inner, eps)
    assert ls.all_done()
    ls.final_tokens_equal()


@pytest.mark.parametrize("shape,lens,W,inner,eps,page,window,sinks",
                         [(rd_inputs.TINY, [32], 4, 1, 0.0, 16, 0, 0), (SMALL, [9, 30], 3, 2, 0.05, 16, 0, 0), (SMALL, [40], 4, 1, 0.0, 32, 7, 2),
                          (SMALL, [70, 1], 5, 1, 0.0, 16, 20, 0)])
def test_float32_lock_step(shape, lens, W, inner, eps, page, window, sinks):
    gm, sess, sm = _setup(shape, False, len(lens), W, 14, page, 16, window, sinks, cap=12, std=0.02 if shape is rd_inputs.TINY else 0.08)
    ls = LockStep(sm, sess, _prefill(sm, sess, shape, lens, 3, 14), F32_TOL)
    _run(ls, W, inner, eps)
    assert ls.near_ties == 0


@pytest.mark.parametrize("lens,W,page,window,sinks", [([40], 16, 16, 0, 0), ([40, 21, 3], 8, 64, 0, 0), ([150, 90], 8, 32, 32, 4)])
def test_bf16_lock_step(lens, W, page, window, sinks):
    gm, sess, sm = _setup(rd_inputs.TWIN, True, len(lens), W, 16, page, 60, window, sinks)
    ls = LockStep(sm, sess, _prefill(sm, sess, rd_inputs.TWIN, lens, 2, 16), BF16_TOL, tie_gap=TIE_GAP)
    _run(ls, W, 1, 0.0)
    assert ls.near_ties <= max(2, int(0.08 * ls.n_drafts))


def test_bf16_window_of_24_rows_with_the_measured_drift():
    """24 recurrences of a row behind a 200-token prompt: two evaluations that round at the same points but sum in
    different orders part by more than the stated 5e-2 + 2e-2 |want| here.  The oracle shows it alone: accumulating in
    float32 instead of float64 moves its latents by 5.0e-2 at step 13 and past the bound from step 14 on (7e-2 at
    step 19).  So the bound cannot be asked as it stands; the GPU, a third such evaluation, is held to the bound plus
    what the two oracles differ by in this very step (largest so far: differences accumulate in the cache), for latents,
    logits, delta and the scores of tied tokens alike."""
    shape, L, W, max_new, window = rd_inputs.TWIN, 200, 24, 16, 64
    gm, sess, sm = _setup(shape, True, 1, W, max_new, 128, 60, window, 0)
    seqs = _prefill(sm, sess, shape, [L], 2, max_new)
    other, _ = make_oracle(shape, seed=0, bf16=True, contract=True, gain_jitter=0.0, max_ctx=256, attn_window=window, dtype=np.float32)
    sm32 = orc.Sampler(other, seed=7, max_iters_per_pos=64)
    sq32 = sm32.prefill(0, rd_inputs.make_prompt(L, shape["vocab"], seed=0), 2, max_new)
    ls = LockStep(sm, sess, seqs, BF16_TOL, tie_gap=TIE_GAP)
    drift = 0.0
    while not ls.all_done():
        info, info32 = sm.df_step(seqs[0], W, 1, 0.0), sm32.df_step(sq32, W, 1, 0.0)
        drift = max(drift, float(np.abs(info["z"] - info32["z"]).max()), float(np.abs(info["logits"] - info32["logits"]).max()))
        ls.tol, ls.tie_gap, ls.delta_tol = Tolerance(5e-2 + drift, 2e-2), TIE_GAP + drift, (5e-2 + drift, 2e-2)
        sess.df_step(W, 1, 0.0)
        ls.compare([info])
        sq32.tokens[:] = seqs[0].tokens                 # both oracles go on from the GPU's tokens
    ls.final_tokens_equal()
    assert drift < 0.3                                   # rounding, not another model


def test_float32_session_equals_the_contiguous_one():
    """Sequential decoder and sampler: same tokens; latents differ by the order of float32 sums only."""
    shape = rd_inputs.TINY
    _, w = make_oracle(shape, seed=1, gain_jitter=0.0, max_ctx=128)
    gm = gpu_model(shape, w)
    prompt = rd_inputs.make_prompt(30, shape["vocab"], seed=2)
    for window in (1, 4):
        kw = dict(batch=1, max_context=128, max_window=window, max_new_tokens=20, seed=3, keep_logits=True)
        a, b = rd.Session(gm, **kw), rd.Session(gm, page_size=16, n_pages=4, **kw)
        for s in (a, b):
            s.prefill(0, prompt, 4)
        while not a.committed(0)[1]:
            for s in (a, b):
                s.ar_step(4) if window == 1 else s.df_step(window, 1, 0.0)
            za, zb = a.debug_read(rd.RD_DBG_LATENTS), b.debug_read(rd.RD_DBG_LATENTS)
            assert np.abs(za - zb).max() <= 1e-4
        assert np.array_equal(a.tokens(0), b.tokens(0))
        st = a.stats(), b.stats()
        assert st[0]["kv_bytes"] == st[1]["kv_bytes"] and st[0]["flops"] == st[1]["flops"]
        ka, kb = a.read_kv(1, 0, 0, 0, 3, 40), b.read_kv(1, 0, 0, 0, 3, 40)
        assert np.abs(ka - kb).max() <= 1e-4 and np.abs(ka).max() > 0
        assert np.array_equal(kb, b.read_kv_noalloc(1, 0, 0, 0, 3, 40))
        assert (b.read_kv(1, 0, 1, 0, 64, 60) == 0).all()              # behind the reserved pages


def test_sequences_share_a_pool_smaller_than_batch_times_context():
    """Four requests through a pool that holds two at a time: release, reuse, the lone run's tokens."""
    shape = rd_inputs.TWIN
    _, w = make_oracle(shape, seed=4, gain_jitter=0.0, max_ctx=64, bf16=True, contract=True)
    gm = gpu_model(shape, w, bf16=True)
    prompts = [rd_inputs.make_prompt(L, shape["vocab"], seed=20 + i) for i, L in enumerate((70, 33, 90, 51))]
    kw = dict(max_context=256, max_window=8, max_new_tokens=12, seed=5)

    def alone(p):
        s = rd.Session(gm, batch=2, page_size=16, n_pages=7, **kw)
        s.prefill(0, p, 2)
        while not s.committed(0)[1]:
            s.df_step(8, 1, 0.0)
        return s.tokens(0)

    want = [alone(p) for p in prompts]
    s = rd.Session(gm, batch=2, page_size=16, n_pages=10, **kw)         # 6 + 3 pages, then 7 + 4 do not fit together
    s.prefill(0, prompts[0], 2)
    s.prefill(1, prompts[1], 2)
    while not (s.committed(0)[1] and s.committed(1)[1]):
        s.df_step(8, 1, 0.0)
    got = [s.tokens(0), s.tokens(1)]
    with pytest.raises(rd.RdError) as err:
        s.prefill(1, np.zeros(200, dtype=np.int32), 2)                   # needs 14 pages: nothing changes
    assert err.value.code == rd.RD_E_CAPACITY and np.array_equal(s.tokens(1), got[1])
    s.release(0)
    s.prefill(1, prompts[2], 2)
    with pytest.raises(rd.RdError) as err:
        s.prefill(0, prompts[3], 2)                                      # 7 held + 4 > 10
    assert err.value.code == rd.RD_E_CAPACITY
    while not s.committed(1)[1]:
        s.df_step(8, 1, 0.0)
    got.append(s.tokens(1))
    s.release(1)
    s.prefill_sliced(0, prompts[3], 2)
    with pytest.raises(rd.RdError) as err:
        s.release(0)
    assert err.value.code == rd.RD_E_STATE
    while s.prefill_pending() or not s.committed(0)[1]:
        s.df_step(8, 1, 0.0)
    got.append(s.tokens(0))
    for i, (a, b) in enumerate(zip(got, want)):
        if i == 1:
            continue      # sequence index 1: its initial states are keyed by the index, no lone run of it here
        assert np.array_equal(a[:len(prompts[i])], b[:len(prompts[i])])
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[3], want[3])   # both ran as sequence 0
    s.release(0)
    with pytest.raises(rd.RdError) as err:
        s.read_kv(1, 0, 0, 0, 0, 4)
    assert err.value.code == rd.RD_E_STATE
    with pytest.raises(rd.RdError) as err:
        s.df_step(8, 1, 0.0)                                             # nothing is running
    assert err.value.code == rd.RD_E_STATE


def test_counters_follow_the_window():
    shape = rd_inputs.TINY
    _, w = make_oracle(shape, seed=1, gain_jitter=0.0, max_ctx=128)
    gm = gpu_model(shape, w)
    s = rd.Session(gm, batch=1, max_context=128, max_window=1, max_new_tokens=3, page_size=16, n_pages=8, attn_window=8, attn_sinks=3)
    s.prefill(0, rd_inputs.make_prompt(50, shape["vocab"], seed=2), 2)
    for _ in range(3):
        s.ar_step(2)
    c, st = gm.cfg, s.stats()
    passes = c.n_prelude + 2 * c.n_core + c.n_coda
    assert st["kv_bytes"] == 3 * passes * (8 + 3 + 1) * 2 * c.hidden * 4     # 11 rows read, one written, per layer and pass


def test_sessions_that_are_refused():
    shape = rd_inputs.TINY
    _, w = make_oracle(shape, seed=1, gain_jitter=0.0, max_ctx=128)
    gm = gpu_model(shape, w)
    kw = dict(batch=2, max_context=64, max_window=4, max_new_tokens=4)
    for bad in (dict(page_size=17, n_pages=4), dict(page_size=8, n_pages=4), dict(page_size=16, n_pages=0), dict(page_size=16, n_pages=4, attn_window=-1),
                dict(page_size=16, n_pages=4, attn_sinks=-1), dict(page_size=16, n_pages=4, latent_slots=3), dict(page_size=0, n_pages=4)):
        with pytest.raises(rd.RdError) as err:
            rd.Session(gm, **(kw | bad))
        assert err.value.code == rd.RD_E_INVALID_ARG
    s = rd.Session(gm, page_size=16, n_pages=4, **kw)
    for call in (lambda: s.set_attention_path(0), lambda: rd.Session(gm, **kw).release(0)):
        with pytest.raises(rd.RdError) as err:
            call()
        assert err.value.code == rd.RD_E_STATE
    with pytest.raises(rd.RdError) as err:
        s.release(2)
    assert err.value.code == rd.RD_E_INVALID_ARG
