"""Pins of the oracle's attention window (config fields attn_window, attn_sinks)."""
import numpy as np
import pytest

import rd_inputs
from helpers import MICRO, SMALL, make_oracle


def _run(n, seed=0, **kw):
    m, _ = make_oracle(SMALL, seed=seed, std=0.1, max_ctx=64, **kw)
    caches = m.new_caches()
    e = m.prelude(rd_inputs.make_prompt(n, SMALL["vocab"], seed=1), np.arange(n), caches)
    return e, caches


def test_a_window_nobody_has_reached_changes_nothing():
    full, _ = _run(20)
    for w, s in ((20, 0), (21, 3), (1000, 0)):
        assert np.array_equal(full, _run(20, attn_window=w, attn_sinks=s)[0])


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (3, 2), (5, 30), (4, 1)])
def test_window_and_sinks_against_a_masked_softmax(window, sinks):
    n = 17
    m, w = make_oracle(MICRO, seed=3, std=0.2, max_ctx=64, attn_window=window, attn_sinks=sinks)
    c = m.cfg
    rng = np.random.default_rng(5)
    x = rng.standard_normal((n, c.hidden))
    cache = m.new_caches()["prelude"]
    got = m.layer("prelude", 0, x, np.arange(n), cache)
    # the attention again, all rows at once under an additive mask
    full, _ = make_oracle(MICRO, seed=3, std=0.2, max_ctx=64)
    plain = full.layer("prelude", 0, x, np.arange(n), full.new_caches()["prelude"])
    p, j = np.arange(n)[:, None], np.arange(n)[None]
    mask = (j <= p) & ((j >= p - window + 1) | (j < sinks))
    K, V = cache.K[0, :n], cache.V[0, :n]
    a = x / np.sqrt((x * x).mean(1, keepdims=True) + c.norm_eps) * m.w["prelude.0.g1"]
    q = (a @ m.w["prelude.0.wq"].T).reshape(n, c.n_heads, c.head_dim)
    z = (q[..., 0::2] + 1j * q[..., 1::2]) * np.exp(1j * np.arange(n)[:, None, None] * c.rope_base ** (-np.arange(0, c.head_dim, 2) / c.head_dim))
    q = np.stack([z.real, z.imag], -1).reshape(q.shape)
    s = np.einsum("phd,jhd->hpj", q, K) / np.sqrt(c.head_dim) + np.where(mask, 0.0, -np.inf)[None]
    e = np.exp(s - s.max(-1, keepdims=True))
    o = np.einsum("hpj,jhd->phd", e / e.sum(-1, keepdims=True), V).reshape(n, -1)
    h = x + o @ m.w["prelude.0.wo"].T
    g2 = h / np.sqrt((h * h).mean(1, keepdims=True) + c.norm_eps) * m.w["prelude.0.g2"]
    gate = g2 @ m.w["prelude.0.wg"].T
    want = h + (gate / (1 + np.exp(-gate)) * (g2 @ m.w["prelude.0.wu"].T)) @ m.w["prelude.0.wd"].T
    assert np.abs(got - want).max() < 1e-5          # the oracle's rotary tables are float32
    if sinks < n - window:
        assert np.abs(got - plain).max() > 1e-6     # and the window is felt
