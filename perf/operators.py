"""Cases for the operators of the paged K/V cache: what a serving step asks of them.

    append   rotary embedding of the new rows' q and k at their positions, K and V written into their pages
    attend   attention of the new rows over the pages of their sequences: causal, grouped heads, rows of many
             sequences in one call; `window` > 0 limits a row to the newest `window` positions and the first `sinks`
    step     both, one after the other, as a layer runs them (the attention's log-sum-exp is not asked for)

A case holds the sizes; ragged lengths follow from its `mix` number, so that work() needs no inputs.  A group is one
sequence's rows of the call: `rows` new rows behind `before` positions that are in the cache already.  `pad` rows at
the end of the call belong to no sequence (position -1) and stay as they are.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
FILL = 0.25                 # what the outputs' padding rows hold before and after
ROPE_BASE = 10000.0


def _case(name, op, dtype, heads, kv_heads, dim, page, groups, rows, before, window=0, sinks=0, pad=0, mix=0, big=0):
    """rows and before are ranges (low, high) drawn per group from `mix`; big > 0: the first group has that many rows."""
    return {"name": name, "op": op, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "groups": groups, "rows_lo": rows[0], "rows_hi": rows[1], "before_lo": before[0], "before_hi": before[1],
            "window": window, "sinks": sinks, "pad": pad, "mix": mix, "big": big}


def listed():
    return [
        # the sequential decoder's token behind a 512-token prompt, 3.5B shape (55 heads of 96): the smallest call
        _case("attend_one_token", "attend", "bf16", 55, 55, 96, 64, 1, (1, 1), (543, 543)),
        # one wavefront of 32 rows behind the same prompt
        _case("attend_wave_32", "attend", "bf16", 55, 55, 96, 64, 1, (32, 32), (511, 511)),
        # four wavefronts behind long prompts, 3.5B shape
        _case("attend_waves_4x32_8k", "attend", "bf16", 55, 55, 96, 128, 4, (32, 32), (8192, 8300), mix=3),
        # a decode batch of a grouped-head model, very ragged, small pages, three padding rows
        _case("attend_tokens_ragged", "attend", "bf16", 32, 8, 128, 16, 64, (1, 1), (16, 16384), pad=3, mix=1),
        # one token behind a very long context: the long axis has to be split
        _case("attend_one_token_131k", "attend", "bf16", 32, 8, 128, 64, 1, (1, 1), (131071, 131071)),
        # a whole prompt at once
        _case("attend_prompt_8k", "attend", "bf16", 32, 8, 128, 64, 1, (8192, 8192), (0, 0)),
        # a slice of a prompt admitted next to running sequences
        _case("attend_slice_and_tokens", "attend", "bf16", 32, 8, 128, 32, 25, (1, 1), (100, 9000), mix=2, big=509),
        # decoding far past the window: only window + sinks are visible
        _case("window_tokens", "attend", "bf16", 32, 8, 128, 64, 48, (1, 1), (5000, 65000), window=4096, sinks=4, mix=4),
        # two prompts under a short window
        _case("window_prompts", "attend", "bf16", 32, 4, 64, 32, 2, (5500, 6500), (0, 1000), window=1024, sinks=16, mix=5),
        # the new tokens of a decode batch into their pages
        _case("append_tokens", "append", "bf16", 32, 8, 128, 16, 64, (1, 1), (16, 16384), mix=1),
        # the rows of a few prompts, ragged
        _case("append_prompts", "append", "bf16", 32, 8, 128, 64, 3, (2500, 2900), (0, 700), pad=5, mix=6),
        # a float32 layer of a small model: append, then attend
        _case("step_f32_waves", "step", "f32", 16, 4, 64, 16, 4, (20, 28), (500, 2000), mix=7),
    ]


def _lengths(case):
    """(rows, positions before them) of every group."""
    rng = random.Random(1000003 * case["mix"] + case["groups"])
    out = []
    for i in range(case["groups"]):
        n = rng.randint(case["rows_lo"], case["rows_hi"])
        lo, hi = case["before_lo"], case["before_hi"]
        b = lo if hi <= lo else int(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1)))) - 1 if lo * 8 < hi else rng.randint(lo, hi)
        out.append((case["big"] if case["big"] and i == 0 else n, max(lo, min(hi, b))))
    return out


def _visible(case, p):
    """Number of keys the row at position p sees."""
    w, s = case["window"], case["sinks"]
    if not w or p < w:
        return p + 1
    return w + min(s, p + 1 - w)


def _keys_read(case, n, b):
    """Keys of a group that at least one of its rows (positions b .. b+n-1) sees."""
    w, s = case["window"], case["sinks"]
    lo = max(0, b - w + 1) if w else 0
    return b + n - lo + min(s if w else 0, lo)


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    groups = _lengths(case)
    rows = sum(n for n, _ in groups)
    nbytes = flops = 0
    if case["op"] in ("append", "step"):
        nbytes += rows * (2 * H + 4 * G) * D * es + 4 * rows
        flops += rows * (H + G) * D * 3
    if case["op"] in ("attend", "step"):
        nbytes += rows * 2 * H * D * es + rows * H * 4 + 4 * rows
        for n, b in groups:
            nbytes += 2 * G * D * es * _keys_read(case, n, b)
            seen = sum(_visible(case, p) for p in range(b, b + n))
            flops += 4 * H * D * seen
    return {"bytes": nbytes, "flops": flops}


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    top = [work(c) for c in listed()]
    top_bytes, top_flops = max(w["bytes"] for w in top), max(w["flops"] for w in top)
    while True:
        op = rng.choice(["attend", "attend", "attend", "append", "step"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kv = rng.choice([1, 2, 3, 4, 5, 8, 16])
        heads = kv * rng.choice([1, 1, 2, 3, 4, 5, 6, 7, 8, 16])
        dim = rng.choice([64, 96, 128])
        page = rng.choice([16, 32, 64, 128])
        kind = rng.choice(["tokens", "waves", "prompts", "slice"])
        if heads > 64:
            continue
        if kind == "tokens":
            groups, rows, big = size(1, 128), (1, 1), 0
        elif kind == "waves":
            groups, w = size(1, 24), size(2, 128)
            rows, big = (max(1, w // 2), w), 0
        elif kind == "prompts":
            groups, n = rng.randint(1, 4), size(64, 8192)
            rows, big = (max(1, n - n // 4), n), 0
        else:
            groups, rows, big = size(2, 48), (1, 1), size(33, 1024)
        hi = size(1, 131072 if kind == "tokens" and groups <= 4 else 32768 if kind == "tokens" else 12000)
        before = (rng.choice([0, hi // 3, hi]), hi)
        window = size(1, 8192) if op != "append" and rng.random() < 0.4 else 0
        sinks = rng.choice([0, 1, 4, 33, 128]) if window else 0
        pad = rng.choice([0, 0, 1, 7])
        case = _case("", op, dtype, heads, kv, dim, page, groups, rows, before, window, sinks, pad, rng.randint(0, 10 ** 6), big)
        del case["name"]
        w = work(case)
        if dtype == "f32" and w["flops"] > top_flops / 16:
            continue
        pool = sum((b + n + page) for n, b in _lengths(case)) * kv * dim * 4
        if w["bytes"] <= top_bytes and w["flops"] <= top_flops and pool <= 3 << 30:
            return case


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    H, G, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    groups = _lengths(case)
    rows = sum(n for n, _ in groups)
    total = rows + case["pad"]
    held = [(n + b + page - 1) // page for n, b in groups]
    n_pages = sum(held) + 2
    stride = max(held) + 1

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32).to(dt)

    s = {"case": case, "groups": groups, "rows": rows, "scale": 1.0 / math.sqrt(D)}
    s["q"], s["k"], s["v"] = normal(total, H, D), normal(total, G, D), normal(total, G, D)
    s["k_pages"], s["v_pages"] = normal(1, n_pages, G, page, D), normal(1, n_pages, G, page, D)
    # the pages of the sequences lie anywhere in the pool; unused table entries hold -1
    order = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
    table = np.full((len(groups), stride), -1, dtype=np.int32)
    at = 0
    for g, n in enumerate(held):
        table[g, :n] = order[at:at + n]
        at += n
    pos = np.concatenate([np.arange(b, b + n, dtype=np.int32) for n, b in groups] + [np.full(case["pad"], -1, dtype=np.int32)])
    start = np.concatenate([[0], np.cumsum([n for n, _ in groups])]).astype(np.int32)
    s["table"] = torch.from_numpy(table).to(DEV)
    s["row_pos"] = torch.from_numpy(pos).to(DEV)
    s["group_start"] = torch.from_numpy(start).to(DEV)
    s["q_rot"] = torch.full((total, H, D), FILL, device=DEV, dtype=dt)
    s["out"] = torch.full((total, H, D), FILL, device=DEV, dtype=dt)
    s["lse"] = torch.full((total, H), FILL, device=DEV, dtype=torch.float32)
    if own:
        import paper_2510_14961_b200 as rd
        stream = torch.cuda.current_stream().cuda_stream
        s["cache"] = rd.PagedCache(n_heads=H, n_kv_heads=G, head_dim=D, page_size=page, n_pages=n_pages, n_layers=1,
                                   max_context=max(n + b for n, b in groups), dtype=rd.RD_BF16 if case["dtype"] == "bf16" else rd.RD_F32,
                                   rope_base=ROPE_BASE, k_pages=s["k_pages"], v_pages=s["v_pages"], stream=stream)
        s["batch"] = rd.PagedRows(s["row_pos"], s["table"], group_start=s["group_start"], max_group_rows=max(n for n, _ in groups))
    return s


# ---- plain form ----------------------------------------------------------------------------------------------
def _where(s, real):
    """Page and offset of every row that belongs to a sequence."""
    page = s["case"]["page"]
    counts = s["group_start"][1:] - s["group_start"][:-1]
    seq = torch.repeat_interleave(torch.arange(counts.numel(), device=DEV), counts.long(), output_size=s["rows"])
    return s["table"][seq, torch.div(real, page, rounding_mode="floor")].long(), real % page


def _rotate(x, cos, sin):
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack([x0 * cos - x1 * sin, x0 * sin + x1 * cos], dim=-1).flatten(-2)


def _append(s):
    D, n = s["case"]["dim"], s["rows"]
    dt = s["q"].dtype
    pos = s["row_pos"][:n].long()
    inv = ROPE_BASE ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)
    ang = pos.double()[:, None] * inv                      # angles in 64 bits: far positions lose their fraction in 32
    cos, sin = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    s["q_rot"][:n] = _rotate(s["q"][:n].float(), cos, sin).to(dt)
    pg, off = _where(s, pos)
    s["k_pages"][0][pg, :, off] = _rotate(s["k"][:n].float(), cos, sin).to(dt)
    s["v_pages"][0][pg, :, off] = s["v"][:n]


def _attend(s, q):
    c = s["case"]
    H, G, D, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    rep = H // G
    r0 = 0
    for g, (n, b) in enumerate(s["groups"]):
        # keys at least one row of the group sees
        lo = max(0, b - c["window"] + 1) if c["window"] else 0
        keys = torch.cat([torch.arange(0, min(c["sinks"] if c["window"] else 0, lo), device=DEV), torch.arange(lo, b + n, device=DEV)])
        pg, off = s["table"][g][torch.div(keys, page, rounding_mode="floor")].long(), keys % page
        K = s["k_pages"][0][pg, :, off].float().transpose(0, 1)            # [G, keys, D]
        V = s["v_pages"][0][pg, :, off].float().transpose(0, 1)
        step = max(1, min(n, (1 << 28) // (H * keys.numel())))
        for i in range(0, n, step):
            m = min(step, n - i)
            a = r0 + i
            qq = q[a:a + m].float().reshape(m, G, rep, D).permute(1, 2, 0, 3).reshape(G, rep * m, D)
            sc = torch.matmul(qq, K.transpose(1, 2)).reshape(G, rep, m, -1) * s["scale"]
            p = torch.arange(b + i, b + i + m, device=DEV)[:, None]
            see = keys[None] <= p
            if c["window"]:
                see &= (keys[None] > p - c["window"]) | (keys[None] < c["sinks"])
            sc = sc.masked_fill(~see, float("-inf"))
            mx = sc.amax(-1, keepdim=True)
            e = torch.exp(sc - mx)
            den = e.sum(-1, keepdim=True)
            o = torch.matmul((e / den).reshape(G, rep * m, -1), V).reshape(G, rep, m, D)
            s["out"][a:a + m] = o.permute(2, 0, 1, 3).reshape(m, H, D).to(s["out"].dtype)
            if c["op"] == "attend":
                s["lse"][a:a + m] = (mx + torch.log(den))[..., 0].permute(2, 0, 1).reshape(m, H)
        r0 += n


def run(s):
    c = s["case"]
    if own:
        cache, batch = s["cache"], s["batch"]
        stream = torch.cuda.current_stream().cuda_stream
        q = s["q"]
        if c["op"] != "attend":
            cache.append(batch, q, s["k"], s["v"], s["q_rot"], stream=stream)
            q = s["q_rot"]
        if c["op"] != "append":
            cache.attend(batch, q, s["out"], s["lse"] if c["op"] == "attend" else None, window=c["window"], sinks=c["sinks"], scale=s["scale"], stream=stream)
    else:
        q = s["q"]
        if c["op"] != "attend":
            _append(s)
            q = s["q_rot"]
        if c["op"] != "append":
            _attend(s, q)
    out = {}
    if c["op"] != "attend":
        out.update(q=s["q_rot"], k_pages=s["k_pages"], v_pages=s["v_pages"])
    if c["op"] != "append":
        out.update(out=s["out"])
    if c["op"] == "attend":                    # a layer has no use for it
        out.update(lse=s["lse"])
    return out


def exact(case, seed):
    """The definition in 64 bits, one sequence and one head at a time, from dense copies of its keys."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    H, G, D, page, w, sinks = case["heads"], case["kv_heads"], case["dim"], case["page"], case["window"], case["sinks"]
    total = s["rows"] + case["pad"]
    kp, vp = s["k_pages"], s["v_pages"]
    out = {}
    q64 = s["q"].double()
    if case["op"] != "attend":
        # z -> z e^(i pos theta_j) on the complex numbers z = x[2j] + i x[2j+1]
        kp, vp = kp.double(), vp.double()
        rot = torch.full((total, H, D), FILL, device=DEV, dtype=torch.float64)
        table = s["table"].cpu().tolist()
        theta = torch.exp(-math.log(ROPE_BASE) * torch.arange(D // 2, device=DEV, dtype=torch.float64) * (2.0 / D))
        r0 = 0
        for g, (n, b) in enumerate(s["groups"]):
            turn = torch.polar(torch.ones(n, 1, D // 2, device=DEV, dtype=torch.float64),
                               torch.arange(b, b + n, device=DEV, dtype=torch.float64)[:, None, None] * theta)

            def rope(x):
                z = torch.view_as_complex(x.double().reshape(n, -1, D // 2, 2).contiguous())
                return torch.view_as_real(z * turn).reshape(n, -1, D)

            rot[r0:r0 + n] = rope(s["q"][r0:r0 + n])
            kk = rope(s["k"][r0:r0 + n])
            vv = s["v"][r0:r0 + n].double()
            p = b
            while p < b + n:                                   # one page after the other
                stop = min(b + n, (p // page + 1) * page)
                kp[0, table[g][p // page], :, p % page:p % page + stop - p] = kk[p - b:stop - b].transpose(0, 1)
                vp[0, table[g][p // page], :, p % page:p % page + stop - p] = vv[p - b:stop - b].transpose(0, 1)
                p = stop
            r0 += n
        out.update(q=rot, k_pages=kp, v_pages=vp)
        # what the attention of a step reads is what the cache and the query buffer hold: their type's values
        q64, kp = rot.to(s["q"].dtype).double(), kp.to(s["q"].dtype)
    if case["op"] != "append":
        o = torch.full((total, H, D), FILL, device=DEV, dtype=torch.float64)
        lse = torch.full((total, H), FILL, device=DEV, dtype=torch.float64)
        r0 = 0
        for g, (n, b) in enumerate(s["groups"]):
            pages = s["table"][g, :(n + b + page - 1) // page].long()
            first = max(0, b - w + 1) if w else 0
            # the sequence's pages in order, cut to its length; a window drops what nobody sees
            keep = torch.arange(b + n, device=DEV)
            if first > sinks:
                keep = torch.cat([keep[:sinks], keep[first:]])
            for h in range(G):
                K = kp[0, pages, h].reshape(-1, D)[keep].double()
                V = vp[0, pages, h].reshape(-1, D)[keep].double()
                step = max(1, min(n, (1 << 26) // keep.numel()))
                for i in range(0, n, step):
                    m = min(step, n - i)
                    pos = torch.arange(b + i, b + i + m, device=DEV)
                    hidden = keep[None, :] > pos[:, None]
                    if w:
                        hidden |= (pos[:, None] - keep[None, :] >= w) & (keep[None, :] >= sinks)
                    for hq in range(h * (H // G), (h + 1) * (H // G)):
                        t = (q64[r0 + i:r0 + i + m, hq] @ K.T) / math.sqrt(D)
                        t[hidden] = -math.inf
                        z = torch.logsumexp(t, dim=1)
                        o[r0 + i:r0 + i + m, hq] = torch.exp(t - z[:, None]) @ V
                        lse[r0 + i:r0 + i + m, hq] = z
            r0 += n
        out.update(out=o)
        if case["op"] == "attend":
            out.update(lse=lse)
    return out
