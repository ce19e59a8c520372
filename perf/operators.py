"""Measured cases of the operators around the attention: the norm and rotation of queries and keys
(forward and backward), appending to a paged key/value cache, attention over that cache.

`listed()` names the cases, `draw()` makes more of the same ranges, `prepare()` makes what a program
holds before the call, `run()` is one pass (`own`: by the library's kernels; otherwise in elementary
torch operations), `exact()` the same result in float64, written apart.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # Training, the headline packed buffer: queries and keys are normed per head and rotated on
        # their way from the fused projection to the attention, and their gradients on the way back.
        dict(name="rope_train_32k", kind="rope", tokens=32768, median=1024, start=0, hq=32, hkv=32, d=128,
             dtype="bf16", wdtype="bf16", norm=True, rot=128, interleaved=False, lens_seed=0),
        # The largest step: 128K tokens, 70B-shaped grouped-query heads.
        dict(name="rope_train_gqa_128k", kind="rope", tokens=131072, median=2048, start=0, hq=64, hkv=8, d=128,
             dtype="bf16", wdtype="f32", norm=True, rot=128, interleaved=False, lens_seed=3),
        # A small full-precision step (convergence checks, unit tests of a training loop).
        dict(name="rope_f32_512", kind="rope", tokens=512, median=128, start=0, hq=8, hkv=4, d=64,
             dtype="f32", wdtype="f32", norm=True, rot=64, interleaved=False, lens_seed=1),
        # A device's share of a 2M-token sequence (far positions), rotation alone, over half of the
        # head, in the interleaved order; an odd number of tokens.
        dict(name="rope_share_8191", kind="rope", tokens=8191, median=0, start=1900000, hq=16, hkv=16, d=64,
             dtype="bf16", wdtype="bf16", norm=False, rot=32, interleaved=True, lens_seed=2),
        # Serving, one step of decoding for 32 sequences: the new keys and values go to the cache.
        dict(name="append_decode_32", kind="append", seqs=32, chunk=1, mix="even", past=8192, page=16, hq=64, hkv=8,
             d=128, dtype="bf16", wdtype="bf16", norm=True, rot=128, interleaved=False, layout="token", lens_seed=4),
        # Serving, prompts of up to 1,024 tokens each.
        dict(name="append_prompts_16", kind="append", seqs=16, chunk=1024, mix="even", past=2048, page=64, hq=32,
             hkv=8, d=128, dtype="bf16", wdtype="bf16", norm=False, rot=128, interleaved=False, layout="head",
             lens_seed=5),
        # The smallest call: one token of one float32 sequence.
        dict(name="append_f32_1", kind="append", seqs=1, chunk=1, mix="even", past=300, page=16, hq=8, hkv=8, d=64,
             dtype="f32", wdtype="f32", norm=True, rot=64, interleaved=False, layout="token", lens_seed=6),
        # Decoding: one query of each of 32 sequences over up to 8K cached keys.
        dict(name="paged_decode_32", kind="paged", seqs=32, chunk=1, mix="even", past=8192, page=16, hq=64, hkv=8,
             d=128, dtype="bf16", layout="token", lens_seed=4),
        # A single user: one query over a 16K-token context.
        dict(name="paged_decode_1", kind="paged", seqs=1, chunk=1, mix="even", past=16384, page=32, hq=32, hkv=8,
             d=128, dtype="bf16", layout="head", lens_seed=7),
        # Chunks of new prompt tokens over what is cached of their sequences.
        dict(name="paged_chunk_8", kind="paged", seqs=8, chunk=1024, mix="even", past=16384, page=64, hq=64, hkv=8,
             d=128, dtype="bf16", layout="token", lens_seed=8),
        # A step of continuous batching: a chunk of one prompt among 16 sequences that decode.
        dict(name="paged_mixed_17", kind="paged", seqs=17, chunk=509, mix="one", past=8192, page=16, hq=48, hkv=8,
             d=128, dtype="bf16", layout="token", lens_seed=9),
        # Full precision, 64-wide heads, short ragged prompts.
        dict(name="paged_f32_3", kind="paged", seqs=3, chunk=200, mix="even", past=700, page=16, hq=8, hkv=4, d=64,
             dtype="f32", layout="token", lens_seed=10),
    ]


HEADS = [(8, 8), (32, 32), (64, 8), (48, 8), (16, 16), (12, 4), (7, 7), (40, 8), (32, 4), (16, 2), (32, 8)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "append", "paged", "paged", "paged"])
    hq, hkv = rng.choice(HEADS)
    d = rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16"] * 4 + ["f32"])
    c = dict(kind=kind, hq=hq, hkv=hkv, d=d, dtype=dtype, lens_seed=rng.randrange(100000))
    if kind != "paged":
        c.update(wdtype=rng.choice(["bf16", "f32"]) if dtype == "bf16" else "f32", norm=rng.random() < 0.7,
                 rot=rng.choice([d, d, d // 2, 16]), interleaved=rng.random() < 0.3)
    if kind == "rope":
        tokens = _log_int(rng, 64, 32768)
        c.update(tokens=tokens, median=_log_int(rng, 16, max(32, tokens // 4)) if rng.random() < 0.7 else 0,
                 start=rng.choice([0, _log_int(rng, 1000, 2000000)]))
        return c
    one = rng.random() < 0.5
    seqs = _log_int(rng, 1, 64)
    chunk = 1 if one else _log_int(rng, 2, 1024)
    # (the plain form holds all scores of a padded batch; appending returns the caches)
    most = 3e9 / (seqs * chunk * hq) if kind == "paged" else 5e8 / (seqs * hkv * d)
    past = _log_int(rng, 16, max(32, min(16384, int(most))))
    c.update(seqs=seqs, chunk=chunk, mix=rng.choice(["even", "even", "one"]) if seqs > 1 and not one else "even",
             past=past, page=rng.choice([16, 16, 32, 64, 128, 256]), layout=rng.choice(["token", "token", "head"]))
    return c


# ---------------------------------------------------------------- what a case stands for


def _segments(c):
    """Lengths of the packed sequences of a training buffer (median 0: one share of a long one)."""
    if not c["median"]:
        return [c["tokens"]]
    r = np.random.default_rng([c["lens_seed"], 5])
    lens, left = [], c["tokens"]
    while left > 0:
        n = int(min(left, max(1, round(math.exp(r.normal(math.log(c["median"]), 1.4))))))
        lens.append(n)
        left -= n
    return lens


def _new_and_total(c):
    """New tokens and tokens after them of each sequence of a serving step."""
    r = np.random.default_rng([c["lens_seed"], 7])
    past = np.exp(r.uniform(math.log(max(1, c["past"] // 8)), math.log(c["past"]), c["seqs"])).astype(int)
    if c["mix"] == "one":
        new = np.ones(c["seqs"], int)
        new[r.integers(c["seqs"])] = c["chunk"]
    else:
        new = r.integers(max(1, c["chunk"] // 4), c["chunk"], size=c["seqs"], endpoint=True)
    return [int(x) for x in new], [int(p) + int(x) for p, x in zip(past, new)]


# ---------------------------------------------------------------- inputs


def _rand(seed, tid, shape, dtype, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + tid * 7919)
    x = torch.empty(shape, dtype=dtype, device="cuda")
    flat = x.view(-1)
    for lo in range(0, flat.numel(), 1 << 28):
        hi = min(flat.numel(), lo + (1 << 28))
        flat[lo:hi] = (torch.randn(hi - lo, generator=g, device="cuda") * std + mean).to(dtype)
    return x


def _rotation(c, seed):
    """Frequencies (base 500,000) and the norms' weights."""
    i = torch.arange(0, c["rot"], 2, dtype=torch.float64)
    freq = torch.pow(torch.tensor(500000.0, dtype=torch.float64), -i / c["rot"]).float().cuda()
    wt = DTYPES[c["wdtype"]]
    wq, wk = (_rand(seed, 50 + j, (c["d"],), wt, 0.2, 1.0) if c["norm"] else None for j in (0, 1))
    return dict(freq=freq, wq=wq, wk=wk, eps=1e-6)


def _rope_inputs(c, seed):
    """The projection's output [T, (hq + 2 hkv) d], of which q and k are views, positions that start
    anew with each sequence, the gradients that the attention's backward hands over."""
    t, dt = c["tokens"], DTYPES[c["dtype"]]
    qkv = _rand(seed, 0, (t, (c["hq"] + 2 * c["hkv"]) * c["d"]), dt)
    q = qkv[:, :c["hq"] * c["d"]].view(t, c["hq"], c["d"])
    k = qkv[:, c["hq"] * c["d"]:(c["hq"] + c["hkv"]) * c["d"]].view(t, c["hkv"], c["d"])
    pos = torch.from_numpy(np.concatenate([np.arange(n, dtype=np.int64) + c["start"] for n in _segments(c)])).cuda()
    return dict(q=q, k=k, pos=pos, gq=_rand(seed, 1, (t, c["hq"], c["d"]), dt, 0.1),
                gk=_rand(seed, 2, (t, c["hkv"], c["d"]), dt, 0.1), **_rotation(c, seed))


def _cache(c, seed, total):
    """Pages of the sequences in a shuffled order, a few more than they need; [pages, page, hkv, d]
    in memory ("token") or [pages, hkv, page, d] ("head"), seen in the first order."""
    n = [-(-x // c["page"]) for x in total]
    pages = sum(n) + 3
    shape = (pages, c["page"], c["hkv"], c["d"]) if c["layout"] == "token" else (pages, c["hkv"], c["page"], c["d"])
    kc, vc = (_rand(seed, 10 + j, shape, DTYPES[c["dtype"]]) for j in (0, 1))
    if c["layout"] == "head":
        kc, vc = kc.permute(0, 2, 1, 3), vc.permute(0, 2, 1, 3)
    ids = np.random.default_rng([seed, 11]).permutation(pages).astype(np.int32)
    table = np.full((len(n), max(n) + 1), -1, np.int32)
    for b, m in enumerate(n):
        table[b, :m] = ids[sum(n[:b]):sum(n[:b]) + m]
    return dict(kc=kc, vc=vc, table=torch.from_numpy(table).cuda(),
                lens=torch.from_numpy(np.asarray(total, np.int32)).cuda())


def _serve_inputs(c, seed):
    new, total = _new_and_total(c)
    t, dt = sum(new), DTYPES[c["dtype"]]
    s = _cache(c, seed, total)
    s["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    s.update(t=t, most_new=max(new), most=max(total))
    if c["kind"] == "paged":
        s["q"] = _rand(seed, 0, (t, c["hq"], c["d"]), dt)
        return s
    qkv = _rand(seed, 0, (t, (c["hq"] + 2 * c["hkv"]) * c["d"]), dt)
    a, b = c["hq"] * c["d"], (c["hq"] + c["hkv"]) * c["d"]
    s.update(q=qkv[:, :a].view(t, c["hq"], c["d"]), k=qkv[:, a:b].view(t, c["hkv"], c["d"]),
             v=qkv[:, b:].view(t, c["hkv"], c["d"]), **_rotation(c, seed))
    return s


def prepare(case, seed):
    c, kind = case, case["kind"]
    s = _rope_inputs(c, seed) if kind == "rope" else _serve_inputs(c, seed)
    s["case"] = c
    # what a program keeps between steps: outputs, and the handles and workspaces of the library
    if kind == "rope":
        dqkv = torch.zeros(c["tokens"], (c["hq"] + 2 * c["hkv"]) * c["d"], dtype=s["q"].dtype, device="cuda")
        a, b = c["hq"] * c["d"], (c["hq"] + c["hkv"]) * c["d"]
        s.update(qo=torch.empty_like(s["gq"]), ko=torch.empty_like(s["gk"]),
                 dq=dqkv[:, :a].view(s["gq"].shape), dk=dqkv[:, a:b].view(s["gk"].shape))
    else:
        s["out"] = torch.empty(s["t"], c["hq"], c["d"], dtype=s["q"].dtype, device="cuda")
        if kind == "paged":
            s["lse"] = torch.empty(c["hq"], s["t"], dtype=torch.float32, device="cuda")
    if own:
        from paper_2502_21231_amd import bs_qkv as Q
        if kind != "paged":
            s["params"] = Q.make_qk_params(s["freq"], c["interleaved"], s["wq"], s["wk"], s["eps"])
        if kind == "rope":
            s["ws"] = Q.alloc_qk_workspace(s["q"], s["k"])
        else:
            s["cache"] = Q.make_paged_cache(s["kc"], s["vc"], s["table"], s["lens"])
        if kind == "paged":
            s["ws"] = Q.alloc_paged_workspace(s["q"], s["cache"], s["most"])
    return s


# ---------------------------------------------------------------- one pass


def _angles(pos, freq):
    a = pos.double()[:, None] * freq.double()
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _turn(x, cos, sin, inter):
    """Rotates the first 2 cos.shape[-1] elements of each head by the angles (sin negated: back)."""
    r = 2 * cos.shape[-1]
    rest = x[..., r:]
    if inter:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, rest], -1)


def _norm_turn(x, w, eps, cos, sin, inter):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w.float()
    return _turn(x, cos, sin, inter)


def _norm_turn_back(x, g, w, eps, cos, sin, inter):
    """Gradients of x and w from that of _norm_turn's result."""
    g = _turn(g.float(), cos, -sin, inter)
    if w is None:
        return g, None
    x = x.float()
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
    xh = x * rstd
    dw = (g * xh).sum((0, 1), dtype=torch.float64).float()
    g = g * w.float()
    return rstd * (g - xh * (g * xh).mean(-1, keepdim=True)), dw


def _tokens(s):
    """Sequence and place in it of each new token, and its position."""
    at = torch.arange(s["t"], device="cuda")
    b = torch.bucketize(at, s["cu"][1:].long(), right=True)
    i = at - s["cu"].long()[b]
    lens = s["lens"].long()
    new = (s["cu"][1:] - s["cu"][:-1]).long()
    return b, i, (lens - new)[b] + i, new, lens


def _attend(s, c):
    page, group, n = c["page"], c["hq"] // c["hkv"], c["seqs"]
    b, i, _, new, lens = _tokens(s)
    j = torch.arange(s["most"], device="cuda")
    slot = s["table"].long()[:, j // page].clamp(min=0)  # [seqs, keys]: page, then place in it
    kk = s["kc"][slot, j % page].float().permute(0, 2, 3, 1).contiguous()  # [seqs, hkv, d, keys]
    vv = s["vc"][slot, j % page].float().transpose(1, 2).contiguous()
    rows = torch.arange(s["most_new"], device="cuda")
    at = (s["cu"][:-1].long()[:, None] + rows).clamp(max=s["t"] - 1)
    qq = s["q"].float()[at].view(n, s["most_new"], c["hkv"], group, c["d"]).transpose(1, 2)
    sc = torch.matmul(qq.reshape(n, c["hkv"], -1, c["d"]), kk).view(n, c["hkv"], s["most_new"], group, -1)
    sc = sc * (1.0 / math.sqrt(c["d"]))
    seen = j[None, None] <= (rows[None, :] + (lens - new)[:, None])[:, :, None]
    sc = sc.masked_fill(~seen[:, None, :, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = (sc - top.clamp(min=-1e30)).exp()
    tot = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, c["hkv"], -1, s["most"]), vv).view(n, c["hkv"], s["most_new"], group, c["d"])
    o = o / tot.clamp(min=1e-30)
    lse = top + tot.log()
    out = o.permute(0, 2, 1, 3, 4)[b, i].reshape(s["t"], c["hq"], c["d"])
    lse = lse[..., 0].permute(0, 2, 1, 3)[b, i].reshape(s["t"], c["hq"]).t()
    s["out"].copy_(out)
    s["lse"].copy_(lse)


def run(state):
    s, c = state, state["case"]
    kind, inter = c["kind"], c["interleaved"] if c["kind"] != "paged" else False
    if own:
        from paper_2502_21231_amd import bs_qkv as Q
        if kind == "rope":
            Q.bs_qk_norm_rope_fwd(s["q"], s["k"], s["pos"], s["params"], s["qo"], s["ko"])
            _, _, dwq, dwk = Q.bs_qk_norm_rope_bwd(s["q"], s["k"], s["pos"], s["params"], s["gq"], s["gk"],
                                                   dq=s["dq"], dk=s["dk"], workspace=s["ws"])
            r = dict(q=s["qo"], k=s["ko"], dq=s["dq"], dk=s["dk"])
            return dict(r, dwq=dwq, dwk=dwk) if c["norm"] else r
        if kind == "append":
            Q.bs_kv_append(s["q"], s["k"], s["v"], s["cache"], s["cu"], s["params"], q_out=s["out"])
            return dict(q=s["out"], kc=s["kc"], vc=s["vc"])
        Q.bs_attn_paged_fwd(s["q"], s["cache"], s["cu"], s["most"], out=s["out"], lse=s["lse"], workspace=s["ws"])
        return dict(out=s["out"], lse=s["lse"])
    if kind == "paged":
        _attend(s, c)
        return dict(out=s["out"], lse=s["lse"])
    if kind == "append":
        b, i, at, _, _ = _tokens(s)
        cos, sin = _angles(at, s["freq"])
        s["out"].copy_(_norm_turn(s["q"], s["wq"], s["eps"], cos, sin, inter))
        slot = s["table"].long()[b, at // c["page"]]
        s["kc"][slot, at % c["page"]] = _norm_turn(s["k"], s["wk"], s["eps"], cos, sin, inter).to(s["k"].dtype)
        s["vc"][slot, at % c["page"]] = s["v"]
        return dict(q=s["out"], kc=s["kc"], vc=s["vc"])
    cos, sin = _angles(s["pos"], s["freq"])
    s["qo"].copy_(_norm_turn(s["q"], s["wq"], s["eps"], cos, sin, inter))
    s["ko"].copy_(_norm_turn(s["k"], s["wk"], s["eps"], cos, sin, inter))
    dq, dwq = _norm_turn_back(s["q"], s["gq"], s["wq"], s["eps"], cos, sin, inter)
    s["dq"].copy_(dq)
    dk, dwk = _norm_turn_back(s["k"], s["gk"], s["wk"], s["eps"], cos, sin, inter)
    s["dk"].copy_(dk)
    r = dict(q=s["qo"], k=s["ko"], dq=s["dq"], dk=s["dk"])
    return dict(r, dwq=dwq, dwk=dwk) if c["norm"] else r


# ---------------------------------------------------------------- work


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    heads = c["hq"] + c["hkv"]
    if c["kind"] == "rope":
        # forward: q and k read and written; backward: their gradients read and written, with norms
        # q and k read again; about 10 operations per element forward and 25 backward
        n = c["tokens"] * heads * c["d"]
        return dict(bytes=n * es * (5 if c["norm"] else 4) + 8 * c["tokens"], flops=35 * n)
    new, total = _new_and_total(c)
    t = sum(new)
    if c["kind"] == "append":
        return dict(bytes=2 * t * (heads + c["hkv"]) * c["d"] * es + 4 * sum(-(-x // c["page"]) for x in new),
                    flops=10 * t * heads * c["d"])
    pairs = sum(n * (x - n) + n * (n + 1) // 2 for n, x in zip(new, total))
    return dict(bytes=2 * t * c["hq"] * c["d"] * es + 4 * t * c["hq"] + 2 * sum(total) * c["hkv"] * c["d"] * es
                + 4 * sum(-(-x // c["page"]) for x in total), flops=4 * c["d"] * c["hq"] * pairs)


# ---------------------------------------------------------------- float64


def _by_matrix(x, w, eps, pos, freq, inter):
    """The norm and rotation of x [T, heads, d] in float64, as complex numbers of modulus one."""
    y = x
    if w is not None:
        y = y / (y.pow(2).sum(-1, keepdim=True) / y.shape[-1] + eps).sqrt() * w.double()
    r = 2 * freq.numel()
    z = torch.polar(torch.ones(pos.numel(), r // 2, dtype=torch.float64, device="cuda"),
                    torch.outer(pos.double(), freq.double()))[:, None]
    even, odd = (slice(0, r, 2), slice(1, r, 2)) if inter else (slice(0, r // 2), slice(r // 2, r))
    turned = torch.complex(y[..., even], y[..., odd]) * z
    out = y.clone()
    out[..., even] = turned.real
    out[..., odd] = turned.imag
    return out


def exact(case, seed):
    c, kind = case, case["kind"]
    if kind == "rope":
        s = _rope_inputs(c, seed)
        got = {}
        for name, x, w, g in (("q", s["q"], s["wq"], s["gq"]), ("k", s["k"], s["wk"], s["gk"])):
            outs, grads = [], []
            ww = w.double().requires_grad_() if w is not None else None
            dw = 0
            for lo in range(0, c["tokens"], 2048):
                at = slice(lo, lo + 2048)
                xx = x[at].double().requires_grad_()
                y = _by_matrix(xx, ww, s["eps"], s["pos"][at], s["freq"], c["interleaved"])
                d = torch.autograd.grad(y, [xx] + ([ww] if w is not None else []), g[at].double())
                outs.append(y.detach())
                grads.append(d[0])
                dw = dw + d[1] if w is not None else 0
            got[name], got["d" + name] = torch.cat(outs), torch.cat(grads)
            if w is not None:
                got["dw" + name] = dw
        return got
    s = _serve_inputs(c, seed)
    new, total = _new_and_total(c)
    table = s["table"].cpu().numpy()
    starts = np.concatenate([[0], np.cumsum(new)])
    place = lambda b, n: (torch.from_numpy(table[b, np.arange(n) // c["page"]]).long().cuda(),  # noqa: E731
                          torch.from_numpy(np.arange(n) % c["page"]).cuda())
    if kind == "append":
        kc, vc = s["kc"].double(), s["vc"].double()
        q = torch.empty(s["t"], c["hq"], c["d"], dtype=torch.float64, device="cuda")
        for b, (n, x) in enumerate(zip(new, total)):
            at = slice(int(starts[b]), int(starts[b]) + n)
            pos = torch.arange(x - n, x, device="cuda")
            p, o = place(b, x)
            q[at] = _by_matrix(s["q"][at].double(), s["wq"], s["eps"], pos, s["freq"], c["interleaved"])
            kc[p[x - n:], o[x - n:]] = _by_matrix(s["k"][at].double(), s["wk"], s["eps"], pos, s["freq"],
                                                  c["interleaved"])
            vc[p[x - n:], o[x - n:]] = s["v"][at].double()
        return dict(q=q, kc=kc, vc=vc)
    out = torch.empty(s["t"], c["hq"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.empty(c["hq"], s["t"], dtype=torch.float64, device="cuda")
    for b, (n, x) in enumerate(zip(new, total)):
        p, o = place(b, x)
        kk, vv = s["kc"][p, o].double(), s["vc"][p, o].double()
        for lo in range(0, n, 512):
            m = min(512, n - lo)
            at = slice(int(starts[b]) + lo, int(starts[b]) + lo + m)
            hidden = torch.arange(x, device="cuda")[None] > torch.arange(x - n + lo, x - n + lo + m, device="cuda")[:, None]
            for h in range(c["hq"]):
                kv = h // (c["hq"] // c["hkv"])
                z = (s["q"][at, h].double() @ kk[:, kv].t() / math.sqrt(c["d"])).masked_fill(hidden, -math.inf)
                lse[h, at] = torch.logsumexp(z, 1)
                out[at, h] = torch.softmax(z, 1) @ vv[:, kv]
    return dict(out=out, lse=lse)
