"""Norm and rotation of queries and keys, and appending to a paged cache, against the float64 oracle.

Tolerances (u = 2^-24, fp32 half step).  Forward: the sum of squares of 128 elements in a tree over 16
partial sums of 8 is within 12 u, its root and reciprocal within 8 u, three products, the rotation's two
products and a sum 3 u, cos and sin within 4e-7 (float32 part of a turn) and the far angles' 1e-6 at 2^31
only: 4e-6 of |a| + |b|, which 1.5 times the row's largest element bounds (rotated pairs: sqrt 2).
Backward: two such sums and five products more, 6e-6 of the terms' magnitude.  A bf16 result is off by half
a bf16 step more.  Weight gradients: a chain of n additions is within n u of the sum of magnitudes; the
terms themselves within 64 u."""
import numpy as np
import pytest
import torch

from oracle import qkv as O
from paper_2502_21231_amd import bs_qkv as Q
from tests.parity_util import f64, half_ulp_bf16

pytestmark = pytest.mark.gpu


def rand(seed, tid, shape, dtype, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed * 1009 + tid)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype)


def close(name, got, want, tol, bf16):
    got, want = f64(got), np.asarray(want)
    assert got.shape == want.shape and np.all(np.isfinite(got)), name
    bound = tol + (half_ulp_bf16(want) if bf16 else 0.0)
    over = np.abs(got - want) - bound
    i = np.unravel_index(np.argmax(over), over.shape)
    assert over[i] <= 0, f"{name}: {got[i]} for {want[i]} at {i}, bound {np.broadcast_to(bound, got.shape)[i]}"


def freqs(rot, base=500000.0):
    return torch.from_numpy((base ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)) if rot else None


# tokens, hq, hkv, d, dtype, weights' dtype (None: no norm; "k": keys only), rot, interleaved, first position
CASES = [
    (37, 8, 2, 128, torch.bfloat16, torch.bfloat16, 128, False, 0),
    (37, 8, 2, 128, torch.bfloat16, torch.float32, 128, True, 1999000),
    (1, 1, 1, 64, torch.float32, torch.float32, 64, False, 2147480000),
    (5, 7, 7, 64, torch.bfloat16, None, 32, True, 12345),
    (5, 12, 4, 128, torch.float32, None, 16, False, -3),
    (130, 3, 1, 128, torch.bfloat16, torch.bfloat16, 0, False, 0),
    (2500, 2, 2, 64, torch.float32, torch.bfloat16, 48, False, 7),
    (3, 40, 8, 128, torch.bfloat16, "k", 112, False, 500),
    (1, 512, 8, 64, torch.bfloat16, torch.float32, 64, True, 1 << 20),
    # several tokens per workgroup, the last one short of them; outputs that are larger than the caches
    (8195, 2, 1, 64, torch.bfloat16, torch.bfloat16, 64, False, 0),
    (4101, 3, 1, 128, torch.float32, torch.float32, 128, True, 3),
    (14001, 8, 2, 128, torch.bfloat16, torch.float32, 96, False, 5),
]


def rope_case(case, seed=0, fused=True):
    T, hq, hkv, d, dt, wdt, rot, inter, start = case
    if fused:  # q and k as parts of a projection's output
        qkv = rand(seed, 0, (T, (hq + 2 * hkv) * d), dt, 2.0)
        q, k = qkv[:, :hq * d].reshape(T, hq, d), qkv[:, hq * d:(hq + hkv) * d].reshape(T, hkv, d)
        buf = qkv.cuda()
        qg, kg = buf[:, :hq * d].view(T, hq, d), buf[:, hq * d:(hq + hkv) * d].view(T, hkv, d)
    else:
        q, k = rand(seed, 0, (T, hq, d), dt), rand(seed, 1, (T, hkv, d), dt)
        qg, kg = q.cuda(), k.cuda()
    wq = rand(seed, 3, (d,), wdt, 0.3, 1.0) if wdt not in (None, "k") else None
    wk = rand(seed, 4, (d,), torch.float32 if wdt == "k" else wdt, 0.3, 1.0) if wdt is not None else None
    f = freqs(rot)
    pos = torch.arange(T, dtype=torch.int64) * 3 % 1000 + start
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    par = Q.make_qk_params(dev(f), inter, dev(wq), dev(wk), 1e-5)
    return q, k, qg, kg, wq, wk, f, pos, par


def ref(x, w, f, pos, inter):
    return O.norm_rope(f64(x), None if w is None else f64(w), float(np.float32(1e-5)), pos.numpy(), None if f is None else f64(f), inter)


@pytest.mark.parametrize("case", CASES)
def test_forward(gpu, case):
    q, k, qg, kg, wq, wk, f, pos, par = rope_case(case)
    qo, ko = Q.bs_qk_norm_rope_fwd(qg, kg, pos.cuda(), par)
    bf = case[4] is torch.bfloat16
    for name, got, x, w in (("q", qo, q, wq), ("k", ko, k, wk)):
        want = ref(x, w, f, pos, case[7])
        close(name, got, want, 6e-6 * np.abs(want).max(-1, keepdims=True), bf)


@pytest.mark.parametrize("case", CASES)
def test_backward(gpu, case):
    T, hq, hkv, d, dt, wdt, rot, inter, start = case
    q, k, qg, kg, wq, wk, f, pos, par = rope_case(case)
    gq, gk = rand(1, 0, (T, hq, d), dt, 0.1), rand(1, 1, (T, hkv, d), dt, 0.1)
    buf = torch.full((T, (hq + hkv) * d + 64), 5.0, dtype=dt, device=gpu)
    dq, dk = buf[:, :hq * d].view(T, hq, d), buf[:, hq * d:(hq + hkv) * d].view(T, hkv, d)
    _, _, dwq, dwk = Q.bs_qk_norm_rope_bwd(qg, kg, pos.cuda(), par, gq.cuda(), gk.cuda(), dq=dq, dk=dk)
    again = Q.bs_qk_norm_rope_bwd(qg, kg, pos.cuda(), par, gq.cuda(), gk.cuda())
    assert torch.equal(dq, again[0]) and torch.equal(dk, again[1])
    assert torch.all(buf[:, (hq + hkv) * d:] == 5.0)
    for name, got, dw, dw2, x, w, g, n in (("q", dq, dwq, again[2], q, wq, gq, hq), ("k", dk, dwk, again[3], k, wk, gk, hkv)):
        dx, dwr, size, mags = O.norm_rope_bwd(f64(x), None if w is None else f64(w), float(np.float32(1e-5)), pos.numpy(),
                                              None if f is None else f64(f), inter, f64(g))
        close("d" + name, got, dx, 6e-6 * size * 1.5, dt is torch.bfloat16)
        if w is None:
            assert dw is None
        else:
            assert torch.equal(dw, dw2)
            chain = -(-T // 256) * -(-n // 16) + 256 + 64
            assert np.all(np.abs(f64(dw) - dwr) <= chain * 2.0 ** -24 * mags)


def test_gradient_against_differences(gpu):
    """The loss's change over a step of the inputs, by float64 differences of the formula, against the kernel's
    gradients: second-order terms of a step of 1e-4 are below 1e-7, float32 gradients within 1e-6."""
    case = (3, 2, 1, 64, torch.float32, torch.float32, 64, False, 11)
    q, k, qg, kg, wq, wk, f, pos, par = rope_case(case, fused=False)
    gq, gk = rand(1, 0, (3, 2, 64), torch.float32), rand(1, 1, (3, 1, 64), torch.float32)
    dq, dk, dwq, dwk = Q.bs_qk_norm_rope_bwd(qg, kg, pos.cuda(), par, gq.cuda(), gk.cuda())
    for x, w, g, dx, dw in ((q, wq, gq, dq, dwq), (k, wk, gk, dk, dwk)):
        rng = np.random.default_rng(0)
        vx, vw = rng.normal(size=x.shape), rng.normal(size=w.shape)
        at = lambda s: float((O.norm_rope(f64(x) + s * vx, f64(w) + s * vw, float(np.float32(1e-5)), pos.numpy(), f64(f), False)  # noqa: E731
                              * f64(g)).sum())
        step = 1e-5
        want = (at(step) - at(-step)) / (2 * step)
        got = float((f64(dx) * vx).sum() + (f64(dw) * vw).sum())
        size = float((np.abs(f64(dx) * vx)).sum() + np.abs(f64(dw) * vw).sum())
        assert abs(got - want) <= 2e-6 * size


def test_in_place_and_empty(gpu):
    case = CASES[0]
    q, k, qg, kg, wq, wk, f, pos, par = rope_case(case, fused=False)
    qo, ko = Q.bs_qk_norm_rope_fwd(qg, kg, pos.cuda(), par)
    gq, gk = qo.clone(), ko.clone()
    want = Q.bs_qk_norm_rope_bwd(qg, kg, pos.cuda(), par, gq, gk)
    got = Q.bs_qk_norm_rope_bwd(qg, kg, pos.cuda(), par, gq, gk, dq=gq, dk=gk)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    Q.bs_qk_norm_rope_fwd(qg, kg, pos.cuda(), par, qg, kg)
    assert torch.equal(qg, qo) and torch.equal(kg, ko)
    # no tokens: no gradients, zero gradients of the weights
    e = qg[:0], kg[:0], pos[:0].cuda()
    a, b, dwq, dwk = Q.bs_qk_norm_rope_bwd(*e, par, qg[:0], kg[:0])
    assert a.shape[0] == 0 and torch.all(dwq == 0) and torch.all(dwk == 0)


def test_unrotated_rest_keeps_infinities(gpu):
    """Without a norm, elements outside the rotation are copied: an infinity there makes no NaN."""
    x = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    x[:, :, 40] = float("inf")
    x[:, :, 50] = float("nan")
    par = Q.make_qk_params(freqs(32).cuda())
    qo, _ = Q.bs_qk_norm_rope_fwd(x.cuda(), x.cuda(), torch.tensor([1, 2]).cuda(), par)
    # (the rotated zeros may be -0: cos 2 < 0)
    assert torch.equal(qo.cpu()[..., 32:].view(torch.int16), x[..., 32:].view(torch.int16)) and torch.all(qo[..., :32] == 0)


def test_replayed_capture(gpu):
    case = CASES[0]
    q, k, qg, kg, wq, wk, f, pos, par = rope_case(case)
    posg, gq, gk = pos.cuda(), rand(1, 0, q.shape, q.dtype).cuda(), rand(1, 1, k.shape, k.dtype).cuda()
    ws = Q.alloc_qk_workspace(qg, kg)
    out = [torch.empty(q.shape, dtype=q.dtype, device=gpu), torch.empty(k.shape, dtype=k.dtype, device=gpu)]
    grads = [torch.empty_like(out[0]), torch.empty_like(out[1]), torch.empty(128, device=gpu), torch.empty(128, device=gpu)]

    def step():
        Q.bs_qk_norm_rope_fwd(qg, kg, posg, par, *out)
        Q.bs_qk_norm_rope_bwd(qg, kg, posg, par, gq, gk, *grads, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        posg.add_(100)
        gq.mul_(0.5)
        for t in out + grads:
            t.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        a = Q.bs_qk_norm_rope_fwd(qg, kg, posg, par)
        b = Q.bs_qk_norm_rope_bwd(qg, kg, posg, par, gq, gk)
        assert all(torch.equal(x, y) for x, y in zip(out + grads, (*a, *b)))


# ---------------------------------------------------------------- append


def make_cache(seed, lens, page, hkv, d, dtype, head_major=False, spare=2, extra_cols=1):
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    ids = rng.permutation(pages)
    table = np.full((len(lens), max(need, default=0) + extra_cols), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = ids[sum(need[:b]):sum(need[:b]) + n]
    shape = (pages, hkv, page, d) if head_major else (pages, page, hkv, d)
    kc, vc = rand(seed, 20, shape, dtype), rand(seed, 21, shape, dtype)
    if head_major:
        kc, vc = kc.permute(0, 2, 1, 3), vc.permute(0, 2, 1, 3)
    return kc, vc, table


def dup(t):
    """On the GPU with the same strides."""
    g = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
    return g.copy_(t)


# lens (after), new, page, hq, hkv, d, dtype, norm, rot, interleaved, head_major, padding rows
APPENDS = [
    ([33, 16, 1, 700], [1, 1, 1, 1], 16, 8, 2, 128, torch.bfloat16, True, 128, False, False, 0),
    ([40, 17, 5], [23, 17, 0], 16, 8, 8, 64, torch.float32, True, 64, True, True, 3),
    ([0, 300, 2], [1, 290, 3], 64, 4, 2, 128, torch.bfloat16, False, 64, False, True, 2),
    ([4096], [77], 256, 7, 7, 64, torch.bfloat16, False, 0, False, False, 0),
    ([5000, 3201], [4999, 3197], 64, 2, 1, 64, torch.bfloat16, True, 64, False, False, 3),
]


@pytest.mark.parametrize("case", APPENDS)
@pytest.mark.parametrize("with_q", [True, False])
def test_append(gpu, case, with_q):
    lens, new, page, hq, hkv, d, dt, norm, rot, inter, hm, pad = case
    T = sum(new) + pad
    kc, vc, table = make_cache(3, lens, page, hkv, d, dt, hm)
    vc[:] = float("nan")  # what the cache holds is neither read nor changed
    qkv = rand(4, 0, (T, (hq + 2 * hkv) * d), dt)
    a, b = hq * d, (hq + hkv) * d
    q, k, v = qkv[:, :a].reshape(T, hq, d), qkv[:, a:b].reshape(T, hkv, d), qkv[:, b:].reshape(T, hkv, d)
    gb = qkv.cuda()
    qg, kg, vg = gb[:, :a].view(T, hq, d), gb[:, a:b].view(T, hkv, d), gb[:, b:].view(T, hkv, d)
    wq, wk = (rand(5, i, (d,), dt, 0.3, 1.0) if norm else None for i in (0, 1))
    f = freqs(rot)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    par = Q.make_qk_params(dev(f), inter, dev(wq), dev(wk), 1e-5)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    kcg, vcg = dup(kc), dup(vc)
    cache = Q.make_paged_cache(kcg, vcg, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    qo = torch.full((T, hq, d), 3.0, dtype=dt, device=gpu)
    got = Q.bs_kv_append(qg if with_q else None, kg, vg, cache, torch.from_numpy(cu).cuda(), par, q_out=qo)
    torch.cuda.synchronize()
    pos = np.concatenate([np.arange(L - n, L) for L, n in zip(lens, new)] + [np.zeros(pad, np.int64)])
    want = lambda x, w: O.norm_rope(f64(x), None if w is None else f64(w), float(np.float32(1e-5)), pos,  # noqa: E731
                                    None if f is None else f64(f), inter)
    bf, n = dt is torch.bfloat16, sum(new)
    if with_q:
        wantq = want(q, wq)[:n]
        close("q_out", got[:n], wantq, 6e-6 * np.abs(wantq).max(-1, keepdims=True), bf)
        assert torch.all(got[n:] == 3.0)
    else:
        assert got is None and torch.all(qo == 3.0)
    kr = want(k, wk)
    _, _, stored = O.append(kr, f64(v), f64(kc), f64(vc), table, lens, cu)
    kh, vh = kcg.cpu(), vcg.cpu()
    for p, s, r in stored:
        close("k", kh[p, s], kr[r], 6e-6 * np.abs(kr[r]).max(-1, keepdims=True), bf)
        assert torch.equal(vh[p, s], v[r])
        kh[p, s], vh[p, s] = kc[p, s], vc[p, s]
    bits = torch.int16 if bf else torch.int32
    for x, y in ((kh, kc), (vh, vc)):  # nothing else changed
        assert torch.equal(x.contiguous().view(bits), y.contiguous().view(bits))
    assert len(stored) == sum(min(a, b) for a, b in zip(lens, new))


def test_append_with_a_table_that_lies(gpu):
    """Pages that do not exist, lengths beyond the table and before the new tokens, offsets out of order: what
    has no place is not stored, and nothing outside the pages is written."""
    page, hkv, d = 16, 2, 64
    store = torch.full((2, 10, page, hkv, d), 7.0, dtype=torch.bfloat16, device=gpu)  # pages 3 .. 6 are the cache
    kc, vc = store[0, 3:7], store[1, 3:7]
    k = rand(0, 0, (6, hkv, d), torch.bfloat16).cuda()
    lens = torch.tensor([17, 40, 2, -5, 2 ** 31 - 1], dtype=torch.int32).cuda()
    table = torch.tensor([[0, 4], [1, 1], [-1, 2], [0, 0], [3, 3]], dtype=torch.int32).cuda()
    cache = Q.make_paged_cache(kc, vc, table, lens)
    cu = torch.tensor([0, 2, 3, 4, 5, 6], dtype=torch.int32).cuda()
    Q.bs_kv_append(None, k, k, cache, cu)
    # sequence 0: token 15 in page 0, token 16's page 4 is not there; 1: token 39 is past the table; 2: page -1
    want = torch.full_like(store, 7.0)
    want[:, 3, 15] = k[0]
    assert torch.equal(store, want)
    for bad in ([0, 9, 3, 1, 2, 6], [4, 4, 4, 4, 4, 4], [0, -1, -1, 100, 3, 2]):
        Q.bs_kv_append(None, k, k, cache, torch.tensor(bad, dtype=torch.int32).cuda())
        torch.cuda.synchronize()
        assert torch.all(store[:, :3] == 7.0) and torch.all(store[:, 7:] == 7.0)


def test_append_then_read_past_2_31_elements(gpu):
    """Pages whose offsets pass 32 bits, in elements and in bytes."""
    page, hkv, d = 256, 8, 128
    pages = (1 << 31) // (page * hkv * d) + 40  # 4.4 GB of bf16 each
    kc, vc = (torch.zeros(pages, page, hkv, d, dtype=torch.bfloat16, device=gpu) for _ in range(2))
    table = torch.tensor([[pages - 1, 0], [pages - 2, 3]], dtype=torch.int32, device=gpu)
    cache = Q.make_paged_cache(kc, vc, table, torch.tensor([200, 260], dtype=torch.int32, device=gpu))
    k, v = rand(0, 0, (3, hkv, d), torch.bfloat16).cuda(), rand(0, 1, (3, hkv, d), torch.bfloat16).cuda()
    Q.bs_kv_append(None, k, v, cache, torch.tensor([0, 1, 3], dtype=torch.int32, device=gpu))
    assert torch.equal(kc[pages - 1, 199], k[0]) and torch.equal(vc[pages - 1, 199], v[0])
    assert torch.equal(kc[3, 2], k[1]) and torch.equal(kc[3, 3], k[2]) and torch.equal(vc[3, 3], v[2])
    assert int((kc != 0).any(-1).sum()) == 3 * hkv
