"""Paged attention shared as a line, over more sequences than a workgroup has threads: sequences of several row blocks
among many others, and one of more new tokens than keys.  Bounds as in test_gpu_paged.py."""
import numpy as np
import pytest
import torch

from paper_2502_21231_amd import bs_attn as B
from paper_2502_21231_amd import bs_qkv as Q
from tests.test_gpu_paged import BF, F32, check, run_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt,tokens,lk", [(F32, 4194300, 2000), (F32, 4194300, 1), (BF, 32760, 700), (BF, 32760, 0)])
def test_more_tokens_than_keys(gpu, dt, tokens, lk):
    """One of 16,384 sequences has up to 4,194,300 new tokens and up to 2,000 keys, so that its first rows see none;
    another, behind it, one query and 1,300 keys."""
    seqs, page, d, at, other = 16384, 16, 64, 5000, 16001
    T = tokens + 1 + 3
    lens, new = np.zeros(seqs, np.int32), np.zeros(seqs, np.int64)
    lens[at], new[at], lens[other], new[other] = lk, tokens, 1300, 1
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    table = torch.full((seqs, 125), -1, dtype=torch.int32, device=gpu)
    n = [-(-lk // page), -(-1300 // page)]
    table[at, :n[0]] = torch.arange(n[0], dtype=torch.int32, device=gpu)
    table[other, :n[1]] = torch.arange(n[0], n[0] + n[1], dtype=torch.int32, device=gpu)
    g = torch.Generator(device=gpu).manual_seed(lk)
    q, k, v = (torch.randn(m, 1, d, generator=g, device=gpu).to(dt) for m in (T, sum(n) * page, sum(n) * page))
    cache = Q.make_paged_cache(k.view(-1, page, 1, d), v.view(-1, page, 1, d), table, torch.from_numpy(lens).cuda())
    out, lse = torch.full((T, 1, d), 3.0, dtype=dt, device=gpu), torch.full((1, T), 3.0, device=gpu)
    ws = Q.alloc_paged_workspace(q, cache, 5000)
    Q.bs_attn_paged_fwd(q, cache, torch.from_numpy(cu).cuda(), 5000, out=out, lse=lse, workspace=ws)
    assert B.bs_read_device_status(ws) == B.BS_OK
    assert not out[:tokens - lk].any() and torch.all(lse[:, :tokens - lk] == -float("inf"))
    # the rows that see keys, and those behind the last sequence
    want = [np.zeros((lk + 1, 1, d)), np.zeros((1, lk + 1)), np.zeros((lk + 1, 1, d))]
    for lo, rows, first, keys in ((0, lk, 0, lk), (lk, 1, n[0] * page, 1300)):
        if rows == 0:
            continue
        kk, vv = k[first:first + keys, 0].double(), v[first:first + keys, 0].double()
        s = q[tokens - lk + lo:, 0][:rows].double() @ kk.t() / 8
        s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(keys - rows + 1), -float("inf"))
        p = s.softmax(1)
        for w, x in zip(want, ((p @ vv)[:, None], s.logsumexp(1)[None], (p @ vv.abs())[:, None])):
            (w[:, lo:lo + rows] if w is want[1] else w[lo:lo + rows])[:] = x.cpu().numpy()
    check(out[tokens - lk:], lse[:, tokens - lk:], want, lk + 1, dt)


def many(seqs, chunks, keys, empty):
    """Lengths of `seqs` sequences of one query each, every `empty`-th of none; {sequence: (new tokens, length)} of others."""
    rng = np.random.default_rng(seqs)
    lens = [int(x) for x in rng.integers(1, keys, seqs)]
    new = [0 if i % empty == 3 else 1 for i in range(seqs)]
    for b, (n, length) in chunks.items():
        new[b], lens[b] = n, length
    return lens, new


# more than 256 sequences, so several per thread; chunks of several row blocks at a thread's first, middle and last one
MANY = [
    (300, {150: (250, 1500)}, 1100, 16, 8, 2, 128, BF),
    (300, {0: (100, 100), 299: (130, 2100)}, 700, 16, 8, 1, 64, BF),
    (1030, {517: (200, 3000), 518: (140, 90), 1029: (300, 1200)}, 60, 16, 2, 1, 64, BF),
    (300, {151: (200, 1300)}, 1100, 16, 4, 2, 64, F32),
    (300, {1: (33, 20), 298: (70, 1400)}, 300, 32, 6, 2, 128, F32),
    (777, {400: (300, 1100), 402: (64, 64)}, 40, 16, 1, 1, 128, F32),
]


@pytest.mark.parametrize("case", MANY, ids=str)
@pytest.mark.parametrize("causal", [True, False])
def test_chunks_among_many_sequences(gpu, case, causal):
    seqs, chunks, keys, page, hq, hkv, d, dt = case
    lens, new = many(seqs, chunks, keys, 5)
    assert dt is F32 or sum(new) + 2 <= 2 * seqs  # (bf16: the line's rule)
    run_case(lens, new, page, hq, hkv, d, dt, causal=causal, pad=2, most=4000)
