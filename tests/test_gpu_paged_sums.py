"""Paged attention where roundings do not average out: one strong key (a sink) before many keys of nearly nothing, all of
one score, so that every weight and every sum is rounded the same way.

Tolerances (u = 2^-24).  A weight: its score is one exact product times scale log2(e) less the maximum, 2 u of at most 12
in log2 units, with the exponential's own step 2e-6; two bf16 parts 2^-17, one 2^-8 (half a step of 8 bits, at a power
of two).  The sum of the weights: chains of 8 and two more additions in a tile, 10 u, then compensated, 2 u: 8e-7.  LSE: a
weight's and the sum's, 3e-6, and the two roundings and log2's step at |lse| below 20, 4 u |lse| = 5e-6."""
import pytest
import torch

from paper_2502_21231_amd import bs_attn as B
from paper_2502_21231_amd import bs_qkv as Q

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def sink(dt, d, keys, T, hq, values, first=None):
    """A call of T queries of hq heads over one KV head's keys, all but the first of one score, which lies 3 to 7 below the
    first's (by the head), with these values [1 or keys, d]; the last T keys are the queries' own.  (out, lse), and in float64 out, lse, and out of |v|."""
    gap = 3 + torch.arange(hq, device="cuda", dtype=torch.float64) % 64 / 16
    q = torch.zeros(T, hq, d, dtype=dt, device="cuda")
    q[:, :, 0] = 8 * gap
    k = torch.zeros(keys, d, dtype=dt, device="cuda")
    k[0, 0] = 1
    v = values.expand(keys, d).to(dt, copy=True)
    if first is not None:
        v[0] = first
    page = 256
    shape = (keys // page, page, 1, d)
    cache = Q.make_paged_cache(k.view(shape), v.view(shape), torch.arange(keys // page, dtype=torch.int32, device="cuda")[None],
                               torch.tensor([keys], dtype=torch.int32, device="cuda"))
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    ws = Q.alloc_paged_workspace(q, cache, keys)
    out, lse = Q.bs_attn_paged_fwd(q, cache, cu, keys, True, 0.125, workspace=ws)
    assert B.bs_read_device_status(ws) == B.BS_OK
    n = torch.arange(keys - T + 1, keys + 1, device="cuda")  # keys that each query sees
    w = torch.exp(-gap)
    total = 1 + w * (n - 1).double()[:, None]

    def attend(x):
        run = x.double().cumsum(0)[n - 1]
        return (x[0].double() + w[:, None] * (run - x[0].double())[:, None]) / total[:, :, None]

    return out, lse, attend(v), (gap + total.log()).t(), attend(v.abs())


def half_step(x):
    """Half the spacing of bf16 numbers at x."""
    return torch.ldexp(torch.ones_like(x), torch.frexp(x.abs())[1] - 9)


@pytest.mark.parametrize("T,hq,keys", [(1, 32, 512), (1, 32, 16384), (8, 4, 1024), (8, 4, 20480), (1, 7, 4096)])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_few_rows_are_not_rounded_to_bf16(gpu, T, hq, keys, d):
    """Values 1 .. 2 behind a sink of value 0: a weight rounded to bf16 shows in full, by up to 2^-8 of the result.  The
    products' sums: 16,384 keys in chains of 16 keys a step, 1,280 steps at most, 4e-5 at half a step each on a sum that
    grows evenly."""
    out, _, want, _, size = sink(BF, d, keys, T, hq, 1 + torch.arange(d, device="cuda")[None] / d, 0.0)
    over = (out.double() - want).abs() - (2.0 ** -17 + 2e-6 + 4e-5) * size - half_step(want)
    assert over.max() <= 0, over.max()


# row blocks that walk all keys (512 of 128 rows), and such as are cut; sequences of few rows
LONG = [(BF, 64, 1 << 17, 1024, 64), (BF, 128, 1 << 20, 1024, 64), (BF, 128, 1 << 20, 1, 32), (BF, 128, 1 << 17, 20, 64),
        (F32, 64, 1 << 17, 1024, 64), (F32, 128, 1 << 17, 1024, 64), (F32, 64, 1 << 20, 8, 8), (F32, 128, 1 << 18, 100, 4)]


def normal(d, keys):
    return 1 + torch.randn(keys, d, generator=torch.Generator(device="cuda").manual_seed(d), device="cuda")


@pytest.mark.parametrize("case", LONG, ids=str)
def test_sum_of_many_weights(gpu, case):
    dt, d, keys, T, hq = case
    out, lse, want, want_lse, size = sink(dt, d, keys, T, hq, normal(d, keys))
    assert ((lse.double() - want_lse).abs() <= 3e-6 + 4 * 2.0 ** -24 * want_lse.abs()).all()
    if dt is BF:
        # O's sums: 16 keys a step, 2^16 steps at 1,048,576 keys, half a step of rounding in each on a sum that grows
        # evenly: u 2^16 / 2 = 2e-3, of one sign only where the values are equal: here they
            # differ, and the steps' roundings are as a walk, u 2^8 = 2e-5
        over = (out.double() - want).abs() - (2.0 ** -8 + 1e-4) * size - half_step(want)
        assert over.max() <= 0, over.max()


@pytest.mark.parametrize("T,hq,d", [(1024, 64, 64), (1024, 64, 128), (300, 64, 64), (1, 16, 128)])
@pytest.mark.parametrize("equal", [True, False])
def test_float32_sums_of_many_products(gpu, T, hq, d, equal):
    """Out.  Within a tile of 32 keys 16 steps from 0, 2 u each, and a weight's 3e-6: 5e-6.  Then one addition a tile to a
    sum that grows evenly, u / 2 of its end each: in the tile form (head_dim 128, 512 row blocks) keys / 32 of them, in
    the few form each of four waves has a fourth of the keys."""
    keys = 1 << 17
    out, _, want, _, size = sink(F32, d, keys, T, hq, torch.ones(1, d, device="cuda") if equal else normal(d, keys))
    steps = keys / 32 / (1 if d == 128 and T == 1024 else 4)
    assert ((out.double() - want).abs() <= (5e-6 + 2.0 ** -25 * steps) * size).all()
