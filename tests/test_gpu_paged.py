"""Attention over a paged key/value cache against the float64 oracle.

Tolerances.  Out: each weight p is rounded to bf16 once for the product (2^-8 relative; float32: not), scores
of a sum of 128 products in float32 are off by a random walk of about 12 u times sum |q k| scale (u = 2^-24;
sum |q k| scale is about 7 for N(0, 1) operands), so p by 1e-5: (2^-8 + 1e-4) times the attention of |v| with the
same weights (the oracle's `size`), plus half a bf16 step of the result; float32: 2e-5 times that.  LSE: 2e-5 +
4 u |lse|, or 1e-4 with bf16 operands whose larger scores the same walk multiplies."""
import numpy as np
import pytest
import torch

from oracle import qkv as O
from paper_2502_21231_amd import bs_attn as B
from paper_2502_21231_amd import bs_qkv as Q
from tests.parity_util import f64, half_ulp_bf16
from tests.test_gpu_qkv import dup, make_cache, rand

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def check(out, lse, want, rows, dtype, walk=1.0):
    """Rows below `rows`; the others still hold 3.  walk: sum |q k| scale over that of N(0, 1) operands."""
    o, l, size = want
    got, gl = f64(out), f64(lse)
    assert np.all(got[rows:] == 3.0) and np.all(gl[:, rows:] == 3.0)
    got, gl, o, l, size = got[:rows], gl[:, :rows], o[:rows], l[:, :rows], size[:rows]
    assert np.all(np.isfinite(got))
    bf = dtype is BF
    bound = ((2.0 ** -8 + 1e-4 * walk) * size + half_ulp_bf16(o)) if bf else 2e-5 * walk * size
    over = np.abs(got - o) - bound
    i = np.unravel_index(np.argmax(over), over.shape) if over.size else None
    assert i is None or over[i] <= 0, f"out {got[i]} for {o[i]} at {i}, bound {bound[i]}"
    assert np.array_equal(np.isneginf(gl), np.isneginf(l)) and not np.any(np.isnan(gl))
    fin = np.isfinite(l)
    assert np.all(np.abs(gl[fin] - l[fin]) <= (1e-4 if bf else 2e-5) * walk + 4 * 2.0 ** -24 * np.abs(l[fin]))


def call(q, kc, vc, table, lens, cu, most, causal=True, scale=None, workspace=None):
    T, hq, d = q.shape
    cache = Q.make_paged_cache(kc, vc, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    out = torch.full((T, hq, d), 3.0, dtype=q.dtype, device="cuda")
    lse = torch.full((hq, T), 3.0, device="cuda")
    ws = workspace
    if ws is None:
        ws = Q.alloc_paged_workspace(q, cache, most)
        ws.fill_(255)  # needs no initialisation
    Q.bs_attn_paged_fwd(q, cache, torch.from_numpy(cu).cuda(), most, causal, scale, out, lse, ws)
    assert B.bs_read_device_status(ws) == B.BS_OK
    return out, lse


def run_case(lens, new, page, hq, hkv, d, dt, hm=False, pad=0, causal=True, seed=0, most=None, edit=None, scale=None,
             nan_tails=True, walk=1.0):
    T = sum(new) + pad
    kc, vc, table = make_cache(seed, lens, page, hkv, d, dt, hm)
    if nan_tails:  # places behind the sequences' ends, pages of no sequence
        for x in (kc, vc):
            used = np.zeros((x.shape[0], page), bool)
            for b, n in enumerate(lens):
                for t in range(n):
                    used[table[b, t // page], t % page] = True
            x[torch.from_numpy(~used)] = float("nan")
    if edit is not None:
        edit(kc, vc, table)
    q = rand(seed, 1, (T, hq, d), dt)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    s = d ** -0.5 if scale is None else scale
    want = O.paged_fwd(f64(q), f64(kc), f64(vc), table, lens, cu, causal, s)
    out, lse = call(q.cuda(), dup(kc), dup(vc), table, lens, cu, most or max(lens, default=0), causal, scale)
    check(out, lse, want, sum(new), dt, walk)


# lens, new, page, hq, hkv, d, dtype
CASES = [
    ([1], [1], 16, 1, 1, 64, BF),
    ([5, 64, 129, 1000], [1, 1, 1, 1], 16, 8, 2, 128, BF),
    ([300, 17, 33], [1, 1, 1], 16, 8, 8, 128, BF),
    ([2000], [1], 32, 16, 1, 64, BF),
    ([700, 3, 90], [1, 1, 1], 64, 64, 1, 128, BF),
    ([513, 127, 128, 40], [30, 127, 1, 40], 16, 6, 2, 64, BF),
    ([900, 257], [200, 257], 64, 8, 1, 128, BF),
    ([333, 640], [333, 129], 256, 7, 7, 128, BF),
    ([777], [300], 16, 12, 4, 64, BF),
    ([4100], [3], 4096, 4, 4, 128, BF),
    ([200, 31, 1], [1, 31, 1], 16, 4, 2, 64, F32),
    ([130, 400], [130, 70], 32, 6, 1, 128, F32),
    ([1100], [1], 16, 3, 3, 128, F32),
    ([65, 66, 67] * 7, [1, 2, 3] * 7, 16, 4, 4, 64, BF),
    ([150], [5], 16, 300, 1, 64, BF),
]


# more of them, where the work is shared otherwise: keys of several workgroups, prompts of many rows, both forms in
# one call, row blocks in parts
SHARED = [
    ([3000, 10, 700], [1, 1, 1], 16, 8, 2, 128, BF),
    ([2900, 2500], [1, 4], 64, 12, 2, 64, BF),
    ([1500, 2100, 40, 9], [1, 150, 1, 1], 16, 12, 4, 128, BF),
    ([600, 1300, 70], [3, 200, 1], 16, 8, 1, 64, BF),
    ([1200, 900], [500, 900], 32, 4, 2, 128, BF),
    ([700], [700], 16, 1, 1, 64, BF),
    ([2000], [40], 16, 32, 1, 128, BF),
    ([1700, 30], [1, 1], 16, 8, 2, 128, F32),
    ([900, 300], [300, 280], 16, 4, 4, 64, F32),
    ([500, 600], [400, 1], 32, 6, 2, 128, F32),
]


@pytest.mark.parametrize("case", CASES + SHARED, ids=str)
@pytest.mark.parametrize("hm", [False, True])
def test_against_oracle(gpu, case, hm):
    run_case(*case, hm=hm, seed=len(case[0]))


# row blocks in many parts, of few and of many rows side by side
PARTS = [
    ([20000], [20], 16, 4, 1, 64, BF),
    ([9000, 2], [16, 2], 64, 8, 1, 128, BF),
    ([40, 3000, 6000, 1], [40, 1, 150, 1], 16, 8, 2, 128, BF),
    ([3000, 2999], [1, 90], 16, 7, 7, 64, BF),
    ([5000], [300], 32, 2, 1, 64, F32),
    ([130, 1300], [130, 300], 16, 4, 4, 128, F32),
]


# float32 with enough row blocks for the tile form: 512 of 128 rows over all KV heads
TILES32 = [
    ([130] * 20 + [1, 40], [130] * 20 + [1, 0], 16, 64, 16, 64, F32),
    ([70, 33, 500, 5], [70, 33, 100, 9], 32, 256, 64, 128, F32),
    ([250, 17], [250, 12], 16, 512, 128, 64, F32),
    ([40, 97, 31], [40, 97, 31], 64, 192, 192, 128, F32),
]


# decoding with a chunk among many single queries, whose work lies on one line
LINES = [
    ([2500] + [1300] * 39, [40] + [1] * 39, 16, 4, 2, 128, BF),
    ([90 * i for i in range(60)], [0] + [1] * 58 + [60], 32, 3, 3, 64, BF),
    ([1100, 3000, 2, 0], [1, 2, 2, 0], 16, 64, 1, 64, BF),
]


@pytest.mark.parametrize("case", LINES, ids=str)
@pytest.mark.parametrize("causal", [True, False])
def test_decoding_with_a_chunk(gpu, case, causal):
    run_case(*case, causal=causal, pad=1)


@pytest.mark.parametrize("case", TILES32, ids=str)
@pytest.mark.parametrize("causal", [True, False])
def test_float32_tiles(gpu, case, causal):
    run_case(*case, causal=causal, pad=3)


def test_float32_tiles_with_missing_pages(gpu):
    def edit(kc, vc, table):
        table[0, 2] = -1
        table[1, 0] = 1 << 20
        table[2, :] = -1

    for d in (64, 128):
        run_case([100, 40, 20], [100, 40, 20], 16, 512, 256, d, F32, edit=edit)


@pytest.mark.parametrize("case", PARTS, ids=str)
@pytest.mark.parametrize("causal", [True, False])
def test_many_parts(gpu, case, causal):
    run_case(*case, causal=causal)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_loose_bound(gpu, case):
    """A max_seqlen_k far above the lengths (a context's, say), which chooses another way to share the work."""
    run_case(*case, seed=1, most=1 << 20)


def test_not_causal(gpu):
    for case in (CASES[1], CASES[5], CASES[10], SHARED[2], SHARED[4], SHARED[8]):
        run_case(*case, seed=2, causal=False)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_without_keys_and_padding(gpu, dt, causal):
    """Sequences without keys, with more rows than keys (the first see none), without rows; padding rows."""
    for most in (300, 5000):
        run_case([0, 5, 300, 0, 80], [1, 9, 0, 0, 200], 16, 8, 2, 128, dt, pad=7, causal=causal, most=most)
    run_case([0, 0], [3, 1], 16, 4, 4, 64, dt, pad=1, causal=causal)
    run_case([300, 64], [1, 70], 32, 4, 1, 64, dt, causal=causal, most=100000 // 3)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("new", [1, 40, 100])
@pytest.mark.parametrize("most", [330, 5000])
def test_missing_pages(gpu, dt, new, most):
    """Pages that are not there hide their keys: first, middle, last ones, all of a sequence's."""
    def edit(kc, vc, table):
        n = kc.shape[0]
        table[0, [0, 5, 6, 7, 8, 20]] = [-1, n, -2 ** 31, 2 ** 31 - 1, -1, n + 5]
        table[1, :] = -1
        table[2, 1:] = -9
    run_case([330, 100, 100], [new] * 3, 16, 8, 2, 128, dt, edit=edit, most=most)
    run_case([330, 100, 100], [new] * 3, 16, 4, 4, 64, dt, edit=edit, hm=True, causal=False, most=most)


@pytest.mark.parametrize("dt", [BF, F32])
def test_shared_and_repeated_pages(gpu, dt):
    """A prefix that sequences share, a page that one sequence lists twice."""
    def edit(kc, vc, table):
        table[1, :3] = table[0, :3]
        table[2, 4] = table[2, 1]
    run_case([100, 90, 90], [1, 20, 3], 16, 8, 2, 64, dt, edit=edit, nan_tails=False)


@pytest.mark.parametrize("new", [1, 33])
def test_large_scores_and_scales(gpu, new):
    """Scores of +-1,000 (a lone key wins), equal scores, a tiny scale."""
    def edit(kc, vc, table):
        kc *= 8
    # sum |q k| scale: 8 times the operands and 128^(1/2) times the scale
    run_case([500, 20], [new, 1], 16, 8, 2, 128, F32, edit=edit, scale=1.0, walk=8 * 128 ** 0.5)
    run_case([500, 20], [new, 1], 16, 8, 2, 128, BF, scale=1e-30)


def test_a_key_of_minus_infinity_has_no_weight(gpu):
    """Scores of -inf (a key that a program blanks by its values): weight 0, as the formula gives."""
    for new in (1, 40):
        def edit(kc, vc, table):
            kc[:] = kc.abs()
            kc[table[0, 2], 3] = float("-inf")
        T, lens, cu = new, [200], np.array([0, new], np.int32)
        kc, vc, table = make_cache(0, lens, 16, 2, 64, BF)
        edit(kc, vc, table)
        q = rand(0, 1, (T, 4, 64), BF).abs()
        want = O.paged_fwd(f64(q), f64(kc), f64(vc), table, lens, cu, True, 0.125)
        out, lse = call(q.cuda(), dup(kc), dup(vc), table, lens, cu, 200)
        check(out, lse, want, T, BF)


def test_many_sequences(gpu):
    """More sequences than one workgroup's threads; single tokens and short chunks, some empty."""
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 40, 1500)]
    new = [int(min(n, x)) for n, x in zip(lens, rng.integers(0, 3, 1500))]
    for most in (40, 5000):
        run_case(lens, new, 16, 2, 1, 64, BF, most=most)
        run_case(lens[:700], new[:700], 16, 2, 2, 64, F32, most=most)
    lens = [int(x) for x in rng.integers(30, 200, 300)]
    new = [int(min(n, x)) for n, x in zip(lens, rng.integers(0, 60, 300))]
    run_case(lens, new, 16, 16, 1, 64, BF)  # 480 rows on average
    run_case(lens, new, 16, 16, 1, 64, F32)
    run_case(lens[:260], new[:260], 16, 8, 1, 64, BF, most=3000)


def test_many_sequences_in_parts_and_float32_tiles(gpu):
    """The same with row blocks in parts, with both forms among them, and as float32 tiles."""
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(0, 900, 300)]
    new = [int(min(n, x)) for n, x in zip(lens, rng.integers(1, 5, 300))]
    run_case(lens, new, 16, 16, 1, 64, BF, most=900)  # some 40 rows on average
    run_case(lens, new, 16, 16, 1, 128, BF, most=100000, pad=5)
    lens = [int(x) for x in rng.integers(0, 200, 290)]
    new = [int(min(n, x)) for n, x in zip(lens, rng.integers(2, 9, 290))]
    run_case(lens, new, 16, 16, 2, 64, F32)
    run_case(lens, new, 32, 16, 2, 128, F32, causal=False)


def test_refused_lengths_write_nothing(gpu):
    kc, vc, table = make_cache(0, [40, 40], 16, 2, 64, BF)
    q = rand(0, 1, (4, 4, 64), BF).cuda()
    kg, vg, tg = kc.cuda(), vc.cuda(), torch.from_numpy(table).cuda()
    ws = None
    for lens, cu, most, code in (([40, 40], [1, 2, 4], 64, 1), ([40, 40], [0, 3, 2], 64, 2), ([40, -1], [0, 2, 4], 64, 2),
                                 ([40, 40], [0, 2, 5], 64, 3), ([40, 30], [0, 2, 4], 39, 4),
                                 ([40, 16 * table.shape[1] + 1], [0, 2, 4], 1000, 4),
                                 ([40, 2 ** 31 - 1], [0, 2, 4], 1000, 4)):
        cache = Q.make_paged_cache(kg, vg, tg, torch.tensor(lens, dtype=torch.int32).cuda())
        out, lse = torch.full_like(q, 3.0), torch.full((4, 4), 3.0, device=gpu)
        ws = Q.alloc_paged_workspace(q, cache, most)
        Q.bs_attn_paged_fwd(q, cache, torch.tensor(cu, dtype=torch.int32).cuda(), most, out=out, lse=lse, workspace=ws)
        with pytest.raises(B.BsError) as e:
            B.bs_read_device_status(ws)
        assert e.value.status == B.BS_ERR_DEVICE_STATUS and f"code {code}" in str(e.value)
        assert torch.all(out == 3.0) and torch.all(lse == 3.0)


def test_refused_arguments(gpu):
    kc, vc, table = make_cache(0, [40], 16, 2, 64, BF)
    kg, vg, tg, lens = kc.cuda(), vc.cuda(), torch.from_numpy(table).cuda(), torch.tensor([40], dtype=torch.int32).cuda()
    cu = torch.tensor([0, 2], dtype=torch.int32).cuda()
    cache = Q.make_paged_cache(kg, vg, tg, lens)
    q = rand(0, 1, (2, 4, 64), BF).cuda()
    with pytest.raises(ValueError):
        Q.make_paged_cache(kg, vg[:, :, :1], tg, lens)
    with pytest.raises(ValueError):
        Q.make_paged_cache(kg, vg.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3), tg, lens)
    with pytest.raises(TypeError):
        Q.make_paged_cache(kg, vg, tg.long(), lens)
    with pytest.raises(ValueError):
        Q.make_paged_cache(kg, vg, tg, torch.zeros(3, dtype=torch.int32).cuda())
    with pytest.raises(B.BsError):  # a page size that is no power of two
        small = Q.make_paged_cache(kg[:, :12], vg[:, :12], tg, lens)
        Q.bs_attn_paged_fwd(q, small, cu, 40)
    with pytest.raises(B.BsError):  # 3 query heads over 2
        Q.bs_attn_paged_fwd(q[:, :3].contiguous(), cache, cu, 40)
    with pytest.raises(ValueError):
        Q.bs_attn_paged_fwd(q.float(), cache, cu, 40)
    with pytest.raises(ValueError):
        Q.bs_attn_paged_fwd(q, cache, torch.tensor([0, 1, 2], dtype=torch.int32).cuda(), 40)
    with pytest.raises(B.BsError):
        Q.bs_attn_paged_fwd(q, cache, cu, 40, scale=-1.0)
    with pytest.raises(B.BsError):
        Q.bs_attn_paged_fwd(q, cache, cu, 40, workspace=torch.empty(16, dtype=torch.uint8, device=gpu))
    with pytest.raises(ValueError, match="is on cpu"):
        Q.bs_attn_paged_fwd(q, cache, cu, 40, workspace=torch.empty(1 << 24, dtype=torch.uint8))


def test_two_streams_and_repeats(gpu):
    """Two calls under way at once, each with a workspace of its own; the same call again gives the same bits."""
    lens, new = [3000, 700, 64], [1, 5, 1]
    kc, vc, table = make_cache(0, lens, 16, 2, 128, BF)
    kg, vg = kc.cuda(), vc.cuda()
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    qs = [rand(i, 1, (7, 16, 128), BF).cuda() for i in range(2)]
    want = [call(q, kg, vg, table, lens, cu, 3000) for q in qs]
    cache = Q.make_paged_cache(kg, vg, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    cug = torch.from_numpy(cu).cuda()
    wss = [Q.alloc_paged_workspace(q, cache, 3000) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = Q.bs_attn_paged_fwd(qs[i], cache, cug, 3000, workspace=wss[i])
    torch.cuda.synchronize()
    for (a, b), (c, d) in zip(got, want):
        assert torch.equal(a, c) and torch.equal(b, d)


@pytest.mark.parametrize("hq,hkv,T,most", [(16, 2, 4, 600), (16, 2, 4, 2000), (8, 8, 90, 600), (8, 2, 90, 4000), (8, 1, 400, 600)])
def test_captured_step_replayed_with_other_lengths(gpu, hq, hkv, T, most):
    """One captured step of a padded batch (append, attention), replayed as the sequences grow and as their
    number of rows changes, against eager calls; a second capture shares the workspace."""
    d, page = 64, 16
    kc, vc = (torch.zeros(200, page, hkv, d, dtype=BF, device=gpu) for _ in range(2))
    table = torch.arange(4 * 40, dtype=torch.int32, device=gpu).view(4, 40)
    lens, cu = torch.zeros(4, dtype=torch.int32, device=gpu), torch.zeros(5, dtype=torch.int32, device=gpu)
    cache = Q.make_paged_cache(kc, vc, table, lens)
    par = Q.make_qk_params((10000.0 ** (-torch.arange(0, d, 2) / d)).float().cuda())
    qkv = rand(0, 0, (T, hq + 2 * hkv, d), BF).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    qo, out = (torch.zeros(T, hq, d, dtype=BF, device=gpu) for _ in range(2))
    lse = torch.zeros(hq, T, device=gpu)
    ws = Q.alloc_paged_workspace(qo, cache, most)

    def step():
        Q.bs_kv_append(q, k, v, cache, cu, par, q_out=qo)
        Q.bs_attn_paged_fwd(qo, cache, cu, most, out=out, lse=lse, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g):
            step()
    rng = np.random.default_rng(0)
    have = np.zeros(4, int)
    for i in range(6):
        new = np.array([1, 1, 1, 1]) if T == 4 else np.array([1, T // 2 if i % 2 and i < 4 else 0, rng.integers(1, 30), 1])
        if i == 3:
            new[1] = 0  # a sequence leaves: its rows and its length
        have = have + new + (100 if i == 2 else 0)
        n = np.where(new == 0, 0, have)
        lens.copy_(torch.from_numpy(n.astype(np.int32)))
        cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)))
        qkv.copy_(rand(i, 5, (T, hq + 2 * hkv, d), BF))
        out.fill_(3.0)
        lse.fill_(3.0)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        a, b = out.clone(), lse.clone()
        want = O.paged_fwd(f64(qo), f64(kc), f64(vc), table.cpu().numpy(), n, cu.cpu().numpy(), True, d ** -0.5)
        check(a, b, want, int(new.sum()), BF)
        out.fill_(3.0)
        lse.fill_(3.0)
        step()
        assert torch.equal(out, a) and torch.equal(lse, b)


@pytest.mark.parametrize("dt", [BF, F32])
def test_serving_gives_what_training_computes(gpu, dt):
    """Prompts run whole through bs_qk_norm_rope_fwd and bs_attn_varlen_fwd, and in pieces through bs_kv_append
    and bs_attn_paged_fwd: prompt chunks, then single tokens.  Both are within their own bounds of the exact
    result, and the keys in the cache are the same bits."""
    hq, hkv, d, page = 8, 2, 128, 16
    total = [150, 67]
    T = sum(total)
    qkv = rand(0, 0, (T, (hq + 2 * hkv) * d), dt).cuda()
    a, b = hq * d, (hq + hkv) * d
    q, k, v = qkv[:, :a].view(T, hq, d), qkv[:, a:b].view(T, hkv, d), qkv[:, b:].view(T, hkv, d)
    w = rand(0, 1, (d,), torch.float32, 0.2, 1.0).cuda()
    par = Q.make_qk_params((10000.0 ** (-torch.arange(0, d, 2) / d)).float().cuda(), q_weight=w, k_weight=w)
    start = np.concatenate([[0], np.cumsum(total)]).astype(np.int32)
    pos = torch.cat([torch.arange(n) for n in total]).cuda()
    qt, kt = Q.bs_qk_norm_rope_fwd(q, k, pos, par)
    cut = torch.from_numpy(start).cuda()
    ot, lt = B.bs_attn_varlen_fwd(qt, kt, v.contiguous(), cut, cut, max(total))
    kc, vc, table = make_cache(0, total, page, hkv, d, dt)
    cache = Q.make_paged_cache(kc.cuda(), vc.cuda(), torch.from_numpy(table).cuda(), torch.zeros(2, dtype=torch.int32).cuda())
    outs, lses, qs = torch.zeros_like(ot), torch.zeros_like(lt), torch.zeros_like(qt)
    at = [0, 0]
    for chunk in ([100, 1], [1, 60], [47, 1], [1, 5], [1, 0]):
        rows = torch.cat([torch.arange(start[i] + at[i], start[i] + at[i] + chunk[i]) for i in range(2)]).cuda()
        at = [x + y for x, y in zip(at, chunk)]
        cache.kv_lens.copy_(torch.tensor(at, dtype=torch.int32))
        cu = torch.tensor([0, chunk[0], sum(chunk)], dtype=torch.int32).cuda()
        qo = Q.bs_kv_append(q[rows], k[rows], v[rows], cache, cu, par)
        o, l = Q.bs_attn_paged_fwd(qo, cache, cu, max(total))
        outs[rows], lses[:, rows], qs[rows] = o, l, qo
    assert at == total
    assert torch.equal(qs, qt)
    for i in range(2):
        t = torch.arange(total[i])
        pages = torch.from_numpy(table[i]).long()[t // page]
        assert torch.equal(cache.k[pages, t % page], kt[start[i]:start[i + 1]])
        assert torch.equal(cache.v[pages, t % page], v[start[i]:start[i + 1]])
    want = O.paged_fwd(f64(qt), f64(cache.k), f64(cache.v), table, total, start, True, d ** -0.5)
    check(outs, lses, want, T, dt)
    check(ot, lt, want, T, dt)


def test_cache_offsets_past_32_bits(gpu):
    """Pages at both ends of a cache of more than 2^31 elements."""
    page, hkv, d = 256, 8, 128
    pages = (1 << 31) // (page * hkv * d) + 40
    big = [torch.zeros(pages, page, hkv, d, dtype=BF, device=gpu) for _ in range(2)]
    lens, new = [600, 300], [1, 40]
    kc, vc, small = make_cache(0, lens, page, hkv, d, BF, extra_cols=0)
    ids = np.array([pages - 1, 0, pages - 2, 1, pages // 2, pages - 3, 5])
    for i in range(kc.shape[0]):
        big[0][ids[i]], big[1][ids[i]] = kc[i].cuda(), vc[i].cuda()
    table = np.where(small >= 0, ids[small], -1).astype(np.int32)
    q = rand(0, 1, (41, 16, d), BF)
    cu = np.array([0, 1, 41], np.int32)
    want = O.paged_fwd(f64(q), f64(kc), f64(vc), small, lens, cu, True, d ** -0.5)
    out, lse = call(q.cuda(), big[0], big[1], table, lens, cu, 600)
    check(out, lse, want, 41, BF)


def test_keys_and_values_in_one_buffer(gpu):
    """Keys and values as halves of one buffer, by page, by token and by head; a table that is a part of a larger."""
    lens, new = [100, 40], [1, 30]
    kc, vc, table = make_cache(0, lens, 16, 2, 64, BF)
    q = rand(0, 1, (31, 4, 64), BF)
    cu = np.array([0, 1, 31], np.int32)
    want = O.paged_fwd(f64(q), f64(kc), f64(vc), table, lens, cu, True, 0.125)
    wide = torch.full((2, table.shape[1] + 5), -1, dtype=torch.int32, device=gpu)
    wide[:, 2:2 + table.shape[1]] = torch.from_numpy(table).cuda()
    for dim in (1, 2, 3):
        both = torch.stack([kc, vc], dim).cuda()
        cache = Q.make_paged_cache(both.select(dim, 0), both.select(dim, 1), wide[:, 2:2 + table.shape[1]],
                                   torch.tensor(lens, dtype=torch.int32).cuda())
        out, lse = torch.full((31, 4, 64), 3.0, dtype=BF, device=gpu), torch.full((4, 31), 3.0, device=gpu)
        Q.bs_attn_paged_fwd(q.cuda(), cache, torch.from_numpy(cu).cuda(), 100, out=out, lse=lse)
        check(out, lse, want, 31, BF)
