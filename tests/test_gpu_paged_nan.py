"""Paged attention over a key of NaN: the rows that see it get NaN in out and LSE (-inf would say that they see no key),
and no other row does."""
import numpy as np
import pytest
import torch

from oracle import qkv as O
from tests.parity_util import f64
from tests.test_gpu_paged import BF, F32, call, check
from tests.test_gpu_qkv import dup, make_cache, rand

pytestmark = pytest.mark.gpu

# lens, new, most: single queries; chunks whole and in parts of their keys, with rows before the key and after it
CASES = [([100, 70], [1, 1], 100), ([3000, 70], [1, 1], 3000), ([90, 40], [60, 40], 100), ([3000, 200], [150, 100], 3000)]


@pytest.mark.parametrize("lens,new,most", CASES)
@pytest.mark.parametrize("hq,hkv,d,dt", [(4, 2, 64, BF), (8, 1, 128, BF), (4, 2, 64, F32), (6, 2, 128, F32), (1024, 512, 64, F32)])
@pytest.mark.parametrize("alone", [False, True])
def test_a_key_of_nan(gpu, lens, new, most, hq, hkv, d, dt, alone):
    """In the first sequence, the key of the chunk's middle row; `alone`: the first key of all, which every row sees, in a
    sequence whose other pages are not there."""
    page = 16
    kc, vc, table = make_cache(3, lens, page, hkv, d, dt)
    at = 0 if alone else lens[0] - 1 - new[0] // 2
    if alone:
        table[0, 1:] = -1
    q = rand(3, 1, (sum(new), hq, d), dt)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    want = O.paged_fwd(f64(q), f64(kc), f64(vc), table, lens, cu, True, d ** -0.5)
    kc[table[0, at // page], at % page, 0] = float("nan")
    out, lse = call(q.cuda(), dup(kc), dup(vc), table, lens, cu, most)
    sees = np.zeros((sum(new), hq), bool)  # only the first KV head's key is one
    sees[:new[0], :hq // hkv] = (np.arange(new[0]) + lens[0] - new[0] >= at)[:, None]
    assert sees.any()
    mask = torch.from_numpy(sees).cuda()
    assert out[mask].isnan().all() and lse.t()[mask].isnan().all()
    out[mask], lse.t()[mask] = torch.from_numpy(want[0]).to(dt).cuda()[mask], torch.from_numpy(want[1]).float().cuda().t()[mask]
    check(out, lse, want, sum(new), dt)
