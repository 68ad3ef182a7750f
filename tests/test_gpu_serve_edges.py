"""GPU checks of the operators of e2s_serve.h at the edges of what their header allows: NaN
beside missing pages, the largest values, overlapping rows, gradients, and memory that
another stream still uses."""
import numpy as np
import pytest

import _serve_helpers as S
from test_gpu_cache import _check_attend, _cuda, _filled, _ints, _match

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
E = pytest.importorskip("paper_2608_23253_amd")

BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("T,max_tokens", [(1, 128), (1, 3000), (4, 2000), (20, 128), (20, 3000)])
def test_nan_key_beside_a_missing_page(T, max_tokens):
    """A token whose page is not there is seen by no query: its weight stays what it was,
    also where a NaN key makes every weight of the tokens that are there NaN."""
    rng = np.random.default_rng(51)
    n, P = 100, 16
    pool, table = _filled(rng, [n, n], 1, P, 64)
    pool.k[table[0, 1], 0, 3, 9] = 0x7F
    table[:, 4] = -1
    there = np.ones(n, bool)
    there[4 * P:5 * P] = False
    q = torch.from_numpy(rng.standard_normal((2, 7, T, 64))).to(BF).cuda()
    was = torch.full((2, 1, max_tokens), 0.25, device="cuda")
    call = E.CacheAttention(E.PagedCache.of(*pool.tensors()), 2, 7, T, max_tokens, BF,
                            causal=False, weights=True)
    out, w = call(q, _cuda(table), _ints([n, n]), weights_in=was, weights_out=was.clone())
    w = w.cpu().numpy()
    assert out[0].isnan().all() and not out[1].isnan().any()
    assert np.isnan(w[0, 0, :n][there]).all()
    assert (w[0, 0, :n][~there] == 0.25).all(), "a weight for tokens that no query sees"
    assert not np.isnan(w[1]).any() and (w[1, 0, :n][~there] == 0.25).all()
