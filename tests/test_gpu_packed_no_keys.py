"""Packs without a key, or without a row, in every call: zeros, a log-sum-exp of -infinity, and weights of the right (empty) shape."""
import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_serving import BF16, F32, INF, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q_lens,k_lens", [([0, 0], None), ([0], None), ([3], [0]), ([130, 0, 2], [0, 0, 0]), ([0, 0], [5, 140])])
@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (4, 2, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("weight_rows", [0, 5])
def test_no_keys_or_no_rows(q_lens, k_lens, Hq, Hkv, D, dtype, weight_rows):
    n, m = sum(q_lens), sum(k_lens or q_lens)
    q, k, v = randn(n, Hq, D, dtype=dtype), randn(m, Hkv, D, dtype=dtype), randn(m, Hkv, D, dtype=dtype)
    with ris.ris_pack_create(q_lens, k_lens) as pack:
        out, lse, *w = ris.ris_attention_packed(pack, q, k, v, return_lse=True, weight_rows=weight_rows)
        ris.ris_device_status()
    assert out.shape == (n, Hq, D) and (out == 0).all() and lse.shape == (Hq, n) and (lse == -INF).all()
    assert len(w) == (weight_rows > 0)
    for x in w:
        assert x.shape == (Hkv, m) and (x == 0).all()


def test_weights_and_their_rows_go_together():
    """Still refused: a place for weights without rows, rows without a place where there are keys."""
    L = ris.lib()
    q, k, v = randn(3, 2, 64), randn(3, 1, 64), randn(3, 1, 64)
    out, kw = torch.empty_like(q), torch.empty(1, 4, device="cuda")
    with ris.ris_pack_create([3]) as pack:
        for rows, place in ((0, kw.data_ptr()), (5, None), (-1, kw.data_ptr())):
            assert L.ris_attention_packed(pack.handle, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), 2, 1, 64, 128, 64, 64, 0, 0,
                                          None, rows, place, None) == ris.RIS_ERR_INVALID
