"""GPU: cross attention where no sequence of the batch has keys: zero rows whatever their count,
with no workspace, which the size query says for such batches."""
import numpy as np
import pytest
import torch

from paper_2603_23049_amd import pcr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,Hq,Hkv,d", [([40], 8, 2, 64), ([300, 1], 8, 2, 64), ([17, 0, 2], 4, 4, 128),
                                           ([1, 1], 40, 2, 64), ([4], 8, 2, 64), ([0, 2000], 16, 2, 128)])
@pytest.mark.parametrize("given", [False, True])
def test_batches_without_keys(rows, Hq, Hkv, d, given):
    B, T = len(rows), sum(rows)
    assert pcr.cross_attn_workspace_bytes(B, T, Hq, Hkv, d, 0) == 0
    pool = pcr.KVPool(torch.zeros(3, Hkv, 16 * d, dtype=torch.bfloat16, device="cuda"),
                      torch.zeros(3, Hkv, 16 * d, dtype=torch.bfloat16, device="cuda"), Hkv, d)
    n, cu = np.zeros(B, np.int32), np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    q = torch.ones(T, Hq, d, dtype=torch.bfloat16, device="cuda")
    out = torch.full((T + 3, Hq, d), 9.0, dtype=torch.bfloat16, device="cuda")
    table = torch.full((B, 2), -1, dtype=torch.int32, device="cuda")
    ws = torch.empty(0, dtype=torch.uint8, device="cuda") if given else None
    pcr.cross_attn(q, pool, table, torch.from_numpy(n).cuda(), torch.from_numpy(cu).cuda(), n, cu, Hq, out, workspace=ws)
    assert (out[:T] == 0).all() and (out[T:] == 9).all()
