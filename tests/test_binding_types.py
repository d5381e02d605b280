"""CPU: the binding of the operators around the pool takes bf16 (or its bits as 16-bit integers)
and refuses other types of 2 bytes, whose bits would be read as bf16."""
import numpy as np
import pytest
import torch

from paper_2603_23049_amd import pcr

CPU = (torch, -1)                        # as if CPU tensors were on the current GPU
Hkv, Hq, d = 2, 4, 64


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int16, torch.uint16])
def test_bf16_and_its_bits_pass(dtype):
    x = torch.zeros(5, 2, 64, dtype=dtype)
    assert pcr._halves(CPU, 640, x, "x") == x.data_ptr() and pcr._rows(CPU, x, 5, 2, 64, "x") == 128


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.int8, torch.int32])
def test_other_types_are_refused(dtype):
    x = torch.zeros(5, 2, 64, dtype=dtype)
    for call in (lambda: pcr._halves(CPU, 640, x, "x"), lambda: pcr._rows(CPU, x, 5, 2, 64, "x")):
        with pytest.raises(ValueError, match=f"x holds {dtype}, not"):
            call()


def test_entry_points_refuse_fp16(monkeypatch):
    monkeypatch.setattr(pcr, "_current_gpu", lambda: CPU)

    def h(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype)

    def i(*shape):
        return torch.zeros(shape, dtype=torch.int32)

    rope = pcr.Rope(np.ones(32))
    n, cu = np.array([5, 9], np.int32), np.array([0, 1, 3], np.int32)
    for bad in ("q", "k", "v", "out", "pool_k", "pool_v"):
        t = {k: torch.float16 if k == bad else torch.bfloat16 for k in ("q", "k", "v", "out", "pool_k", "pool_v")}
        pool = pcr.KVPool(h(4, Hkv, 16 * d, dtype=t["pool_k"]), h(4, Hkv, 16 * d, dtype=t["pool_v"]), Hkv, d)
        with pytest.raises(ValueError, match="float16"):
            pcr.rope_append_kv(rope, pool, h(5, Hq, d, dtype=t["q"]), h(5, Hkv, d, dtype=t["k"]),
                               h(5, Hkv, d, dtype=t["v"]), i(5), i(5), Hq, h(5, Hq, d, dtype=t["out"]))
        if bad in ("k", "v"):
            continue
        with pytest.raises(ValueError, match="float16"):
            pcr.cross_attn(h(3, Hq, d, dtype=t["q"]), pool, i(2, 4), i(2), i(3), n, cu, Hq, h(3, Hq, d, dtype=t["out"]))
        if bad in ("q", "out"):
            with pytest.raises(ValueError, match="float16"):
                pcr.rope_rows(rope, h(5, Hq, d, dtype=t["q"]), i(5), h(5, Hq, d, dtype=t["out"]))
