"""GPU: a serving step in which sequences are refused for want of blocks, followed through the
calls that take host lengths. The host reads how many sequences were served and counts no rows for
the others; the rest of the step runs on the served ones, nothing of the others is written,
and once blocks are released the next step serves them."""
import numpy as np
import pytest
import torch

import opref
from oracle import attention as oattn
from paper_2603_23049_amd import pcr, synth
from gpuio import MAX_ABS, MEAN_ABS, error_stats, u16
from test_gpu_operator_step import BS, Pool, _i32, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (16, 4, 128)])
def test_refused_sequences_through_a_step(Hq, Hkv, d):
    gen = torch.Generator(device="cuda").manual_seed(d)
    B, f = 4, (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    rope = pcr.Rope(f)
    enc_len = np.array([40, 0, 90, 17], np.int32)
    enc = Pool(B, 6, 20, Hkv, d, gen, 1)
    slots, _, _ = enc.assign(enc_len, int(enc_len.sum()))
    pcr.append_kv(enc.kv, _rand(gen, int(enc_len.sum()), Hkv, d), _rand(gen, int(enc_len.sum()), Hkv, d), slots)
    pool = Pool(B, 8, 11, Hkv, d, gen, 2)
    lens = np.zeros(B, np.int32)
    # 3 + 1 + 5 blocks of 11 leave 2: sequence 2 (one more needs 3) is refused in the second step, and 3 with it
    for step, (new, served) in enumerate([([40, 5, 70, 0], 4), ([1, 12, 50, 3], 2), ([0, 1, 50, 3], 4)]):
        new = np.array(new, np.int32)
        cap = int(new.sum()) + 3
        k_before, v_before, bt_before = pool.kv.k.clone(), pool.kv.v.clone(), pool.bt.clone()
        slots, pos, cu = pool.assign(new, cap)
        assert pool.status.tolist()[0] == served, step                 # the host's one look at the device
        rows = np.where(np.arange(B) < pool.status.tolist()[0], new, 0).astype(np.int32)
        h_cu, prefix = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32), lens.copy()
        T = int(h_cu[-1])
        lens = lens + rows
        assert np.array_equal(cu.cpu().numpy(), h_cu) and np.array_equal(pool.lens.cpu().numpy(), lens)
        q, k, v = _rand(gen, cap, Hq, d), _rand(gen, cap, Hkv, d), _rand(gen, cap, Hkv, d)
        q_rot = torch.empty_like(q)
        pcr.rope_append_kv(rope, pool.kv, q, k, v, pos[None], slots, Hq, q_rot)
        out, x_out = torch.full_like(q, 9.0), torch.full_like(q, 9.0)
        pcr.prefix_prefill_attn(q_rot, pool.kv, pool.bt, _i32(prefix), cu, prefix, h_cu, Hq, out)
        pcr.cross_attn(q_rot, enc.kv, enc.bt, enc.lens, cu, enc_len, h_cu, Hq, x_out)
        torch.cuda.synchronize()
        assert (out[T:] == 9).all() and (x_out[T:] == 9).all()
        s = slots.cpu().long()
        assert (s[:T] >= 0).all() and (s[T:] == -1).all() and (pos[T:] == 0).all()
        assert torch.equal(pool.bt[served:], bt_before[served:])
        untouched = torch.ones(pool.n, BS, dtype=torch.bool)
        untouched[s[:T] // BS, s[:T] % BS] = False
        for now, was, view in ((pool.kv.k, k_before, (Hkv, BS, d)), (pool.kv.v, v_before, (Hkv, d, BS))):
            slot = 2 if view[1] == BS else 3
            now, was = (x.cpu().view(-1, *view).movedim(slot, 1)[untouched].contiguous() for x in (now, was))
            assert torch.equal(now.view(torch.int16), was.view(torch.int16))
        w = oattn.attention(u16(q_rot[:T].view(torch.int16)), u16(pool.kv.k.view(torch.int16)),
                            u16(pool.kv.v.view(torch.int16)), pool.bt.cpu().numpy(), prefix, h_cu, Hkv, BS)
        mx, mean = error_stats(synth.bf16_bits_to_f32(u16(out[:T].view(torch.int16))).astype(np.float64), w)
        assert mx <= MAX_ABS and mean <= MEAN_ABS, (step, mx, mean)
        xw, dev = opref.cross(q_rot[:T].cpu().double(), enc.kv.k.cpu().double(), enc.kv.v.cpu().double(),
                              enc.bt.cpu().numpy(), enc_len, h_cu, Hkv, d ** -0.5)
        assert ((x_out[:T].cpu().double() - xw).abs() <=
                1.25 * dev * 2.0 ** -8 / (1 - 2.0 ** -8) + xw.abs() * 2.0 ** -8 + 1e-30).all(), step
        if step == 1:                                                  # the first sequence ends
            keep = lens.copy()
            keep[0] = 0
            pcr.release_blocks(pool.lens, _i32(keep), pool.bt, pool.free, pool.count, pool.n, pool.count, pool.status)
            pool.lens.copy_(_i32(keep))
            lens = keep
