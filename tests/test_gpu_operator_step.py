"""GPU: the operators together as a serving step of an encoder-decoder model uses them. Encoder
states go into a pool of their own through assigned blocks; then, per step, blocks are
assigned for the new tokens, Q and K are rotated and K/V written, causal attention runs over
prefix and new tokens, and cross attention reads the encoder's states: a prompt, then single
tokens, then rejected tokens are released and their blocks taken again. Every step's outputs
are checked against the definitions in 64 bits, from the pool's own contents."""
import numpy as np
import pytest
import torch

import opref
from oracle import attention as oattn
from paper_2603_23049_amd import pcr, synth
from gpuio import MAX_ABS, MEAN_ABS, error_stats, u16

pytestmark = pytest.mark.gpu
BS = 16


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)


class Pool:
    """One layer's pool with its block tables and free blocks on the GPU."""

    def __init__(self, B, max_blocks, num_blocks, Hkv, d, gen, seed):
        self.kv = pcr.KVPool(_rand(gen, num_blocks, Hkv, BS * d), _rand(gen, num_blocks, Hkv, BS * d), Hkv, d)
        self.bt = _i32(np.full((B, max_blocks), -1))
        self.free = _i32(np.random.Generator(np.random.PCG64(seed)).permutation(num_blocks))
        self.count = _i32([num_blocks])
        self.lens = _i32(np.zeros(B))
        self.status = _i32([0, 0, 0])
        self.n = num_blocks

    def assign(self, new, cap):
        B = len(new)
        slots, pos, cu = _i32(np.zeros(cap)), _i32(np.zeros(cap)), _i32(np.zeros(B + 1))
        pcr.assign_blocks(self.lens, _i32(new), self.bt, self.free, self.count, self.n, slots, cu, self.lens,
                          self.count, self.status, positions=pos)
        return slots, pos, cu


@pytest.mark.parametrize("Hq,Hkv,d,axes", [(8, 2, 64, 1), (16, 4, 128, 3)])
def test_encoder_decoder_steps(Hq, Hkv, d, axes):
    gen = torch.Generator(device="cuda").manual_seed(d)
    B, scale = 3, 1.0 / d ** 0.5
    enc_len = np.array([70, 0, 333], np.int32)
    enc = Pool(B, 24, 40, Hkv, d, gen, 1)
    slots, _, _ = enc.assign(enc_len, int(enc_len.sum()))
    pcr.append_kv(enc.kv, _rand(gen, int(enc_len.sum()), Hkv, d), _rand(gen, int(enc_len.sum()), Hkv, d), slots)

    f = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    axis = (np.arange(d // 2) % axes).astype(np.int32)
    rope = pcr.Rope(f, axis, axes)
    pool = Pool(B, 12, 30, Hkv, d, gen, 2)
    lens = np.zeros(B, np.int32)
    steps = [[40, 5, 100], [1, 1, 1], [3, 1, 0], [1, 1, 1]]
    for i, new in enumerate(steps):
        new = np.array(new, np.int32)
        T, cap = int(new.sum()), int(new.sum()) + (7 if i else 0)      # padded rows in the later steps
        slots, pos, cu = pool.assign(new, cap)
        qkv = _rand(gen, cap, (Hq + 2 * Hkv) * d)
        q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([Hq * d, Hkv * d, Hkv * d], dim=1))
        positions = torch.stack([pos // (a + 1) for a in range(axes)])
        q_rot = torch.empty(cap, Hq, d, dtype=torch.bfloat16, device="cuda")
        pcr.rope_append_kv(rope, pool.kv, q, k, v, positions, slots, Hq, q_rot)
        h_cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        out, x_out = torch.zeros_like(q_rot), torch.zeros_like(q_rot)
        prefix = lens.copy()
        pcr.prefix_prefill_attn(q_rot, pool.kv, pool.bt, _i32(prefix), cu, prefix, h_cu, Hq, out)
        pcr.cross_attn(q_rot, enc.kv, enc.bt, enc.lens, cu, enc_len, h_cu, Hq, x_out)
        torch.cuda.synchronize()
        lens = lens + new
        assert np.array_equal(pool.lens.cpu().numpy(), lens) and np.array_equal(cu.cpu().numpy(), h_cu)
        assert (slots[T:].cpu() == -1).all() and pool.status.cpu().tolist()[0::2] == [B, T]
        # the rotation, and what the pool holds of it
        want, size = opref.rotate(q.cpu().double(), positions.cpu(), f, axis, 0)
        assert ((q_rot.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -19).all()
        s = slots[:T].cpu().long()
        k_in = pool.kv.k.cpu().view(-1, Hkv, BS, d)[s // BS, :, s % BS].double()
        want, size = opref.rotate(k[:T].cpu().double(), positions[:, :T].cpu(), f, axis, 0)
        assert ((k_in - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -19).all()
        assert torch.equal(pool.kv.v.cpu().view(-1, Hkv, d, BS)[s // BS, :, :, s % BS], v[:T].cpu())
        # both attentions, from the pools as they are
        w = oattn.attention(u16(q_rot[:T].view(torch.int16)), u16(pool.kv.k.view(torch.int16)),
                            u16(pool.kv.v.view(torch.int16)), pool.bt.cpu().numpy(), prefix, h_cu, Hkv, BS)
        got = synth.bf16_bits_to_f32(u16(out[:T].view(torch.int16))).astype(np.float64)
        mx, mean = error_stats(got, w)
        assert mx <= MAX_ABS and mean <= MEAN_ABS, (i, mx, mean)
        xw, dev = opref.cross(q_rot[:T].cpu().double(), enc.kv.k.cpu().double(), enc.kv.v.cpu().double(),
                              enc.bt.cpu().numpy(), enc_len, h_cu, Hkv, scale)
        err = (x_out[:T].cpu().double() - xw).abs()
        assert (err <= 1.25 * dev * 2.0 ** -8 / (1 - 2.0 ** -8) + xw.abs() * 2.0 ** -8 + 1e-30).all(), i
        assert (out[T:] == 0).all() and (x_out[T:] == 0).all()
        if i == 2:                                            # two tokens rejected, one sequence ends
            keep = np.maximum(lens - np.array([2, 0, 0]), 0).astype(np.int32)
            keep[2] = 0
            before = int(pool.count)
            pcr.release_blocks(pool.lens, _i32(keep), pool.bt, pool.free, pool.count, pool.n, pool.count, pool.status)
            freed = sum(-(-int(a) // BS) - -(-int(b) // BS) for a, b in zip(lens, keep))
            assert int(pool.count) == before + freed and pool.status.cpu().tolist() == [B, freed, freed]
            pool.lens.copy_(_i32(keep))
            lens = keep
