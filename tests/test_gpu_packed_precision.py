"""Precision of the sums over a 4-bit cache against 64 bits: bf16 at 64 channels and fp32, whose softmax weights keep all of fp32's bits.

The output's own rounding hides what the sums lose, so the draft's values cancel: a chain of five nodes with one key and one query, whose
values take away what the cached tokens sum up to, each the rest of the one before (a bf16 value has 8 bits: four of them leave 2^-32 of the sum).
The last node's result is nearly 0, and shows the error of the sums themselves.

Bound: the worst case of fp32 sums, as a share of sum |w v|: weights off by their scores' error (twice: in the sum and in what it is divided
by) and 2^-23 of their own, n + 64 roundings.  Weights of 8 bits are off by up to 2^-9, n of them by 2^-9 / sqrt(3 n) in the mean."""
import math

import numpy as np
import pytest
import torch

import compact_reference as ref

pytestmark = pytest.mark.gpu

CASES = [   # tokens per sequence, query heads per KV head, block size, kept list
    ([8], 1, 16, False), ([8], 8, 16, True), ([5, 40], 3, 24, True), ([64], 16, 64, False), ([3, 31], 16, 7, True), ([200, 90], 8, 32, False),
    ([41500, 33, 0, 64, 12], 16, 64, False)]   # (equal shares of all chunks)
N = 5


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 64), (torch.float32, 64), (torch.float32, 128)], ids=["bf16-64", "f32-64", "f32-128"])
@pytest.mark.parametrize("lens,G,B,kept", CASES)
def test_weights_keep_their_bits(gpu_lib, dtype, D, lens, G, B, kept):
    sp, Hkv, bt = gpu_lib, 1 if len(lens) > 2 else 2, len(lens)
    T = -(-max(lens) // B) * B
    h, k, v = ref.cache(sp, bt, Hkv, T, D, B, dtype, seed=sum(lens), lens=lens)
    g = torch.Generator().manual_seed(G)
    q1 = torch.randn((bt, Hkv, D), generator=g).bfloat16().double()
    kd1 = torch.randn((bt, Hkv, D), generator=g).bfloat16().double()
    vd = torch.zeros((bt, N, Hkv, D), dtype=torch.float64)
    want, size, reach = np.zeros((bt, Hkv, D)), np.zeros((bt, Hkv, D)), np.zeros((bt, Hkv))
    for b, L in enumerate(lens):
        for i in range(Hkv):
            K, V, qq = k[b, i, :L], v[b, i, :L], q1[b, i].numpy()
            z, zd = K @ qq / math.sqrt(D), float(kd1[b, i].numpy() @ qq) / math.sqrt(D)
            top = max([zd] + z.tolist())
            w, wd = np.exp(z - top), math.exp(zd - top)
            rest = w @ V if L else np.zeros((D,))
            size[b, i] = w @ np.abs(V) if L else 0
            for j in range(N - 1):
                x = torch.from_numpy(-rest / wd).bfloat16().double()
                vd[b, j, i] = x
                rest = rest + wd * x.numpy()
                size[b, i] += wd * np.abs(x.numpy())
            den = w.sum() + N * wd
            want[b, i], size[b, i] = rest / den, size[b, i] / den
            reach[b, i] = max((np.abs(K) @ np.abs(qq)).max() if L else 0, float(np.abs(kd1[b, i].numpy()) @ np.abs(qq))) / math.sqrt(D)
    q = q1[:, None, :, None].expand(bt, N, Hkv, G, D).reshape(bt, N, Hkv * G, D).to(dtype).contiguous().cuda()
    kd = kd1[:, None].expand(bt, N, Hkv, D).to(dtype).contiguous().cuda()
    tree = sp.Tree(q, kd, vd.to(dtype).cuda(), torch.arange(-1, N - 1, dtype=torch.int32, device="cuda").expand(bt, N).contiguous())
    idx = cnt = None
    if kept:
        idx = torch.arange(T // B, dtype=torch.int32, device="cuda").expand(bt, Hkv, T // B).contiguous()
        cnt = torch.full((bt, Hkv), T // B, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    ws = torch.zeros((sp.specpv_packed_workspace_bytes(h, tree, sp.SelectCfg(0, 0, T // B)),), dtype=torch.uint8, device="cuda")
    sp.specpv_packed_verify_attn(h, tree, idx, cnt, out, None, ws)
    got = out[:, N - 1].double().cpu().numpy().reshape(bt, Hkv, G, D)
    for b, L in enumerate(lens):
        bound = size[b] * (2 * ref.score_error(reach[b], D)[:, None] + 2.0 ** -23 + (L + N + 64) * 2.0 ** -24) + np.abs(want[b]) * ref.half_step(dtype)
        e = np.abs(got[b] - want[b][:, None]).max(1)
        assert (e <= bound).all(), (b, float((e / np.maximum(bound, 1e-300)).max()), float((e / np.maximum(size[b], 1e-300)).max()))
