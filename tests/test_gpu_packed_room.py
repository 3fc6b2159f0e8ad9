"""Packed caches whose memory ends inside their last block, and lengths that claim more: the rows that there are, and no others."""
import pytest
import torch

import compact_reference as ref
from test_gpu_packed_attn import _lists, _tree, check

pytestmark = pytest.mark.gpu


def _cut(sp, batch, Hkv, T, room, D, B, dtype, layout, lens):
    """A cache of T rows whose allocation goes on for `room` rows in all, NaNs under large scales among them."""
    h, k, v = ref.cache(sp, batch, Hkv, room, D, B, dtype, layout, seed=T, lens=lens)
    t_dim = 2 if layout == "bhtd" else 1
    for s in (h.k_scale, h.v_scale):
        s.narrow(t_dim, T, room - T).fill_(255)
    cut = lambda x: x.narrow(t_dim, 0, T)  # noqa: E731
    return sp.PackedKV(*(cut(x) for x in (h.k, h.v, h.k_scale, h.v_scale)), h.ctx_len, B, layout=layout, dtype=dtype), k, v


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D,B,layout,T,lens", [(64, 24, "bhtd", 40, [45, 40, 39]), (128, 64, "bthd", 700, [2 ** 31 - 1, 703, 5]), (128, 1024, "bhtd", 1000, [1024, 1001, 0]),
                                               (64, 32, "bhtd", 33, [64, 63, 33])])
def test_attention(gpu_lib, dtype, D, B, layout, T, lens):
    sp = gpu_lib
    nb = -(-T // B)
    h, k, v = _cut(sp, 3, 2, T, nb * B, D, B, dtype, layout, lens)
    assert h.max_blocks == nb and h.c.tokens == T
    tree, tv, parent = _tree(sp, 3, 7, 0, 4, 2, D, dtype, T)
    ws = torch.zeros((sp.specpv_packed_workspace_bytes(h, tree, sp.SelectCfg(0, 0, nb + 1)),), dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(tree.q) for _ in "ab"]
    sp.specpv_packed_verify_attn(h, tree, None, None, out[0], None, ws)
    check(sp, _handle(sp, h, T), (k, v), tree, tv, parent)
    sp.specpv_packed_verify_attn(_handle(sp, h, T), tree, None, None, out[1], None, ws)
    assert torch.equal(*out) and torch.isfinite(out[0]).all()
    idx, cnt = _lists(3, 2, [[list(range(nb))[::-1] + [nb], [nb - 1]] for _ in lens])
    sp.specpv_packed_verify_attn(h, tree, idx, cnt, out[0], None, ws)
    sp.specpv_packed_verify_attn(_handle(sp, h, T), tree, idx, cnt, out[1], None, ws)
    assert torch.equal(*out) and torch.isfinite(out[0]).all()


def _handle(sp, h, T):
    """The same cache under lengths that its memory has room for."""
    return sp.PackedKV(h.k, h.v, h.k_scale, h.v_scale, h.ctx_len.clamp(max=T), h.B, layout="bhtd" if h.k.shape[1] == h.Hkv else "bthd", dtype=h.dtype)


@pytest.mark.parametrize("dtype,D,M,Hq,T,lens", [(torch.bfloat16, 128, 2, 4, 91500, [91520, 91501, 40000]), (torch.float32, 64, 60, 10, 13000, [2 ** 30, 1, 13056]),
                                                 (torch.bfloat16, 64, 128, 16, 5690, [5696, 33, 700])])
def test_shares_of_batches(gpu_lib, dtype, D, M, Hq, T, lens):
    sp = gpu_lib
    nb = -(-T // 64)
    h, k, v = _cut(sp, 3, 2 if Hq < 16 else 1, T, nb * 64, D, 64, dtype, "bhtd", lens)
    tree, tv, parent = _tree(sp, 3, M, 0, Hq, h.Hkv, D, dtype, M)
    ws = torch.zeros((sp.specpv_packed_workspace_bytes(h, tree),), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(tree.q), torch.zeros(tree.q.shape[:3], device="cuda")
    sp.specpv_packed_verify_attn(h, tree, None, None, out, lse, ws)
    want, want_lse = check(sp, _handle(sp, h, T), (k, v), tree, tv, parent)
    # (the shares are dealt by whole blocks, which both lengths have as many of)
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gather(gpu_lib, dtype):
    sp = gpu_lib
    T, B, D = 40, 24, 64
    h, k, v = _cut(sp, 2, 2, T, 48, D, B, dtype, "bhtd", [45, 30])
    idx, cnt = _lists(2, 2, [[[1, 0], [1]], [[0, 1], [1, 2]]])
    n = idx.shape[-1]
    for sel in (None, idx):
        rows = (2 if sel is None else n) * B
        got, want = ([torch.full((2, 2, rows, D), 9.0, dtype=dtype, device="cuda") for _ in "kv"] + [torch.full((2,), -1, dtype=torch.int32, device="cuda")] for _ in "ab")
        sp.specpv_packed_gather_blocks(h, sel, None if sel is None else cnt, *got)
        sp.specpv_packed_gather_blocks(_handle(sp, h, T), sel, None if sel is None else cnt, *want)
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[0]).all()
        assert got[2].tolist() == ([40, 30] if sel is None else [48, 30])      # (the list [1, 0] ends with a whole block)
    whole = [torch.full((2, 2, 48, D), 9.0, dtype=dtype, device="cuda") for _ in "kv"]
    sp.specpv_packed_gather_blocks(h, None, None, *whole)
    for o, x in zip(whole, (k, v)):
        assert torch.equal(o[0, :, :40].double().cpu(), torch.from_numpy(x[0, :, :40])) and not o[0, :, 40:].any()


def test_a_cache_that_fills_up(gpu_lib):
    """Rows appended past the end are left out while the caller's length moves on: attention goes by what is there."""
    sp = gpu_lib
    T, B, D = 40, 24, 64
    h, _, _ = _cut(sp, 1, 2, T, 48, D, B, torch.bfloat16, "bhtd", [30])
    g = torch.Generator().manual_seed(2)
    x = [torch.randn((1, 2, 15, D), generator=g).bfloat16().cuda() for _ in "kv"]
    sp.specpv_pack_tokens(sp.KV(x[0], x[1], torch.tensor([15], dtype=torch.int32, device="cuda"), 16), h, dst_begin=h.ctx_len)
    h.ctx_len.add_(15)
    tree, tv, parent = _tree(sp, 1, 5, 0, 4, 2, D, torch.bfloat16, 3)
    vals = [torch.from_numpy(ref.unpack(c.cpu().numpy(), s.cpu().numpy())) for c, s in ((h.k, h.k_scale), (h.v, h.v_scale))]
    want, lse = check(sp, _handle(sp, h, T), [a.numpy() for a in vals], tree, tv, parent)
    ws = torch.zeros((sp.specpv_packed_workspace_bytes(h, tree),), dtype=torch.uint8, device="cuda")
    out, l = torch.zeros_like(want), torch.zeros_like(lse)
    sp.specpv_packed_verify_attn(h, tree, None, None, out, l, ws)
    assert torch.equal(out, want) and torch.equal(l, lse)
