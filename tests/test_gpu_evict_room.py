"""Evictions that may keep more tokens than the source has room for: every sequence stays whole, and nothing of the rest is touched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_weights", [True, False], ids=["weights", "rows"])
@pytest.mark.parametrize("T,n,stale", [(20000, 32768, 0), (20000, 24577, 5), (16400, 70001, 19999), (4000, 9001, 3), (16384, 16500, 0)])
def test_more_than_the_source_has_room_for(gpu_lib, T, n, stale, with_weights):
    """keep_idx holds token numbers of an earlier call before this one: -1 behind the last kept token takes their place in every entry."""
    sp, B, D, Hkv = gpu_lib, 16, 64, 2
    lens = [T, 17, 0]
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn((3, Hkv, T, D), generator=g, device="cuda").bfloat16() for _ in "kv")
    w = torch.rand((3, Hkv, T), generator=g, device="cuda")
    src = sp.KV(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"), B)
    cap = -(-n // B) * B
    dst = sp.KV(*(torch.full((3, Hkv, cap, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"), torch.full((3,), -9, dtype=torch.int32, device="cuda"), B)
    idx = torch.full((3, Hkv, n), stale, dtype=torch.int32, device="cuda")
    nw = torch.full((3, Hkv, cap), 4.0, device="cuda") if with_weights else None
    ws = torch.zeros((sp.specpv_evict_workspace_bytes(src),), dtype=torch.uint8, device="cuda")
    sp.specpv_evict_tokens(src, w, 4, 100, n - 104, dst, idx, nw, ws)
    assert dst.ctx_len.tolist() == lens
    at = torch.arange(n, device="cuda")
    for b, L in enumerate(lens):
        assert torch.equal(idx[b], torch.where(at < L, at, -1).to(torch.int32).expand(Hkv, n))
        for to, x in ((dst.k, k), (dst.v, v)):
            assert torch.equal(to[b, :, :L], x[b, :, :L]) and (to[b, :, L:] == 5.0).all()
        if with_weights:
            assert torch.equal(nw[b, :, :L], w[b, :, :L]) and not nw[b, :, L:].any()
