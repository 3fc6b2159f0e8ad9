"""Eviction by accumulated weight: kept tokens, their rows and weights, exactly."""
import numpy as np
import pytest
import torch

import compact_reference as ref

pytestmark = pytest.mark.gpu


def run(sp, w, lens, ns, nr, k, dtype=torch.bfloat16, D=64, B=16, layout="bhtd", dst_B=24, spare=30, with_weights=True, seed=0, ws=None):
    """w [batch, Hkv, T] on the host.  Checks everything and returns keep_idx."""
    batch, Hkv, T = w.shape
    g = torch.Generator().manual_seed(seed)
    kk, vv = (torch.randn((batch, Hkv, T, D), generator=g).to(dtype) for _ in "kv")
    dev = lambda t: (t if layout == "bhtd" else t.permute(0, 2, 1, 3)).contiguous().cuda()  # noqa: E731
    src = sp.KV(dev(kk), dev(vv), torch.tensor(lens, dtype=torch.int32, device="cuda"), B, layout=layout)
    n = ns + nr + k
    cap = -(-(n + spare) // dst_B) * dst_B
    old = [torch.full((batch, Hkv, cap, D), 5.0, dtype=dtype) for _ in "kv"]
    dst = sp.KV(dev(old[0]), dev(old[1]), torch.full((batch,), -9, dtype=torch.int32, device="cuda"), dst_B, layout=layout)
    idx = torch.full((batch, Hkv, n), -7, dtype=torch.int32, device="cuda")
    nw = torch.full((batch, Hkv, cap), 4.0, device="cuda") if with_weights else None
    ws = torch.zeros((sp.specpv_evict_workspace_bytes(src),), dtype=torch.uint8, device="cuda") if ws is None else ws
    sp.specpv_evict_tokens(src, w.cuda(), ns, nr, k, dst, idx, nw, ws)
    torch.cuda.synchronize()
    assert not ws[:65536].any()
    got = [x if layout == "bhtd" else x.permute(0, 2, 1, 3) for x in (dst.k, dst.v)]
    got = [x.cpu() for x in got]
    hi, hw = idx.cpu(), None if nw is None else nw.cpu()
    assert dst.ctx_len.tolist() == [min(L, n) for L in lens]
    for b, L in enumerate(lens):
        for h in range(Hkv):
            kept = ref.kept_tokens(w[b, h].tolist(), L, ns, nr, k)
            assert hi[b, h].tolist() == kept + [-1] * (n - len(kept)), (b, h)
            for x, y, o in zip(got, (kk, vv), old):
                assert torch.equal(x[b, h, :len(kept)], y[b, h, kept]) and torch.equal(x[b, h, len(kept):], o[b, h, len(kept):])
            if hw is not None:
                a, c = hw[b, h, :len(kept)], w[b, h, kept]
                assert np.array_equal(a.numpy(), c.numpy(), equal_nan=True) and not hw[b, h, len(kept):].any()
    return idx


def _weights(shape, seed=0):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(2.5 * torch.randn(shape, generator=g) - 6)
    return w * (torch.rand(shape, generator=g) > 0.1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D,layout,B", [(64, "bhtd", 16), (128, "bthd", 16), (128, "bhtd", 7)])
def test_batches(gpu_lib, dtype, D, layout, B):
    T = -(-400 // B) * B
    run(gpu_lib, _weights((4, 2, T)), [400, 61, 60, 0], 4, 16, 41, dtype, D, B, layout)


@pytest.mark.parametrize("ns,nr,k", [(0, 0, 1), (0, 0, 100), (5, 0, 0), (0, 9, 0), (3, 4, 0), (0, 200, 55), (200, 55, 1), (1, 1, 254)])
def test_parts(gpu_lib, ns, nr, k):
    run(gpu_lib, _weights((1, 3, 272), ns + k), [257], ns, nr, k)


@pytest.mark.parametrize("L,k", [(20000, 5000), (20001, 19000), (9000, 1), (131072, 16384), (4097, 4096), (70000, 333)])
def test_long_sequences(gpu_lib, L, k):
    T = -(-L // 16) * 16
    run(gpu_lib, _weights((1, 2, T), k), [L], 4, 64, min(k, L - 69), D=64, with_weights=L % 2 == 0)


@pytest.mark.parametrize("what", ["equal", "zero", "few", "signs", "one bit", "special"])
def test_ties_and_signs(gpu_lib, what):
    """Equal weights go by their place; negative ones (nothing forbids them) and zeros of both signs; infinities; NaN last of all."""
    g = torch.Generator().manual_seed(3)
    T = 6000
    w = {"equal": torch.full((1, 2, T), 0.3), "zero": torch.zeros((1, 2, T)), "few": torch.randint(0, 4, (1, 2, T), generator=g).float() * 0.25,
         "signs": torch.randn((1, 2, T), generator=g).bfloat16().float(), "one bit": 1.0 + torch.randint(0, 3, (1, 2, T), generator=g) * 2.0 ** -23,
         "special": torch.rand((1, 2, T), generator=g)}[what]
    if what in ("zero", "signs"):
        w[..., ::3] = -0.0
        w[..., 1::5] = 0.0
    if what == "special":
        w[0, 0, 7::11], w[0, 0, 100], w[0, 0, 3::13] = float("nan"), float("inf"), -float("inf")
        w[0, 1] = float("nan")
    for ns, nr, k in ((2, 10, 1000), (0, 0, 1), (1, 1, T - 3), (4, 4, 5800)):
        run(gpu_lib, w, [T], ns, nr, k, seed=1)


def test_weights_of_one_exponent(gpu_lib):
    """Keys that differ in their last bits only, and keys spread over all exponents."""
    g = torch.Generator().manual_seed(5)
    near = (torch.full((1, 1, 50000), 0x3f800000, dtype=torch.int32) + torch.randint(0, 700, (1, 1, 50000), generator=g).to(torch.int32)).view(torch.float32)
    far = torch.randint(0, 0x7f800000, (1, 1, 50000), generator=g).to(torch.int32).view(torch.float32)
    for w in (near, far):
        run(gpu_lib, w, [49999], 4, 32, 12345)


def test_one_workspace_many_calls(gpu_lib):
    """Calls of different shapes one after the other in a workspace of the largest."""
    sp = gpu_lib
    ws = torch.zeros((max(65536 * 4, 1 << 22),), dtype=torch.uint8, device="cuda")
    for i, (b, h, T, k) in enumerate([(2, 4, 5008, 700), (1, 1, 160, 20), (3, 2, 20000, 9999), (2, 4, 5008, 701)]):
        run(sp, _weights((b, h, T), i), [T - j for j in range(b)], 4, 8, k, ws=ws)


def test_binding_refuses(gpu_lib):
    sp = gpu_lib
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i1 = lambda: torch.zeros((1,), dtype=torch.int32, device="cuda")  # noqa: E731
    src, dst = sp.KV(z(1, 2, 64, 64), z(1, 2, 64, 64), i1(), 16), sp.KV(z(1, 2, 32, 64), z(1, 2, 32, 64), i1(), 16)
    w, idx = torch.zeros((1, 2, 64), device="cuda"), torch.zeros((1, 2, 20), dtype=torch.int32, device="cuda")
    ws = torch.zeros((sp.specpv_evict_workspace_bytes(src),), dtype=torch.uint8, device="cuda")
    sp.specpv_evict_tokens(src, w, 2, 8, 10, dst, idx, None, ws)
    for a in ((w[..., :48], 2, 8, 10, dst, idx), (w, 2, 8, 11, dst, idx), (w.double(), 2, 8, 10, dst, idx), (w, 2, 8, 10, dst, idx.long()),
              (w, 2, 8, 10, dst, idx, torch.zeros((1, 2, 64), device="cuda")), (w, 2, 8, 10, sp.KV(z(1, 1, 32, 64), z(1, 1, 32, 64), i1(), 16), idx)):
        with pytest.raises(ValueError):
            sp.specpv_evict_tokens(src, *a, **({} if len(a) > 6 else dict(dst_weights=None)), workspace=ws)
    for kw in (dict(dst=src), dict(ws=None), dict(ws=ws[:1000])):
        with pytest.raises(sp.SpecPVError):
            sp.specpv_evict_tokens(src, w, 2, 8, 10, kw.get("dst", dst), idx, None, kw["ws"] if "ws" in kw else ws)


def test_memory_that_ends_inside_the_last_block(gpu_lib):
    """A destination whose blocks would hold the kept tokens, but whose memory does not, is refused."""
    sp = gpu_lib
    z = lambda t: torch.zeros((1, 2, t, 64), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i1 = lambda: torch.zeros((1,), dtype=torch.int32, device="cuda")  # noqa: E731
    src = sp.KV(z(64), z(64), i1(), 16)
    w, idx = torch.zeros((1, 2, 64), device="cuda"), torch.zeros((1, 2, 20), dtype=torch.int32, device="cuda")
    ws = torch.zeros((sp.specpv_evict_workspace_bytes(src),), dtype=torch.uint8, device="cuda")
    sp.specpv_evict_tokens(src, w, 2, 8, 10, sp.KV(z(20), z(20), i1(), 16), idx, None, ws)
    with pytest.raises(ValueError):
        sp.specpv_evict_tokens(src, w, 2, 8, 10, sp.KV(z(19), z(19), i1(), 16), idx, None, ws)
