"""Rows into the 4-bit cache and out of it: codes, scales and summaries equal to the definition's bit for bit."""
import numpy as np
import pytest
import torch

import compact_reference as ref

pytestmark = pytest.mark.gpu
KEEP = 0x5a


class Target:
    """A packed cache full of a pattern, in a given layout, with unused bytes between its rows."""

    def __init__(self, sp, batch, Hkv, T, D, B, dtype, layout="bhtd", wide=1, lens=None):
        shape = (batch, Hkv, T) if layout == "bhtd" else (batch, T, Hkv)
        self.big = [torch.full(shape + (w * wide,), KEEP, dtype=torch.uint8, device="cuda") for w in (D // 2, D // 2, D // 32, D // 32)]
        self.k, self.v, self.ks, self.vs = (t[..., :t.shape[-1] // wide] for t in self.big)
        self.layout = layout
        self.h = sp.PackedKV(self.k, self.v, self.ks, self.vs, torch.tensor(lens or [T] * batch, dtype=torch.int32, device="cuda"), B, layout=layout, dtype=dtype)

    def host(self):
        t = [x if self.layout == "bhtd" else x.permute(0, 2, 1, 3) for x in (self.k, self.v, self.ks, self.vs)]
        return [x.cpu().numpy() for x in t]


def _source(sp, batch, Hkv, n, D, dtype, layout="bhtd", seed=0, lens=None, scale=True):
    g = torch.Generator().manual_seed(seed)
    x = [torch.randn((batch, Hkv, n, D), generator=g) * (torch.exp(2 * torch.randn((1, Hkv, 1, D), generator=g)) if scale else 1) for _ in "kv"]
    x = [y.to(dtype) for y in x]
    y = [t if layout == "bhtd" else t.permute(0, 2, 1, 3) for t in x]
    y = [t.contiguous().cuda() for t in y]
    lens = torch.tensor(lens or [n] * batch, dtype=torch.int32, device="cuda")
    return sp.KV(y[0], y[1], lens, 16, layout=layout), x[0].double().numpy(), x[1].double().numpy()


def _expect(host, src, place):
    """The target's arrays after rows `place` = [(b, token, source row)] of src = (k, v)."""
    k, v, ks, vs = (a.copy() for a in host)
    for b, t, r in place:
        for g in range(k.shape[1]):
            for c, s, x in ((k, ks, src[0]), (v, vs, src[1])):
                codes, scales = ref.pack_row(x[b, g, r])
                c[b, g, t] = codes[0::2] | (codes[1::2] << 4)
                s[b, g, t] = scales
    return k, v, ks, vs


def _same(target, want):
    for got, w, name in zip(target.host(), want, ("k", "v", "k_scale", "v_scale")):
        assert np.array_equal(got, w), (name, np.argwhere(got != w)[:5].tolist())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout,wide", [("bhtd", 1), ("bthd", 1), ("bhtd", 2)])
def test_whole_cache(gpu_lib, dtype, D, layout, wide):
    sp = gpu_lib
    lens = [37, 0, 1]
    src, k, v = _source(sp, 3, 2, 40, D, dtype, layout, 1, lens)
    t = Target(sp, 3, 2, 48, D, 16, dtype, layout, wide, lens)
    want = _expect(t.host(), (k, v), [(b, i, i) for b in range(3) for i in range(lens[b])])
    sp.specpv_pack_tokens(src, t.h)
    _same(t, want)
    for big in t.big:      # between the rows
        assert wide == 1 or (big[..., big.shape[-1] // 2:] == KEEP).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_ranges_and_counts(gpu_lib, dtype):
    sp = gpu_lib
    src, k, v = _source(sp, 4, 2, 30, 64, dtype, "bhtd", 2, [30, 20, 30, 30])
    t = Target(sp, 4, 2, 40, 64, 8, dtype)
    host = t.host()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    # 5 rows from 7 on to 3; 12 asked for, 2 there; none; six that end behind the cache's last token
    sp.specpv_pack_tokens(src, t.h, dst_begin=i32(3, 0, 5, 37), src_begin=i32(7, 18, 2, 0), n_rows=i32(5, 12, 0, 6), max_rows=30)
    place = [(0, 3 + i, 7 + i) for i in range(5)] + [(1, i, 18 + i) for i in range(2)] + [(3, 37 + i, i) for i in range(3)]
    host = _expect(host, (k, v), place)
    _same(t, host)
    # at most max_rows; a begin in front of the cache: what lies in front of it is left out
    sp.specpv_pack_tokens(src, t.h, dst_begin=i32(20, -3, 20, 20), src_begin=i32(0, 0, 0, 29), max_rows=4)
    place = [(0, 20 + i, i) for i in range(4)] + [(1, 0, 3)] + [(2, 20 + i, i) for i in range(4)] + [(3, 20, 29)]
    _same(t, _expect(host, (k, v), place))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_listed_rows(gpu_lib, dtype, D):
    """Accepted candidates out of a token-major buffer; rows that are not there leave their tokens as they were, a row may come twice."""
    sp = gpu_lib
    src, k, v = _source(sp, 2, 3, 26, D, dtype, "bthd", 3)
    t = Target(sp, 2, 3, 64, D, 24, dtype)
    rows = [[3, 4, 9, 9, -1, 25, 26, 0], [5, 6, 7, 8, 9, 10, 11, 12]]
    n, begin = [8, 3], [20, 61]
    sp.specpv_pack_tokens(src, t.h, dst_begin=torch.tensor(begin, dtype=torch.int32, device="cuda"), src_rows=torch.tensor(rows, dtype=torch.int32, device="cuda"),
                          n_rows=torch.tensor(n, dtype=torch.int32, device="cuda"))
    place = [(b, begin[b] + i, rows[b][i]) for b in range(2) for i in range(n[b]) if 0 <= rows[b][i] < 26]
    fresh = Target(sp, 2, 3, 64, D, 24, dtype)
    _same(t, _expect(fresh.host(), (k, v), place))


def test_every_bf16_value(gpu_lib):
    """Each of the 65536 bf16 values as a group's largest magnitude and under larger ones, and its negative."""
    sp = gpu_lib
    bits = torch.arange(65536, dtype=torch.int32)
    x = bits.to(torch.int16).view(torch.bfloat16)
    rows = torch.zeros((65536, 64), dtype=torch.bfloat16)
    rows[:, 0] = x
    rows[:, 1] = -x
    rows[:, 2] = (x.float() * 0.37).bfloat16()
    rows[:, 32] = x
    rows[:, 33] = (x.float().abs() * 2.6).clamp(max=3e38).bfloat16()     # (NaN stays NaN)
    rows[:, 34] = (x.float() * 0.11).bfloat16()
    rows = rows.view(1, 1, 65536, 64)
    n = torch.tensor([65536], dtype=torch.int32, device="cuda")
    t = Target(sp, 1, 1, 65536, 64, 64, torch.bfloat16)
    sp.specpv_pack_tokens(sp.KV(rows.cuda(), rows.cuda(), n, 64), t.h)
    k, v, ks, vs = t.host()
    assert np.array_equal(k, v) and np.array_equal(ks, vs)
    y = rows.double().numpy()[0, 0].reshape(65536, 2, 32)
    top = np.abs(y).max(-1)
    fine = np.isfinite(y).all(-1)
    with np.errstate(all="ignore"):
        e = np.clip(np.ceil(np.log2(np.maximum(top, 2.0 ** -140) / 7)), -124, 125)
        e = np.where(top > 7 * 2.0 ** e, e + 1, np.where(top <= 7 * 2.0 ** (e - 1), e - 1, e)).clip(-124, 125)
        d = np.abs(np.abs(y)[..., None] / 2.0 ** e[..., None, None] - ref.GRID)
    assert np.array_equal(ks[0, 0], np.where(fine, e + 127, 255))
    best = d.min(-1, keepdims=True)
    first, last = (d == best).argmax(-1), 7 - (d == best)[..., ::-1].argmax(-1)
    code = np.where(first % 2 == 0, first, last) | (np.signbit(y) * 8)
    got = np.stack((k[0, 0] & 15, k[0, 0] >> 4), -1).reshape(65536, 2, 32)
    assert np.array_equal(got[fine], code[fine])
    # and back: bf16 holds every value, NaN where the group had none
    out = torch.zeros((1, 1, 65536, 64), dtype=torch.bfloat16, device="cuda")
    sp.specpv_packed_gather_blocks(t.h, None, None, out, torch.zeros_like(out))
    want = ref.unpack(k[0, 0], ks[0, 0])
    assert np.array_equal(out[0, 0].double().cpu().numpy(), want, equal_nan=True)
    assert np.isnan(want.reshape(65536, 2, 32)).all(-1)[~fine].all()


@pytest.mark.parametrize("dtype,D,Bk", [(torch.bfloat16, 128, 16), (torch.bfloat16, 64, 64), (torch.float32, 128, 24), (torch.float32, 64, 1), (torch.bfloat16, 128, 100),
                                        (torch.float32, 64, 300)])
def test_summaries(gpu_lib, dtype, D, Bk):
    """Two calls one behind the other, the second in the middle of a block: the summaries of block_summarize over the same keys."""
    sp = gpu_lib
    lens = [333, 70]
    src, k, _ = _source(sp, 2, 2, 340, D, dtype, "bhtd", 5, lens)
    T = -(-340 // Bk) * Bk
    t = Target(sp, 2, 2, T, D, Bk, dtype)
    full = sp.KV(src.k, src.v, src.ctx_len, Bk)
    want = [torch.full(full.summary_shape(), 7.0, dtype=dtype, device="cuda") for _ in "xn"]
    got = [torch.full(t.h.summary_shape(), 7.0, dtype=dtype, device="cuda") for _ in "xn"]
    sp.specpv_block_summarize(full, 0, -1, *want)
    cut = torch.tensor([111, 70], dtype=torch.int32, device="cuda")
    sp.specpv_pack_tokens(src, t.h, n_rows=cut, kmax=got[0], kmin=got[1])
    sp.specpv_pack_tokens(src, t.h, dst_begin=cut, src_begin=cut, kmax=got[0], kmin=got[1])
    nb = full.max_blocks
    for a, b in zip(got, want):
        assert torch.equal(a[:, :, :nb], b) and (a[:, :, nb:] == 7.0).all()
    assert np.array_equal(t.host()[0][0, :, :333], _expect(t.host(), (k, k), [(0, i, i) for i in range(333)])[0][0, :, :333])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D,Bk,layout,gap", [(128, 64, "bhtd", 0), (64, 24, "bthd", 0), (128, 7, "bhtd", 5)])
def test_gather(gpu_lib, dtype, D, Bk, layout, gap):
    sp = gpu_lib
    T = 11 * Bk
    lens = [T - 3, Bk + 1, 0]
    h, k, v = ref.cache(sp, 3, 2, T, D, Bk, dtype, layout, gap, seed=4, lens=lens)
    idx = torch.tensor([[[0, 5, 10, -1, 3, 99], [10, 10, 2, 0, 1, 4]], [[0, 1, 2, 3, 4, 5], [1, 0, -5, 7, 7, 7]], [[0, 0, 0, 0, 0, 0], [1, 2, 3, 4, 5, 6]]],
                       dtype=torch.int32, device="cuda")
    cnt = torch.tensor([[5, 6], [6, 2], [6, 0]], dtype=torch.int32, device="cuda")
    out = [torch.full((3, 2, 6 * Bk, D), 9.0, dtype=dtype, device="cuda") for _ in "kv"]
    ln = torch.full((3,), -1, dtype=torch.int32, device="cuda")
    sp.specpv_packed_gather_blocks(h, idx, cnt, out[0], out[1], ln)
    most = [0, 0, 0]
    for b in range(3):
        for g in range(2):
            want = np.zeros((2, 6 * Bk, D))
            for i in range(int(cnt[b, g])):
                e = int(idx[b, g, i])
                n = min(Bk, lens[b] - e * Bk)
                if e < 0 or n <= 0:
                    continue
                want[0, i * Bk:i * Bk + n], want[1, i * Bk:i * Bk + n] = k[b, g, e * Bk:e * Bk + n], v[b, g, e * Bk:e * Bk + n]
                most[b] = max(most[b], i * Bk + n)
            for o, w in zip(out, want):
                assert np.array_equal(o[b, g].double().cpu().numpy(), w), (b, g)
    assert ln.tolist() == most
    out = [torch.full((3, 2, T, D), 9.0, dtype=dtype, device="cuda") for _ in "kv"]
    sp.specpv_packed_gather_blocks(h, None, None, out[0], out[1], ln)
    for b in range(3):
        for o, w in zip(out, (k, v)):
            assert np.array_equal(o[b, :, :lens[b]].double().cpu().numpy(), w[b, :, :lens[b]]) and not o[b, :, lens[b]:].any()
    assert ln.tolist() == lens


@pytest.mark.parametrize("dtype,Bk", [(torch.bfloat16, 32), (torch.float32, 48), (torch.bfloat16, 64), (torch.float32, 128)])
def test_more_blocks_than_workgroups(gpu_lib, dtype, Bk):
    """A long prompt in two calls, cut inside a block: codes as from a cache of blocks of 16, summaries as from block_summarize."""
    sp = gpu_lib
    n = 9000
    src, _, _ = _source(sp, 2, 4, n, 64, dtype, "bthd", 6, [n, n - 700])
    T = -(-n // 384) * 384
    a, b = Target(sp, 2, 4, T, 64, Bk, dtype), Target(sp, 2, 4, T, 64, 16, dtype)
    cut = torch.tensor([4501, 4501], dtype=torch.int32, device="cuda")
    got = [torch.full(a.h.summary_shape(), 7.0, dtype=dtype, device="cuda") for _ in "xn"]
    want = [torch.full(a.h.summary_shape(), 7.0, dtype=dtype, device="cuda") for _ in "xn"]
    sp.specpv_pack_tokens(src, a.h, n_rows=cut, kmax=got[0], kmin=got[1])
    sp.specpv_pack_tokens(src, a.h, dst_begin=cut, src_begin=cut, kmax=got[0], kmin=got[1])
    sp.specpv_pack_tokens(src, b.h)
    for x, y in zip(a.host(), b.host()):
        assert np.array_equal(x, y)
    whole = [torch.zeros((2, T, 4, 64), dtype=dtype, device="cuda") for _ in "kv"]
    for x, y in zip(whole, (src.k, src.v)):
        x[:, :n] = y if y.shape[1] == n else y.permute(0, 2, 1, 3)
    sp.specpv_block_summarize(sp.KV(whole[0], whole[1], src.ctx_len, Bk, layout="bthd"), 0, -1, *want)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_length_beyond_the_source(gpu_lib):
    """A source whose length claims more rows than it has room for gives those that it has."""
    sp = gpu_lib
    src, k, v = _source(sp, 1, 2, 16, 64, torch.bfloat16, "bhtd", 8, [40])
    t = Target(sp, 1, 2, 48, 64, 16, torch.bfloat16)
    want = _expect(t.host(), (k, v), [(0, i, i) for i in range(16)])
    sp.specpv_pack_tokens(src, t.h, max_rows=40)
    _same(t, want)
    rows = torch.tensor([[20, 15, 16, 39]], dtype=torch.int32, device="cuda")
    sp.specpv_pack_tokens(src, t.h, src_rows=rows, dst_begin=torch.tensor([30], dtype=torch.int32, device="cuda"))
    _same(t, _expect(want, (k, v), [(0, 31, 15)]))


def test_memory_that_ends_inside_the_last_block(gpu_lib):
    """Rows that max_blocks counts and the allocation does not have are not written."""
    sp = gpu_lib
    src, k, v = _source(sp, 1, 2, 60, 64, torch.bfloat16, "bhtd", 9)
    big = [torch.full((1, 2, 60, w), KEEP, dtype=torch.uint8, device="cuda") for w in (32, 32, 2, 2)]
    h = sp.PackedKV(*(t[:, :, :40] for t in big), torch.zeros((1,), dtype=torch.int32, device="cuda"), 24, dtype=torch.bfloat16)
    assert h.max_blocks * h.B == 48
    kmax, kmin = (torch.zeros(h.summary_shape(), dtype=torch.bfloat16, device="cuda") for _ in "xn")
    sp.specpv_pack_tokens(src, h, kmax=kmax, kmin=kmin)
    want = _expect([np.full(t.shape, KEEP, dtype=np.uint8) for t in big], (k, v), [(0, i, i) for i in range(40)])
    for t, w in zip(big, want):
        assert np.array_equal(t.cpu().numpy(), w)
    assert np.array_equal(kmax[0, :, 1].double().cpu().numpy(), k[0, :, 24:40].max(1))
