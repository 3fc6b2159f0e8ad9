"""Accumulated attention weights against 64 bits."""
import numpy as np
import pytest
import torch

import compact_reference as ref

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, sp, dtype, D, Hq, Hkv, M, B, lens, layout="bhtd", n_key=0, seed=0):
        g = torch.Generator().manual_seed(seed)
        batch = len(lens)
        T = -(-max(max(lens), 1) // B) * B
        self.q = torch.randn((batch, M, Hq, D), generator=g).to(dtype)
        self.k = torch.randn((batch, Hkv, T, D), generator=g).to(dtype)
        k = self.k if layout == "bhtd" else self.k.permute(0, 2, 1, 3).contiguous()
        k = k.cuda()
        self.kv = sp.KV(k, k, torch.tensor(lens, dtype=torch.int32, device="cuda"), B, layout=layout)
        parent = torch.arange(-1, M + n_key - 1, dtype=torch.int32).expand(batch, -1).contiguous().cuda() if n_key else None
        self.tree = sp.Tree(self.q.cuda(), parent=parent)
        self.lse = (torch.randn((batch, M, Hq), generator=g) * 0.3 + np.log(max(max(lens), 1))).float()
        self.lens, self.T, self.G = lens, T, Hq // Hkv
        self.w = torch.rand((batch, Hkv, T), generator=g)

    def check(self, sp, nodes=None, n_nodes=None, idx=None, cnt=None):
        w = self.w.cuda()
        lse = self.lse.cuda()
        sp.specpv_accumulate_weights(self.kv, self.tree, lse, w, nodes, n_nodes, idx, cnt)
        got = w.double().cpu().numpy()
        before, q, k, ls = self.w.double().numpy(), self.q.double().numpy(), self.k.double().numpy(), self.lse.double().numpy()
        for b, L in enumerate(self.lens):
            rows = range(q.shape[1])
            if nodes is not None:
                rows = [r for r in nodes[b, :max(0, int(n_nodes[b]))].tolist() if 0 <= r < q.shape[1]]
            for g in range(got.shape[1]):
                h = slice(g * self.G, (g + 1) * self.G)
                t = ref.listed_tokens(L, self.kv.B, None if idx is None else idx[b, g].tolist(), None if cnt is None else cnt[b, g])
                add, off = ref.weights_of(q[b, :, h], k[b, g], ls[b, :, h], rows, t, self.T)
                # the weights' own error; as many roundings as there are rows, and one for each addition to what was there
                n = len(rows) * self.G + 2
                bound = off + add * n * 2.0 ** -24 + (before[b, g] + add) * 4 * 2.0 ** -24
                e = np.abs(got[b, g] - before[b, g] - add)
                assert (e <= bound).all(), (b, g, float(e.max()), int((e > bound).sum()))
                untouched = np.setdiff1d(np.arange(self.T), t)
                assert np.array_equal(got[b, g][untouched], before[b, g][untouched])
        return w


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,M,B,lens,layout", [(4, 1, 1, 16, [1], "bhtd"), (10, 2, 13, 24, [300, 0, 33], "bthd"), (3, 3, 40, 64, [513], "bhtd"), (16, 1, 20, 7, [260, 259], "bhtd")])
def test_every_row(gpu_lib, dtype, D, Hq, Hkv, M, B, lens, layout):
    Case(gpu_lib, dtype, D, Hq, Hkv, M, B, lens, layout, seed=M).check(gpu_lib)


@pytest.mark.parametrize("dtype,M,Hq", [(torch.bfloat16, 128, 16), (torch.float32, 110, 8)])
def test_more_rows_than_fit_at_a_time(gpu_lib, dtype, M, Hq):
    Case(gpu_lib, dtype, 128, Hq, 1, M, 64, [200], seed=1).check(gpu_lib)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_nodes_and_lists(gpu_lib, dtype):
    c = Case(gpu_lib, dtype, 128, 8, 2, 9, 16, [150, 40, 20], n_key=4, seed=2)
    nodes = torch.tensor([[0, 3, 3, 8, -1], [9, 2, 1, 100, 4], [0, 1, 2, 3, 4]], dtype=torch.int32, device="cuda")
    n = torch.tensor([5, 3, 0], dtype=torch.int32, device="cuda")
    c.check(gpu_lib, nodes, n)
    idx = torch.tensor([[[9, 0, 0, 4, -1, 99], [1, 2, 3, 4, 5, 6]], [[2, 1, 0, 3, 0, 0], [0, 0, 0, 0, 0, 0]], [[0, 1, 2, 3, 4, 5], [1, 0, 0, 0, 0, 0]]],
                       dtype=torch.int32, device="cuda")
    cnt = torch.tensor([[6, 6], [4, 0], [2, 1]], dtype=torch.int32, device="cuda")
    c.check(gpu_lib, nodes, n, idx, cnt)
    c.check(gpu_lib, None, None, idx, cnt)


def test_lists_of_single_tokens(gpu_lib):
    c = Case(gpu_lib, torch.bfloat16, 64, 4, 1, 3, 1, [500], seed=3)
    idx = torch.randperm(500, generator=torch.Generator().manual_seed(1))[:301].to(torch.int32).view(1, 1, 301).cuda()
    c.check(gpu_lib, idx=idx, cnt=torch.tensor([[300]], dtype=torch.int32, device="cuda"))


def test_infinite_sums(gpu_lib):
    """A row that attended nothing (-inf) adds nothing, one whose sum is infinite weighs nothing, NaN stays with its KV head."""
    sp = gpu_lib
    c = Case(sp, torch.bfloat16, 64, 4, 2, 2, 16, [70], seed=4)
    c.lse[0, 0, 0], c.lse[0, 1, 1] = -np.inf, np.inf
    c.check(sp)
    c.lse[0, 0, 3] = float("nan")
    w = c.w.cuda()
    sp.specpv_accumulate_weights(c.kv, c.tree, c.lse.cuda(), w)
    assert w[0, 1, :70].isnan().all() and not w[0, 0].isnan().any() and not w[0, 1, 70:].isnan().any()


def test_rows_behind_the_sequence(gpu_lib):
    """NaN keys that the sequence does not have change nothing."""
    sp = gpu_lib
    c = Case(sp, torch.float32, 128, 4, 1, 5, 16, [37], seed=5)
    c.kv.k[:, :, 37:] = float("nan")
    c.check(sp)


def test_the_same_bits_twice(gpu_lib):
    sp = gpu_lib
    c = Case(sp, torch.bfloat16, 128, 8, 2, 30, 16, [900], seed=6)
    idx = torch.randint(0, 57, (1, 2, 80), generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()   # blocks twice and more
    cnt = torch.full((1, 2), 80, dtype=torch.int32, device="cuda")
    runs = [c.check(sp, idx=idx, cnt=cnt) for _ in range(3)]
    assert all(torch.equal(r, runs[0]) for r in runs)


def test_binding_refuses(gpu_lib):
    sp = gpu_lib
    c = Case(sp, torch.bfloat16, 64, 4, 2, 3, 16, [30])
    w, lse = c.w.cuda(), c.lse.cuda()
    nodes, n = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.ones((1,), dtype=torch.int32, device="cuda")
    for bad in ((lse[:, :2], w, None, None), (lse.double(), w, None, None), (lse, w[..., :16], None, None), (lse, w, nodes, None), (lse, w, None, n), (lse, w, nodes.long(), n),
                (lse, w, nodes[0], n)):
        with pytest.raises(ValueError):
            sp.specpv_accumulate_weights(c.kv, c.tree, *bad)


@pytest.mark.parametrize("dtype,D,batch,Hq,M,layout", [(torch.bfloat16, 128, 4, 6, 43, "bhtd"), (torch.bfloat16, 128, 8, 16, 40, "bthd"), (torch.float32, 128, 4, 8, 33, "bhtd"),
                                                       (torch.bfloat16, 64, 16, 6, 43, "bthd"), (torch.float32, 64, 16, 10, 40, "bhtd")])
def test_many_rows_of_many_tokens(gpu_lib, dtype, D, batch, Hq, M, layout):
    """128 rows and more for room enough to give every CU tokens, most of it not used; whole caches, some rows, and lists."""
    T = 8192
    c = Case(gpu_lib, dtype, D, Hq, 2, M, 16, [T - 1, 100, 0, 33] + [5] * (batch - 4), layout, seed=M + D)
    c.check(gpu_lib)
    g = torch.Generator().manual_seed(7)
    nodes = torch.randint(-2, M + 2, (batch, M + 3), generator=g).to(torch.int32).cuda()
    n = torch.randint(0, M + 4, (batch,), generator=g).to(torch.int32)
    n[0] = M + 3
    idx = torch.randint(-1, T // 16 + 1, (batch, 2, T // 16), generator=g).to(torch.int32)
    idx[1:, :, 1::2] = 0
    cnt = torch.randint(0, T // 16 + 1, (batch, 2), generator=g).to(torch.int32)
    c.check(gpu_lib, nodes, n.cuda())
    c.check(gpu_lib, idx=idx.cuda(), cnt=cnt.cuda())


@pytest.mark.parametrize("dtype,D,Hq,M,lens,layout", [(torch.bfloat16, 128, 6, 33, [700, 0, 33], "bhtd"), (torch.bfloat16, 64, 16, 100, [65], "bthd"), (torch.float32, 128, 8, 64, [321, 32], "bthd"),
                                                      (torch.float32, 64, 10, 128, [1, 200], "bhtd")])
def test_many_rows_of_few_tokens(gpu_lib, dtype, D, Hq, M, lens, layout):
    """Wavefronts that share the rows of the same tokens: whole caches, some rows, lists with blocks twice."""
    c = Case(gpu_lib, dtype, D, Hq, 2, M, 16, lens, layout, seed=M)
    c.check(gpu_lib)
    g = torch.Generator().manual_seed(8)
    n = torch.tensor([M, M // 2 + 1, 0][:len(lens)], dtype=torch.int32, device="cuda")
    c.check(gpu_lib, torch.randint(-1, M + 1, (len(lens), M), generator=g).to(torch.int32).cuda(), n)
    idx = torch.randint(-1, max(lens) // 16 + 2, (len(lens), 2, 7), generator=g).to(torch.int32).cuda()
    cnt = torch.randint(0, 8, (len(lens), 2), generator=g).to(torch.int32).cuda()
    c.check(gpu_lib, idx=idx, cnt=cnt)
