"""Infinite keys, and query rows that count for nothing whatever is in them: no NaN where the definition has a number."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# every form of the kernel: one to sixteen wavefronts to the tokens, rows that fill no tile of 32 and rows that do
CASES = [(torch.bfloat16, 128, 1, 4, 1, 1, 64), (torch.float32, 64, 1, 10, 2, 13, 300), (torch.float32, 128, 1, 4, 1, 5, 96), (torch.bfloat16, 128, 2, 10, 2, 27, 500),
         (torch.bfloat16, 64, 1, 16, 1, 33, 260), (torch.float32, 128, 1, 8, 2, 30, 320), (torch.bfloat16, 128, 1, 8, 2, 32, 900), (torch.bfloat16, 128, 4, 12, 4, 49, 16384),
         (torch.float32, 64, 2, 12, 4, 33, 16384), (torch.bfloat16, 128, 4, 12, 4, 61, 8192), (torch.bfloat16, 64, 2, 12, 4, 33, 16384)]


def _case(dtype, D, batch, Hq, Hkv, M, T, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + M)
    q = torch.randn((batch, M, Hq, D), generator=g, device="cuda").abs().clamp(min=0.01).to(dtype)      # (an infinite key's products have its sign)
    k = torch.randn((batch, Hkv, T, D), generator=g, device="cuda").to(dtype)
    lse = torch.rand((batch, M, Hq), generator=g, device="cuda") + 9.0
    return q, k, lse, torch.rand((batch, Hkv, T), generator=g, device="cuda")


def _run(sp, q, k, lse, w, **over):
    T = k.shape[2]
    room = torch.zeros(w.shape[:2] + (-(-T // 16) * 16,), device="cuda")      # (whole blocks)
    room[..., :T] = w
    kv = sp.KV(k, k, torch.full((q.shape[0],), T, dtype=torch.int32, device="cuda"), 16)
    sp.specpv_accumulate_weights(kv, sp.Tree(q), lse, room, **over)
    assert not room[..., T:].any()
    return room[..., :T].contiguous()


def _lists(k):
    n = -(-k.shape[2] // 16)
    idx = torch.arange(n, dtype=torch.int32, device="cuda").expand(k.shape[0], k.shape[1], n).contiguous()
    return dict(sel_idx=idx, sel_count=torch.full(k.shape[:2], n, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("lists", [False, True], ids=["whole", "lists"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_infinite_keys(gpu_lib, case, lists):
    """exp(-inf - lse) = 0 for keys whose products are all -inf, exp(inf - lse) = inf for +inf; the other tokens' bits are those beside finite keys."""
    sp = gpu_lib
    q, k, lse, w = _case(*case)
    T, over = k.shape[2], _lists(k) if lists else {}
    want = _run(sp, q, k, lse, w, **over)
    low, high = torch.arange(3, T, 37, device="cuda"), torch.arange(5, T, 41, device="cuda")
    k[:, :, low, 7] = -float("inf")
    k[:, :, high, 11] = float("inf")
    both = torch.isin(low, high)
    got = _run(sp, q, k, lse, w, **over)
    assert torch.equal(got[:, :, low[~both]], w[:, :, low[~both]])
    only = high[~torch.isin(high, low)]
    assert (got[:, :, only] == float("inf")).all()
    rest = torch.ones((T,), dtype=torch.bool, device="cuda")
    rest[low], rest[high] = False, False
    assert torch.equal(got[:, :, rest], want[:, :, rest]) and torch.isfinite(want).all()


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_rows_that_give_nothing(gpu_lib, case):
    """Rows of padding: their log-sum-exp is -inf, and what stands in their query rows may be anything.  Bits as of zeros there."""
    sp = gpu_lib
    q, k, lse, w = _case(*case, seed=50)
    M, Hq = q.shape[1:3]
    dead = torch.rand((q.shape[0], M, Hq), generator=torch.Generator().manual_seed(1)) < 0.4
    dead[0, 0, 0] = True
    dead = dead.cuda()
    lse = torch.where(dead, -float("inf"), lse)
    q = torch.where(dead[..., None], 0.0, q)
    want = _run(sp, q, k, lse, w)
    assert torch.isfinite(want).all()
    for bad in (float("nan"), float("inf"), -float("inf")):
        got = _run(sp, torch.where(dead[..., None], bad, q), k, lse, w)
        assert torch.equal(got, want), bad


def test_nodes_that_are_none(gpu_lib):
    """Entries outside the tree beside infinite keys."""
    sp = gpu_lib
    q, k, lse, w = _case(torch.bfloat16, 128, 2, 8, 2, 9, 200)
    k[:, :, 50, 3] = -float("inf")
    nodes = torch.tensor([[0, -1, 3, 99], [-5, 8, 8, 2]], dtype=torch.int32, device="cuda")
    n = torch.tensor([4, 3], dtype=torch.int32, device="cuda")
    got = _run(sp, q, k, lse, w, nodes=nodes, n_nodes=n)
    assert torch.isfinite(got).all() and torch.equal(got[:, :, 50], w[:, :, 50]) and (got[:, :, 49] > w[:, :, 49]).all()


def test_an_infinite_sum_beside_infinite_products(gpu_lib):
    """A row whose log-sum-exp is +inf weighs finite keys nothing, and exp(inf - inf) is no number."""
    sp = gpu_lib
    q, k, lse, w = _case(torch.float32, 64, 1, 4, 2, 3, 40)
    lse[0, 1, 1] = float("inf")
    k[0, 0, 8, 0] = float("inf")
    got = _run(sp, q, k, lse, w)
    assert got[0, 0, 8].isnan() and torch.isfinite(got[0, 0, :8]).all() and torch.isfinite(got[0, 0, 9:]).all() and torch.isfinite(got[0, 1]).all()
