"""Evictions from sources with room for more than 16384 tokens (a first digit, candidates, threshold and places in launches of their own):
ties, signs, infinities and NaN across the workgroups' 4096 tokens, and more chunks of those than a workgroup has threads."""
import pytest
import torch

from test_gpu_evict import run

pytestmark = pytest.mark.gpu


def _special(what, T):
    g = torch.Generator().manual_seed(T)
    w = {"equal": torch.full((1, 2, T), 0.3), "zero": torch.zeros((1, 2, T)), "few": torch.randint(0, 4, (1, 2, T), generator=g).float() * 0.25,
         "signs": torch.randn((1, 2, T), generator=g).bfloat16().float(), "negative": -torch.rand((1, 2, T), generator=g),
         "one bit": 1.0 + torch.randint(0, 3, (1, 2, T), generator=g) * 2.0 ** -23, "special": torch.rand((1, 2, T), generator=g)}[what]
    if what in ("zero", "signs"):
        w[..., ::3] = -0.0
        w[..., 1::5] = 0.0
    if what == "special":
        w[0, 0, 7::11], w[0, 0, 100], w[0, 0, T - 300], w[0, 0, 3::13] = float("nan"), float("inf"), float("inf"), -float("inf")
        w[0, 1] = float("nan")
    return w


@pytest.mark.parametrize("what", ["equal", "zero", "few", "signs", "negative", "one bit", "special"])
@pytest.mark.parametrize("T,L", [(40000, 39001), (24576, 24576), (32768, 20479)])
def test_ties_and_signs(gpu_lib, what, T, L):
    """The threshold among equal keys of several chunks; sequences that end inside one; NaN kept last, and by place."""
    w = _special(what, T)
    w[..., L:] = float("inf")                 # (behind the sequence: not candidates)
    for ns, nr, k in ((2, 10, 12000), (0, 0, 1), (1, 1, L - 3), (4096, 4096, 9000), (0, 0, L - 1), (5000, 3, 0)):
        run(gpu_lib, w, [L], ns, nr, k, seed=1)


@pytest.mark.parametrize("k", [3, 2000, 700000])
@pytest.mark.parametrize("what", ["few", "signs", "special"])
def test_more_chunks_than_threads(gpu_lib, what, k):
    """More than 2^20 tokens: 257 chunks, the last of 1234 tokens."""
    T = (1 << 20) + 1248
    run(gpu_lib, _special(what, T)[:, :1], [(1 << 20) + 1234], 4, 64, k, spare=0, with_weights=k < 10000)
