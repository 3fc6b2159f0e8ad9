"""Packed attention with more row tiles of all (sequence, KV head) pairs than the chip has CUs: one split each, of four wavefronts."""
import pytest
import torch

import compact_reference as ref
from test_gpu_packed_attn import _lists, _tree, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,M,Hq,batch,B", [(torch.bfloat16, 128, 60, 16, 9, 16), (torch.bfloat16, 64, 60, 16, 9, 32), (torch.float32, 128, 37, 16, 8, 24), (torch.float32, 64, 60, 16, 9, 64)])
def test_more_columns_than_cus(gpu_lib, dtype, D, M, Hq, batch, B):
    sp, Hkv = gpu_lib, 4
    T = -(-300 // B) * B
    lens = [T - 7 * b for b in range(batch)]
    h, k, v = ref.cache(sp, batch, Hkv, T, D, B, dtype, seed=M + D, lens=lens)
    tree, tv, parent = _tree(sp, batch, M, 3, Hq, Hkv, D, dtype, M)
    check(sp, h, (k, v), tree, tv, parent)
    n = T // B
    idx, cnt = _lists(batch, Hkv, [[[(3 * i + g + b) % n for i in range(1 + (b + g) % 4)] for g in range(Hkv)] for b in range(batch)])
    check(sp, h, (k, v), tree, tv, parent, idx, cnt)
