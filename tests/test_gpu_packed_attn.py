"""Verify attention over the 4-bit cache against 64 bits on the values that it stands for."""
import numpy as np
import pytest
import torch

import compact_reference as ref
import oracle
import workloads

pytestmark = pytest.mark.gpu


def _tree(sp, batch, M, n_key, Hq, Hkv, D, dtype, seed, kind="bounded", size=1.0):
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn((batch, M, Hq, D), generator=g) * size).to(dtype)
    kd, vd = (torch.randn((batch, M + n_key, Hkv, D), generator=g).to(dtype) for _ in "kv")
    rng = np.random.default_rng(seed)
    parent = torch.tensor([oracle.extend_parents(workloads.make_tree(M, kind, rng).tolist(), n_key) for _ in range(batch)], dtype=torch.int32)
    return sp.Tree(q.cuda(), kd.cuda(), vd.cuda(), parent.cuda()), [x.double().numpy() for x in (q, kd, vd)], parent.numpy()


def _lists(batch, Hkv, rows, dev="cuda"):
    """rows[b][g]: entries; padded with -1."""
    n = max(1, max(len(r) for b in rows for r in b))
    idx = torch.tensor([[r + [-1] * (n - len(r)) for r in b] for b in rows], dtype=torch.int32, device=dev)
    return idx, torch.tensor([[len(r) for r in b] for b in rows], dtype=torch.int32, device=dev)


def check(sp, h, kv, tree, tv, parent, idx=None, cnt=None, with_lse=True, ws=None):
    dtype = h.dtype
    out = torch.full(tree.q.shape, 3.0, dtype=dtype, device="cuda")
    lse = torch.full(tree.q.shape[:3], 3.0, device="cuda") if with_lse else None
    if ws is None:
        ws = torch.zeros((sp.specpv_packed_workspace_bytes(h, tree, sp.SelectCfg(0, 0, idx.shape[-1]) if idx is not None else None),), dtype=torch.uint8, device="cuda")
    sp.specpv_packed_verify_attn(h, tree, idx, cnt, out, lse, ws)
    got, glse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    lens, D = h.ctx_len.tolist(), h.D
    G = tree.Hq // h.Hkv
    step, inner = ref.half_step(dtype), ref.half_step(dtype) if dtype == torch.bfloat16 else 2.0 ** -23
    for b in range(h.batch):
        for g in range(h.Hkv):
            t = ref.listed_tokens(lens[b], h.B, None if idx is None else idx[b, g].tolist(), None if cnt is None else cnt[b, g])
            q, kd, vd = tv[0][b, :, g * G:(g + 1) * G], tv[1][b, :, g], tv[2][b, :, g]
            O, lo, size, reach = ref.attention(q, kv[0][b, g], kv[1][b, g], kd, vd, parent[b], tree.n_key_only, t)
            n = len(t) + tree.M
            # weights: the scores' error, their rounding in front of the product with V, the sums' n roundings; a split's result in
            # 16 bits (fp16: 2^-11 of the value, or half of its least step, 2^-24, which is more for results below 2^-14 and does not
            # grow where splits are averaged); the output's own
            half = dtype == torch.bfloat16
            off = size * (2 * ref.score_error(reach, D)[..., None] + inner + (n + 64) * 2.0 ** -24 + (2.0 ** -11 if half else 0)) + np.abs(O) * step + (2.0 ** -25 if half else 0)
            e = np.abs(got[b, :, g * G:(g + 1) * G] - O)
            assert (e <= off).all(), (b, g, float((e / off).max()), float(e.max()))
            if lse is not None:
                off = ref.score_error(reach, D) + (n + 64) * 2.0 ** -24 + 4 * np.abs(lo) * 2.0 ** -24
                e = np.abs(glse[b, :, g * G:(g + 1) * G] - lo)
                assert (e <= off).all(), (b, g, float((e / off).max()))
    return out, lse


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,M,B,lens", [(4, 1, 1, 16, [1]), (8, 2, 3, 64, [0, 31, 33]), (10, 2, 17, 24, [700, 5]), (16, 1, 9, 64, [1000]), (3, 3, 33, 7, [129, 128])])
def test_whole_cache(gpu_lib, dtype, D, Hq, Hkv, M, B, lens):
    sp = gpu_lib
    T = -(-max(max(lens), 1) // B) * B
    h, k, v = ref.cache(sp, len(lens), Hkv, T, D, B, dtype, seed=M, lens=lens)
    tree, tv, parent = _tree(sp, len(lens), M, 0, Hq, Hkv, D, dtype, 7 * M)
    check(sp, h, (k, v), tree, tv, parent)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D,B,layout,n_key", [(128, 64, "bhtd", 0), (128, 64, "bhtd", 18), (64, 16, "bthd", 5), (128, 24, "bthd", 0), (64, 5, "bhtd", 1)])
def test_lists(gpu_lib, dtype, D, B, layout, n_key):
    """Out of order, padded, repeated, outside the sequence; one list is empty, one has only what is not there."""
    sp = gpu_lib
    lens = [9 * B + 2, 3 * B]
    h, k, v = ref.cache(sp, 2, 2, 10 * B, D, B, dtype, layout, seed=B, lens=lens)
    tree, tv, parent = _tree(sp, 2, 11, n_key, 8, 2, D, dtype, 3 * B)
    idx, cnt = _lists(2, 2, [[[9, 0, 4, 4, -1, 77, 2], []], [[1, 2], [3, 9, -2]]])
    check(sp, h, (k, v), tree, tv, parent, idx, cnt)
    cnt[0, 0] = 3                     # the count cuts the list
    check(sp, h, (k, v), tree, tv, parent, idx, cnt, with_lse=False)
    cnt[0, 1] = -4
    check(sp, h, (k, v), tree, tv, parent, idx, cnt)


@pytest.mark.parametrize("dtype,M,Hq,Hkv,T", [(torch.bfloat16, 128, 16, 1, 640), (torch.bfloat16, 60, 8, 2, 3000), (torch.bfloat16, 1, 8, 2, 20000), (torch.float32, 128, 16, 1, 320),
                                              (torch.float32, 2, 4, 1, 9000)])
def test_many_rows_and_long_caches(gpu_lib, dtype, M, Hq, Hkv, T):
    sp = gpu_lib
    h, k, v = ref.cache(sp, 1, Hkv, T, 128, 64 if T % 64 == 0 else 40, dtype, seed=T, lens=[T - 1])
    tree, tv, parent = _tree(sp, 1, M, 0, Hq, Hkv, 128, dtype, T, size=2.0)
    check(sp, h, (k, v), tree, tv, parent)


def test_weights_that_a_late_token_dwarfs(gpu_lib):
    """Scores that grow along the cache by more than any slack of the running maximum, then shrink; the sums stay right."""
    sp = gpu_lib
    h, k, v = ref.cache(sp, 1, 1, 2048, 64, 32, torch.float32, seed=3)
    tree, tv, parent = _tree(sp, 1, 4, 0, 2, 1, 64, torch.float32, 5, size=9.0)
    out, lse = check(sp, h, (k, v), tree, tv, parent)
    assert float(lse.max()) > 60


def test_rows_behind_the_sequence_are_not_read(gpu_lib):
    """NaN scales in every row that no list names or the sequence does not have; and in a row that counts, NaN comes out."""
    sp = gpu_lib
    for dtype in (torch.float32, torch.bfloat16):
        for D in (64, 128):
            h, k, v = ref.cache(sp, 2, 2, 256, D, 16, dtype, seed=6, lens=[100, 33])
            keep = torch.zeros((2, 256), dtype=torch.bool)
            idx, cnt = _lists(2, 2, [[[0, 2, 6], [0, 2, 6]], [[2, 1], [2, 1]]])
            for b, L in ((0, 100), (1, 33)):
                for i in idx[b, 0].tolist():
                    if i >= 0:
                        keep[b, i * 16:min(L, i * 16 + 16)] = True
            for sc in (h.k_scale, h.v_scale):
                sc.copy_(torch.where(keep[:, None, :, None].cuda(), sc, 255))
            tree, tv, parent = _tree(sp, 2, 5, 0, 4, 2, D, dtype, 8)
            out, lse = check(sp, h, (k, v), tree, tv, parent, idx, cnt)
            h.k_scale[0, 1, 97, 0] = 255       # an attended key of one head
            ws = torch.zeros((sp.specpv_packed_workspace_bytes(h, tree, sp.SelectCfg(0, 0, 3)),), dtype=torch.uint8, device="cuda")
            bad, bl = torch.zeros_like(out), torch.zeros_like(lse)
            sp.specpv_packed_verify_attn(h, tree, idx, cnt, bad, bl, ws)
            assert bad[0, :, 2:].isnan().all() and bl[0, :, 2:].isnan().all()
            assert torch.equal(bad[0, :, :2], out[0, :, :2]) and torch.equal(bad[1], out[1]) and torch.equal(bl[1], lse[1])


def test_a_smaller_workspace_serves(gpu_lib):
    """Any size that holds one split is taken and gives a right result; too little is refused."""
    sp = gpu_lib
    h, k, v = ref.cache(sp, 1, 2, 4096, 128, 64, torch.bfloat16, seed=1)
    tree, tv, parent = _tree(sp, 1, 12, 0, 8, 2, 128, torch.bfloat16, 1)
    full = sp.specpv_packed_workspace_bytes(h, tree)
    one = 65536 + 12 * 8 * (256 + 8) + 512
    assert one < full
    for size in (one, (one + full) // 2, full):
        check(sp, h, (k, v), tree, tv, parent, ws=torch.zeros((size,), dtype=torch.uint8, device="cuda"))
    with pytest.raises(sp.SpecPVError) as e:
        sp.specpv_packed_verify_attn(h, tree, None, None, torch.zeros_like(tree.q), None, torch.zeros((65536,), dtype=torch.uint8, device="cuda"))
    assert e.value.status == -2


def test_binding_refuses(gpu_lib):
    sp = gpu_lib
    h, _, _ = ref.cache(sp, 1, 2, 64, 128, 16, torch.bfloat16)
    tree, _, _ = _tree(sp, 1, 3, 0, 4, 2, 128, torch.bfloat16, 1)
    ws = torch.zeros((1 << 20,), dtype=torch.uint8, device="cuda")
    idx, cnt = _lists(1, 2, [[[0], [1]]])
    for bad in (dict(out=torch.zeros_like(tree.q).float()), dict(out=torch.zeros_like(tree.q)[:, :2]), dict(lse=torch.zeros((1, 3, 5), device="cuda")),
                dict(idx=idx.long(), cnt=cnt), dict(idx=idx, cnt=cnt[:, :1]), dict(cnt=cnt), dict(tree=sp.Tree(tree.q.float()))):
        a = dict(dict(out=torch.zeros_like(tree.q), lse=None, idx=None, cnt=None, tree=tree), **bad)
        with pytest.raises(ValueError):
            sp.specpv_packed_verify_attn(h, a["tree"], a["idx"], a["cnt"], a["out"], a["lse"], ws)
    with pytest.raises(ValueError):
        sp.specpv_packed_gather_blocks(h, idx, cnt, torch.zeros((1, 2, 32, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 2, 16, 128), dtype=torch.bfloat16, device="cuda"))
    src = sp.KV(torch.zeros((1, 2, 8, 128), device="cuda"), torch.zeros((1, 2, 8, 128), device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda"), 8)
    with pytest.raises(ValueError):
        sp.specpv_pack_tokens(src, h)                        # fp32 rows, a cache for bf16
    with pytest.raises(ValueError):
        sp.PackedKV(h.k, h.v, h.k_scale[:, :, ::2], h.v_scale[:, :, ::2], h.ctx_len, 16)


@pytest.mark.parametrize("dtype,D,M,Hq,Hkv,lens", [(torch.bfloat16, 128, 60, 8, 2, [40000]), (torch.bfloat16, 64, 1, 4, 1, [20000]), (torch.float32, 64, 9, 8, 2, [30001]),
                                                   (torch.bfloat16, 128, 2, 16, 8, list(range(1, 300, 15))), (torch.float32, 64, 9, 16, 8, list(range(0, 300, 15)))])
def test_splits_of_every_kind(gpu_lib, dtype, D, M, Hq, Hkv, lens):
    """One workgroup a CU and two, the most splits that there are, and a number of columns that leaves a third of the CUs idle."""
    sp = gpu_lib
    T = -(-max(lens) // 64) * 64
    h, k, v = ref.cache(sp, len(lens), Hkv, T, D, 64, dtype, seed=M, lens=lens)
    tree, tv, parent = _tree(sp, len(lens), M, 0, Hq, Hkv, D, dtype, M + D)
    check(sp, h, (k, v), tree, tv, parent)


@pytest.mark.parametrize("dtype,D,M,Hq,Hkv,lens,Bk", [(torch.bfloat16, 128, 2, 4, 2, [91600, 0, 40000], 64), (torch.bfloat16, 64, 128, 16, 1, [5701, 33, 0, 64, 700], 24),
                                                      (torch.bfloat16, 128, 60, 10, 2, [1, 9000, 4000, 8999], 64), (torch.float32, 64, 60, 10, 2, [9000, 1, 33], 40),
                                                      (torch.float32, 128, 40, 4, 1, [9000, 20, 5120], 64), (torch.bfloat16, 64, 1, 4, 2, [0, 0, 91600], 16),
                                                      (torch.bfloat16, 64, 128, 16, 1, [7999, 33, 0, 64, 700], 24), (torch.bfloat16, 128, 60, 10, 2, [1, 12000, 4000, 8999], 64),
                                                      (torch.float32, 64, 60, 10, 2, [13000, 1, 33], 40), (torch.float32, 128, 40, 4, 1, [21500, 20, 5120], 64)])
def test_shares_of_batches(gpu_lib, dtype, D, M, Hq, Hkv, lens, Bk):
    """Long whole caches of three sequences and more, some of them empty or nearly so; in less workspace; and none left at all."""
    sp = gpu_lib
    T = -(-max(lens) // Bk) * Bk
    h, k, v = ref.cache(sp, len(lens), Hkv, T, D, Bk, dtype, "bthd" if M == 60 else "bhtd", seed=M, lens=lens)
    tree, tv, parent = _tree(sp, len(lens), M, 0, Hq, Hkv, D, dtype, M + D)
    check(sp, h, (k, v), tree, tv, parent)
    full = sp.specpv_packed_workspace_bytes(h, tree)
    rows = len(lens) * Hq * M          # results of one split and their sums, each in whole 256 bytes
    one = 65536 + sum(-(-x // 256) * 256 for x in (rows * D * (2 if dtype == torch.bfloat16 and D == 128 else 4), rows * 8))
    assert one <= full
    for size in (one, one + (full - one) // 3):
        check(sp, h, (k, v), tree, tv, parent, ws=torch.zeros((size,), dtype=torch.uint8, device="cuda"))
    h.ctx_len.zero_()
    check(sp, h, (k, v), tree, tv, parent)


@pytest.mark.parametrize("M", [3, 12])
def test_rows_far_apart(gpu_lib, M):
    """Rows 64 MiB from each other, which a chunk's 32-bit offsets do not reach: the same bits as from the same rows side by side."""
    sp = gpu_lib
    h, k, v = ref.cache(sp, 1, 1, 48, 128, 16, torch.bfloat16, seed=M, lens=[45])
    far = []
    for t, wide in ((h.k, 1 << 26), (h.v, 1 << 26), (h.k_scale, 1 << 22), (h.v_scale, 1 << 22)):
        far.append(torch.empty((1, 1, 48, wide), dtype=torch.uint8, device="cuda")[..., :t.shape[-1]])
        far[-1].copy_(t)
    f = sp.PackedKV(*far, h.ctx_len, 16)
    tree, tv, parent = _tree(sp, 1, M, 0, 4, 1, 128, torch.bfloat16, M)
    want = check(sp, h, (k, v), tree, tv, parent)
    got = check(sp, f, (k, v), tree, tv, parent)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    idx, cnt = _lists(1, 1, [[[2, 0, 0]]])
    assert torch.equal(check(sp, f, (k, v), tree, tv, parent, idx, cnt)[0], check(sp, h, (k, v), tree, tv, parent, idx, cnt)[0])


@pytest.mark.parametrize("dtype,D,M,n_key,Hq,Hkv,lens", [(torch.bfloat16, 128, 60, 5, 10, 2, [1, 12000, 4000, 8999]), (torch.float32, 64, 60, 17, 10, 2, [13000, 0, 33]),
                                                         (torch.bfloat16, 64, 20, 3, 8, 2, [700, 90]), (torch.bfloat16, 128, 3, 18, 8, 2, [3000])])
def test_key_only_nodes_over_whole_caches(gpu_lib, dtype, D, M, n_key, Hq, Hkv, lens):
    sp = gpu_lib
    T = -(-max(lens) // 64) * 64
    h, k, v = ref.cache(sp, len(lens), Hkv, T, D, 64, dtype, seed=M, lens=lens)
    tree, tv, parent = _tree(sp, len(lens), M, n_key, Hq, Hkv, D, dtype, M + D)
    check(sp, h, (k, v), tree, tv, parent)
