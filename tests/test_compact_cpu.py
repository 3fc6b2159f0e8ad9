"""Refusals of the 4-bit cache's calls, the accumulated weights and the eviction: every bad argument is an error code before
anything is launched (made-up addresses, no GPU), and the reference's own format against hand-worked values."""
import ctypes

import numpy as np
import pytest
import torch

import compact_reference as ref
import paper_2512_02337_amd as specpv
from paper_2512_02337_amd import binding
from test_abi_cpu import _cfg, _kv, _tree

B, vp = ctypes.byref, ctypes.c_void_p


def _packed(**over):
    d = dict(k=0x1000, v=0x2000, k_scale=0x3004, v_scale=0x4008, stride_b=1 << 20, stride_h=1 << 16, stride_t=64, ctx_len=0x5000, batch=1, n_kv_heads=8,
             head_dim=128, block_size=64, max_blocks=16, dtype=1)
    d.update(over)
    return binding._PackedKV(**d)


BAD_PACKED = [dict(k=None), dict(k_scale=None), dict(v_scale=None), dict(ctx_len=None), dict(head_dim=96), dict(dtype=2), dict(stride_t=32), dict(stride_t=96),
              dict(stride_h=(1 << 16) + 16), dict(stride_b=-64), dict(k=0x1008), dict(v_scale=0x4002), dict(batch=0), dict(n_kv_heads=0), dict(block_size=0),
              dict(max_blocks=0)]


def test_format_of_the_reference():
    codes, scales = ref.pack_row([7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.0, -0.3] + [0.0] * 22)
    assert scales.tolist() == [127]
    assert codes[:10].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 9]
    assert ref.pack_row([7.0001] + [0] * 31)[1].tolist() == [128] and ref.pack_row([0.0] * 32)[1].tolist() == [3]
    assert ref.pack_row([3.4e38] + [0] * 31)[1].tolist() == [252] and ref.pack_row([1e-45] + [0] * 31)[0][0] == 0
    assert ref.pack_row([np.inf] + [1.0] * 63)[1].tolist() == [255, 127 - 2]
    assert ref.unpack(np.array([0x9f] + [0] * 15, dtype=np.uint8), np.array([128], dtype=np.uint8))[:2].tolist() == [-12.0, -1.0]


@pytest.mark.parametrize("bad", BAD_PACKED, ids=lambda d: "%s=%s" % next(iter(d.items())))
def test_packed_descriptors(bad):
    lib = specpv.load()
    p = _packed(**bad)
    assert lib.specpv_packed_workspace_bytes(B(p), B(_tree()), B(_cfg())) == 0
    assert lib.specpv_pack_tokens(B(_kv()), None, None, None, 4, B(p), None, None, None, None) == -1
    assert lib.specpv_packed_verify_attn(B(p), B(_tree()), None, None, 0, vp(0x300), None, vp(0x8000), 1 << 40, None) == -1
    assert lib.specpv_packed_gather_blocks(B(p), None, None, 0, vp(0x100), vp(0x200), None, None) == -1
    assert lib.specpv_packed_select_blocks(B(p), B(_tree()), vp(16), vp(32), B(_cfg()), vp(0x100), vp(0x200), None, vp(0x8000), 1 << 30, None) == -1


def test_pack_arguments():
    lib = specpv.load()
    ok = dict(kv=_kv(), src_begin=None, src_rows=None, n_rows=None, max_rows=4, p=_packed(), dst_begin=None, kmax=None, kmin=None)

    def call(**over):
        a = dict(ok, **over)
        return lib.specpv_pack_tokens(B(a["kv"]), a["src_begin"], a["src_rows"], a["n_rows"], a["max_rows"], B(a["p"]), a["dst_begin"], a["kmax"], a["kmin"], None)
    assert call(max_rows=0) == -1
    assert call(src_rows=vp(0x100), src_begin=vp(0x200)) == -1
    assert call(kmax=vp(16)) == -1 and call(kmin=vp(16)) == -1 and call(kmax=vp(16), kmin=vp(24)) == -1
    assert call(p=_packed(batch=2)) == -1 and call(p=_packed(n_kv_heads=4)) == -1 and call(p=_packed(dtype=0)) == -1
    assert call(kv=_kv(head_dim=64, stride_t=64)) == -1
    assert call(kv=_kv(batch=70000), p=_packed(batch=70000)) == -3
    assert call(p=_packed(max_blocks=1 << 25)) == -3


def test_packed_attention_arguments():
    lib = specpv.load()
    need = lib.specpv_packed_workspace_bytes(B(_packed()), B(_tree()), B(_cfg()))
    assert need > 0 and lib.specpv_packed_workspace_bytes(B(_packed()), None, None) > 0

    def call(p=None, tree=None, idx=vp(0x100), cnt=vp(0x200), n=7, out=vp(0x300), ws=vp(0x8000), bytes_=need):
        return lib.specpv_packed_verify_attn(B(p or _packed()), B(tree or _tree()), idx, cnt, n, out, None, ws, bytes_, None)
    assert call(tree=_tree(M=129)) == -3 and call(tree=_tree(M=0)) == -1 and call(tree=_tree(kd=None)) == -1 and call(tree=_tree(n_q_heads=30)) == -1
    assert call(out=None) == -1 and call(out=vp(0x308)) == -1 and call(cnt=None) == -1 and call(n=-1) == -1
    assert call(n=(1 << 24) + 1) == -3 and call(n=1 << 24, p=_packed(block_size=128)) == -3
    assert call(ws=None) == -2 and call(bytes_=1000) == -2
    assert lib.specpv_packed_gather_blocks(B(_packed()), vp(0x100), None, 3, vp(0x100), vp(0x200), None, None) == -1
    assert lib.specpv_packed_gather_blocks(B(_packed()), vp(0x100), vp(0x300), 0, vp(0x100), vp(0x200), None, None) == -1
    assert lib.specpv_packed_gather_blocks(B(_packed()), None, None, 0, vp(0x108), vp(0x200), None, None) == -1
    assert lib.specpv_packed_select_blocks(B(_packed()), B(_tree()), vp(16), vp(32), B(_cfg(k_blocks=-1)), vp(0x100), vp(0x200), None, vp(0x8000), need, None) == -1


def test_weights_arguments():
    lib = specpv.load()

    def call(kv=None, tree=None, lse=vp(0x100), nodes=None, n_nodes=None, most=0, idx=None, cnt=None, n=0, w=vp(0x200)):
        return lib.specpv_accumulate_weights(B(kv or _kv()), B(tree or _tree(kd=None, vd=None, parent=None)), lse, nodes, n_nodes, most, idx, cnt, n, w, None)
    assert call(lse=None) == -1 and call(w=None) == -1 and call(kv=_kv(head_dim=96)) == -1 and call(tree=_tree(M=129)) == -3
    assert call(nodes=vp(0x300)) == -1 and call(nodes=vp(0x300), n_nodes=vp(0x400)) == -1 and call(nodes=vp(0x300), n_nodes=vp(0x400), most=129) == -3
    assert call(idx=vp(0x300)) == -1 and call(idx=vp(0x300), cnt=vp(0x400), n=-1) == -1 and call(idx=vp(0x300), cnt=vp(0x400), n=1 << 25) == -3
    assert call(kv=_kv(batch=70000)) == -3


def test_eviction_arguments():
    lib = specpv.load()
    need = lib.specpv_evict_workspace_bytes(B(_kv()))
    assert need > 0 and lib.specpv_evict_workspace_bytes(B(_kv(head_dim=96))) == 0
    other = dict(k=0x11000, v=0x12000, ctx_len=0x13000)

    def call(kv=None, w=vp(0x100), ns=4, nr=8, k=20, dst=None, nw=vp(0x200), idx=vp(0x300), ws=vp(0x8000), bytes_=need):
        return lib.specpv_evict_tokens(B(kv or _kv()), w, ns, nr, k, B(dst or _kv(**other)), nw, idx, ws, bytes_, None)
    assert call(w=None) == -1 and call(idx=None) == -1 and call(ns=-1) == -1 and call(nr=-1) == -1 and call(k=-1) == -1 and call(ns=0, nr=0, k=0) == -1
    assert call(dst=_kv(**dict(other, k=0x1000))) == -1 and call(dst=_kv(**dict(other, v=0x2000))) == -1 and call(dst=_kv(**dict(other, ctx_len=0x3000))) == -1
    assert call(nw=vp(0x100)) == -1                                  # weights in place
    assert call(k=16 * 64) == -1                                     # no room for 1036 tokens in 1024
    assert call(k=(1 << 31) - 1, nr=(1 << 31) - 1) == -1
    assert call(dst=_kv(batch=2, **other)) == -1 and call(dst=_kv(dtype=0, **other)) == -1 and call(dst=_kv(n_kv_heads=4, **other)) == -1
    assert call(ws=None) == -2 and call(bytes_=need - 1) == -2


def test_binding_refuses():
    """Shapes and types that the C side cannot see (CPU tensors are refused by each descriptor)."""
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    one = torch.zeros((1,), dtype=torch.int32)
    with pytest.raises(ValueError):
        specpv.PackedKV(u8(1, 2, 64, 64), u8(1, 2, 64, 64), u8(1, 2, 64, 4), u8(1, 2, 64, 4), one, 16)           # not on the GPU
    with pytest.raises(ValueError):
        specpv.PackedKV(u8(1, 2, 64, 64), u8(1, 2, 64, 64), u8(1, 2, 64, 8), u8(1, 2, 64, 8), one, 16)           # scales
    with pytest.raises(ValueError):
        specpv.PackedKV(u8(1, 2, 64, 64).float(), u8(1, 2, 64, 64), u8(1, 2, 64, 4), u8(1, 2, 64, 4), one, 16)
    with pytest.raises(ValueError):
        specpv.PackedKV(u8(1, 2, 64, 64), u8(1, 2, 64, 64), u8(1, 2, 64, 4), u8(1, 2, 64, 4), one, 16, dtype=torch.float16)


def test_workspaces_off_their_alignment():
    lib = specpv.load()
    assert lib.specpv_packed_verify_attn(B(_packed()), B(_tree()), None, None, 0, vp(0x300), None, vp(0x8008), 1 << 40, None) == -1
    assert lib.specpv_evict_tokens(B(_kv()), vp(0x100), 4, 8, 20, B(_kv(k=0x11000, v=0x12000, ctx_len=0x13000)), vp(0x200), vp(0x300), vp(0x8004), 1 << 30, None) == -1


def test_rows_of_a_packed_allocation():
    lib = specpv.load()
    p = _packed(tokens=-1)
    assert lib.specpv_packed_workspace_bytes(B(p), B(_tree()), B(_cfg())) == 0
    assert lib.specpv_pack_tokens(B(_kv()), None, None, None, 4, B(p), None, None, None, None) == -1
    assert lib.specpv_packed_workspace_bytes(B(_packed(tokens=1000)), B(_tree()), B(_cfg())) == lib.specpv_packed_workspace_bytes(B(_packed()), B(_tree()), B(_cfg())) > 0


def test_counts_without_lists():
    """A count or a list by itself is refused (a list of no entries may come as a null pointer, and none of them means all)."""
    lib = specpv.load()
    assert lib.specpv_packed_verify_attn(B(_packed()), B(_tree()), None, vp(0x200), 0, vp(0x300), None, vp(0x8000), 1 << 40, None) == -1
    assert lib.specpv_packed_gather_blocks(B(_packed()), None, vp(0x200), 0, vp(0x100), vp(0x200), None, None) == -1
    tree = _tree(kd=None, vd=None, parent=None)
    assert lib.specpv_accumulate_weights(B(_kv()), B(tree), vp(0x100), None, None, 0, None, vp(0x400), 0, vp(0x200), None) == -1
    assert lib.specpv_accumulate_weights(B(_kv()), B(tree), vp(0x100), None, vp(0x400), 0, None, None, 0, vp(0x200), None) == -1
