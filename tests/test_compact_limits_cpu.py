"""Sizes beyond what the compact cache's launches count in, told on the host (made-up addresses, no GPU)."""
import ctypes

import pytest
import torch

import paper_2512_02337_amd as specpv
from test_abi_cpu import _tree
from test_compact_cpu import _packed

B, vp = ctypes.byref, ctypes.c_void_p
cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="the plans follow the GPU's count of CUs, 256 without one")


def _slots(batch, Hkv, blocks, M=1, G=4):
    """Partial results (of all rows of a KV head each) that a batch of whole caches asks room for; bf16, 128 channels."""
    p = _packed(batch=batch, n_kv_heads=Hkv, max_blocks=blocks, block_size=1024, stride_h=0, stride_b=0)
    need = specpv.load().specpv_packed_workspace_bytes(B(p), B(_tree(M=M, n_q_heads=Hkv * G)), None)
    up = lambda x: (x + 255) & ~255  # noqa: E731
    for n in range(1, 300 + batch * Hkv * 65):
        if 65536 + up(n * M * G * 256) + up(n * M * G * 8) == need:
            return n
    raise AssertionError(need)


@cpu_only
def test_chunks_of_all_sequences_are_counted_in_32_bits():
    """Rooms of 2^30 tokens, which sequences and heads may share (strides of 0): 2^25 chunks each.  Beyond 2^30 chunks in all, what the
    shares of a batch are dealt by would wrap around: splits of each pair instead."""
    assert _slots(3, 2, 1 << 16) == 256 + 6                    # shares, as below
    assert _slots(3, 10, 1 << 20) == 256 + 30                  # 30 * 2^25 chunks: less than 2^30
    for batch, Hkv, splits in ((4, 8, 8), (16, 16, 1), (64, 2, 2), (64, 64, 1)):
        assert _slots(batch, Hkv, 1 << 20) == splits * batch * Hkv, (batch, Hkv)


def test_more_pairs_than_the_second_launch_has_room_for():
    """Refused before the first one is enqueued."""
    def call(batch, Hkv):
        p = _packed(batch=batch, n_kv_heads=Hkv, stride_h=0, stride_b=0)
        return specpv.load().specpv_packed_verify_attn(B(p), B(_tree(M=1, n_q_heads=Hkv)), None, None, 0, vp(0x300), None, vp(0x8000), 1 << 60, None)
    assert call(65536, 8) == -3 and call(1, 524281) == -3
