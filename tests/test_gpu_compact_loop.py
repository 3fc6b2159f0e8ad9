"""The 4-bit cache, the weights and the eviction together, as a decode loop uses them; captured and replayed; on another stream."""
import numpy as np
import pytest
import torch

import compact_reference as ref
import oracle
import workloads

pytestmark = pytest.mark.gpu
B, Hq, Hkv, D, M = 16, 8, 2, 128, 7


def _randn(g, *shape):
    return torch.randn(shape, generator=g).bfloat16().cuda()


class Loop:
    """A sequence that is packed, cut by its weights, and decoded on: two refresh steps with a partial step between them."""

    def __init__(self, sp, L=900, keep=(4, 60, 260)):
        self.sp, self.keep = sp, keep
        g = torch.Generator().manual_seed(11)
        self.g = g
        T = -(-L // B) * B
        i1 = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")  # noqa: E731
        self.kv = sp.KV(_randn(g, 1, Hkv, T, D), _randn(g, 1, Hkv, T, D), i1(L), B)
        n = sum(keep)
        room = -(-(n + 64) // B) * B
        self.small = sp.KV(torch.zeros((1, Hkv, room, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, Hkv, room, D), dtype=torch.bfloat16, device="cuda"), i1(0), B)
        z = lambda w: torch.zeros((1, Hkv, room, w), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.packed = sp.PackedKV(z(D // 2), z(D // 2), z(D // 32), z(D // 32), i1(0), B)
        self.weights, self.new_weights = torch.zeros((1, Hkv, T), device="cuda"), torch.zeros((1, Hkv, room), device="cuda")
        self.keep_idx = torch.zeros((1, Hkv, n), dtype=torch.int32, device="cuda")
        self.kmax, self.kmin = (torch.zeros(self.packed.summary_shape(), dtype=torch.bfloat16, device="cuda") for _ in "xn")
        self.cfg = sp.SelectCfg(1, 2, 5, n_extra_slots=4)
        self.idx, self.cnt = torch.zeros((1, Hkv, self.cfg.n_sel), dtype=torch.int32, device="cuda"), torch.zeros((1, Hkv), dtype=torch.int32, device="cuda")
        rng = np.random.default_rng(4)
        self.parent = torch.tensor([workloads.make_tree(M, "bounded", rng).tolist()], dtype=torch.int32, device="cuda")
        self.steps = [dict(q=_randn(g, 1, M, Hq, D), kd=_randn(g, 1, M, Hkv, D), vd=_randn(g, 1, M, Hkv, D), out=torch.zeros((1, M, Hq, D), dtype=torch.bfloat16, device="cuda"),
                           lse=torch.zeros((1, M, Hq), device="cuda")) for _ in range(3)]
        for s in self.steps:
            s["tree"] = sp.Tree(s["q"], s["kd"], s["vd"], self.parent)
            s["buf"] = sp.KV(s["kd"], s["vd"], i1(M), B, layout="bthd")
        self.accepted, self.n_accepted = torch.tensor([[0, 2, 3]], dtype=torch.int32, device="cuda"), i1(3)
        sizes = [sp.specpv_workspace_bytes(self.kv, self.steps[0]["tree"], self.cfg), sp.specpv_packed_workspace_bytes(self.packed, self.steps[0]["tree"], self.cfg),
                 sp.specpv_evict_workspace_bytes(self.kv)]
        self.ws = torch.zeros((max(sizes),), dtype=torch.uint8, device="cuda")

    def run(self):
        sp, (ns, nr, k) = self.sp, self.keep
        s0, s1, s2 = self.steps
        self.weights.zero_()
        # a full pass over the whole cache; what its accepted rows attended; the cache cut by it; what is left in 4 bits
        sp.specpv_partial_verify_attn(self.kv, s0["tree"], None, None, s0["out"], s0["lse"], self.ws)
        sp.specpv_accumulate_weights(self.kv, s0["tree"], s0["lse"], self.weights, self.accepted, self.n_accepted)
        sp.specpv_evict_tokens(self.kv, self.weights, ns, nr, k, self.small, self.keep_idx, self.new_weights, self.ws)
        sp.specpv_pack_tokens(self.small, self.packed, kmax=self.kmax, kmin=self.kmin)
        self.packed.ctx_len.copy_(self.small.ctx_len)
        # the accepted rows join it; a full pass that chooses blocks, a partial one over those
        sp.specpv_pack_tokens(s0["buf"], self.packed, dst_begin=self.packed.ctx_len, src_rows=self.accepted, n_rows=self.n_accepted, kmax=self.kmax, kmin=self.kmin)
        self.packed.ctx_len.add_(self.n_accepted)
        sp.specpv_packed_verify_attn(self.packed, s1["tree"], None, None, s1["out"], s1["lse"], self.ws)
        sp.specpv_packed_select_blocks(self.packed, s1["tree"], self.kmax, self.kmin, self.cfg, self.idx, self.cnt, None, self.ws)
        sp.specpv_packed_verify_attn(self.packed, s2["tree"], self.idx, self.cnt, s2["out"], s2["lse"], self.ws)
        return [s[x] for s in self.steps for x in ("out", "lse")] + [self.weights, self.new_weights, self.keep_idx, self.idx, self.cnt, self.packed.k, self.packed.k_scale,
                                                                    self.packed.v, self.packed.v_scale, self.kmax, self.kmin, self.small.ctx_len, self.packed.ctx_len]

    def values(self):
        return [ref.unpack(c.cpu().numpy(), s.cpu().numpy()) for c, s in ((self.packed.k, self.packed.k_scale), (self.packed.v, self.packed.v_scale))]


def _attention(step, parent, k, v, tokens_of):
    """Over heads, in 64 bits: out, lse."""
    f = lambda t: t.double().cpu().numpy()[0]  # noqa: E731
    q, kd, vd = f(step["q"]), f(step["kd"]), f(step["vd"])
    O, l = np.zeros(q.shape), np.zeros(q.shape[:2])
    G = Hq // Hkv
    for g in range(Hkv):
        h = slice(g * G, (g + 1) * G)
        O[:, h], l[:, h], _, _ = ref.attention(q[:, h], k[g], v[g], kd[:, g], vd[:, g], parent, 0, tokens_of(g))
    return O, l


def test_a_decode_loop(gpu_lib):
    sp = gpu_lib
    loop = Loop(sp)
    loop.run()
    torch.cuda.synchronize()
    par, n = loop.parent[0].tolist(), sum(loop.keep)
    k, v = (t.double().cpu().numpy()[0] for t in (loop.kv.k, loop.kv.v))
    s0, s1, s2 = loop.steps
    O, l = _attention(s0, par, k, v, lambda g: np.arange(900))
    assert np.abs(s0["out"].double().cpu().numpy()[0] - O).max() < 2e-2
    # weights by the definition's own sums; which tokens stay by the library's weights (near ties are its own affair)
    q, G = s0["q"].double().cpu().numpy()[0], Hq // Hkv
    for g in range(Hkv):
        w, off = ref.weights_of(q[:, g * G:(g + 1) * G], k[g], l[:, g * G:(g + 1) * G], [0, 2, 3], np.arange(900), 912)
        got = loop.weights[0, g].double().cpu().numpy()
        assert (np.abs(got - w) <= off + w * 1e-4).all()       # (1e-4: the log-sum-exp that it was given)
        kept = ref.kept_tokens(loop.weights[0, g].tolist(), 900, *loop.keep)
        assert loop.keep_idx[0, g].tolist() == kept
        # the packed rows are the kept ones and, behind them, the accepted candidates
        kd = s0["kd"].double().cpu().numpy()[0]
        rows = np.concatenate((k[g, kept], kd[[0, 2, 3], g]))
        for t in (0, 5, n - 1, n, n + 2):
            codes, scales = ref.pack_row(rows[t])
            assert np.array_equal(ref.unpack(loop.packed.k[0, g, t].cpu().numpy(), loop.packed.k_scale[0, g, t].cpu().numpy()),
                                  ref.unpack((codes[0::2] | (codes[1::2] << 4)).astype(np.uint8), scales))
        nb = -(-(n + 3) // B)
        for i in range(nb):
            assert np.array_equal(loop.kmax[0, g, i].double().cpu().numpy(), rows[i * B:(i + 1) * B].max(0))
            assert np.array_equal(loop.kmin[0, g, i].double().cpu().numpy(), rows[i * B:(i + 1) * B].min(0))
    assert loop.packed.ctx_len.tolist() == [n + 3]
    pk, pv = loop.values()
    O, l = _attention(s1, par, pk[0], pv[0], lambda g: np.arange(n + 3))
    assert np.abs(s1["out"].double().cpu().numpy()[0] - O).max() < 2e-2 and np.abs(s1["lse"].double().cpu().numpy()[0] - l).max() < 1e-4
    O, l = _attention(s2, par, pk[0], pv[0], lambda g: ref.listed_tokens(n + 3, B, loop.idx[0, g].tolist(), loop.cnt[0, g]))
    assert np.abs(s2["out"].double().cpu().numpy()[0] - O).max() < 2e-2 and np.abs(s2["lse"].double().cpu().numpy()[0] - l).max() < 1e-4
    # the lists are what an ordinary cache with these summaries would have
    assert loop.cnt.tolist() == [[8, 8]] and all(loop.idx[0, g, 0] == 0 and loop.idx[0, g, 7] == -(-(n + 3) // B) - 1 for g in range(Hkv))


def test_captured_and_replayed(gpu_lib):
    sp = gpu_lib
    loop = Loop(sp)
    want = [t.clone() for t in loop.run()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        loop.run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        outs = loop.run()
    for i in range(4):
        for t in outs:
            t.zero_() if t is not loop.packed.ctx_len else None
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), i
        torch.randn(1000, device="cuda").sum().item()      # eager work between the replays


def test_another_stream(gpu_lib):
    """Calls go to the stream that is current."""
    sp = gpu_lib
    a, b = Loop(sp), Loop(sp)
    want = [t.clone() for t in a.run()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        got = b.run()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_nothing_is_allocated(gpu_lib):
    loop = Loop(gpu_lib)
    loop.run()
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    loop.run()
    torch.cuda.synchronize()
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before


def test_two_graphs_in_one_workspace(gpu_lib):
    """Graphs of different shapes that share a workspace, replayed in turn, and an eager call between them."""
    sp = gpu_lib
    loops = [Loop(sp), Loop(sp, 20000, (2, 33, 9000))]
    ws = loops[0].ws if loops[0].ws.numel() > loops[1].ws.numel() else loops[1].ws
    want, graphs = [], []
    for loop in loops:
        loop.ws = ws
        want.append([t.clone() for t in loop.run()])
    torch.cuda.synchronize()
    for loop in loops:
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            loop.run()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs = loop.run()
        loop.outs = outs
    for i in range(3):
        for j in (0, 1, 1, 0):
            for t in loops[j].outs:
                t.zero_() if t is not loops[j].packed.ctx_len else None
            graphs[j].replay()
        loops[i & 1].run()
        torch.cuda.synchronize()
        for loop, w in zip(loops, want):
            assert all(torch.equal(a, b) for a, b in zip(loop.outs, w)), i


def test_offsets_beyond_32_bits(gpu_lib):
    """Rows 64 KiB apart, 4.5 GB from first to last: the same bits as from the same rows side by side."""
    sp = gpu_lib
    T, L, Dh = 70032, 70021, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = [torch.randn((1, T, 1, Dh), generator=g, device="cuda").bfloat16() for _ in "kv"]
    i1 = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")  # noqa: E731
    near = sp.KV(rows[0], rows[1], i1(L), 24, layout="bthd")
    apart = [torch.empty((1, T, 1, 32768), dtype=torch.bfloat16, device="cuda")[..., :Dh] for _ in "kv"]
    for a, b in zip(apart, rows):
        a.copy_(b)
    far = sp.KV(apart[0], apart[1], i1(L), 24, layout="bthd")
    q = torch.randn((1, 5, 4, Dh), generator=g, device="cuda").bfloat16()
    kd, vd = (torch.randn((1, 5, 1, Dh), generator=g, device="cuda").bfloat16() for _ in "kv")
    tree = sp.Tree(q, kd, vd, torch.arange(-1, 4, dtype=torch.int32, device="cuda")[None])
    lse = torch.full((1, 5, 4), 12.0, device="cuda")
    ends = [torch.zeros((1, 1, T), device="cuda") for _ in "ab"]
    for kv, w in zip((near, far), ends):
        sp.specpv_accumulate_weights(kv, tree, lse, w)
    assert torch.equal(*ends) and ends[0][0, 0, L - 1] > 0
    kept = []
    for kv, w in zip((near, far), ends):
        dst = sp.KV(*(torch.zeros((1, 5000, 1, Dh), dtype=torch.bfloat16, device="cuda") for _ in "kv"), i1(0), 20, layout="bthd")
        idx = torch.zeros((1, 1, 5000), dtype=torch.int32, device="cuda")
        sp.specpv_evict_tokens(kv, w, 4, 100, 4896, dst, idx, None, torch.zeros((sp.specpv_evict_workspace_bytes(kv),), dtype=torch.uint8, device="cuda"))
        kept.append((dst.k, dst.v, idx))
    assert all(torch.equal(a, b) for a, b in zip(*kept)) and int(kept[0][2][0, 0, -1]) == L - 1
    del far, apart
    z = lambda wide, w: torch.empty((1, T, 1, wide), dtype=torch.uint8, device="cuda")[..., :w]  # noqa: E731
    packs = [sp.PackedKV(z(32, 32), z(32, 32), z(2, 2), z(2, 2), i1(L), 24, layout="bthd"),
             sp.PackedKV(z(65536, 32), z(65536, 32), z(4096, 2), z(4096, 2), i1(L), 24, layout="bthd")]
    sel, cnt = torch.tensor([[[2917, 0, 5, 2900, 1400, -1]]], dtype=torch.int32, device="cuda"), torch.tensor([[6]], dtype=torch.int32, device="cuda")
    ws = torch.zeros((sp.specpv_packed_workspace_bytes(packs[0], tree, sp.SelectCfg(0, 0, 6)),), dtype=torch.uint8, device="cuda")
    got = []
    for p in packs:
        sp.specpv_pack_tokens(near, p)
        o = [torch.zeros((1, 1, 6 * 24, Dh), dtype=torch.bfloat16, device="cuda") for _ in "kv"] + [torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(lse)]
        sp.specpv_packed_gather_blocks(p, sel, cnt, o[0], o[1])
        sp.specpv_packed_verify_attn(p, tree, sel, cnt, o[2], None, ws)
        sp.specpv_packed_verify_attn(p, tree, None, None, o[3], o[4], ws)
        got.append(o)
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][0].abs().sum() > 0 and torch.isfinite(got[0][4]).all()
    last = got[0][0][0, 0, :L - 2917 * 24].float()
    assert (last - rows[0][0, 2917 * 24:L, 0].float()).abs().max() < 1.0       # 4 bits: at most half of the last step, 2^e with e <= 0


def test_lists_of_no_entries(gpu_lib):
    """Tensors without an element have no address: refused, not taken for no list at all."""
    sp = gpu_lib
    h, _, _ = ref.cache(sp, 1, 2, 64, 128, 16, torch.bfloat16)
    q = torch.zeros((1, 3, 4, 128), dtype=torch.bfloat16, device="cuda")
    kd = torch.zeros((1, 3, 2, 128), dtype=torch.bfloat16, device="cuda")
    tree = sp.Tree(q, kd, kd, torch.tensor([[-1, 0, 1]], dtype=torch.int32, device="cuda"))
    none, cnt = torch.zeros((1, 2, 0), dtype=torch.int32, device="cuda"), torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    ws = torch.zeros((1 << 20,), dtype=torch.uint8, device="cuda")
    empty = torch.zeros((1, 2, 0, 128), dtype=torch.bfloat16, device="cuda")
    kv = sp.KV(*(torch.zeros((1, 2, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"), torch.ones((1,), dtype=torch.int32, device="cuda"), 16)
    lse, w = torch.zeros((1, 3, 4), device="cuda"), torch.zeros((1, 2, 64), device="cuda")
    for call in (lambda: sp.specpv_packed_verify_attn(h, tree, none, cnt, torch.zeros_like(q), None, ws), lambda: sp.specpv_packed_gather_blocks(h, none, cnt, empty, empty),
                 lambda: sp.specpv_accumulate_weights(kv, tree, lse, w, None, None, none, cnt),
                 lambda: sp.specpv_accumulate_weights(kv, tree, lse, w, torch.zeros((1, 0), dtype=torch.int32, device="cuda"), torch.ones((1,), dtype=torch.int32, device="cuda")),
                 lambda: sp.specpv_pack_tokens(kv, h, src_rows=torch.zeros((1, 0), dtype=torch.int32, device="cuda"))):
        with pytest.raises(sp.SpecPVError):
            call()
    assert not w.any()


def test_replays_follow_the_lengths(gpu_lib):
    """A batch whose sequences grow and shrink between the replays of one graph: each replay gives what an eager call gives."""
    sp = gpu_lib
    g = torch.Generator(device="cuda").manual_seed(9)
    T, Hk, Dh = 13056, 2, 64
    rows = [torch.randn((3, Hk, T, Dh), generator=g, device="cuda").bfloat16() for _ in "kv"]
    lens = torch.tensor([13000, 700, 1], dtype=torch.int32, device="cuda")
    z = lambda w: torch.zeros((3, Hk, T, w), dtype=torch.uint8, device="cuda")  # noqa: E731
    p = sp.PackedKV(z(32), z(32), z(2), z(2), torch.full((3,), T, dtype=torch.int32, device="cuda"), 64)
    full = sp.KV(rows[0], rows[1], torch.full((3,), T, dtype=torch.int32, device="cuda"), 64)
    sp.specpv_pack_tokens(full, p)
    p.ctx_len.copy_(lens)
    kv = sp.KV(rows[0], rows[1], p.ctx_len, 64)
    q = torch.randn((3, 60, 10, Dh), generator=g, device="cuda").bfloat16()
    kd, vd = (torch.randn((3, 60, Hk, Dh), generator=g, device="cuda").bfloat16() for _ in "kv")
    tree = sp.Tree(q, kd, vd, torch.arange(-1, 59, dtype=torch.int32, device="cuda").expand(3, -1).contiguous())
    ws = torch.zeros((max(sp.specpv_packed_workspace_bytes(p, tree), sp.specpv_evict_workspace_bytes(kv)),), dtype=torch.uint8, device="cuda")
    dst = sp.KV(*(torch.zeros((3, Hk, 704, Dh), dtype=torch.bfloat16, device="cuda") for _ in "kv"), torch.zeros((3,), dtype=torch.int32, device="cuda"), 64)
    o = dict(out=torch.zeros_like(q), lse=torch.zeros((3, 60, 10), device="cuda"), w=torch.zeros((3, Hk, T), device="cuda"),
             idx=torch.zeros((3, Hk, 700), dtype=torch.int32, device="cuda"), k=dst.k, v=dst.v, n=dst.ctx_len)

    def run():
        o["w"].zero_()
        sp.specpv_packed_verify_attn(p, tree, None, None, o["out"], o["lse"], ws)
        sp.specpv_accumulate_weights(kv, tree, o["lse"], o["w"])
        sp.specpv_evict_tokens(kv, o["w"], 4, 96, 600, dst, o["idx"], None, ws)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for now in ([13000, 700, 1], [5, 13056, 6000], [0, 0, 0], [13056, 13056, 13056], [699, 701, 700]):
        p.ctx_len.copy_(torch.tensor(now, dtype=torch.int32))
        for t in o.values():
            t.zero_()
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in o.values()]
        for t in o.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o.values(), want)), now
        assert o["n"].tolist() == [min(L, 700) for L in now]
