"""aspd_norm_rope_append against the float64 oracle: norms per head, rotary positions on one and several axes, rows at any stride,
the cache, the positions of slots; and the whole way from new tokens to attention."""
import numpy as np
import pytest
import torch

import aspd_workloads as W
from oracle import TokenTable
from oracle.scores import attend_scored, norm_rotate
from scores_drive import check, score_error

pytestmark = pytest.mark.gpu

EPS = 1e-6
U = 2.0 ** -24


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_08895_amd import binding
    binding.lib()
    return binding


def _type(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _bound(y, dtype):
    """|error| of y = (a c - b s, b c + a s): a and b carry the roundings of a sum of D squares (32 U covers D = 128, added in
    runs of 16 and a tree), of the root, the weight and the products, the cosine and sine one each; then the result's own."""
    D = y.shape[-1]
    a, b = np.abs(y[..., :D // 2]), np.abs(y[..., D // 2:])
    pair = np.sqrt(a * a + b * b)   # the rotation keeps it
    return 48 * U * np.concatenate([pair, pair], -1) * np.sqrt(2) + (2.0 ** -8 if dtype == "bf16" else U) * np.abs(y)


class _Call:
    """Rows of random values at random places of a cache, one call's worth."""

    def __init__(self, A, dtype, hq, hkv, hd, NQ, layout="packed", B=5, seed=0, sigma=1.0, lost=0.0):
        g = torch.Generator().manual_seed(seed + NQ)
        rng = np.random.default_rng(seed + NQ + hd)
        t = _type(dtype)
        widths = [hq * hd, hkv * hd, hkv * hd]
        if layout == "fused":
            parts = (torch.randn(NQ, sum(widths), generator=g) * sigma).to(t).cuda().split(widths, 1)
        elif layout == "odd":        # rows and starts off 16-byte boundaries
            parts = [(torch.randn(NQ, w + 3, generator=g) * sigma).to(t).cuda()[:, 1:w + 1] for w in widths]
        else:
            parts = [(torch.randn(NQ, w, generator=g) * sigma).to(t).cuda() for w in widths]
        self.q, self.k, self.v = (p.unflatten(1, (-1, hd)) for p in parts)
        blocks = NQ // 16 + 3
        self.pools = [torch.randn(blocks, hkv, 16, hd, generator=g).to(t).cuda() for _ in range(2)]
        self.kv = A.KVCache(*self.pools, torch.zeros(B, 1, dtype=torch.int32, device="cuda"), hq)
        self.state = A.BatchState(B, 4 * NQ + 4, "cuda")
        self.step = A.Step(NQ, B, B, "cuda")
        self.pos = rng.integers(0, 100_000, NQ).astype(np.int32)
        self.seq = rng.integers(0, B, NQ).astype(np.int32)
        self.slot = rng.permutation(4 * NQ)[:NQ].astype(np.int32)
        place = rng.permutation(blocks * 16)[:NQ].astype(np.int64)
        self.lost = rng.random(NQ) < lost
        self.place = np.where(self.lost, np.where(self.pos % 2 == 0, -1, blocks * 16), place)
        for name, x in (("position_ids", self.pos), ("q_seq", self.seq), ("logical_slot", self.slot), ("slot_mapping", self.place)):
            getattr(self.step, name).copy_(torch.from_numpy(x))
        self.before = [x.double().cpu().numpy().copy() for x in (self.q, self.k, self.v, *self.pools)]
        self.dtype, self.hd, self.NQ, self.B, self.rng, self.g = dtype, hd, NQ, B, rng, g

    def weight(self, shift=0):     # `shift` elements off a 16-byte boundary
        return (1 + 0.3 * torch.randn(self.hd + shift, generator=self.g)).to(_type(self.dtype)).cuda()[shift:]

    def check(self, q_got, positions, theta, qw=None, kw=None, offset=0.0, slot_pos=None, eps=EPS):
        q, k, v, kp, vp = self.before
        w = [None if x is None else x.double().cpu().numpy() for x in (qw, kw)]
        want = norm_rotate(q, positions, theta, w[0], eps, offset)
        got = q_got.double().cpu().numpy()[:self.NQ]
        off = np.abs(got - want)
        bound = _bound(want, self.dtype)
        print(f"[{self.dtype} rows {self.NQ}] q {np.max(off / np.maximum(bound, 1e-300)):.3f} of the bound", flush=True)
        assert (off <= bound).all()
        kp, vp = kp.copy(), vp.copy()
        k_new = norm_rotate(k, positions, theta, w[1], eps, offset)
        bound = np.zeros_like(kp)
        for r in np.flatnonzero(~self.lost):
            blk, at = divmod(int(self.place[r]), 16)
            kp[blk, :, at], vp[blk, :, at] = k_new[r], v[r]
            bound[blk, :, at] = _bound(k_new[r], self.dtype)
        assert (np.abs(self.pools[0].double().cpu().numpy() - kp) <= bound).all()    # (0 where nothing was written)
        assert np.array_equal(self.pools[1].double().cpu().numpy(), vp)
        if slot_pos is not None:
            table = np.full((self.B, self.state.owner_stride), -7)
            table[self.seq, self.slot] = self.pos
            assert np.array_equal(slot_pos.cpu().numpy(), table)


SHAPES = [("bf16", 32, 8, 128), ("bf16", 6, 6, 64), ("bf16", 7, 1, 128), ("f32", 40, 5, 128), ("f32", 4, 2, 64), ("bf16", 1, 1, 64)]


@pytest.mark.parametrize("dtype,hq,hkv,hd", SHAPES)
@pytest.mark.parametrize("layout", ["packed", "fused", "odd"])
@pytest.mark.parametrize("NQ", [1, 7, 300])
def test_rows_of_any_layout(A, dtype, hq, hkv, hd, layout, NQ):
    """Norms of both, one and neither; tokens without a place are turned and written nowhere."""
    for qn, kn, offset in ((True, True, 0.0), (True, False, 1.0), (False, False, 0.0)):
        c = _Call(A, dtype, hq, hkv, hd, NQ, layout, lost=0.1)
        qw, kw = c.weight() if qn else None, c.weight() if kn else None
        slot_pos = torch.full((c.B, c.state.owner_stride), -7, dtype=torch.int32, device="cuda")
        out = torch.full((NQ + 2, hq, hd), -5.0, dtype=_type(dtype), device="cuda")
        got = A.aspd_norm_rope_append(c.kv, c.state, c.step, A.Rotary(1e6, q_weight=qw, k_weight=kw, norm_eps=EPS, weight_offset=offset),
                                      c.q, c.k, c.v, q_out=out, slot_pos=slot_pos)
        assert got is out
        c.check(got, c.pos, 1e6, qw, kw, offset, slot_pos)
        assert bool((out[NQ:] == -5.0).all())                                       # rows behind the last
        assert np.array_equal(c.q.double().cpu().numpy(), c.before[0])              # its inputs are left as they are
        assert np.array_equal(c.k.double().cpu().numpy(), c.before[1])


@pytest.mark.parametrize("layout", ["packed", "fused", "odd"])
def test_where_the_queries_stand(A, layout):
    c = _Call(A, "bf16", 8, 2, 128, 33, layout)
    qw = c.weight()
    got = A.aspd_norm_rope_append(c.kv, c.state, c.step, A.Rotary(1e4, q_weight=qw, norm_eps=EPS), c.q, c.k, c.v)
    assert got is c.q
    c.check(got, c.pos, 1e4, qw)
    if layout == "packed":     # q_out may be q
        c = _Call(A, "bf16", 8, 2, 128, 33, layout)
        c.check(A.aspd_norm_rope_append(c.kv, c.state, c.step, A.Rotary(1e4), c.q, c.k, c.v, q_out=c.q), c.pos, 1e4)


@pytest.mark.parametrize("dtype,hq,hkv,hd", SHAPES[:2] + SHAPES[3:5])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
def test_axes(A, dtype, hq, hkv, hd, axes):
    """Sections, turns, and any assignment of pairs to axes; positions of any sign; a wider array than the step's rows."""
    half = hd // 2
    rng = np.random.default_rng(axes)
    pairs = [half // axes + (half % axes if a == 0 else 0) for a in range(axes)]
    for of_pair in (A.axes_in_sections(pairs), A.axes_in_turn(pairs), rng.integers(0, axes, half).tolist(), None):
        c = _Call(A, dtype, hq, hkv, hd, 41, "fused")
        where = rng.integers(-50, 90_000, size=(axes, 60)).astype(np.int32)
        qw, kw = c.weight(), c.weight()
        got = A.aspd_norm_rope_append(c.kv, c.state, c.step,
                                      A.Rotary(1e6, axis_of_pair=of_pair, axis_pos=torch.from_numpy(where).cuda(), q_weight=qw, k_weight=kw,
                                               norm_eps=EPS), c.q, c.k, c.v, q_out=torch.empty_like(c.q, memory_format=torch.contiguous_format))
        of = np.zeros(half, dtype=int) if of_pair is None else np.array(list(of_pair))
        c.check(got, where[of][:, :41].T, 1e6, qw, kw)


def test_offsets_of_sequences_and_no_rotation(A):
    c = _Call(A, "bf16", 8, 4, 64, 50, "fused")
    offset = np.array([-1000, 0, 7, 90_000, -1], dtype=np.int32)
    slot_pos = torch.full((c.B, c.state.owner_stride), -7, dtype=torch.int32, device="cuda")
    got = A.aspd_norm_rope_append(c.kv, c.state, c.step, A.Rotary(1e4, pos_offset=torch.from_numpy(offset).cuda()), c.q, c.k, c.v,
                                  q_out=torch.empty(50, 8, 64, dtype=torch.bfloat16, device="cuda"), slot_pos=slot_pos)
    c.check(got, c.pos + offset[c.seq], 1e4, slot_pos=slot_pos)      # (slots keep the position ids of Eq. 4)
    for kw in (None, True):
        c = _Call(A, "f32", 8, 4, 64, 50)
        kw = c.weight() if kw else None
        c.check(A.aspd_norm_rope_append(c.kv, c.state, c.step, A.Rotary(0.0, k_weight=kw, norm_eps=EPS), c.q, c.k, c.v), c.pos, 0, None, kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_of_zeros_and_of_large_values(A, dtype):
    """A head of zeros stays zeros, one of large values is normed like any other, an infinity stays in its head."""
    c = _Call(A, dtype, 8, 2, 128, 9)
    c.q[0] = 0
    c.k[1] = 0
    c.q[2] *= 1e15
    c.q[3] *= 1e-15
    c.before[0], c.before[1] = c.q.double().cpu().numpy(), c.k.double().cpu().numpy()
    qw, kw = c.weight(), c.weight()
    how = A.Rotary(1e4, q_weight=qw, k_weight=kw, norm_eps=EPS)
    fresh = torch.empty_like(c.q)
    c.check(A.aspd_norm_rope_append(c.kv, c.state, c.step, how, c.q, c.k, c.v, q_out=fresh), c.pos, 1e4, qw, kw)
    assert not fresh[0].any()
    c.q[5, 3, 7] = float("inf")
    again = A.aspd_norm_rope_append(c.kv, c.state, c.step, how, c.q, c.k, c.v, q_out=torch.empty_like(c.q))
    same = torch.ones(9, 8, dtype=torch.bool, device="cuda")
    same[5, 3] = False
    assert torch.equal(again[same], fresh[same])


def test_as_aspd_rope_append_without_anything_new(A):
    for dtype in ("bf16", "f32"):
        a, b = (_Call(A, dtype, 32, 8, 128, 77) for _ in range(2))
        A.aspd_rope_append(a.kv, a.step, a.q, a.k, a.v, 1e6)
        A.aspd_norm_rope_append(b.kv, b.state, b.step, A.Rotary(1e6), b.q, b.k, b.v)
        b.check(b.q, b.pos, 1e6)
        # fp32 arithmetic of the same formula: apart by the roundings of either
        assert (a.q.double() - b.q.double()).abs().max().item() <= (2.0 ** -7 if dtype == "bf16" else 8 * U) * 8


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_off_a_boundary(A, dtype):
    c = _Call(A, dtype, 8, 2, 128, 21, "fused")
    qw, kw = c.weight(1), c.weight(3)
    out = torch.empty(21, 8, 128, dtype=_type(dtype), device="cuda")
    c.check(A.aspd_norm_rope_append(c.kv, c.state, c.step, A.Rotary(1e4, q_weight=qw, k_weight=kw, norm_eps=EPS), c.q, c.k, c.v, q_out=out),
            c.pos, 1e4, qw, kw)


@pytest.mark.parametrize("hq,hkv,hd", [(16, 4, 128), (6, 6, 64)])
def test_whole_sequences_from_their_tokens(A, hq, hkv, hd):
    """A re-prefill: metadata of whole sequences, one append, one attention call, on an empty cache."""
    from gpu_drive import GpuBatch
    from oracle.sequence_layout import replay_layout
    from test_gpu_sequence import _build
    wl = W.random_small(9, num_q_heads=hq, num_kv_heads=hkv, head_dim=hd, batch=3, prefix_range=(60, 300))
    gb = GpuBatch(wl)
    gb.kv.k.fill_(float("nan"))
    gb.kv.v.fill_(float("nan"))
    layouts = W.random_layouts(wl, seed=4, fill=0.8)
    tt, meta = replay_layout(wl.block_tables, 16, layouts)
    step = _build(A, gb, layouts)
    g = torch.Generator().manual_seed(6)
    weights, rotary = _chain_rotary(A, wl, g, 1e4)
    widths = [hq * hd, hkv * hd, hkv * hd]
    q, k, v = (x.unflatten(1, (-1, hd)) for x in (torch.randn(meta.NQ, sum(widths), generator=g) * 2).bfloat16().cuda().split(widths, 1))
    slot_pos = A.new_slot_pos(gb.state)
    q_out = A.aspd_norm_rope_append(gb.kv, gb.state, step, rotary, q, k, v, q_out=torch.empty(meta.NQ, hq, hd, dtype=torch.bfloat16, device="cuda"),
                                    slot_pos=slot_pos)
    slopes = (2.0 ** (-8.0 * np.arange(1, hq + 1) / hq)).astype(np.float32)
    lse = torch.empty(meta.NQ, hq, dtype=torch.float32, device="cuda")
    out = A.aspd_attn_full_sequence(gb.kv, gb.state, step, q_out, gb.workspace, lse=lse,
                                    scores=A.Scores(8.0, torch.from_numpy(slopes).cuda(), slot_pos))
    want = norm_rotate(q.double().cpu().numpy(), meta.position_ids, 1e4, weights[0].double().numpy(), EPS)
    assert (np.abs(q_out.double().cpu().numpy() - want) <= _bound(want, "bf16")).all()
    assert np.array_equal(slot_pos.cpu().numpy()[meta.q_seq, meta.logical_slot], meta.position_ids)
    ref = attend_scored(tt, meta, q_out.cpu(), gb.kv.k.cpu(), gb.kv.v.cpu(), softcap=8.0, slopes=slopes, score_error=score_error(hd, 8.0))
    check(out, lse, ref, "bf16", label="whole sequences")


def test_a_step_without_tokens_and_a_side_stream(A):
    c = _Call(A, "bf16", 8, 2, 64, 20, "fused")
    c.step.NQ = 0
    out = torch.full((20, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    A.aspd_norm_rope_append(c.kv, c.state, c.step, A.Rotary(1e4), c.q, c.k, c.v, q_out=out)
    assert bool((out == 3.0).all())
    c.step.NQ = 20
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    A.aspd_norm_rope_append(c.kv, c.state, c.step, A.Rotary(1e4), c.q, c.k, c.v, q_out=out, stream=side)
    side.synchronize()
    c.check(out, c.pos, 1e4)


def _chain_rotary(A, wl, g, theta):
    w = [(1 + 0.2 * torch.randn(wl.head_dim, generator=g)).to(wl.torch_dtype) for _ in range(2)]
    return w, A.Rotary(theta, q_weight=w[0].cuda(), k_weight=w[1].cuda(), norm_eps=EPS)


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 32, 8, 128), ("bf16", 12, 4, 64), ("f32", 8, 2, 128)])
@pytest.mark.parametrize("theta,cap,bias", [(1e6, 10.0, False), (0.0, 0.0, True), (1e4, 5.0, True)])
def test_from_new_tokens_to_attention(A, dtype, hq, hkv, hd, theta, cap, bias):
    """Prompts, a branch prefix, decode steps, the merge and a serial step through the operators, from an empty cache: every
    token's key, value and position come from the append, and every step's attention is the oracle's on what is cached."""
    from gpu_drive import GpuBatch
    wl = W.random_small(7, dtype=dtype, num_q_heads=hq, num_kv_heads=hkv, head_dim=hd, batch=3, prefix_range=(20, 200), branches_range=(1, 4))
    gb = GpuBatch(wl)
    gb.kv.k.fill_(float("nan"))          # what nobody appends nobody reads
    gb.kv.v.fill_(float("nan"))
    tt = TokenTable(wl.block_tables, 16)
    slot_pos = A.new_slot_pos(gb.state)
    g = torch.Generator().manual_seed(3)
    weights, rotary = _chain_rotary(A, wl, g, theta)
    slopes = (2.0 ** (-8.0 * np.arange(1, hq + 1) / hq)).astype(np.float32)
    scores = A.Scores(softcap=cap, slopes=torch.from_numpy(slopes).cuda() if bias else None, slot_pos=slot_pos if bias else None)

    def layer(step, meta, fn, label):
        widths = [hq * hd, hkv * hd, hkv * hd]
        qkv = (torch.randn(meta.NQ, sum(widths), generator=g) * 2).to(wl.torch_dtype)
        q, k, v = (x.unflatten(1, (-1, hd)) for x in qkv.cuda().split(widths, 1))
        q_out = torch.empty(meta.NQ, hq, hd, dtype=wl.torch_dtype, device="cuda")
        A.aspd_norm_rope_append(gb.kv, gb.state, step, rotary, q, k, v, q_out=q_out, slot_pos=slot_pos)
        out = torch.empty_like(q_out)
        lse = torch.empty(meta.NQ, hq, dtype=torch.float32, device="cuda")
        fn(gb.kv, gb.state, step, q_out, gb.workspace, out=out, lse=lse, scores=scores)
        torch.cuda.synchronize()
        want = norm_rotate(q.double().cpu().numpy(), meta.position_ids, theta, weights[0].double().numpy(), EPS)
        assert (np.abs(q_out.double().cpu().numpy() - want) <= _bound(want, dtype)).all()
        k_want = norm_rotate(k.double().cpu().numpy(), meta.position_ids, theta, weights[1].double().numpy(), EPS)
        at = torch.from_numpy(meta.slot_mapping).cuda()
        assert (np.abs(gb.kv.k[at // 16, :, at % 16].double().cpu().numpy() - k_want) <= _bound(k_want, dtype)).all()
        for r in range(meta.NQ):
            assert int(slot_pos[int(meta.q_seq[r]), int(meta.logical_slot[r])]) == int(meta.position_ids[r])
        ref = attend_scored(tt, meta, q_out.cpu(), gb.kv.k.cpu(), gb.kv.v.cpu(), softcap=cap, slopes=slopes if bias else None,
                            score_error=score_error(hd, cap))
        check(out, lse, ref, dtype, label=label)

    layer(gb.serial(wl.prefix_len), tt.append_serial(wl.prefix_len), A.aspd_attn_serial_decode, "prompt")
    tt.open_parallel(wl.num_branches)
    gb.open_parallel()
    new = np.minimum(wl.branch_len, 6)
    layer(gb.parallel(new), tt.append_parallel(new), A.aspd_attn_branch_chunk, "prefix of the branches")
    for _ in range(2):
        one = np.ones(wl.NB, dtype=np.int32)
        layer(gb.parallel(one), tt.append_parallel(one), A.aspd_attn_parallel_decode, "decode")
    gb.merge()
    tt.merge()
    one = np.ones(wl.B, dtype=np.int32)
    layer(gb.serial(one), tt.append_serial(one), A.aspd_attn_serial_decode, "serial")
    assert gb.fault() == 0


def test_a_captured_layer(A):
    """Metadata, append and attention of one step in a graph, replayed with the state put back and eager work in between."""
    from gpu_drive import GpuBatch
    wl = W.random_small(8, num_q_heads=16, num_kv_heads=4, head_dim=128, batch=4, prefix_range=(200, 900))
    gb = GpuBatch(wl)
    gb.serial(wl.prefix_len)
    gb.open_parallel()
    gb.parallel(np.minimum(wl.branch_len, 20))
    st = gb.state
    slot_pos = torch.randint(0, 900, (st.B, st.owner_stride), dtype=torch.int32, device="cuda")
    _, rotary = _chain_rotary(A, wl, torch.Generator().manual_seed(1), 1e6)
    scores = A.Scores(softcap=20.0, slopes=torch.full((16,), 0.01, device="cuda"), slot_pos=slot_pos)
    live = [st.stage_base, st.seq_len, st.branch_len, st.slot_owner, st.main_pos]
    snap = [t.clone() for t in live]
    ones = gb._dev_i32(np.ones(wl.NB))
    step = A.Step(wl.NB, wl.NB, wl.B, "cuda", max_new_per_seq=int(wl.num_branches.max()))
    step.plan = torch.empty(A.aspd_plan_bytes(gb.kv, wl.B, wl.NB), dtype=torch.uint8, device="cuda")
    q, k, v = (torch.randn(wl.NB, h, 128, device="cuda").bfloat16() for h in (16, 4, 4))
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    pools = [gb.kv.k.clone(), gb.kv.v.clone(), slot_pos.clone()]

    def layer():
        for dst, src in zip(live, snap):
            dst.copy_(src)
        A.aspd_build_branch_meta(gb.kv, st, A.STAGE_PARALLEL, ones, step=step)
        A.aspd_norm_rope_append(gb.kv, st, step, rotary, q, k, v, q_out=q_out, slot_pos=slot_pos)
        A.aspd_attn_parallel_decode(gb.kv, st, step, q_out, gb.workspace, out=out, scores=scores)

    layer()
    torch.cuda.synchronize()
    want = [t.clone() for t in (q_out, out, gb.kv.k, gb.kv.v, slot_pos)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for _ in range(4):
        for dst, src in zip((gb.kv.k, gb.kv.v, slot_pos), pools):
            dst.copy_(src)
        q_out.fill_(float("nan"))
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((q_out, gb.kv.k, gb.kv.v, slot_pos), (want[0], want[2], want[3], want[4])):
            assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(ref))
        assert (out.float() - want[1].float()).abs().max().item() <= 2 ** -7 * want[1].float().abs().max().item()
