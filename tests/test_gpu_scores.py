"""Attention on changed scores (a tanh cap, a bias by distance) against the float64 oracle: every kernel that takes such a call
(streaming, row-splitting, whole sequences, fp32), both head sizes, and the places where it can go wrong."""
import numpy as np
import pytest
import torch

import aspd_workloads as W
from oracle import TokenTable
from oracle.scores import attend_scored
from oracle.sequence_layout import replay_layout
from scores_drive import check, compare, score_error, slot_positions

pytestmark = pytest.mark.gpu

CHANGES = [(20.0, False), (0.0, True), (3.0, True)]
HEADS = [("bf16", 32, 8, 128), ("bf16", 8, 8, 64), ("bf16", 28, 4, 128), ("f32", 4, 4, 64), ("f32", 8, 2, 128)]


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_08895_amd import binding
    binding.lib()
    return binding


def _both(wl, A, held, pos_mode="same_seq", lib_mode=None):
    """Prefix and `held` tokens per branch on both sides."""
    from gpu_drive import GpuBatch
    gb = GpuBatch(wl)
    tt = TokenTable(wl.block_tables, 16, pos_mode=pos_mode)
    if lib_mode is not None:
        gb.state.pos_mode = lib_mode
    tt.append_serial(wl.prefix_len)
    gb.serial(wl.prefix_len)
    tt.open_parallel(wl.num_branches)
    gb.open_parallel()
    tt.append_parallel(held)
    gb.parallel(held)
    return gb, tt


def _step(A, gb, tt, wl, kind, rng, hint=True):
    """The next step of that kind on both sides: (step, meta, call)."""
    if kind == "serial":
        tt.merge()
        gb.merge()
        new = np.ones(wl.B, dtype=np.int32)
        meta = tt.append_serial(new)
        step = A.aspd_build_branch_meta(gb.kv, gb.state, A.STAGE_SERIAL, gb._dev_i32(new), NQ=meta.NQ, max_new_per_seq=1 if hint else 0)
        return step, meta, A.aspd_attn_serial_decode
    new = np.ones(wl.NB, dtype=np.int32) if kind == "decode" else rng.integers(0, 19, size=wl.NB).astype(np.int32)
    if kind == "chunk":
        new[0] = 19
    meta = tt.append_parallel(new)
    most = int(np.bincount(meta.q_seq, minlength=wl.B).max())
    step = A.aspd_build_branch_meta(gb.kv, gb.state, A.STAGE_PARALLEL, gb._dev_i32(new), NQ=meta.NQ, max_new_per_seq=most if hint else 0)
    return step, meta, A.aspd_attn_parallel_decode if kind == "decode" else A.aspd_attn_branch_chunk


@pytest.mark.parametrize("cap,bias", CHANGES)
@pytest.mark.parametrize("kind", ["decode", "chunk", "serial"])
@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS)
def test_steps(A, dtype, hq, hkv, hd, kind, cap, bias):
    """Ragged batches of short and mid-sized sequences, hinted and not; unwritten slots, unmapped blocks and the positions of
    slots not in use hold anything."""
    for seed, lo, hi in ((3, 0, 60), (4, 150, 800)):
        rng = np.random.default_rng(seed)
        wl = W.random_small(seed, dtype=dtype, num_q_heads=hq, num_kv_heads=hkv, head_dim=hd, batch=3, prefix_range=(lo, hi),
                            branches_range=(1, 7))
        held = np.minimum(wl.branch_len, 20)
        gb, tt = _both(wl, A, held)
        # K and V of slots nobody has written
        tail = [(s, j) for s in range(wl.B) for j in range(len(tt.pos[s]) + 160, wl.max_blocks_per_seq * 16) if wl.block_tables[s, j // 16] >= 0]
        for s, j in tail[::3]:
            gb.kv.k[int(wl.block_tables[s, j // 16]), :, j % 16] = float("nan")
            gb.kv.v[int(wl.block_tables[s, j // 16]), :, j % 16] = float("inf")
        step, meta, fn = _step(A, gb, tt, wl, kind, rng, hint=seed == 4)
        compare(A, gb, tt, wl, step, meta, fn, cap, bias, sigma=4.0, label=f"{kind} {dtype} {hq}/{hkv}x{hd} seed {seed}")
        assert gb.fault() == 0


@pytest.mark.parametrize("cap,bias", CHANGES)
@pytest.mark.parametrize("hq,hkv,hd,batch,prefix", [(32, 8, 128, 1, 6000), (4, 4, 64, 2, 9000), (6, 2, 128, 3, 2500)])
def test_few_long_sequences_split_over_workgroups(A, hq, hkv, hd, batch, prefix, cap, bias):
    """Parts of an item are merged in the launch or behind it."""
    wl = W.random_small(11, num_q_heads=hq, num_kv_heads=hkv, head_dim=hd, batch=batch, prefix_range=(prefix, prefix + 99),
                        branches_range=(3, 6))
    gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20))
    rng = np.random.default_rng(1)
    for kind in ("decode", "chunk", "serial"):
        step, meta, fn = _step(A, gb, tt, wl, kind, rng)
        compare(A, gb, tt, wl, step, meta, fn, cap, bias, sigma=4.0, label=f"{kind} {hq}/{hkv}x{hd} {prefix}")


@pytest.mark.parametrize("cap,bias", CHANGES)
@pytest.mark.parametrize("hq,hkv,hd", [(32, 8, 128), (8, 8, 64), (12, 4, 128)])
def test_prompts(A, hq, hkv, hd, cap, bias):
    """Whole prompts as one serial append: several row groups a sequence, one of them a single token, one empty."""
    wl = W.make_workload("prompts", 21, dtype="bf16", num_q_heads=hq, num_kv_heads=hkv, head_dim=hd, sigma=0.5, prefix_range=None,
                         branches_range=None, branch_len_range=None, batch=5, pool_factor=1.2, extra_tokens_per_branch=0,
                         extra_tokens_per_seq=3, prefix_len=[700, 1, 0, 333, 64], num_branches=[1] * 5, branch_len=[1] * 5)
    from gpu_drive import GpuBatch
    gb = GpuBatch(wl)
    tt = TokenTable(wl.block_tables, 16)
    meta = tt.append_serial(wl.prefix_len)
    step = A.aspd_build_branch_meta(gb.kv, gb.state, A.STAGE_SERIAL, gb._dev_i32(wl.prefix_len), NQ=meta.NQ, max_new_per_seq=700)
    compare(A, gb, tt, wl, step, meta, A.aspd_attn_serial_decode, cap, bias, sigma=4.0, label=f"prompts {hq}/{hkv}x{hd}")


def _sequences(A, wl, layouts, shared=False):
    from gpu_drive import GpuBatch
    from test_gpu_sequence import _build
    gb = GpuBatch(wl)
    tt, meta = replay_layout(wl.block_tables, 16, layouts)
    step = _build(A, gb, layouts)
    step.shared_mask = int(shared)
    return gb, tt, step, meta


@pytest.mark.parametrize("cap,bias", CHANGES)
@pytest.mark.parametrize("hq,hkv,hd,batch,hi,fill", [(32, 8, 128, 3, 900, 1.0), (8, 8, 64, 5, 400, 0.7), (28, 4, 128, 2, 1800, 1.0),
                                                     (4, 1, 64, 1, 3000, 1.0), (3, 3, 128, 6, 50, 0.5)])
def test_whole_sequences(A, hq, hkv, hd, batch, hi, fill, cap, bias):
    """Stages, empty runs, row groups cut into pieces (one long sequence); twice, bit for bit."""
    wl = W.random_small(31 + hi, num_q_heads=hq, num_kv_heads=hkv, head_dim=hd, batch=batch, prefix_range=(hi // 2, hi))
    layouts = W.random_layouts(wl, seed=hi, fill=fill)
    gb, tt, step, meta = _sequences(A, wl, layouts)
    rows = None if meta.NQ < 700 else np.sort(np.random.default_rng(3).choice(meta.NQ, 700, replace=False))
    out, lse, q, scores = compare(A, gb, tt, wl, step, meta, A.aspd_attn_full_sequence, cap, bias, rows=rows, sigma=4.0,
                                  label=f"sequences {hq}/{hkv}x{hd} {hi}")
    again = A.aspd_attn_full_sequence(gb.kv, gb.state, step, q.to(gb.dev), gb.workspace, scores=scores)
    assert torch.equal(out, again)


@pytest.mark.parametrize("cap,bias", CHANGES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_mask(A, dtype, cap, bias):
    wl = W.random_small(41, dtype=dtype, num_q_heads=8, num_kv_heads=2, head_dim=128, batch=3, prefix_range=(5, 300))
    gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20))
    new = np.ones(wl.NB, dtype=np.int32)
    meta = tt.append_parallel(new)
    step = A.Step(meta.NQ, wl.NB, wl.B, gb.dev, max_new_per_seq=8)
    step.shared_mask = 1
    A.aspd_build_branch_meta(gb.kv, gb.state, A.STAGE_PARALLEL, gb._dev_i32(new), step=step)
    compare(A, gb, tt, wl, step, meta, A.aspd_attn_parallel_decode, cap, bias, shared_mask=True, sigma=3.0, label="shared mask")
    if dtype == "bf16":
        layouts = W.random_layouts(wl, seed=9, fill=0.8)
        gb, tt, step, meta = _sequences(A, wl, layouts, shared=True)
        compare(A, gb, tt, wl, step, meta, A.aspd_attn_full_sequence, cap, bias, shared_mask=True, sigma=3.0, label="shared sequences")


@pytest.mark.parametrize("mode,lib", [("same_max", "POS_SAME_MAX"), (("fix", 40), 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distances_are_those_of_the_position_paradigm(A, dtype, mode, lib):
    wl = W.random_small(51, dtype=dtype, num_q_heads=8, num_kv_heads=4, head_dim=64, batch=3, prefix_range=(5, 200))
    gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20), pos_mode=mode, lib_mode=getattr(A, lib) if isinstance(lib, str) else A.POS_FIX_N(lib))
    rng = np.random.default_rng(4)
    for kind in ("decode", "serial"):
        step, meta, fn = _step(A, gb, tt, wl, kind, rng)
        assert np.array_equal(step.position_ids.cpu().numpy()[:meta.NQ], meta.position_ids)
        compare(A, gb, tt, wl, step, meta, fn, 0.0, True, label=f"{kind} {mode}")


@pytest.mark.parametrize("cap", [2.0 ** -10, 0.5, 2.0 ** 10])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, 0.7])
def test_smallest_and_largest_caps_and_a_scale(A, dtype, cap, scale):
    """Far beyond the cap every score is the cap and its sign, far below it the cap changes nothing."""
    wl = W.random_small(61, dtype=dtype, num_q_heads=8, num_kv_heads=4, head_dim=128, batch=2, prefix_range=(100, 400))
    gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20))
    rng = np.random.default_rng(5)
    for kind in ("decode", "chunk"):
        step, meta, fn = _step(A, gb, tt, wl, kind, rng)
        compare(A, gb, tt, wl, step, meta, fn, cap, False, scale=scale, sigma=6.0, label=f"{kind} cap {cap} scale {scale}")


@pytest.mark.parametrize("kind", ["decode", "chunk"])
def test_slopes_of_any_sign_and_size(A, kind):
    """Zero, negative (far keys count more), and so steep that a row is its own key alone."""
    wl = W.random_small(71, num_q_heads=8, num_kv_heads=2, head_dim=128, batch=3, prefix_range=(300, 2000))
    gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20))
    step, meta, fn = _step(A, gb, tt, wl, kind, np.random.default_rng(6))
    slopes = np.array([0.0, -0.01, 1000.0, 1e-6, -1.0, 0.3, 3e4, -3e4], dtype=np.float32)
    out, _, _, _ = compare(A, gb, tt, wl, step, meta, fn, 0.0, True, slopes=slopes, label=f"slopes {kind}")
    own = torch.from_numpy(meta.slot_mapping)
    v = wl.v_cache[own // 16, :, own % 16]
    assert torch.equal(out[:, 6].cpu(), v[:, 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_a_change_it_is_the_plain_call(A, dtype):
    wl = W.random_small(81, dtype=dtype, num_q_heads=8, num_kv_heads=2, head_dim=128, batch=2, prefix_range=(300, 900))
    gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20))
    step, meta, fn = _step(A, gb, tt, wl, "chunk", np.random.default_rng(7))
    q = wl.draw_q(meta.NQ).to(gb.dev)
    assert torch.equal(fn(gb.kv, gb.state, step, q, gb.workspace), fn(gb.kv, gb.state, step, q, gb.workspace, scores=A.Scores()))


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 17), ("f32", 1)])
def test_steps_of_serial_and_parallel_sequences(A, dtype, new):
    """MIXED: branch tokens of two sequences and main-branch tokens of one, a second stage behind a merged one."""
    from gpu_drive import GpuBatch
    wl = W.random_small(85, dtype=dtype, num_q_heads=8, num_kv_heads=2, head_dim=128, batch=3, prefix_range=(90, 700), branches_range=(3, 3),
                        extra_tokens_per_branch=60)
    gb = GpuBatch(wl)
    tt = TokenTable(wl.block_tables, 16)
    tt.append_serial(wl.prefix_len)
    gb.serial(wl.prefix_len)
    fn = A.aspd_attn_parallel_decode if new == 1 else A.aspd_attn_branch_chunk
    for count in ([2, 0, 3], [3, 2, 0]):
        tt.open_parallel(count)
        gb.renumber(count)
        for tokens in (5, new):
            nb = np.full(sum(count), tokens, dtype=np.int32)
            nm = np.array([tokens if k == 0 else 0 for k in count], dtype=np.int32)
            meta = tt.append_mixed(nb, nm)
            step = gb.mixed(nb, nm)
            compare(A, gb, tt, wl, step, meta, fn if tokens == new else A.aspd_attn_branch_chunk, 12.0, True, sigma=3.0,
                    label=f"mixed {dtype} {tokens}")
        tt.merge()
        gb.merge()
    assert gb.fault() == 0


def test_a_long_context(A):
    """70 000 tokens: positions and offsets of a long cache, a bias that fades, sampled rows."""
    wl = W.make_workload("long", 91, dtype="bf16", num_q_heads=4, num_kv_heads=1, head_dim=64, sigma=0.5, prefix_range=None,
                         branches_range=None, branch_len_range=None, batch=1, pool_factor=1.0, extra_tokens_per_branch=24,
                         extra_tokens_per_seq=4, prefix_len=[70_000], num_branches=[3], branch_len=[4, 1, 9])
    gb, tt = _both(wl, A, wl.branch_len)
    rng = np.random.default_rng(8)
    slopes = np.array([1e-4, 1e-3, 0.0, -1e-4], dtype=np.float32)
    for kind in ("decode", "chunk"):
        step, meta, fn = _step(A, gb, tt, wl, kind, rng)
        compare(A, gb, tt, wl, step, meta, fn, 30.0, True, slopes=slopes, sigma=4.0, label=f"long {kind}")


@pytest.mark.parametrize("kind", ["decode", "chunk", "sequences"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_replayed(A, kind, dtype):
    """A captured call, replayed with eager calls on the same workspace in between."""
    if dtype == "f32" and kind == "sequences":
        pytest.skip("whole sequences are bf16 only")
    wl = W.random_small(101, dtype=dtype, num_q_heads=8, num_kv_heads=2, head_dim=64, batch=3, prefix_range=(50, 1200))
    if kind == "sequences":
        gb, tt, step, meta = _sequences(A, wl, W.random_layouts(wl, seed=5))
        fn = A.aspd_attn_full_sequence
    else:
        gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20))
        step, meta, fn = _step(A, gb, tt, wl, kind, np.random.default_rng(9))
    out, lse, q, scores = compare(A, gb, tt, wl, step, meta, fn, 10.0, True, sigma=3.0, label=f"eager {kind}", repeat=2)
    q = q.to(gb.dev)
    got, got_lse = torch.empty_like(out), torch.empty_like(lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn(gb.kv, gb.state, step, q, gb.workspace, out=got, lse=got_lse, scores=scores)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fn(gb.kv, gb.state, step, q, gb.workspace, out=got, lse=got_lse, scores=scores)
    for _ in range(4):
        got.fill_(float("nan"))
        got_lse.fill_(float("nan"))
        fn(gb.kv, gb.state, step, q, gb.workspace)      # the plain call, on the same workspace
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (got.float() - out.float()).abs().max().item() <= 2 ** -7 * out.float().abs().max().item()
        assert (got_lse - lse).abs().max().item() <= 1e-4


def test_two_streams(A):
    """Two batches at once, a workspace each."""
    sides = []
    for seed in (111, 112):
        wl = W.random_small(seed, num_q_heads=16, num_kv_heads=4, head_dim=128, batch=4, prefix_range=(300, 1500))
        gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20))
        step, meta, fn = _step(A, gb, tt, wl, "decode", np.random.default_rng(seed))
        out, lse, q, scores = compare(A, gb, tt, wl, step, meta, fn, 10.0, True, sigma=3.0, label=f"alone {seed}")
        sides.append((gb, step, fn, out, q.to(gb.dev), scores, torch.empty_like(out), torch.cuda.Stream()))
    for _ in range(4):
        torch.cuda.synchronize()
        for gb, step, fn, _, q, scores, got, stream in sides:
            with torch.cuda.stream(stream):
                for _ in range(4):
                    fn(gb.kv, gb.state, step, q, gb.workspace, out=got, scores=scores)
        torch.cuda.synchronize()
        for _, _, _, out, _, _, got, _ in sides:
            assert (got.float() - out.float()).abs().max().item() <= 2 ** -7 * out.float().abs().max().item()


def test_a_grid_of_few_workgroups(A):
    """Many segments a workgroup, several windows of block ids."""
    wl = W.random_small(121, num_q_heads=8, num_kv_heads=4, head_dim=64, batch=3, prefix_range=(9000, 12000), branches_range=(2, 3))
    gb, tt = _both(wl, A, np.minimum(wl.branch_len, 20))
    new = np.ones(wl.NB, dtype=np.int32)
    meta = tt.append_parallel(new)
    step = A.aspd_build_branch_meta(gb.kv, gb.state, A.STAGE_PARALLEL, gb._dev_i32(new), NQ=meta.NQ, max_new_per_seq=3, max_workgroups=2)
    compare(A, gb, tt, wl, step, meta, A.aspd_attn_parallel_decode, 10.0, True, sigma=3.0, label="two workgroups")


@pytest.mark.parametrize("tokens", [3, 90])     # the streaming, the row-splitting kernel
def test_rows_of_a_refused_sequence_may_hold_anything(A, tokens):
    """One sequence of the step outgrows its block table and is refused: its rows of the step keep what was there, and the others
    are attended as if it were not there."""
    from gpu_drive import GpuBatch
    wl = W.random_small(131, num_q_heads=8, num_kv_heads=2, head_dim=128, batch=3, prefix_range=(150, 300))
    gb = GpuBatch(wl)
    tt = TokenTable(wl.block_tables, 16)
    room = [16 * int((row >= 0).sum()) for row in wl.block_tables]
    have = np.array([room[0] - 100, room[1] - 100, room[2] - 100], dtype=np.int32)
    tt.append_serial(have)
    gb.serial(have)
    new = np.array([tokens, 200, tokens], dtype=np.int32)
    step = A.Step(int(new.sum()), wl.B, wl.B, gb.dev, max_new_per_seq=200 if tokens > 3 else 6)
    for t in (step.logical_slot, step.position_ids, step.q_branch, step.kv_len):
        t.fill_(0x3fffffff)
    A.aspd_build_branch_meta(gb.kv, gb.state, A.STAGE_SERIAL, gb._dev_i32(new), step=step)
    assert gb.fault() & A.FAULT_BLOCK_TABLE
    keep = np.r_[0:tokens, tokens + 200:2 * tokens + 200]
    meta = tt.append_serial(np.array([tokens, 0, tokens], dtype=np.int32))
    assert np.array_equal(step.logical_slot.cpu().numpy()[keep], meta.logical_slot)
    q = wl.draw_q(step.NQ)
    slopes = np.full(8, 0.05, dtype=np.float32)
    scores = A.Scores(softcap=10.0, slopes=torch.from_numpy(slopes).to(gb.dev), slot_pos=slot_positions(gb, tt))
    lse = torch.zeros(step.NQ, 8, device=gb.dev)
    out = A.aspd_attn_serial_decode(gb.kv, gb.state, step, q.to(gb.dev), gb.workspace, lse=lse, scores=scores)
    ref = attend_scored(tt, meta, q[keep], wl.k_cache, wl.v_cache, softcap=10.0, slopes=slopes, score_error=score_error(128, 10.0))
    check(out[keep], lse[keep], ref, "bf16", label=f"beside a refused sequence, {tokens} tokens")
