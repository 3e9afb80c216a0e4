"""What the calls on changed scores and the norm-and-rotary append refuse, before anything would be launched (no GPU needed):
through the C ABI and through the binding."""
import ctypes as C

import pytest
import torch

from paper_2508_08895_amd import binding as A
from test_library_abi import _kv

_STATE = dict(B=2, NB=2, stage_base_d=0x10, seq_len_d=0x20, cu_branches_d=0x30, branch_len_d=0x40, slot_owner_d=0x50, owner_stride=64)
_STEP = dict(NQ=2, cu_new_d=0x10, cu_seq_new_d=0x10, q_seq_d=0x10, q_branch_d=0x10, position_ids_d=0x10, logical_slot_d=0x10,
             slot_mapping_d=0x10, kv_len_d=0x10)


def _append(kv=None, state=None, step=None, q=0x100, qs=0, k=0x200, ks=0, v=0x300, vs=0, q_out=0x400, slot_pos=0x500, no_state=False, **how):
    L = A.lib()
    st, sp = A.aspd_state(**{**_STATE, **(state or {})}), A.aspd_step(**{**_STEP, **(step or {})})
    h = A.aspd_rotary(**{**dict(rope_theta=1e4, norm_eps=1e-6), **how})
    kvs = kv or _kv()
    return L.aspd_norm_rope_append(C.byref(kvs), None if no_state else C.byref(st), C.byref(sp), C.byref(h), q, qs, k, ks, v, vs, q_out,
                                   slot_pos, None)


def test_append_refuses():
    bad = A.ERR_INVALID_ARG
    assert _append(kv=_kv(head_dim=96)) == A.ERR_UNSUPPORTED
    assert _append(kv=_kv(dtype=3)) == A.ERR_UNSUPPORTED
    assert _append(q=None) == bad and _append(k=None) == bad and _append(v=None) == bad
    for theta in (1.0, 0.5, -3.0, float("nan"), float("inf")):
        assert _append(rope_theta=theta) == bad, theta
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert _append(q_weight_d=0x600, norm_eps=eps) == bad
        assert _append(k_weight_d=0x600, norm_eps=eps) == bad
    assert _append(q_weight_d=0x600, weight_offset=float("nan")) == bad
    assert _append(qs=32 * 128 - 1) == bad and _append(ks=8 * 128 - 1) == bad and _append(vs=-8) == bad
    assert _append(q_out=0x100, qs=32 * 128 + 8) == bad                       # in place, but not packed
    assert _append(step=dict(NQ=-1)) == bad
    for name in ("position_ids_d", "slot_mapping_d", "q_seq_d", "logical_slot_d"):
        assert _append(step={name: None}) == bad, name
    assert _append(no_state=True) == bad                                      # slot_pos needs its sizes
    assert _append(state=dict(owner_stride=0)) == bad
    assert _append(slot_pos=None, pos_offset_d=0x700, no_state=True) == bad
    assert _append(slot_pos=None, pos_offset_d=0x700, step=dict(q_seq_d=None)) == bad
    axes = dict(axis_pos_d=0x700, axis_stride=2, num_axes=3)
    assert _append(**{**axes, "axis_stride": 1}) == bad
    assert _append(**{**axes, "num_axes": 0}) == bad
    assert _append(**{**axes, "num_axes": 5}) == A.ERR_UNSUPPORTED
    assert _append(**axes, pos_offset_d=0x800) == bad                         # one or the other
    of_pair = (C.c_uint8 * 64)(*([2] * 63 + [3]))
    assert _append(**axes, axis_of_pair=C.cast(of_pair, C.c_void_p)) == bad   # an axis that is not there
    L = A.lib()
    kv, sp, st = _kv(), A.aspd_step(**_STEP), A.aspd_state(**_STATE)
    assert L.aspd_norm_rope_append(C.byref(kv), C.byref(st), C.byref(sp), None, 0x100, 0, 0x200, 0, 0x300, 0, 0x400, None, None) == bad
    assert L.aspd_norm_rope_append(C.byref(kv), C.byref(st), None, None, 0x100, 0, 0x200, 0, 0x300, 0, 0x400, None, None) == bad
    assert _append(step=dict(NQ=0), q=None) == A.OK                           # nothing to do, nothing launched


_CALLS = ("aspd_attn_parallel_decode_scored", "aspd_attn_branch_chunk_scored", "aspd_attn_serial_decode_scored")


@pytest.mark.parametrize("name", _CALLS)
def test_scored_calls_refuse(name):
    L = A.lib()

    def attn(kv=None, state=None, step=None, q=0x100, ws=0x300, no_scores=False, **sc):
        kvs, st, sp = kv or _kv(), A.aspd_state(**{**_STATE, **(state or {})}), A.aspd_step(**{**_STEP, **(step or {})})
        s = A.aspd_scores(**sc)
        return getattr(L, name)(C.byref(kvs), C.byref(st), C.byref(sp), None if no_scores else C.byref(s), q, 0x200, None, 0.0, ws, 1 << 30, None)

    bad = A.ERR_INVALID_ARG
    assert attn(no_scores=True) == bad
    for cap in (-1.0, float("nan"), float("inf")):
        assert attn(softcap=cap) == bad, cap
    for cap in (2.0 ** -11, 2.0 ** 10 * 1.0001, 1e30, 1e-30):
        assert attn(softcap=cap) == A.ERR_UNSUPPORTED, cap
    assert attn(slopes_d=0x600) == bad                                        # distances need positions
    ok = dict(slopes_d=0x600, slot_pos_d=0x700)
    assert attn(**ok, step=dict(position_ids_d=None)) == bad
    assert attn(**ok, state=dict(owner_stride=60)) == bad                     # fewer than the block table's slots
    # and what the call of the same name refuses
    assert attn(**ok, q=0x104) == bad and attn(**ok, ws=0x310) == bad and attn(**ok, kv=_kv(head_dim=96)) == A.ERR_UNSUPPORTED
    assert attn(**ok, step=dict(NQ=0), q=None) == A.OK


def test_scored_sequences_refuse_a_step_of_another_kind():
    L = A.lib()
    kv, st, sp, sc = _kv(), A.aspd_state(**_STATE), A.aspd_step(**_STEP), A.aspd_scores(softcap=1.0)
    fn = L.aspd_attn_full_sequence_scored
    assert fn(C.byref(kv), C.byref(st), C.byref(sp), None, 0x100, 0x200, None, 0.0, 0x300, 1 << 30, None) == A.ERR_INVALID_ARG
    assert fn(C.byref(kv), C.byref(st), C.byref(sp), C.byref(sc), 0x100, 0x200, None, 0.0, 0x300, 1 << 30, None) == A.ERR_INVALID_ARG
    kv = _kv(dtype=A.F32)
    assert fn(C.byref(kv), C.byref(st), C.byref(sp), C.byref(sc), 0x100, 0x200, None, 0.0, 0x300, 1 << 30, None) == A.ERR_UNSUPPORTED


class _Stream:
    cuda_stream = 0


def _objects():
    kv = A.KVCache(torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16),
                   torch.zeros(3, 4, dtype=torch.int32), 8)
    return kv, A.BatchState(3, 64, "cpu"), A.Step(6, 3, 3, "cpu")


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


@pytest.mark.parametrize("what,over", [
    ("q", dict(q=_t(6, 8, 32))), ("q", dict(q=_t(5, 8, 64))), ("q", dict(q=_t(6, 512))), ("q", dict(q=_t(6, 8, 64, dtype=torch.float32))),
    ("q", dict(q=_t(6, 64, 8).transpose(1, 2))), ("q", dict(q=_t(6, 16, 64)[:, ::2])), ("q", dict(q=_t(1, 8, 64).expand(6, 8, 64))),
    ("q", dict(q=None)), ("q", dict(q=3)), ("k_new", dict(k=_t(6, 8, 64))), ("v_new", dict(v=_t(6, 2, 64).to_sparse())),
    ("q_out", dict(q_out=_t(6, 9, 64)[:, :8])), ("slot_pos", dict(slot_pos=_t(3, 64))), ("slot_pos", dict(slot_pos=_t(3, 60, dtype=torch.int32))),
    ("slot_pos", dict(slot_pos=_t(2, 64, dtype=torch.int32))), ("slot_pos", dict(slot_pos=_t(3, 128, dtype=torch.int32)[:, ::2])),
    ("q_weight", dict(how=dict(q_weight=_t(63)))), ("k_weight", dict(how=dict(k_weight=_t(64, dtype=torch.float32)))),
    ("k_weight", dict(how=dict(k_weight=_t(128)[::2]))), ("pos_offset", dict(how=dict(pos_offset=_t(2, dtype=torch.int32)))),
    ("pos_offset", dict(how=dict(pos_offset=_t(3, dtype=torch.int64)))), ("axis_pos", dict(how=dict(axis_pos=_t(3, 5, dtype=torch.int32)))),
    ("axis_pos", dict(how=dict(axis_pos=_t(18, dtype=torch.int32)))), ("axis_pos", dict(how=dict(axis_pos=_t(6, 3, dtype=torch.int32).t()))),
    ("axis_of_pair", dict(how=dict(axis_pos=_t(3, 6, dtype=torch.int32), axis_of_pair=[0] * 31)))])
def test_binding_names_the_argument_it_refuses(what, over):
    kv, st, sp = _objects()
    how = A.Rotary(1e4, **over.pop("how", {}))
    a = dict(q=_t(6, 8, 64), k=_t(6, 2, 64), v=_t(6, 2, 64), q_out=None, slot_pos=None)
    a.update(over)
    with pytest.raises(ValueError, match=f"^{what}: "):
        A.aspd_norm_rope_append(kv, st, sp, how, a["q"], a["k"], a["v"], q_out=a["q_out"], slot_pos=a["slot_pos"], stream=_Stream)


def test_binding_raises_what_the_library_says():
    kv, st, sp = _objects()
    q, k = _t(6, 8, 64), _t(6, 2, 64)
    with pytest.raises(A.AspdError, match="aspd_norm_rope_append: invalid argument"):
        A.aspd_norm_rope_append(kv, st, sp, A.Rotary(1.0), q, k, k, stream=_Stream)
    with pytest.raises(A.AspdError, match="aspd_norm_rope_append: unsupported"):
        A.aspd_norm_rope_append(kv, st, sp, A.Rotary(1e4, axis_pos=_t(5, 6, dtype=torch.int32)), q, k, k, stream=_Stream)
    with pytest.raises(TypeError):
        A.aspd_norm_rope_append(kv, st, sp, A.Rotary("1"), q, k, k, stream=_Stream)
    ws = torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(A.AspdError, match="aspd_attn_serial_decode_scored: invalid argument"):
        A.aspd_attn_serial_decode(kv, st, sp, q, ws, stream=_Stream, scores=A.Scores(softcap=-1.0))
    with pytest.raises(ValueError, match="^slopes: "):
        A.aspd_attn_serial_decode(kv, st, sp, q, ws, stream=_Stream, scores=A.Scores(slopes=_t(8)))
    with pytest.raises(ValueError, match="^slopes: "):
        A.aspd_attn_serial_decode(kv, st, sp, q, ws, stream=_Stream, scores=A.Scores(slopes=_t(7, dtype=torch.float32)))
    with pytest.raises(ValueError, match="^slot_pos: "):
        A.aspd_attn_serial_decode(kv, st, sp, q, ws, stream=_Stream, scores=A.Scores(slopes=_t(8, dtype=torch.float32), slot_pos=_t(3, 64)))
    sp.NQ = 0
    assert A.aspd_attn_serial_decode(kv, st, sp, q, ws, out=q, stream=_Stream, scores=A.Scores(softcap=5.0)) is q
    assert A.aspd_norm_rope_append(kv, st, sp, A.Rotary(1e4), q, k, k, stream=_Stream) is q


def test_axes_of_pairs():
    assert list(A.axes_in_sections([2, 3, 1])) == [0, 0, 1, 1, 1, 2]
    assert list(A.axes_in_turn([4, 2, 2])) == [0, 1, 2, 0, 1, 2, 0, 0]
    assert list(A.axes_in_turn([8])) == [0] * 8
    assert A.Rotary(1e4, axis_of_pair=[0, 1]).axis_of_pair == b"\x00\x01"
