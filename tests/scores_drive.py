"""Test helper: attention calls on changed scores against the float64 oracle, element by element, with the bound that the
arithmetic gives.

A weight is rounded to the cache's type once (bf16: 2^-8 of it) and so is the output; a score is off by the rounding of its
products' sum (D additions in fp32), of the cap (2^-23 of the cap by its formula in bf16 kernels, of the score in fp32 ones) and
of its way into the exponent, by a few halves of 2^-23 of its size.  An error e_j of score j moves the output by no more than
sum p_j e_j |v_j| + |out| sum p_j e_j.  Sums over n keys in fp32 add n 2^-24 at most."""
import numpy as np
import torch

from oracle.scores import attend_scored

U = 2.0 ** -24


def score_error(D, cap):
    """`spread`: |slope| times how far the positions of a sequence's rows of the step lie apart.  Where many rows are taken
    together the bias is a sum of two, slope (p_j - p) and slope (p - p_r), p the position of one of the rows: each no larger
    than |bias| + spread and rounded like it."""
    def of(s_abs, s, bias, spread):
        return U * (D * s_abs + 2 * cap + 8 * (np.abs(s) + np.abs(bias) + 2 * spread) + 8)
    return of


def slot_positions(gb, tt, garbage=True):
    """slot_pos of the batch as the token table has it; slots not in use hold anything."""
    st = gb.state
    rng = np.random.default_rng(5)
    host = rng.integers(-2 ** 31, 2 ** 31, size=(st.B, st.owner_stride), dtype=np.int64) if garbage else np.zeros((st.B, st.owner_stride))
    for s in range(st.B):
        host[s, :len(tt.pos[s])] = tt.pos[s]
    return torch.from_numpy(host.astype(np.int32)).to(gb.dev)


def compare(A, gb, tt, wl, step, meta, fn, cap, bias, rows=None, scale=0.0, shared_mask=False, label="", sigma=1.0, slot_pos=None,
            slopes=None, repeat=1):
    """One call of `fn`, checked; returns what it gave."""
    q = (wl.draw_q(meta.NQ).float() * sigma).to(wl.torch_dtype)
    Hq, D = wl.num_q_heads, wl.head_dim
    if bias and slopes is None:
        slopes = (2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq)).astype(np.float32)
    scores = A.Scores(softcap=cap, slopes=torch.from_numpy(slopes).to(gb.dev) if bias else None,
                      slot_pos=(slot_positions(gb, tt) if slot_pos is None else slot_pos) if bias else None)
    for _ in range(repeat):
        out = torch.full((meta.NQ, Hq, D), float("nan"), dtype=q.dtype, device=gb.dev)
        lse = torch.full((meta.NQ, Hq), float("nan"), dtype=torch.float32, device=gb.dev)
        fn(gb.kv, gb.state, step, q.to(gb.dev), gb.workspace, out=out, lse=lse, sm_scale=scale, scores=scores)
        torch.cuda.synchronize()
    ref = attend_scored(tt, meta, q, wl.k_cache, wl.v_cache, softcap=cap, slopes=slopes if bias else None, scale=scale or None,
                        rows=rows, shared_mask=shared_mask, score_error=score_error(D, cap))
    check(out, lse, ref, wl.dtype, rows, label)
    return out, lse, q, scores


def check(out, lse, ref, dtype, rows=None, label=""):
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    sel = np.arange(out.shape[0]) if rows is None else np.asarray(rows)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    want, mass, err = ref["out"][sel], ref["mass"][sel], ref["error"][sel][..., None]
    n = ref["keys"][sel][:, None]
    sums = (n[..., None] + 16) * U
    bound = half * (mass + np.abs(want)) + ref["error_mass"][sel] + np.abs(want) * err + sums * (mass + np.abs(want))
    off = np.abs(out[sel] - want)
    lse_bound = ref["error"][sel] + (n + 16) * U + 4 * U * np.abs(ref["lse"][sel])
    lse_off = np.abs(lse[sel] - ref["lse"][sel])
    print(f"[{label}] rows={sel.size} out {np.nanmax(off / bound):.3f} and lse {np.nanmax(lse_off / lse_bound):.3f} of the bound", flush=True)
    assert np.isfinite(out[sel]).all() and np.isfinite(lse[sel]).all(), label
    assert (off <= bound).all(), (label, float((off / bound).max()))
    assert (lse_off <= lse_bound).all(), (label, float((lse_off / lse_bound).max()))
