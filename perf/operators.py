"""What the operators around a layer's positions and scores are measured on: the way of new queries, keys and values into
attention (a norm per head, rotary positions on one or several axes, the append to the paged cache) and the attention calls
on capped and distance-biased scores.

A case is one call of one layer over a batch whose step is prepared, as a decoding program has it when it reaches the
layer.  Kinds of step:
  decode     one token per branch of sequences in a parallel stage
  serial     the stage has been merged, one main-branch token per sequence
  chunk      several tokens per branch (a forced branch prefix, teacher-forced pieces)
  prefill    prompts: all tokens of a batch of empty sequences
  sequences  whole multi-stage sequences, every token a row
Formulas: row r of sequence s, heads h, keys j in the cache of s,
  append     x' = x / sqrt(mean(x^2) + eps) * w per head of q and k, pair (i, i + D/2) turned by position(axis(i)) theta^(-2i/D);
             q' returned, k' and v to the cache at the token's slot, the token's position to slot_pos
  attention  s = scale q.k;  s = cap tanh(s / cap) with a cap;  s += slope[h] (slot_pos[j] - position[r]) with slopes;
             softmax over the keys r may see (its own branch and everything before its stage), times v; log-sum-exp
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
THETA = 1e6
EPS = 1e-6

_7B = dict(dtype="bf16", hq=32, hkv=8, hd=128)       # the benchmark configurations' heads
_SMALL = dict(dtype="bf16", hq=16, hkv=4, hd=64)
_F32 = dict(dtype="f32", hq=4, hkv=4, hd=64)


def _case(op, kind, name=None, *, batch, prefix, branches=(1, 1), held=(0, 0), new=(1, 1), shape=1, dtype, hq, hkv, hd, **how):
    c = dict(op=op, kind=kind, batch=batch, prefix_lo=prefix[0], prefix_hi=prefix[1], branches_lo=branches[0], branches_hi=branches[1],
             held_lo=held[0], held_hi=held[1], new_lo=new[0], new_hi=new[1], shape=shape, dtype=dtype, hq=hq, hkv=hkv, hd=hd, **how)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call there is: three branches of one short sequence in fp32; a launch is all of it
        _case("append", "decode", "append_tiny_f32", batch=1, prefix=(64, 64), branches=(3, 3), held=(4, 15), axes=1, norm=True,
              fused=False, **_F32),
        # one step of a serving batch, queries, keys and values as one projection leaves them; sequences that began with
        # images, whose text positions lag behind their token counts
        _case("append", "decode", "append_decode", batch=64, prefix=(500, 2500), branches=(2, 10), held=(24, 144), axes=3, norm=True,
              fused=True, **_7B),
        # prompts with images: time, height and width are axes of their own
        _case("append", "prefill", "append_images", batch=8, prefix=(90, 2000), axes=3, norm=True, fused=True, **_7B),
        # teacher forcing: all tokens of whole sequences at once (bandwidth)
        _case("append", "sequences", "append_sequences", batch=24, prefix=(700, 7000), branches=(1, 8), axes=1, norm=True, fused=True,
              **_7B),
        # configuration 1 with a distance bias in the place of rotary positions: latency, fp32
        _case("attention", "decode", "bias_tiny_f32", batch=1, prefix=(64, 64), branches=(3, 3), held=(4, 15), cap=0.0, bias=True,
              **_F32),
        # configuration 2, one user's conversation, scores capped: the latency of interactive decoding
        _case("attention", "decode", "cap_single", batch=1, prefix=(2048, 2048), branches=(4, 4), held=(63, 63), cap=50.0, bias=False,
              **_7B),
        # configuration 5, a large serving batch: the bandwidth of the cache reads
        _case("attention", "decode", "cap_batch64", batch=64, prefix=(1024, 8192), branches=(2, 10), held=(24, 144), cap=50.0,
              bias=False, **_7B),
        # after the merge, one token per sequence of an odd batch, smaller heads, both changes of the scores
        _case("attention", "serial", "both_serial_hd64", batch=27, prefix=(37, 3001), branches=(1, 5), held=(1, 90), cap=30.0, bias=True,
              **_SMALL),
        # a stage opens: branch prefixes of ragged length behind mid-sized contexts
        _case("attention", "chunk", "bias_stage_open", batch=12, prefix=(200, 5000), branches=(2, 5), new=(5, 21), cap=0.0, bias=True,
              **_7B),
        # the 16-token chunk over a batch
        _case("attention", "chunk", "cap_chunk", batch=32, prefix=(1024, 8192), branches=(2, 10), held=(8, 128), new=(16, 16), cap=50.0,
              bias=False, **_7B),
        # a few short sequences rebuilt whole
        _case("attention", "sequences", "both_short_sequences", batch=3, prefix=(301, 1500), branches=(2, 5), cap=30.0, bias=True, **_7B),
        # teacher forcing over longer ones: matrix products and the softmax between them
        _case("attention", "sequences", "cap_sequences", batch=8, prefix=(1100, 6000), branches=(1, 8), cap=50.0, bias=False, **_7B),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    shape = rng.randrange(1 << 20)
    heads = rng.choice([_7B, _7B, _7B, _SMALL, dict(dtype="bf16", hq=28, hkv=4, hd=128), dict(dtype="bf16", hq=6, hkv=6, hd=64)])
    f32 = rng.random() < 0.15  # fp32 is for small calls
    if f32:
        heads = rng.choice([_F32, dict(dtype="f32", hq=8, hkv=2, hd=128)])
    if rng.random() < 0.4:
        kind = rng.choice(["decode", "serial", "chunk", "prefill", "sequences"])
        hi = log_int(20, 600 if f32 else 7000)
        batch = log_int(1, max(1.5, min(64, (2000 if f32 else 60_000) / hi)))
        return _case("append", kind, batch=batch, prefix=(max(1, hi // rng.randint(1, 9)), hi), branches=(1, rng.randint(2, 9)),
                     held=(0, rng.randint(1, 150)), new=(2, rng.randint(3, 24)) if kind == "chunk" else (1, 1), shape=shape,
                     axes=rng.choice([1, 1, 2, 3]), norm=rng.random() < 0.8, fused=rng.random() < 0.6, **heads)
    kind = rng.choice(["decode", "decode", "serial", "chunk", "prefill", "sequences"])
    if f32 and kind in ("prefill", "sequences"):
        kind = "decode"
    how = rng.choice([dict(cap=round(rng.uniform(5, 60), 1), bias=False), dict(cap=0.0, bias=True),
                      dict(cap=round(rng.uniform(5, 60), 1), bias=True)])
    if kind in ("prefill", "sequences"):
        hi = log_int(60, 6000)
        batch = log_int(1, max(1.5, min(48, 9e9 / (heads["hq"] * hi * hi))))
        return _case("attention", kind, batch=batch, prefix=(max(1, hi // rng.randint(2, 9)), hi), branches=(1, rng.randint(2, 9)),
                     shape=shape, **how, **heads)
    hi = log_int(40, 600) if f32 else log_int(60, 16000)
    batch = log_int(1, 6) if f32 else log_int(1, max(1.5, min(64, (120_000 if kind == "chunk" else 300_000) / hi)))
    return _case("attention", kind, batch=batch, prefix=(max(1, hi // rng.randint(1, 8)), hi), branches=(rng.randint(1, 3), rng.randint(3, 10)),
                 held=(rng.randint(0, 20), rng.randint(21, 60 if f32 else 200)),
                 new=(rng.randint(2, 8), rng.randint(9, 24)) if kind == "chunk" else (1, 1), shape=shape, **how, **heads)


# ------------------------------------------------------------------------------------------------ lengths
def _sequences(case):
    """Per sequence its runs of tokens in cache order, (stage, branch, first position, tokens), branch 0 the main one, and how
    many leading runs were in the cache before the step.  From the case alone."""
    r = random.Random(case["shape"])
    kind, out = case["kind"], []
    for n in [r.randint(case["prefix_lo"], case["prefix_hi"]) for _ in range(case["batch"])]:
        if kind == "prefill":
            out.append(([(0, 0, 0, n)], 0))
            continue
        if kind == "sequences":
            stages = r.randint(0, 3)
            w = [r.random() + 0.05 for _ in range(2 * stages + 1)]
            part = [int(n * x / sum(w)) for x in w]
            part[0] += n - sum(part)
            runs, at = [], 0
            for i, m in enumerate(part):
                if i % 2 == 0:
                    runs.append((i, 0, at, m))
                else:
                    k = r.randint(case["branches_lo"], case["branches_hi"])
                    cut = [0] + sorted(r.randint(0, m) for _ in range(k - 1)) + [m]
                    runs += [(i, b + 1, at, cut[b + 1] - cut[b]) for b in range(k)]
                at += m
            out.append((runs, 0))
            continue
        held = [r.randint(case["held_lo"], case["held_hi"]) for _ in range(r.randint(case["branches_lo"], case["branches_hi"]))]
        new = [r.randint(case["new_lo"], case["new_hi"]) for _ in held]
        runs = [(0, 0, 0, n)] + [(1, b + 1, n, h) for b, h in enumerate(held)]
        old = len(runs)
        if kind == "serial":
            runs.append((2, 0, n + sum(held), 1))
        else:
            runs += [(1, b + 1, n + h, m) for b, (h, m) in enumerate(zip(held, new))]
        out.append((runs, old))
    return out


def _tokens(runs):
    """stage, branch, position of every token of a sequence, in cache order."""
    n = np.array([x[3] for x in runs])
    first = np.repeat(np.cumsum(n) - n, n)
    within = np.arange(n.sum()) - first
    return (np.repeat([x[0] for x in runs], n), np.repeat([x[1] for x in runs], n), np.repeat([x[2] for x in runs], n) + within)


def _seen(case):
    """(tokens in the caches, new tokens, keys that the new tokens attend)."""
    tokens = rows = keys = 0
    for runs, old in _sequences(case):
        start, total = {}, 0
        before = {}
        for i, (stage, branch, _, n) in enumerate(runs):
            start.setdefault(stage, total)
            if i >= old:
                seen = total if branch == 0 else start[stage] + before.get((stage, branch), 0)
                keys += n * seen + n * (n + 1) // 2
                rows += n
            before[(stage, branch)] = before.get((stage, branch), 0) + n
            total += n
        tokens += total
    return tokens, rows, keys


# ------------------------------------------------------------------------------------------------ state
class _State:
    pass


def _axis_of_pair(case):
    """Which axis a pair turns by: sections of the head, the first axis (time) a quarter of it."""
    half, axes = case["hd"] // 2, case["axes"]
    t = half if axes == 1 else half // 4
    return [0 if i < t else 1 + (i - t) * (axes - 1) // (half - t) for i in range(half)]


def _inputs(case, seed):
    """The arrays of one call, on the GPU."""
    st = _State()
    dev = torch.device("cuda")
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, sigma=1.0):
        return torch.randn(*shape, generator=gen, device=dev, dtype=dtype) * sigma

    def i32(x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(dev)

    seqs = _sequences(case)
    B = len(seqs)
    total = [sum(x[3] for x in runs) for runs, _ in seqs]
    blocks = [(t + BLOCK - 1) // BLOCK for t in total]
    # a pool with some room to spare, its blocks dealt to the sequences at random
    pool = sum(blocks) + sum(blocks) // 8 + 1
    order = np.random.default_rng(seed).permutation(pool)
    tables = np.zeros((B, max(blocks)), dtype=np.int32)
    width = max(blocks) * BLOCK
    owner = np.zeros((B, width), dtype=np.uint8)
    slot_pos = np.zeros((B, width), dtype=np.int32)
    q_seq, slot, pos, tag, base, at = [], [], [], [], [], 0
    for s, ((runs, old), n) in enumerate(zip(seqs, blocks)):
        tables[s, :n] = order[at:at + n]
        at += n
        stage, branch, p = _tokens(runs)
        m, first = len(stage), sum(x[3] for x in runs[:old])
        owner[s, :m] = branch
        slot_pos[s, :m] = p
        q_seq.append(np.full(m - first, s))
        slot.append(np.arange(first, m))
        pos.append(p[first:])
        tag.append(branch[first:])
        start = {}
        for k, x in enumerate(runs):
            start.setdefault(x[0], sum(y[3] for y in runs[:k]))
        base.append(np.array([start.get(i, 0) for i in range(max(start) + 1)])[stage[first:]])
    q_seq, slot, pos, tag, base = (np.concatenate(x) for x in (q_seq, slot, pos, tag, base))
    rows = len(q_seq)
    count = np.bincount(q_seq, minlength=B)
    st.case, st.B, st.rows, st.count, st.seqs = case, B, rows, count, seqs
    st.tables, st.owner, st.slot_pos = i32(tables), torch.from_numpy(owner).to(dev), i32(slot_pos)
    st.q_seq, st.slot, st.pos, st.tag, st.base = (i32(x) for x in (q_seq, slot, pos, tag, base))
    st.slot_mapping = torch.from_numpy(tables[q_seq, slot // BLOCK].astype(np.int64) * BLOCK + slot % BLOCK).to(dev)
    st.k_cache, st.v_cache = normal(pool, hkv, BLOCK, hd), normal(pool, hkv, BLOCK, hd)
    if case["op"] == "append":
        width = [hq * hd, hkv * hd, hkv * hd]
        if case["fused"]:
            parts = normal(rows, sum(width), sigma=2.0).split(width, dim=1)
        else:
            parts = [normal(rows, w, sigma=2.0) for w in width]
        st.q, st.k_new, st.v_new = (x.unflatten(1, (-1, hd)) for x in parts)
        st.q_out = torch.empty(rows, hq, hd, device=dev, dtype=dtype)
        st.q_weight, st.k_weight = (1 + normal(hd, sigma=0.2), 1 + normal(hd, sigma=0.2)) if case["norm"] else (None, None)
        st.axis_of_pair = _axis_of_pair(case)
        st.axis_pos = st.offset = None
        if case["axes"] > 1:
            # a decoding step: every axis goes on from where the prompt's image left it; a prompt: a grid in the middle of it
            if case["kind"] in ("prefill", "sequences"):
                g = np.random.default_rng(seed + 1)
                side = max(1, int(math.sqrt(rows / 4)))
                st.axis_pos = i32(np.stack([pos // 2] + [pos // 2 + g.integers(0, side, rows) for _ in range(case["axes"] - 1)]))
            else:
                st.offset = i32(-np.random.default_rng(seed + 1).integers(0, case["prefix_lo"] // 2 + 1, B))
        st.slot_pos.zero_()
        return st
    # with a cap, scores that reach half of it, as those of models trained with one do
    st.q = normal(rows, hq, hd, sigma=6.0 if case["cap"] else 2.0)
    st.slopes = None
    if case["bias"]:
        st.slopes = torch.exp2(-8.0 * torch.arange(1, hq + 1, device=dev, dtype=torch.float32) / hq)
    st.out = torch.empty_like(st.q)
    st.lse = torch.empty(rows, hq, device=dev, dtype=torch.float32)
    return st


def _handles(st):
    """What a program of the framework keeps: the cache and the batch state, the step with its plan, the workspace."""
    from paper_2508_08895_amd import binding as A

    case, seqs, dev = st.case, st.seqs, st.tables.device

    def dev_i32(x):
        return torch.tensor([int(v) for v in x] or [0], dtype=torch.int32, device=dev)

    st.A = A
    st.kv = A.KVCache(st.k_cache, st.v_cache, st.tables, case["hq"])
    st.state = state = A.BatchState(st.B, st.owner.shape[1], dev)
    kind = case["kind"]
    if kind == "sequences" and case["dtype"] == "f32":
        # (whole sequences are planned for bf16 attention only: in fp32 a program names the rows of the step itself)
        st.step = A.Step(st.rows, 0, st.B, dev)
        for name, rows in (("position_ids", st.pos), ("q_seq", st.q_seq), ("logical_slot", st.slot), ("slot_mapping", st.slot_mapping)):
            getattr(st.step, name).copy_(rows)
    elif kind == "sequences":
        runs = [x for r, _ in seqs for x in r]
        st.step = A.aspd_build_sequence_meta(st.kv, state, dev_i32(np.cumsum([0] + [len(r) for r, _ in seqs])),
                                             dev_i32([x[1] for x in runs]), dev_i32([x[3] for x in runs]), st.rows)
        st.attention = A.aspd_attn_full_sequence
    elif kind == "prefill":
        st.step = A.aspd_build_branch_meta(st.kv, state, A.STAGE_SERIAL, dev_i32(st.count), NQ=st.rows, max_new_per_seq=int(st.count.max()))
        st.attention = A.aspd_attn_serial_decode
    else:
        first = [r[0][3] for r, _ in seqs]
        held = [[x[3] for x in r[1:old]] for r, old in seqs]
        A.aspd_build_branch_meta(st.kv, state, A.STAGE_SERIAL, dev_i32(first), NQ=sum(first), plan=False)
        state.open_parallel(torch.from_numpy(np.cumsum([0] + [len(h) for h in held]).astype(np.int32)))
        flat = [n for h in held for n in h]
        A.aspd_build_branch_meta(st.kv, state, A.STAGE_PARALLEL, dev_i32(flat), NQ=sum(flat), plan=False)
        if kind == "serial":
            A.aspd_build_branch_meta(st.kv, state, A.STAGE_MERGE, None)
            st.step = A.aspd_build_branch_meta(st.kv, state, A.STAGE_SERIAL, dev_i32([1] * st.B), NQ=st.rows, max_new_per_seq=1)
            st.attention = A.aspd_attn_serial_decode
        else:
            new = [x[3] for r, old in seqs for x in r[old:]]
            st.step = A.aspd_build_branch_meta(st.kv, state, A.STAGE_PARALLEL, dev_i32(new), NQ=st.rows,
                                               max_new_per_seq=int(st.count.max()))
            st.attention = A.aspd_attn_branch_chunk if kind == "chunk" else A.aspd_attn_parallel_decode
    if case["op"] == "append":
        st.rotary = A.Rotary(THETA, axis_of_pair=st.axis_of_pair if case["axes"] > 1 else None, axis_pos=st.axis_pos,
                             pos_offset=st.offset, q_weight=st.q_weight, k_weight=st.k_weight, norm_eps=EPS)
    else:
        st.workspace = A.new_workspace(st.kv, st.B, st.rows)
        st.scores = A.Scores(softcap=case["cap"], slopes=st.slopes, slot_pos=st.slot_pos if case["bias"] else None)


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _handles(st)
    elif case["op"] == "attention":
        # rows of a sequence side by side, the last one again behind them, and where a row is found there
        first = np.cumsum(st.count) - st.count
        most = int(st.count.max())
        dev = st.tables.device
        st.side = torch.from_numpy(first[:, None] + np.minimum(np.arange(most), np.maximum(st.count, 1)[:, None] - 1)).to(dev)
        seq = np.repeat(np.arange(st.B), st.count)
        st.back = torch.from_numpy(seq * most + np.arange(st.rows) - first[seq]).to(dev)
    return st


def run(st):
    if st.case["op"] == "append":
        if own:
            st.A.aspd_norm_rope_append(st.kv, st.state, st.step, st.rotary, st.q, st.k_new, st.v_new, q_out=st.q_out, slot_pos=st.slot_pos)
        else:
            _append(st)
        return {"q": st.q_out, "k_cache": st.k_cache, "v_cache": st.v_cache, "slot_pos": st.slot_pos}
    if own:
        st.attention(st.kv, st.state, st.step, st.q, st.workspace, out=st.out, lse=st.lse, scores=st.scores)
        return {"out": st.out, "lse": st.lse}
    out, lse = _attend(st)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------------------ plain forms
def _append(st):
    hd = st.case["hd"]
    pair = torch.arange(hd // 2, device=st.q.device)
    if st.axis_pos is not None:
        pos = st.axis_pos[torch.tensor(st.axis_of_pair, device=st.q.device)].t()   # [rows][pairs]
    else:
        pos = st.pos if st.offset is None else st.pos + st.offset[st.q_seq.long()]
        pos = pos[:, None]
    angle = pos.double() * torch.exp(-(2.0 / hd) * math.log(THETA) * pair.double())
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        a, b = x[..., : hd // 2], x[..., hd // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    st.q_out.copy_(turned(st.q, st.q_weight))
    block, within = st.slot_mapping // BLOCK, st.slot_mapping % BLOCK
    st.k_cache[block, :, within] = turned(st.k_new, st.k_weight).to(st.k_cache.dtype)
    st.v_cache[block, :, within] = st.v_new
    st.slot_pos[st.q_seq.long(), st.slot.long()] = st.pos


def _attend(st):
    c = st.case
    hq, hkv, hd = c["hq"], c["hkv"], c["hd"]
    g = hq // hkv
    tables = st.tables.long()

    def keys(pool):
        return pool[tables].transpose(1, 2).flatten(2, 3).float()                 # [B][hkv][T][hd]

    k, v = keys(st.k_cache), keys(st.v_cache)
    B, T = k.shape[0], k.shape[2]
    q = st.q[st.side].float()                                                     # [B][R][hq][hd]
    R = q.shape[1]
    q = q.view(B, R, hkv, g, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, R * g, hd)
    s = torch.matmul(q, k.transpose(2, 3)).mul_(1 / math.sqrt(hd))
    if c["cap"]:
        s.div_(c["cap"]).tanh_().mul_(c["cap"])
    s = s.view(B, hkv, R, g, T)
    if st.slopes is not None:
        distance = (st.slot_pos[:, None, :] - st.pos[st.side][:, :, None]).float()
        s.addcmul_(distance[:, None, :, None, :], st.slopes.view(1, hkv, 1, g, 1))
    j = torch.arange(T, device=q.device)
    slot, tag, base = (x[st.side][:, :, None] for x in (st.slot, st.tag, st.base))
    seen = (j <= slot) & ((tag == 0) | (j < base) | (st.owner[:, None, :] == tag))
    s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, hkv, R * g, T), v).view(B, hkv, R, g, hd) / total
    lse = (m + torch.log(total)).squeeze(-1)
    out = o.permute(0, 2, 1, 3, 4).reshape(B * R, hq, hd)[st.back].to(st.q.dtype)
    return out, lse.permute(0, 2, 1, 3).reshape(B * R, hq)[st.back]


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    st = _inputs(case, seed)
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    dev = st.q.device
    if case["op"] == "append":
        # complex numbers: pair i of a head is a + ib and turns by e^(i angle)
        axis = torch.tensor(st.axis_of_pair, device=dev)
        where = st.pos[:, None].expand(-1, hd // 2) if st.axis_pos is None else torch.stack([st.axis_pos[a] for a in axis.tolist()], 1)
        if st.offset is not None:
            where = where + torch.repeat_interleave(st.offset, torch.from_numpy(st.count).to(dev))[:, None]
        omega = THETA ** (-torch.arange(0, hd, 2, device=dev, dtype=torch.float64) / hd)
        out = {"q": None, "slot_pos": None, "k_cache": st.k_cache.double(), "v_cache": st.v_cache.double()}

        def rotated(x, weight):
            got = torch.empty(x.shape, dtype=torch.float64, device=dev)
            for at in range(0, x.shape[0], 1 << 15):
                y = x[at:at + (1 << 15)].double()
                if weight is not None:
                    y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / hd + EPS) * weight.double()
                turn = torch.polar(torch.ones((), dtype=torch.float64, device=dev), where[at:at + (1 << 15)].double() * omega)
                z = torch.complex(y[..., : hd // 2], y[..., hd // 2:].contiguous()) * turn[:, None]
                got[at:at + (1 << 15)] = torch.cat([z.real, z.imag], -1)
            return got

        out["q"] = rotated(st.q, st.q_weight)
        k = rotated(st.k_new, st.k_weight)
        for name, x in (("k_cache", k), ("v_cache", st.v_new.double())):
            pool = out[name].transpose(1, 2).contiguous()                          # [blocks][16][hkv][hd]
            pool.view(-1, hkv, hd)[st.slot_mapping] = x
            out[name] = pool.transpose(1, 2).contiguous()
        return out
    out = torch.empty(st.rows, hq, hd, dtype=torch.float64, device=dev)
    lse = torch.empty(st.rows, hq, dtype=torch.float64, device=dev)
    row = 0
    for s, (runs, old) in enumerate(st.seqs):
        stage, branch, pos = (torch.from_numpy(x).to(dev) for x in _tokens(runs))
        n, first = len(stage), sum(x[3] for x in runs[:old])
        at = st.tables[s, torch.arange(n, device=dev) // BLOCK].long() * BLOCK + torch.arange(n, device=dev) % BLOCK
        k, v = (x.transpose(1, 2).reshape(-1, hkv, hd)[at] for x in (st.k_cache, st.v_cache))
        for lo in range(first, n, 4096):
            hi = min(n, lo + 4096)
            i = torch.arange(lo, hi, device=dev)[:, None]
            j = torch.arange(n, device=dev)[None]
            # the definition's cases: a main-branch token sees all before it, a branch's its own branch and the other stages
            seen = (j <= i) & ((branch[i] == 0) | (stage[j] != stage[i]) | (branch[j] == branch[i]))
            far = (pos[j] - pos[i]).double()
            r = slice(row + lo - first, row + hi - first)
            for h in range(hq):
                x = st.q[r, h].double() @ k[:, h // (hq // hkv)].double().t() / math.sqrt(hd)
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                if st.slopes is not None:
                    x = x + st.slopes[h].double() * far
                x = torch.where(seen, x, -math.inf)
                lse[r, h] = torch.logsumexp(x, -1)
                out[r, h] = torch.softmax(x, -1) @ v[:, h // (hq // hkv)].double()
        row += n - first
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------------------ what it takes
def work(case):
    """append: queries, keys and values of the new tokens read and written once.  attention: the cache of the sequences once,
    queries read, outputs and log-sum-exps written; two products of the visible scores."""
    tokens, rows, keys = _seen(case)
    elt = 4 if case["dtype"] == "f32" else 2
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    if case["op"] == "append":
        return {"bytes": 2 * rows * (hq + 2 * hkv) * hd * elt + 4 * rows * (5 + (case["axes"] if case["axes"] > 1 else 0)),
                "flops": rows * (hq + hkv) * hd * (7 if case["norm"] else 3)}
    return {"bytes": 2 * tokens * hkv * hd * elt + rows * hq * (2 * hd * elt + 4) + (4 * tokens if case["bias"] else 0),
            "flops": 4 * hd * hq * keys}
