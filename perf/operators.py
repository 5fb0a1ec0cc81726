"""Measured cases of the paged key/value cache: rotary positions, the append, the attention, the shared prefix.

Four operators, each by a `kind`:

  rope     rotary positions of [tokens][heads][dh] vectors (dv_rope), forward or inverse (the gradient's direction)
  append   keys and values of new tokens into a paged cache, rotated on the way, and the tokens' rotated queries
           (dv_paged_append)
  attn     decode attention of each token over its sequence's pages (dv_paged_attn)
  prefix   the same where all sequences share a long prefix, which is attended once for the batch (dv_paged_attn with
           shared_pages)

With `own` false, run() computes them in elementary torch operations in 32 bits (angles in 64); with `own` true it
makes the calls of the binding. exact() computes them in 64 bits, sequence by sequence.

Values: queries and keys are of unit scale times 1.5 and 1, so softmax rows are neither flat nor one-hot; fresh
queries, keys and values are slices of one projection's output, as a layer produces them. Pages of a sequence lie
anywhere in the pool.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f16": torch.float16, "f32": torch.float32}
BYTES = {"f16": 2, "f32": 4}


def listed():
    return [
        # One decode step's queries of a full serving batch (the 96 heads of the OPT-175B layer shape): latency.
        dict(name="rope_decode_b32", kind="rope", tokens=32, heads=96, dh=128, rot=128, layout="half", rule="plain",
             dtype="f32", far=2048, inverse=False),
        # Prompts at far positions of a context extended by parts, half of each head rotated, adjacent pairs.
        dict(name="rope_prompt_far_f16", kind="rope", tokens=6001, heads=32, dh=128, rot=64, layout="interleaved",
             rule="parts", dtype="f16", far=1000000, inverse=False),
        # The gradient's direction at odd sizes, positions interpolated.
        dict(name="rope_inverse_odd", kind="rope", tokens=777, heads=13, dh=80, rot=32, layout="half", rule="linear",
             dtype="f32", far=9000, inverse=True),
        # One token of each of 32 sequences, two slots of the batch idle: the append of every decode step.
        dict(name="append_decode_b32", kind="append", seqs=32, idle=2, lo=1, hi=1, start=300, q_heads=96, heads=96,
             dh=128, rot=128, layout="half", page=16, ktype="f16", itype="f32"),
        # Whole prompts of different lengths, grouped heads, fp16 activations.
        dict(name="append_prompts_gqa", kind="append", seqs=12, idle=0, lo=100, hi=1500, start=700, q_heads=64,
             heads=8, dh=128, rot=128, layout="interleaved", page=64, ktype="f16", itype="f16"),
        # A few drafted tokens a sequence into an fp32 cache without rotation (learned positions), odd pages and heads.
        dict(name="append_odd_f32", kind="append", seqs=5, idle=1, lo=1, hi=9, start=333, q_heads=0, heads=7, dh=56,
             rot=0, layout="half", page=10, ktype="f32", itype="f32"),
        # The smallest model's step (OPT-125m heads), one sequence of 128 rows, fp32: launches are all of it.
        dict(name="attn_125m_b1_f32", kind="attn", seqs=1, tokens=1, q_heads=12, heads=12, sel=0, dh=64, lo=128,
             hi=128, page=16, ktype="f32", prefix=0),
        # The attention of a full serving batch with a head set for each token (32 of the OPT-175B layer's 96 heads).
        dict(name="attn_175b_b32_sets", kind="attn", seqs=32, tokens=1, q_heads=96, heads=96, sel=32, dh=128, lo=512,
             hi=2048, page=16, ktype="f16", prefix=0),
        # Long contexts with grouped heads: eight query heads read each key and value.
        dict(name="attn_gqa_long_b6", kind="attn", seqs=6, tokens=1, q_heads=64, heads=8, sel=0, dh=128, lo=8000,
             hi=50000, page=64, ktype="f16", prefix=0),
        # Ragged small contexts, odd head width, pages that end inside every tile, two drafted tokens a sequence.
        dict(name="attn_odd_drafts", kind="attn", seqs=7, tokens=2, q_heads=15, heads=5, sel=0, dh=80, lo=2, hi=3001,
             page=24, ktype="f16", prefix=0),
        # 32 users of one long system prompt (OPT-6.7B heads): the prompt's keys and values are read once.
        dict(name="prefix_b32", kind="prefix", seqs=32, tokens=1, q_heads=32, heads=32, sel=0, dh=128, lo=16, hi=700,
             page=16, ktype="f16", prefix=8192),
        # 16 users of a longer document, grouped heads, four drafted tokens each: 512 query rows meet every key.
        dict(name="prefix_gqa_drafts", kind="prefix", seqs=16, tokens=4, q_heads=64, heads=8, sel=0, dh=128, lo=100,
             hi=2000, page=32, ktype="f16", prefix=16384),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _load(c):
    """What a case costs the plain form (elements gathered and scored), to keep drawn cases below the listed ones."""
    if c["kind"] in ("attn", "prefix"):
        n, k = c["sel"] or c["heads"], c["seqs"] * c["tokens"]
        return k * n * c["hi"] * c["dh"] + c["prefix"] * k * c["q_heads"] * 8
    return 0


def draw(rng):
    """One more case: 1 to 64 tokens against contexts of 1 to 50000 rows, prompts up to thousands of tokens, head widths 40
    to 256, one to eight query heads a key head, head sets, pages of 1 to 128 rows, both types and layouts."""
    every = listed()
    most = {k: max(work(c)["bytes"] for c in every if c["kind"] == k) for k in ("rope", "append", "attn", "prefix")}
    heavy = max(_load(c) for c in every)
    while True:
        kind = rng.choice(["rope", "append", "attn", "attn", "attn", "prefix", "prefix"])
        dh = rng.choice([40, 64, 64, 80, 96, 128, 128, 128, 192, 256])
        layout = rng.choice(["half", "interleaved"])
        rot = rng.choice([dh, dh, dh // 2 // 2 * 2, 32])
        ktype = rng.choice(["f16", "f16", "f16", "f32"])
        group = rng.choice([1, 1, 2, 4, 5, 8])
        heads = _log(rng, 1, 96 if group == 1 else 16)
        page = rng.choice([1, 8, 10, 16, 16, 24, 32, 64, 128])
        if kind == "rope":
            c = dict(kind=kind, tokens=_log(rng, 1, 6000), heads=heads, dh=dh, rot=rot, layout=layout,
                     rule=rng.choice(["plain", "linear", "ntk", "parts"]), dtype=rng.choice(["f16", "f32"]),
                     far=_log(rng, 1, 1000000), inverse=rng.random() < 0.3)
        elif kind == "append":
            lo = _log(rng, 1, 300)
            c = dict(kind=kind, seqs=_log(rng, 1, 48), idle=rng.randint(0, 2), lo=lo, hi=lo * rng.randint(1, 5),
                     start=_log(rng, 1, 3000), q_heads=heads * group if rng.random() < 0.8 else 0, heads=heads, dh=dh,
                     rot=rot if rng.random() < 0.8 else 0, layout=layout, page=page, ktype=ktype,
                     itype=rng.choice(["f16", "f32"]))
        else:
            lo = _log(rng, 1, 20000 if kind == "attn" else 500)
            sel = max(1, int(heads * group * rng.uniform(0.2, 0.6))) if rng.random() < 0.3 and heads > 1 else 0
            c = dict(kind=kind, seqs=_log(rng, 1, 32), tokens=rng.choice([1, 1, 1, 2, 4]), q_heads=heads * group,
                     heads=heads, sel=sel, dh=dh, lo=lo, hi=int(lo * rng.uniform(1, 5)), page=page, ktype=ktype,
                     prefix=0 if kind == "attn" else _log(rng, 64, 16384) // page * page or page)
            if c["seqs"] * c["tokens"] * c["q_heads"] < 4:
                continue
        if _pool(c) * c["heads"] * dh * BYTES[c.get("ktype", "f16")] * 2 > 3e9:
            continue
        if work(c)["bytes"] <= most[kind] and _load(c) <= heavy:
            return c


# ------------------------------------------------------------------------------------------------ sizes of a case
def _spread(lo, hi, n):
    """n lengths from lo to hi, evenly spread."""
    return [lo] if n == 1 and lo == hi else [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _tokens(c):
    return sum(_spread(c["lo"], c["hi"], c["seqs"]))


def _private(c):
    """Rows of each token of a sequence behind the shared prefix, summed over the tokens."""
    return sum(max(n - i, 0) for n in _spread(c["lo"], c["hi"], c["seqs"]) for i in range(c["tokens"]))


def _pool(c):
    """Rows of the page pool."""
    if c["kind"] == "rope":
        return 0
    page = c["page"]
    if c["kind"] == "append":
        own_pages = sum(-(-(c["start"] + n) // page) for n in _spread(c["lo"], c["hi"], c["seqs"]))
    else:
        own_pages = sum(-(-n // page) for n in _spread(c["lo"], c["hi"], c["seqs"])) + c["prefix"] // page
    return (own_pages + 3) * page


def work(case):
    c = case
    if c["kind"] == "rope":
        n = c["tokens"] * c["heads"] * c["dh"]
        return {"bytes": 2 * n * BYTES[c["dtype"]], "flops": 3 * c["tokens"] * c["heads"] * c["rot"]}
    if c["kind"] == "append":
        t, kv, q = _tokens(c), 2 * c["heads"] * c["dh"], c["q_heads"] * c["dh"]
        return {"bytes": t * (kv * (BYTES[c["itype"]] + BYTES[c["ktype"]]) + q * 2 * BYTES[c["itype"]]),
                "flops": 3 * t * (c["heads"] + c["q_heads"]) * c["rot"]}
    tokens, sel = c["seqs"] * c["tokens"], c["sel"] or c["q_heads"]
    private = _private(c)
    # Keys and values: each row once for every sequence and key head that is used, a shared row once for the batch.
    seq_rows = sum(_spread(c["lo"], c["hi"], c["seqs"]))
    used = c["heads"] * min(1.0, sel / c["heads"]) if c["sel"] else c["heads"]
    rows = seq_rows * used + c["prefix"] * c["heads"]
    small = tokens * sel * (2 * c["dh"] + 1) * 4
    return {"bytes": rows * 2 * c["dh"] * BYTES[c["ktype"]] + small,
            "flops": 4 * c["dh"] * sel * (private + tokens * c["prefix"])}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _freq(rot, rule, base=10000.0):
    """Radians a position of each rotated pair: plain, positions interpolated (linear), a larger base (ntk), or by
    parts: pairs that turn often in the original context keep their frequency, the slow ones are interpolated."""
    i = np.arange(rot // 2, dtype=np.float64)
    factor, orig, low, high = 8.0, 4096.0, 1.0, 32.0
    if rule == "ntk" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2.0 * i / rot)
    if rule == "linear":
        f = f / factor
    if rule == "parts":
        g = np.clip((orig * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        f = f * (g + (1.0 - g) / factor)
    return f


def _table(c, g, lengths, shared):
    """Block table [seqs][pages]: the shared pages first, then pages of a sequence's own, anywhere in the pool."""
    page, n = c["page"], len(lengths)
    counts = [-(-x // page) for x in lengths]
    width = shared + max(counts + [1])
    free = torch.randperm(_pool(c) // page, generator=g, device=DEV).to(torch.int32).cpu().numpy()
    table = np.zeros((n, width), dtype=np.int32)
    table[:, :shared] = free[:shared]
    at = shared
    for s, k in enumerate(counts):
        table[s, shared:shared + k] = free[at:at + k]
        at += k
    return torch.from_numpy(table).to(DEV)


def prepare(case, seed):
    c, g = case, _gen(seed)
    rng = np.random.default_rng(seed)
    if c["kind"] == "rope":
        x = torch.randn((c["tokens"], c["heads"], c["dh"]), generator=g, dtype=DTYPES[c["dtype"]], device=DEV)
        pos = torch.randint(0, c["far"], (c["tokens"],), generator=g, device=DEV).to(torch.int32)
        return {"c": c, "x": x, "pos": pos, "freq": torch.from_numpy(_freq(c["rot"], c["rule"])).to(DEV),
                "mscale": 0.1 * math.log(8.0) + 1.0 if c["rule"] == "parts" else 1.0, "out": torch.empty_like(x)}
    lengths = _spread(c["lo"], c["hi"], c["seqs"])
    rng.shuffle(lengths)
    shape = (_pool(c) // c["page"], c["heads"], c["page"], c["dh"])
    K = torch.randn(shape, generator=g, dtype=DTYPES[c["ktype"]], device=DEV)
    V = torch.randn(shape, generator=g, dtype=DTYPES[c["ktype"]], device=DEV)
    if c["kind"] == "append":
        start = rng.integers(0, c["start"] + 1, c["seqs"])
        table = _table(c, g, [c["start"] + n for n in lengths], 0)
        pos = np.concatenate([s + np.arange(n) for s, n in zip(start, lengths)] + [np.full(c["idle"], -1)])
        seq = np.concatenate([np.full(n, i) for i, n in enumerate(lengths)] + [np.zeros(c["idle"], dtype=int)])
        t, dh, hq, hk = len(pos), c["dh"], c["q_heads"], c["heads"]
        qkv = torch.randn((t, (hq + 2 * hk) * dh), generator=g, dtype=DTYPES[c["itype"]], device=DEV)
        q = qkv[:, :hq * dh].view(t, hq, dh) if hq else None
        k = qkv[:, hq * dh:(hq + hk) * dh].view(t, hk, dh)
        v = qkv[:, (hq + hk) * dh:].view(t, hk, dh)
        return {"c": c, "K": K, "V": V, "table": table, "q": q, "k": k, "v": v,
                "q_out": torch.zeros((t, hq, dh), dtype=qkv.dtype, device=DEV) if hq else None,
                "pos": torch.from_numpy(pos.astype(np.int32)).to(DEV),
                "seq": torch.from_numpy(seq.astype(np.int32)).to(DEV),
                "freq": torch.from_numpy(_freq(c["rot"], "plain")).to(DEV) if c["rot"] else None}
    shared = c["prefix"] // c["page"]
    table = _table(c, g, lengths, shared)
    n = c["tokens"]
    pos = np.concatenate([c["prefix"] + np.maximum(np.arange(x - n, x), -1 - c["prefix"]) for x in lengths])
    seq = np.repeat(np.arange(c["seqs"]), n)
    heads = None
    if c["sel"]:
        order = torch.rand((len(pos), c["q_heads"]), generator=g, device=DEV).argsort(dim=1)
        heads = order[:, :c["sel"]].sort(dim=1).values.to(torch.int32).contiguous()
    q = torch.randn((len(pos), c["sel"] or c["q_heads"], c["dh"]), generator=g, device=DEV).mul_(1.5)
    return {"c": c, "K": K, "V": V, "table": table, "q": q, "heads": heads, "shared": shared,
            "max_len": c["prefix"] + max(lengths), "scale": 1.0 / math.sqrt(c["dh"]),
            "pos": torch.from_numpy(pos.astype(np.int32)).to(DEV),
            "seq": torch.from_numpy(seq.astype(np.int32)).to(DEV), "out": torch.empty_like(q),
            "lse": torch.empty(q.shape[:2], device=DEV)}


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, pos, freq, layout, mscale=1.0, inverse=False):
    """x [tokens][heads][dh] in 32 bits, its first 2 len(freq) elements rotated; angles in 64 bits."""
    angle = pos.double()[:, None, None] * freq
    cos, sin = (angle.cos() * mscale).float(), (angle.sin() * (-mscale if inverse else mscale)).float()
    x, rot = x.float(), 2 * len(freq)
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_append(s):
    c, live = s["c"], s["pos"] >= 0
    pos, seq = s["pos"][live].long(), s["seq"][live].long()
    pages, rows = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    turn = (lambda x: _rotate(x, s["pos"], s["freq"], c["layout"])) if c["rot"] else (lambda x: x.float())
    s["K"][pages, :, rows] = turn(s["k"])[live].to(s["K"].dtype)
    s["V"][pages, :, rows] = s["v"][live].to(s["V"].dtype)
    if s["q"] is None:
        return s["K"], s["V"]
    s["q_out"][live] = turn(s["q"])[live].to(s["q_out"].dtype)
    return s["K"], s["V"], s["q_out"]


def _plain_attn(s):
    """Softmax over [shared rows | own rows]; the shared rows' products are taken once for all tokens."""
    c, q, pos = s["c"], s["q"], s["pos"].long()
    t, n, dh = q.shape
    group, p0, page = c["q_heads"] // c["heads"], c["prefix"], c["page"]
    own_pages = s["table"][:, s["shared"]:].long()[s["seq"].long()]                     # [t][pages]
    if s["heads"] is None:
        pick = torch.arange(c["heads"], device=DEV).expand(t, -1)
    else:
        pick, group = s["heads"].long() // group, 1
    gather = lambda X: X[own_pages[:, None, :], pick[:, :, None]].flatten(2, 3).float()  # [t][pick][rows][dh]
    k, v = gather(s["K"]), gather(s["V"])
    at = p0 + torch.arange(k.shape[2], device=DEV)
    seen = at[None, :] <= pos[:, None]                                                  # [t][rows]
    qg = q.view(t, -1, group, dh)
    score = torch.matmul(qg, k.transpose(2, 3)).reshape(t, n, -1) * s["scale"]
    score = torch.where(seen[:, None, :], score, -math.inf)
    if p0:
        # every query head of a key head over all tokens at once; heads that a token does not use are dropped again
        full = q if s["heads"] is None else torch.zeros((t, c["q_heads"], dh), device=DEV).scatter_(
            1, s["heads"].long()[:, :, None].expand(-1, -1, dh), q)
        pages = s["table"][0, :s["shared"]].long()
        kp, vp = (X[pages].transpose(0, 1).flatten(1, 2).float() for X in (s["K"], s["V"]))   # [heads][p0][dh]
        fq = full.view(t, c["heads"], -1, dh).transpose(0, 1).flatten(1, 2)             # [heads][t * group][dh]
        fs = torch.matmul(fq, kp.transpose(1, 2)).view(c["heads"], t, -1, p0).transpose(0, 1).flatten(1, 2)
        ps = fs if s["heads"] is None else fs.gather(1, s["heads"].long()[:, :, None].expand(-1, -1, p0))
        ps = torch.where((torch.arange(p0, device=DEV)[None, :] <= pos[:, None])[:, None, :], ps * s["scale"], -math.inf)
        score = torch.cat([ps, score], dim=-1)
    top = score.amax(dim=-1, keepdim=True)
    w = (score - torch.where(top.isinf(), 0.0, top)).exp()
    total = w.sum(dim=-1, keepdim=True)
    wr = w[..., p0:].reshape(t, -1, group, w.shape[-1] - p0)
    out = torch.matmul(wr, v).reshape(t, n, dh)
    if p0:
        wp = w[..., :p0]
        if s["heads"] is not None:
            wp = torch.zeros((t, c["q_heads"], p0), device=DEV).scatter_(
                1, s["heads"].long()[:, :, None].expand(-1, -1, p0), wp)
        fo = torch.matmul(wp.view(t, c["heads"], -1, p0).transpose(0, 1).flatten(1, 2), vp)
        fo = fo.view(c["heads"], t, -1, dh).transpose(0, 1).flatten(1, 2)
        out = out + (fo if s["heads"] is None else fo.gather(1, s["heads"].long()[:, :, None].expand(-1, -1, dh)))
    none = total == 0
    out = torch.where(none, 0.0, out / torch.where(none, 1.0, total))
    return out, (top + total.log()).squeeze(-1)


# ------------------------------------------------------------------------------------------------ a pass
def _handles(s):
    """The cache and rotation objects that a program keeps beside its tensors."""
    from paper_2310_17157_amd import binding as dv
    c = s["c"]
    layout = dv.DV_ROPE_HALF if c.get("layout") == "half" else dv.DV_ROPE_INTERLEAVED
    s["dv"] = dv
    if s.get("freq") is not None:
        s["rotary"] = dv.Rotary(s["freq"], layout=layout, mscale=s.get("mscale", 1.0))
    if c["kind"] != "rope":
        s["kv"] = dv.PagedKV(s["K"], s["V"], s["table"])
    if c["kind"] in ("attn", "prefix"):
        s["ws"] = torch.empty(dv.paged_attn_workspace_bytes(
            s["kv"], len(s["pos"]), c["q_heads"], s["max_len"], n_heads=c["sel"], shared_pages=s["shared"]),
            dtype=torch.uint8, device=DEV)


def run(state):
    s = state
    c = s["c"]
    if own:
        if "dv" not in s:
            _handles(s)
        dv = s["dv"]
        if c["kind"] == "rope":
            return dv.dv_rope(s["rotary"], s["x"], s["pos"], inverse=c["inverse"], out=s["out"])
        if c["kind"] == "append":
            dv.dv_paged_append(s["kv"], s["k"], s["v"], s["pos"], seq=s["seq"], rotary=s.get("rotary"), q=s["q"],
                               q_out=s["q_out"])
            return (s["K"], s["V"]) if s["q"] is None else (s["K"], s["V"], s["q_out"])
        return dv.dv_paged_attn(s["kv"], s["q"], s["pos"], s["max_len"], s["scale"], seq=s["seq"], heads=s["heads"],
                                q_heads=c["q_heads"], shared_pages=s["shared"], out=s["out"], lse=s["lse"], ws=s["ws"])
    if c["kind"] == "rope":
        return _rotate(s["x"], s["pos"], s["freq"], c["layout"], s["mscale"], c["inverse"]).to(s["x"].dtype)
    return _plain_append(s) if c["kind"] == "append" else _plain_attn(s)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _turn64(x, pos, freq, layout, mscale, inverse):
    """Rotation as a product of complex numbers."""
    x = x.double()
    r = 2 * len(freq)
    pairs = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if layout == "half" else x[..., :r].unflatten(-1, (r // 2, 2))
    z = torch.view_as_complex(pairs.contiguous())
    a = pos.double()[:, None, None] * freq * (-1 if inverse else 1)
    z = torch.view_as_real(z * torch.polar(torch.full_like(a, mscale), a))
    z = z.transpose(-1, -2).flatten(-2) if layout == "half" else z.flatten(-2)
    return torch.cat([z, x[..., r:]], dim=-1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rope":
        return _turn64(s["x"], s["pos"], s["freq"], c["layout"], s["mscale"], c["inverse"])
    page = c["page"]
    pos, seq, table = (s[k].cpu().numpy() for k in ("pos", "seq", "table"))
    if c["kind"] == "append":
        K, V = s["K"].double(), s["V"].double()
        k, q = s["k"].double(), None if s["q"] is None else s["q"].double()
        if c["rot"]:
            k = _turn64(s["k"], s["pos"], s["freq"], c["layout"], 1.0, False)
            q = None if q is None else _turn64(s["q"], s["pos"], s["freq"], c["layout"], 1.0, False)
        at = [i for i in range(len(pos)) if pos[i] >= 0]
        flat = torch.tensor([int(table[seq[i], pos[i] // page]) * page + int(pos[i]) % page for i in at], device=DEV)
        at = torch.tensor(at, device=DEV)
        for X, x in ((K, k), (V, s["v"].double())):
            rows = X.transpose(1, 2).flatten(0, 1)
            rows[flat] = x[at]
            X.copy_(rows.unflatten(0, (-1, page)).transpose(1, 2))
        if q is None:
            return K, V
        q_out = torch.zeros_like(q)
        q_out[at] = q[at]
        return K, V, q_out
    group = c["q_heads"] // c["heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    kept = {}
    for i in range(len(pos)):
        n = int(pos[i]) + 1
        if n <= 0:
            continue
        if int(seq[i]) not in kept:
            pages = torch.from_numpy(table[seq[i]]).long().to(DEV)
            kept = {int(seq[i]): [X[pages].transpose(0, 1).flatten(1, 2) for X in (s["K"], s["V"])]}
        Ks, Vs = kept[int(seq[i])]
        q = s["q"][i].double()
        for h in range(c["heads"]):
            mine = (torch.arange(group, device=DEV) + h * group if s["heads"] is None
                    else (s["heads"][i].long() // group == h).nonzero()[:, 0])
            if len(mine):
                x = q[mine] @ Ks[h, :n].double().t() * s["scale"]
                out[i, mine] = torch.softmax(x, dim=-1) @ Vs[h, :n].double()
                lse[i, mine] = torch.logsumexp(x, dim=-1)
    return out, lse
