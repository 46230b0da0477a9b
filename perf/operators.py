"""Cases and plain forms of the token-memory operators.

A frame's BEV maps (and any other tokens) are kept as rows of a key/value
memory that later queries attend to.  Three operators serve it:

    append   where the new tokens of every sequence go: offsets, memory rows,
             key spans and new lengths, from the lengths alone
             (rtcc_memory_append);
    prepare  per-head RMS norm of queries and keys and their rotation by
             (t, y, x) positions in one pass, keys, values and coordinates
             written to their memory rows (rtcc_qkv_prepare);
    attend   attention over spans of the memory with tanh-capped scores, a
             distance bias, causal / prefix / sequence masks and absent
             agents' slots (rtcc_memory_attention).

run() computes a case by elementary torch operations in 32 bits, or, where
`own` is set, by the framework's calls.  exact() is the definition in 64 bits.
"""
import math
import random

import torch

own = False

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # one decision step of 61 tracked requests: every sequence grows by at most a token
        dict(name="append_step", op="append", seqs=61, max_new=1, capacity=16384),
        # ragged bursts of many sequences (up to 200 rows each) into their slots
        dict(name="append_burst", op="append", seqs=2048, max_new=200, capacity=1000),
        # the same step's 61 tokens: grouped heads, one position axis (latency)
        dict(name="prepare_step", op="prepare", tokens=61, rows=61 * 64, heads=32, kv=8, dim=128, dtype="bf16",
             pt=64, py=0, px=0, inter=False, packed=True, drop=0),
        # one agent's 128 x 128 map of the 3-agent workload: 384 channels as 6 heads
        dict(name="prepare_map", op="prepare", tokens=16384, rows=16384, heads=6, kv=6, dim=64, dtype="fp16",
             pt=8, py=12, px=12, inter=False, packed=False, drop=0),
        # all five 352 x 100 maps of the long-range workload at once
        dict(name="prepare_frame", op="prepare", tokens=176000, rows=176000, heads=6, kv=6, dim=64, dtype="bf16",
             pt=8, py=12, px=12, inter=True, packed=True, drop=0),
        # odd count and head size, partial rotation, tokens that have no row
        dict(name="prepare_odd", op="prepare", tokens=12345, rows=12500, heads=10, kv=5, dim=80, dtype="fp16",
             pt=4, py=9, px=11, inter=True, packed=True, drop=7),
        # one query over a short memory: the latency of a call
        dict(name="attend_token", op="attend", seqs=1, q=1, k=4097, slots=0, absent=0, heads=6, kv=6, dim=64,
             dtype="fp16", causal=False, prefix=0, cap=0.0, dist=False, ragged=False, gap=0),
        # a decision step of 61 sequences with ragged histories: single tokens, grouped heads, capped scores
        dict(name="attend_step", op="attend", seqs=61, q=1, k=16384, slots=0, absent=0, heads=32, kv=8, dim=128,
             dtype="bf16", causal=True, prefix=0, cap=30.0, dist=False, ragged=True, gap=40),
        # 300 object queries over the eight 352 x 100 maps of the stress workload, one agent absent
        dict(name="attend_objects", op="attend", seqs=1, q=300, k=281600, slots=8, absent=1, heads=6, kv=6, dim=64,
             dtype="fp16", causal=False, prefix=0, cap=0.0, dist=True, ragged=False, gap=0),
        # the ego map of the 3-agent workload (128 x 128 cells) over all three agents' maps
        dict(name="attend_map", op="attend", seqs=1, q=16384, k=49152, slots=3, absent=0, heads=6, kv=6, dim=64,
             dtype="fp16", causal=False, prefix=0, cap=50.0, dist=True, ragged=False, gap=0),
        # packed ragged sequences, causal after a prefix all may see, grouped heads
        dict(name="attend_packed", op="attend", seqs=7, q=2100, k=2500, slots=0, absent=0, heads=16, kv=4, dim=128,
             dtype="bf16", causal=True, prefix=333, cap=30.0, dist=False, ragged=True, gap=0),
        # 17 new tokens of each of 9 sequences over their histories, odd head size
        dict(name="attend_chunk", op="attend", seqs=9, q=17, k=5001, slots=0, absent=0, heads=12, kv=4, dim=80,
             dtype="bf16", causal=True, prefix=100, cap=0.0, dist=True, ragged=True, gap=13),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "prepare", "prepare", "attend", "attend", "attend", "attend"])
    if op == "append":
        return dict(op=op, seqs=_log(rng, 1, 4096), max_new=_log(rng, 1, 300), capacity=_log(rng, 1, 20000))
    kv = rng.choice([1, 2, 3, 4, 5, 6, 8])
    group = rng.choice([1, 1, 2, 3, 4, 8]) if kv <= 4 else rng.choice([1, 1, 2, 4])
    dim = rng.choice([16, 32, 40, 64, 64, 64, 72, 80, 96, 104, 128, 128, 128])
    dtype = rng.choice(["fp16", "bf16"])
    if op == "prepare":
        most = max(1, 176000 * 18 * 64 // ((kv * group + 2 * kv) * dim))
        tokens = _log(rng, 1, min(most, 176000))
        half = dim // 2
        cut = sorted(rng.randint(0, half) for _ in range(3))
        if rng.random() < 0.5:
            cut[2] = half
        return dict(op=op, tokens=tokens, rows=tokens + rng.randint(0, 99), heads=kv * group, kv=kv, dim=dim,
                    dtype=dtype, pt=cut[0], py=cut[1] - cut[0], px=cut[2] - cut[1], inter=rng.random() < 0.5,
                    packed=rng.random() < 0.5, drop=rng.choice([0, 0, 5]))
    cap = rng.choice([0.0, 0.0, 20.0, 30.0, 50.0])
    dist = rng.random() < 0.4
    kind = rng.choice(["step", "step", "chunk", "packed", "map", "objects"])
    c = dict(op=op, seqs=1, q=1, k=1, slots=0, absent=0, heads=kv * group, kv=kv, dim=dim, dtype=dtype, causal=False,
             prefix=0, cap=cap, dist=dist, ragged=False, gap=0)
    if kind == "step":
        c.update(seqs=_log(rng, 1, 80), causal=True, ragged=rng.random() < 0.7, gap=rng.randint(0, 50))
        c.update(k=_log(rng, 1, max(1, 61 * 16384 * 8 * 128 // (c["seqs"] * kv * group * dim))))
        c["k"] = min(c["k"], 100000)
    elif kind == "chunk":
        c.update(seqs=_log(rng, 1, 16), q=_log(rng, 2, 100), k=_log(rng, 1, 10000), causal=rng.random() < 0.7,
                 ragged=rng.random() < 0.7, gap=rng.randint(0, 30))
        c["prefix"] = rng.choice([0, c["k"] // 3])
    elif kind == "packed":
        c.update(seqs=_log(rng, 1, 12), q=_log(rng, 64, 3000), causal=True, ragged=rng.random() < 0.7)
        c.update(k=c["q"] + rng.choice([0, 0, rng.randint(0, 500)]))
        c["prefix"] = rng.choice([0, 0, c["k"] // 4])
    elif kind == "map":
        c["slots"] = rng.randint(2, 5)
        c.update(q=_log(rng, 256, 12000), absent=rng.choice([0, 0, 1]))
        c.update(k=c["slots"] * _log(rng, 100, 8000))
        c.update(k=c["k"] // c["slots"] * c["slots"])
    else:
        c["slots"] = rng.randint(2, 8)
        c.update(q=_log(rng, 2, 500), k=c["slots"] * _log(rng, 300, 30000), absent=rng.choice([0, 1]))
    # no more score elements, products or cached bytes than the largest listed case
    h = c["heads"]
    while h * c["seqs"] * c["q"] * c["k"] * max(dim, 64) > 6 * 16384 * 49152 * 64 and c["q"] > 1:
        c["q"] = (c["q"] + 1) // 2
    return c


# ---------------------------------------------------------------------------
# sizes of a case (host arithmetic; the sequences' lengths come from the case,
# the values from the seed)
# ---------------------------------------------------------------------------

def _spans(c):
    """Per sequence: tokens, keys, prefix; where its keys begin; rows in all.

    A sequence's history lies in a region of its own; regions have gaps of
    `gap` stale rows.  Ragged: lengths from half (queries) or 1/16th (keys) of
    the largest up; the first sequence has the largest.  Packed sequences never
    have fewer keys than tokens."""
    rng = random.Random("%d %d %d" % (c["seqs"], c["q"], c["k"]))
    n, held, prefix, begin, at = [], [], [], [], 0
    for i in range(c["seqs"]):
        q, k = c["q"], c["k"]
        if c["ragged"] and i:
            q = rng.randint((c["q"] + 1) // 2, c["q"])
            k = rng.randint(max(1, c["k"] // 16), c["k"])
            if c["k"] >= c["q"]:
                k = max(k, q)
        n.append(q)
        held.append(k)
        prefix.append(min(k, rng.randint(0, c["prefix"]) if i else c["prefix"]) if c["prefix"] else 0)
        begin.append(at + c["gap"])
        at += k + c["gap"]
    return n, held, prefix, begin, at + c["gap"]


def _pairs(c):
    """Visible (query, key) pairs of one head, and visible keys."""
    n, held, prefix, _, _ = _spans(c)
    pairs, keys = 0, 0
    for q, k, p in zip(n, held, prefix):
        if c["slots"]:
            k = k // c["slots"] * (c["slots"] - c["absent"])
        if c["causal"]:
            pairs += sum(min(k, max(0, p, k - q + 1 + i)) for i in range(q))
        else:
            pairs += q * k
        keys += k
    return pairs, keys


def work(c):
    if c["op"] == "append":
        tokens = c["seqs"] * c["max_new"]
        return {"bytes": 4 * (2 * c["seqs"] + 4 * c["seqs"] + 1 + 3 * tokens), "flops": 0}
    if c["op"] == "prepare":
        per = (c["heads"] + 2 * c["kv"]) * c["dim"]
        rot = (c["heads"] + c["kv"]) * c["dim"]
        return {"bytes": c["tokens"] * (4 * per + 12 + 4 + 8), "flops": c["tokens"] * rot * 7}
    pairs, keys = _pairs(c)
    tokens = sum(_spans(c)[0])
    d = c["dim"]
    return {"bytes": 4 * tokens * c["heads"] * d + 4 * keys * c["kv"] * d + 4 * tokens * c["heads"]
            + (8 * (keys + tokens) if c["dist"] else 0),
            "flops": pairs * c["heads"] * 4 * d}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    return {"append": _prepare_append, "prepare": _prepare_prepare, "attend": _prepare_attend}[case["op"]](case, seed)


def _prepare_append(c, seed):
    g = _gen(seed)
    n = c["seqs"]
    # one new row each in a step of single tokens with a few sequences idle; bursts are uniform
    new = torch.randint(0, c["max_new"] + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    if c["max_new"] == 1:
        new = (torch.rand(n, generator=g, device="cuda") < 0.9).int()
    held = torch.randint(0, c["capacity"] + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    slot = torch.randperm(n, generator=g, device="cuda").int()
    tokens = n * c["max_new"]
    e = lambda k: torch.empty(k, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(case=c, new=new, held=held, slot=slot, offsets=e(n + 1), rows=e(tokens), seq=e(tokens), pos=e(tokens),
                begin=e(n), end=e(n), length=e(n))


def _prepare_prepare(c, seed):
    g = _gen(seed)
    n, hq, hk, d, dt = c["tokens"], c["heads"], c["kv"], c["dim"], DT[c["dtype"]]
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    # a projection's output: channels of unlike scale; packed = one [q | k | v] row per token
    x = (rand(n, hq + 2 * hk, d) * (0.5 + 2 * torch.rand(hq + 2 * hk, 1, generator=g, device="cuda"))).to(dt)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    if not c["packed"]:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    # frame number and BEV coordinates in metres (cells of 0.8 m), as one axis a plain token count
    if c["py"] + c["px"]:
        w = max(1, int(math.sqrt(n)))
        at = torch.arange(n, device="cuda")
        off = float(torch.rand(1, generator=g, device="cuda").item()) * 50
        pos = torch.stack([(at % 7).float(), 0.8 * (at // w).float() - 40 + off, 0.8 * (at % w).float() - 140], 1)
    else:
        pos = torch.zeros(n, 3, device="cuda")
        pos[:, 0] = torch.randint(0, 100000, (n,), generator=g, device="cuda").float()
    rows = torch.randperm(c["rows"], generator=g, device="cuda")[:n].int()
    if c["drop"]:
        rows[::c["drop"]] = -1
    z = lambda *s: torch.zeros(*s, device="cuda", dtype=dt)  # noqa: E731
    return dict(case=c, q=q, k=k, v=v, pos=pos.contiguous(), rows=rows, q_gain=1 + 0.2 * rand(d), k_gain=1 + 0.2 * rand(d),
                q_out=z(n, hq, d), k_mem=z(c["rows"], hk, d), v_mem=z(c["rows"], hk, d),
                coord=torch.zeros(c["rows"], 2, device="cuda"))


def _prepare_attend(c, seed):
    g = _gen(seed)
    n, held, prefix, begin, rows = _spans(c)
    hq, hk, d, dt = c["heads"], c["kv"], c["dim"], DT[c["dtype"]]
    tokens = sum(n)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    # normed and rotated vectors have about unit mean square; the gains spread the scores
    q = (1.5 * rand(tokens, hq, d)).to(dt)
    k = rand(rows, hk, d).to(dt)
    v = rand(rows, hk, d).to(dt)
    s = dict(case=c, q=q, k=k, v=v, begin=_i32(begin), end=_i32([b + m for b, m in zip(begin, held)]),
             offsets=_i32([sum(n[:i]) for i in range(len(n) + 1)]), prefix=_i32(prefix) if c["prefix"] else None,
             present=None, slopes=None, q_pos=None, k_pos=None, max_q=max(n), max_k=max(held),
             out=torch.zeros(tokens, hq, d, dtype=dt, device="cuda"), lse=torch.zeros(tokens, hq, device="cuda"),
             workspace=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"))
    if c["slots"]:
        p = torch.ones(c["slots"], dtype=torch.int32, device="cuda")
        if c["absent"]:
            p[1 + int(seed) % (c["slots"] - 1)] = 0
        s["present"] = p
    if c["dist"]:
        # metres: cells of 0.8 m for maps, the row number for sequences of tokens
        s["slopes"] = torch.tensor([0.25 * 2.0 ** (-i * 6 / hq) for i in range(hq)], device="cuda")
        if c["slots"]:
            per = c["k"] // c["slots"]
            w = max(1, int(math.sqrt(per)))
            at = torch.arange(rows, device="cuda") % per
            s["k_pos"] = torch.stack([0.8 * (at // w).float(), 0.8 * (at % w).float()], 1).contiguous()
            s["k_pos"] += 3 * rand(1, 2)
            if c["q"] > 1000:
                a = torch.arange(tokens, device="cuda")
                s["q_pos"] = torch.stack([0.8 * (a // w).float(), 0.8 * (a % w).float()], 1).contiguous()
            else:
                s["q_pos"] = (torch.rand(tokens, 2, generator=g, device="cuda") * 0.8 * w).contiguous()
        else:
            k_pos, q_pos = torch.zeros(rows, 2), torch.zeros(tokens, 2)
            at = 0
            for m, b, h in zip(n, begin, held):
                k_pos[b:b + h, 1] = torch.arange(h).float()
                q_pos[at:at + m, 1] = torch.arange(h - m, h).float()
                at += m
            s["k_pos"], s["q_pos"] = k_pos.cuda(), q_pos.cuda()
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        return {"append": _own_append, "prepare": _own_prepare, "attend": _own_attend}[c["op"]](s, c)
    return {"append": _plain_append, "prepare": _plain_prepare, "attend": _plain_attend}[c["op"]](s, c)


THETA, EPS = 10000.0, 1e-6


def _ptr(t):
    return None if t is None else t.data_ptr()


def _own_append(s, c):
    from paper_2608_08330_gb300 import rtcc as R
    stream = torch.cuda.current_stream().cuda_stream
    R.check(R.rtcc_memory_append(c["seqs"], c["capacity"], s["rows"].numel(), s["new"].data_ptr(), s["held"].data_ptr(),
                                 s["slot"].data_ptr(), s["offsets"].data_ptr(), s["rows"].data_ptr(),
                                 s["seq"].data_ptr(), s["pos"].data_ptr(), s["begin"].data_ptr(), s["end"].data_ptr(),
                                 s["length"].data_ptr(), stream))
    return [s["offsets"], s["rows"], s["seq"], s["pos"], s["begin"], s["end"], s["length"]]


def _plain_append(s, c):
    new, held, cap, n = s["new"].long(), s["held"].long(), c["capacity"], s["rows"].numel()
    offsets = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.cumsum(new, 0)])
    at = torch.arange(n, device="cuda")
    seq = torch.searchsorted(offsets[1:].contiguous(), at, right=True)
    live = seq < c["seqs"]
    seq = torch.where(live, seq, 0)
    pos = held[seq] + at - offsets[seq]
    begin = s["slot"].long() * cap
    length = torch.minimum(held + new, torch.full_like(held, cap))
    rows = torch.where(live & (pos < cap), begin[seq] + pos, -1)
    seq, pos = torch.where(live, seq, -1), torch.where(live, pos, -1)
    return [t.int() for t in (offsets, rows, seq, pos, begin, begin + length, length)]


def _own_prepare(s, c):
    from paper_2608_08330_gb300 import rtcc as R
    q, k, v = s["q"], s["k"], s["v"]
    cfg = R.prepare_config(c["heads"], c["kv"], c["dim"], R.BF16 if c["dtype"] == "bf16" else R.FP16, c["tokens"],
                           c["rows"], q.stride()[:2], k.stride()[:2], v.stride()[:2], s["q_out"].stride()[:2],
                           s["k_mem"].stride()[:2], s["v_mem"].stride()[:2], (c["pt"], c["py"], c["px"]),
                           interleaved=c["inter"], theta=THETA, eps=EPS)
    R.check(R.rtcc_qkv_prepare(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), s["q_gain"].data_ptr(),
                               s["k_gain"].data_ptr(), s["pos"].data_ptr(), s["rows"].data_ptr(), s["q_out"].data_ptr(),
                               s["k_mem"].data_ptr(), s["v_mem"].data_ptr(), s["coord"].data_ptr(),
                               torch.cuda.current_stream().cuda_stream))
    return [s["q_out"], s["k_mem"], s["v_mem"], s["coord"]]


def _plain_norm_rotate(x, gain, pos, c):
    """RMS norm over each head, gain, rotation of the pairs by position x frequency."""
    d, per = c["dim"], (c["pt"], c["py"], c["px"])
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    rot = sum(per)
    if not rot:
        return x
    freq = [torch.pow(torch.tensor(THETA, device="cuda"), -torch.arange(m, device="cuda").float() / max(m, 1)) for m in per]
    angle = torch.cat([pos[:, a:a + 1] * f for a, f in enumerate(freq)], 1)[:, None]
    cos, sin = torch.cos(angle), torch.sin(angle)
    a, b = (x[..., 0:2 * rot:2], x[..., 1:2 * rot:2]) if c["inter"] else (x[..., :rot], x[..., rot:2 * rot])
    u, w = a * cos - b * sin, a * sin + b * cos
    y = torch.stack([u, w], -1).flatten(-2) if c["inter"] else torch.cat([u, w], -1)
    return torch.cat([y, x[..., 2 * rot:d]], -1)


def _plain_prepare(s, c):
    s["q_out"].copy_(_plain_norm_rotate(s["q"], s["q_gain"], s["pos"], c))
    k = _plain_norm_rotate(s["k"], s["k_gain"], s["pos"], c).to(s["k"].dtype)
    keep = s["rows"] >= 0
    rows = s["rows"][keep].long()
    s["k_mem"][rows] = k[keep]
    s["v_mem"][rows] = s["v"][keep]
    s["coord"][rows] = s["pos"][keep][:, 1:]
    return [s["q_out"], s["k_mem"], s["v_mem"], s["coord"]]


def _own_attend(s, c):
    from paper_2608_08330_gb300 import rtcc as R
    q, k, v, out = s["q"], s["k"], s["v"], s["out"]
    cfg = R.attn_config(c["heads"], c["kv"], c["dim"], R.BF16 if c["dtype"] == "bf16" else R.FP16, q.shape[0], k.shape[0],
                        q.stride()[:2], k.stride()[:2], v.stride()[:2], out.stride()[:2], c["seqs"], s["max_q"],
                        s["max_k"], causal=c["causal"], n_slots=c["slots"],
                        slot_rows=c["k"] // c["slots"] if c["slots"] else 0, scale=1 / math.sqrt(c["dim"]), cap=c["cap"])
    R.check(R.rtcc_memory_attention(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), s["offsets"].data_ptr(),
                                    s["begin"].data_ptr(), s["end"].data_ptr(), _ptr(s["prefix"]), _ptr(s["present"]),
                                    _ptr(s["slopes"]), _ptr(s["q_pos"]), _ptr(s["k_pos"]), out.data_ptr(),
                                    s["lse"].data_ptr(), s["workspace"].data_ptr(), s["workspace"].numel(),
                                    torch.cuda.current_stream().cuda_stream))
    return [out, s["lse"]]


def _plain_attend(s, c):
    """All sequences padded to the longest: scores, cap, bias, mask, softmax, product."""
    hq, hk, d, tokens, rows = c["heads"], c["kv"], c["dim"], s["q"].shape[0], s["k"].shape[0]
    grp = hq // hk
    off, begin, end = s["offsets"].long(), s["begin"].long(), s["end"].long()
    i = torch.arange(s["max_q"], device="cuda")
    j = torch.arange(s["max_k"], device="cuda")
    n, m = (off[1:] - off[:-1])[:, None], (end - begin)[:, None]
    qi = (off[:-1, None] + i).clamp(max=tokens - 1)                       # [B, Q]
    kj = (begin[:, None] + j).clamp(max=rows - 1)                         # [B, L]
    q = s["q"].float()[qi].reshape(-1, s["max_q"], hk, grp, d).permute(0, 2, 3, 1, 4)   # [B, hk, grp, Q, d]
    k = s["k"].float()[kj].permute(0, 2, 3, 1)[:, :, None]                # [B, hk, 1, d, L]
    x = torch.matmul(q, k) * (1 / math.sqrt(d))
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if c["dist"]:
        dist = (s["q_pos"][qi][:, :, None] - s["k_pos"][kj][:, None]).abs().sum(-1)     # [B, Q, L]
        x = x - s["slopes"].reshape(1, hk, grp, 1, 1) * dist[:, None, None]
    see = (j < m)[:, None].expand(-1, s["max_q"], -1)
    if c["causal"]:
        last = (m - n)[:, :, None] + i[None, :, None]
        lead = s["prefix"].long()[:, None, None] if s["prefix"] is not None else 0
        see = see & ((j[None, None] <= last) | (j[None, None] < lead))
    if c["slots"]:
        see = see & (s["present"][(kj // (c["k"] // c["slots"])).clamp(max=c["slots"] - 1)] != 0)[:, None]
    x = torch.where(see[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    v = s["v"].float()[kj].permute(0, 2, 1, 3)[:, :, None]                # [B, hk, 1, L, d]
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = torch.log(total) + top
    at = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(off[1:].contiguous(), at, right=True)
    pick = seq * s["max_q"] + at - off[seq]
    o = o.permute(0, 3, 1, 2, 4).reshape(-1, hq, d)[pick]
    lse = lse[..., 0].permute(0, 3, 1, 2).reshape(-1, hq)[pick]
    return [o.to(s["q"].dtype), lse]


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return None
    return {"prepare": _exact_prepare, "attend": _exact_attend}[case["op"]](s, case)


def _exact_turn(x, gain, pos, c):
    x = x.double()
    x = gain.double() * x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / c["dim"] + EPS)
    rot = c["pt"] + c["py"] + c["px"]
    if rot == 0:
        return x
    exps, axis = [], []
    for a, m in enumerate((c["pt"], c["py"], c["px"])):
        exps += [p / m for p in range(m)]
        axis += [a] * m
    freq = torch.tensor([THETA ** -e for e in exps], dtype=torch.float64, device="cuda")
    angle = pos.double()[:, axis] * freq
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    first = torch.arange(rot, device="cuda") * (2 if c["inter"] else 1)
    second = first + (1 if c["inter"] else rot)
    z = torch.complex(x[..., first], x[..., second]) * turn
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_prepare(s, c):
    q = _exact_turn(s["q"], s["q_gain"], s["pos"], c)
    k = _exact_turn(s["k"], s["k_gain"], s["pos"], c)
    live = torch.nonzero(s["rows"] >= 0)[:, 0]
    at = s["rows"].long()[live]
    k_mem = torch.zeros(c["rows"], c["kv"], c["dim"], dtype=torch.float64, device="cuda").index_copy_(0, at, k[live])
    v_mem = torch.zeros_like(k_mem).index_copy_(0, at, s["v"].double()[live])
    coord = torch.zeros(c["rows"], 2, dtype=torch.float64, device="cuda").index_copy_(0, at, s["pos"].double()[live, 1:])
    return [q, k_mem, v_mem, coord]


def _exact_attend(s, c):
    pairs, _ = _pairs(c)
    if pairs * c["heads"] * c["dim"] > 6 * 16384 * 49152 * 64 * 2:
        return None
    n, held, prefix, begin, _ = _spans(c)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    at = 0
    for m, h, p, b in zip(n, held, prefix, begin):
        for a in range(c["heads"]):
            kk = s["k"][b:b + h, a // (c["heads"] // c["kv"])].double()
            vv = s["v"][b:b + h, a // (c["heads"] // c["kv"])].double()
            gone = torch.zeros(h, dtype=torch.bool, device="cuda")
            if c["slots"]:
                gone = s["present"].repeat_interleave(c["k"] // c["slots"])[:h] == 0
            for lo in range(0, m, 2048):
                hi = min(m, lo + 2048)
                x = s["q"][at + lo:at + hi, a].double() @ kk.T / math.sqrt(c["dim"])
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                if c["dist"]:
                    x -= s["slopes"][a].double() * torch.cdist(s["q_pos"][at + lo:at + hi].double(),
                                                               s["k_pos"][b:b + h].double(), p=1)
                if c["causal"]:
                    r = torch.arange(lo, hi, device="cuda")[:, None] + (h - m)
                    y = torch.arange(h, device="cuda")[None]
                    x.masked_fill_((y > r) & (y >= p), -math.inf)
                x.masked_fill_(gone[None], -math.inf)
                t = torch.logsumexp(x, 1)
                w = torch.exp(x - t[:, None]).nan_to_num(0.0)
                out[at + lo:at + hi, a] = w @ vv
                lse[at + lo:at + hi, a] = t
        at += m
    return [out, lse]
