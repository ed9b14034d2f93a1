"""Measured cases of cross attention: packed query rows and single tokens over an encoder's states of another length.

  prefill  a packed batch's rows, each segment over its own range of key rows (CrossPlan.run, padoc_cross_attn)
  bwd      its gradients: of q, and of k and v summed over every segment that reads them (CrossPlan.run_bwd,
           padoc_cross_attn_bwd)
  decode   one token of each live stream over its page's states (CrossPlan.run on the streams' segments)

A segment is a range of query rows with a range of key rows. Pages are segments of their own; with regions a page has a
segment of layout rows over all of its states and one for each branch over the states of the branch's crop, so that key
rows are shared between segments. A page without an image has no key rows: its outputs are 0, its log-sum-exps -inf.

Sizes follow the repository's workloads: 16 query heads over 2 KV heads of 128 dims (the fp32 bring-up page 4 over 1 of
64; 16 over 16 of 64 as encoder-decoders have them), packed batches of 32k rows of 8 pages, serving batches of some 670
streams of 32 pages, images of 10 to 40 by 40 patches and more. The encoder's batch is padded: each page's states start
at a multiple of the longest page's. k and v of a state lie behind one another, as a fused projection leaves them.
"""
import math
import random

import torch

own = False

DEV = "cuda"


def _case(name, op, pages, rows, keys, *, hq=16, hkv=2, d=128, dtype="bf16", ragged=True, regions=0, empty=0):
    """rows, keys: query rows and states of the longest page; ragged: the other pages are shorter; regions: branches of a
    page over crops of its states; empty: every so many pages one has no states (0: none)."""
    return {"name": name, "op": op, "pages": pages, "rows": rows, "keys": keys, "hq": hq, "hkv": hkv, "d": d,
            "dtype": dtype, "ragged": ragged, "regions": regions, "empty": empty}


def listed():
    return [
        # the training forward of a packed batch of 32k rows over images of up to 2560 states
        _case("prefill_packed", "prefill", 8, 4096, 2560, ragged=False),
        # an encoder-decoder's head layout: as many KV heads as query heads, of 64 dims, ragged pages, one without an image
        _case("prefill_mha64", "prefill", 9, 2049, 1201, hkv=16, d=64, empty=5),
        # one page of odd length over one image of 24 x 40 patches and a token
        _case("prefill_page", "prefill", 1, 2617, 961),
        # the fp32 bring-up page
        _case("prefill_tiny_f32", "prefill", 1, 368, 260, hq=4, hkv=1, d=64, dtype="f32"),
        # the backward of the packed batch
        _case("bwd_packed", "bwd", 8, 4096, 2560, ragged=False),
        # layout-grounded pages: 24 branches a page, each over its region's crop of the page's states
        _case("bwd_regions", "bwd", 8, 2300, 1601, regions=24),
        # the backward in the encoder-decoder's layout
        _case("bwd_mha64", "bwd", 9, 2049, 1201, hkv=16, d=64, empty=5),
        # one decode step of the serving batch: 32 pages of up to 30 streams over up to 4096 states
        _case("decode_step", "decode", 32, 30, 4096),
        # the same streams in the encoder-decoder's layout, smaller images
        _case("decode_mha64", "decode", 32, 30, 1201, hkv=16, d=64),
        # a single user's token over one image: latency
        _case("decode_one", "decode", 1, 1, 961),
        # the branches of one page over the states of a whole document: few rows, a long axis
        _case("decode_document", "decode", 1, 24, 150_001),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["prefill", "bwd", "decode"])
    hq, hkv, d = rng.choice([(16, 2, 128), (16, 2, 128), (16, 16, 64), (8, 8, 128), (4, 1, 64), (12, 4, 64), (14, 2, 128), (10, 2, 64)])
    c = _case("", op, log_int(1, 32), 1, 1, hq=hq, hkv=hkv, d=d, dtype=rng.choice(["bf16"] * 5 + ["f32"]),
              ragged=rng.random() < 0.8, empty=rng.choice([0, 0, 4]))
    del c["name"]
    if op == "decode":
        c["rows"] = rng.randint(1, 40)
        c["keys"] = log_int(8, 4096 if c["pages"] > 1 else 150_000)
    else:
        c["rows"] = log_int(1, 4096)
        c["keys"] = log_int(8, 4096)
        c["regions"] = rng.choice([0, 0, rng.randint(2, 16)]) if c["rows"] >= 64 else 0
    # no more than the packed batch's work, in fp32 a sixteenth of it
    most = 16 * 128 * 32768 * 2560 / (16 if c["dtype"] == "f32" else 1)
    while c["pages"] * c["rows"] * c["keys"] * hq * d > most or c["pages"] * c["keys"] * hkv * d * (2 if c["dtype"] == "f32" else 1) > 2 ** 27:
        if c["pages"] > 1:
            c["pages"] //= 2
        else:
            c["keys"] //= 2
    return c


def _segments(case):
    """[(first query row, query rows, first key row, key rows)], query rows, key rows."""
    rng = random.Random(case["pages"] * 1_000_003 + case["rows"] * 1009 + case["keys"])
    segments, q = [], 0
    for p in range(case["pages"]):
        short = case["ragged"] and case["pages"] > 1
        n = rng.randint(max(1, case["rows"] * 2 // 5), case["rows"]) if short else case["rows"]
        e = rng.randint(max(1, case["keys"] // 4), case["keys"]) if short else case["keys"]
        if case["empty"] and p % case["empty"] == case["empty"] - 1:
            e = 0
        base = p * case["keys"]
        if not case["regions"]:
            segments.append((q, n, base, e))
            q += n
            continue
        layout = min(n, max(1, n // 8))
        segments.append((q, layout, base, e))
        q, left = q + layout, n - layout
        for r in range(case["regions"]):
            m = left // (case["regions"] - r)
            if m == 0:
                continue
            size = min(e, max(1, e // 12 + rng.randint(0, e // 6 + 1))) if e else 0
            segments.append((q, m, base + rng.randint(0, e - size), size))
            q, left = q + m, left - m
    return segments, q, case["pages"] * case["keys"]


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt, hq, hkv, d = _dtype(case), case["hq"], case["hkv"], case["d"]
    segments, rows, keys = _segments(case)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=dt)  # noqa: E731
    q, kv = randn(rows, hq, d), randn(keys, 2 * hkv, d)
    st = {"case": case, "segments": segments, "q": q, "k": kv[:, :hkv], "v": kv[:, hkv:], "scale": 1 / math.sqrt(d)}
    seg = torch.tensor(segments, dtype=torch.int64, device=DEV)
    # the segments side by side: the rows of each, padded to the longest, and which of them are its own
    i = torch.arange(max(s[1] for s in segments), device=DEV)
    j = torch.arange(max(1, max(s[3] for s in segments)), device=DEV)
    st["q_in"], st["k_in"] = i < seg[:, 1:2], j < seg[:, 3:4]
    st["q_at"] = torch.where(st["q_in"], seg[:, 0:1] + i, 0)
    st["k_at"] = torch.where(st["k_in"], seg[:, 2:3] + j, 0)
    if case["op"] == "bwd":     # what the forward left
        st["dout"] = randn(rows, hq, d)
        st["out"], st["lse"] = _forward(st)
    if own:
        from paper_2608_06146_gb300.engine import CrossPlan
        st["plan"] = CrossPlan(segments, hq, hkv, d, dt, DEV, training=case["op"] == "bwd")
        new = lambda n, h: torch.empty((n, h, d), dtype=dt, device=DEV)  # noqa: E731
        if case["op"] == "bwd":
            st["dq"], dkv = new(rows, hq), new(keys, 2 * hkv)
            st["dk"], st["dv"] = dkv[:, :hkv], dkv[:, hkv:]
        else:
            st["o"], st["l"] = new(rows, hq), torch.empty((rows, hq), dtype=torch.float32, device=DEV)
    return st


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------

def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    if st["case"]["op"] == "bwd":
        st["plan"].run_bwd(st["q"], st["k"], st["v"], st["out"], st["dout"], st["lse"], st["scale"], st["dq"], st["dk"], st["dv"])
        return {"dq": st["dq"], "dk": st["dk"], "dv": st["dv"]}
    st["plan"].run(st["q"], st["k"], st["v"], st["scale"], st["o"], st["l"])
    return {"out": st["o"], "lse": st["l"]}


def _run_plain(st):
    if st["case"]["op"] == "bwd":
        dq, dk, dv = _backward(st)
        return {"dq": dq, "dk": dk, "dv": dv}
    out, lse = _forward(st)
    return {"out": out, "lse": lse}


def _query_side(st, x):
    """Rows [rows][hq][d] as [segments][hkv][rows of a segment x group][d] in 32 bits."""
    c = st["case"]
    s, n = st["q_at"].shape
    return x[st["q_at"]].float().view(s, n, c["hkv"], c["hq"] // c["hkv"], c["d"]).transpose(1, 2).flatten(2, 3)


def _key_side(st, x):
    return x[st["k_at"]].float().transpose(1, 2)


def _rows_back(st, x):
    """The inverse of _query_side: the segments' own rows in their order."""
    c = st["case"]
    s, n = st["q_at"].shape
    x = x.unflatten(2, (n, c["hq"] // c["hkv"])).transpose(1, 2).flatten(2, 3)
    return x[st["q_in"]]


def _scores(st, q, k):
    return (q @ k.transpose(-1, -2)).mul_(st["scale"]).masked_fill_(~st["k_in"][:, None, None], -math.inf)


def _forward(st):
    q, k, v = _query_side(st, st["q"]), _key_side(st, st["k"]), _key_side(st, st["v"])
    s = _scores(st, q, k)
    top = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    return _rows_back(st, out).to(_dtype(st["case"])), _rows_back(st, lse)[..., 0]


def _backward(st):
    dt = _dtype(st["case"])
    q, k, v, g = _query_side(st, st["q"]), _key_side(st, st["k"]), _key_side(st, st["v"]), _query_side(st, st["dout"])
    s, n = st["q_at"].shape
    lse = st["lse"][st["q_at"]].view(s, n, st["case"]["hkv"], -1).transpose(1, 2).flatten(2, 3)[..., None]
    p = _scores(st, q, k).sub_(lse.clamp_min(torch.finfo(torch.float32).min)).exp_()
    p = p.mul_(_own_rows(st)[:, None, :, None])
    dv = p.transpose(-1, -2) @ g
    dp = g @ v.transpose(-1, -2)
    ds = dp.sub_((p * dp).sum(-1, keepdim=True)).mul_(p).mul_(st["scale"])
    dq, dk = ds @ k, ds.transpose(-1, -2) @ q
    return _rows_back(st, dq).to(dt), _keys_back(st, dk).to(dt), _keys_back(st, dv).to(dt)


def _own_rows(st):
    return st["q_in"].repeat_interleave(st["case"]["hq"] // st["case"]["hkv"], 1)


def _keys_back(st, x):
    """Sums over the segments that share a key row."""
    c = st["case"]
    total = torch.zeros((c["pages"] * c["keys"], c["hkv"], c["d"]), dtype=torch.float32, device=DEV)
    return total.index_add_(0, st["k_at"][st["k_in"]], x.transpose(1, 2)[st["k_in"]])


# ------------------------------------------------------------------------------------------------
# The definition in 64 bits
# ------------------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    train = case["op"] == "bwd"
    q, k, v = (st[n].double().requires_grad_(train) for n in "qkv")
    grads = [torch.zeros_like(t, requires_grad=False) for t in (q, k, v)]
    out = torch.zeros_like(q, requires_grad=False)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    group = case["hq"] // case["hkv"]
    for qb, qn, kb, kn in st["segments"]:
        if kn == 0:
            continue
        for h in range(case["hq"]):     # one head at a time
            with torch.set_grad_enabled(train):
                s = q[qb:qb + qn, h] @ k[kb:kb + kn, h // group].T / math.sqrt(case["d"])
                o = torch.softmax(s, -1) @ v[kb:kb + kn, h // group]
            if train:
                for total, got in zip(grads, torch.autograd.grad((o * st["dout"][qb:qb + qn, h].double()).sum(), (q, k, v))):
                    total += got
            else:
                out[qb:qb + qn, h], lse[qb:qb + qn, h] = o, torch.logsumexp(s, -1)
    return {"dq": grads[0], "dk": grads[1], "dv": grads[2]} if train else {"out": out, "lse": lse}


def work(case):
    segments, rows, keys = _segments(case)
    hq, hkv, d, e = case["hq"], case["hkv"], case["d"], 4 if case["dtype"] == "f32" else 2
    pairs = sum(s[1] * s[3] for s in segments)
    read = {}       # the states of each page that a segment reads
    for s in segments:
        read.setdefault(s[2] // case["keys"], set()).update(range(s[2], s[2] + s[3]))
    seen = sum(len(r) for r in read.values())
    if case["op"] == "bwd":
        return {"bytes": (4 * rows * hq * d + 2 * (seen + keys) * hkv * d) * e + 4 * rows * hq, "flops": 10 * pairs * hq * d}
    return {"bytes": (2 * rows * hq * d + 2 * seen * hkv * d) * e + 4 * rows * hq, "flops": 4 * pairs * hq * d}
