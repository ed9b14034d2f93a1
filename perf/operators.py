"""Measured cases of the operators between a model's projections and the attention kernels, and of the cache's block copies.

  rotary       RMS norm of the query and key heads (or none) and rotary positions with several axes, packed rows
               (padoc_qk_rotary)
  rotary_bwd   its gradients: of the rows and of the two norm weights (padoc_qk_rotary_bwd)
  append       the same on a step's or a prefix's rows, written into the paged cache and the decode call's query
               order (padoc_append_rotary_inputs)
  append_e4m3  into the FP8 cache (padoc_append_rotary_inputs_e4m3)
  copy         blocks copied by (source, destination) pairs in every layer's pool (padoc_copy_kv_blocks, _e4m3)

Sizes follow the repository's workloads: 16 query heads over 2 KV heads of 128 dims (the fp32 bring-up page 4 over 1
of 64), packed batches of about 32k tokens, serving batches of some 670 streams, prefixes of 1024 to 4096 tokens,
blocks of 16 tokens. A row's q, k and v lie behind one another, as a fused projection leaves them.
"""
import math

import torch

own = False

DEV = "cuda"
BS = 16
BASE = 5e6      # rotary base frequency
EPS = 1e-6


def _case(name, op, rows, *, hq=16, hkv=2, d=128, rot=128, dtype="bf16", axes=3, layout="sections", adjacent=False,
          norm=True, far=0, kv="bf16", blocks=0, layers=1, run=1):
    """rows: packed rows, inputs or copied blocks; rot: rotated dims of a head; layout: how the axes share the
    frequencies; far: position of the first token; blocks: blocks of a pool; run: consecutive tokens of a stream."""
    return {"name": name, "op": op, "rows": rows, "hq": hq, "hkv": hkv, "d": d, "rot": rot, "dtype": dtype, "axes": axes,
            "layout": layout, "adjacent": adjacent, "norm": norm, "far": far, "kv": kv, "blocks": blocks,
            "layers": layers, "run": run}


def listed():
    return [
        # the training forward of a packed batch of 32k tokens of pages with an image, head norms, interleaved axes
        _case("rotary_packed", "rotary", 32768, layout="interleaved"),
        # the fp32 bring-up page: a small call, one axis, no norm
        _case("rotary_tiny_f32", "rotary", 368, hq=4, hkv=1, d=64, rot=64, dtype="f32", axes=1, norm=False),
        # one page of odd length far into a long document, adjacent pairs, half of each head rotated, without a norm
        _case("rotary_far_page", "rotary", 2617, rot=64, axes=1, adjacent=True, norm=False, far=1_000_003),
        # the backward of the packed batch, with the weights' gradients
        _case("rotary_bwd_packed", "rotary_bwd", 32768, layout="interleaved"),
        # the backward of one page, rotation only
        _case("rotary_bwd_page", "rotary_bwd", 3313, norm=False),
        # one decode step of the serving batch (32 pages): a new token for each of 672 streams
        _case("append_step", "append", 672, layout="interleaved", blocks=4096),
        # a single user's step: the latency of one token
        _case("append_one", "append", 1, layout="interleaved", blocks=256),
        # a page's prefix written to the cache, an odd number of tokens, no norm
        _case("append_prefix", "append", 4001, norm=False, blocks=1024, run=4001),
        # the decode step over the FP8 cache, and a page's prefix into it
        _case("append_e4m3_step", "append_e4m3", 672, layout="interleaved", blocks=4096, kv="e4m3"),
        _case("append_e4m3_prefix", "append_e4m3", 4001, blocks=1024, run=4001, kv="e4m3"),
        # 64 branches forked: their last blocks copied in the pools of 8 layers
        _case("copy_fork", "copy", 64, blocks=2048, layers=8),
        # a serving batch's FP8 pool compacted: the upper blocks moved down
        _case("copy_compact_e4m3", "copy", 6001, blocks=12290, kv="e4m3"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotary", "rotary_bwd", "append", "append_e4m3", "copy"])
    hq, hkv = rng.choice([(16, 2), (16, 2), (4, 1), (6, 6), (7, 1), (32, 4)])
    d = rng.choice([128, 128, 64, 80])
    rot = rng.choice([d, d, d // 2 // 16 * 16])
    axes = rng.choice([1, 2, 3, 3])
    c = _case("", op, 1, hq=hq, hkv=hkv, d=d, rot=rot, dtype=rng.choice(["bf16", "bf16", "f32"]), axes=axes,
              layout=rng.choice(["sections", "interleaved"]), adjacent=rng.random() < 0.3, norm=rng.random() < 0.6,
              far=rng.choice([0, rng.randrange(1_000_000)]))
    del c["name"]
    if op in ("rotary", "rotary_bwd"):
        c["rows"] = log_int(1, 32768 * 20 // ((hq + 2 * hkv) * (2 if c["dtype"] == "f32" else 1)))
    elif op in ("append", "append_e4m3"):
        c["rows"] = log_int(1, 4096)
        c["run"] = rng.choice([1, 1, rng.randint(2, 40), c["rows"]])
        if op == "append_e4m3":
            c["kv"], c["dtype"], c["d"], c["rot"] = "e4m3", "bf16", 128, rng.choice([128, 128, 64])
            c["hkv"], c["hq"] = rng.choice([(2, 16), (1, 8), (4, 32)])
        c["blocks"] = -(-c["rows"] // c["run"]) * (c["run"] // BS + 2) + 8
    else:
        c["kv"] = rng.choice(["bf16", "e4m3"])
        c["d"] = 128 if c["kv"] == "e4m3" else c["d"]
        c["dtype"] = "bf16" if c["kv"] == "e4m3" else c["dtype"]
        c["layers"] = rng.randint(1, 12)
        block = work(dict(c, rows=1))["bytes"]
        c["rows"] = log_int(1, max(1, int(4e8 / block)))
        c["blocks"] = 2 * c["rows"] + rng.randint(0, 200)
    return c


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _frequencies(case):
    """(inverse frequencies, axis of each), one for each rotated pair."""
    n = case["rot"] // 2
    inv = [BASE ** (-i / n) for i in range(n)]
    if case["layout"] == "sections":
        axis = [i * case["axes"] // n for i in range(n)]
    else:
        axis = [i % case["axes"] for i in range(n)]
    return inv, axis


def _positions(case, rows, g):
    """Pages of an image (the axes count its frames, rows and columns) and text (the axes run together)."""
    r = torch.arange(rows, device=DEV)
    page = r // 2500
    p = r % 2500
    w = 40
    side = int(torch.randint(10, 40, (1,), generator=g, device=DEV))
    image, base = p < side * w, case["far"] + 5 * page
    text = base + max(side, w) + p - side * w
    axes = torch.stack([base, base + p // w, base + p % w, base], 1)
    if case["axes"] == 1:
        axes = (case["far"] + p)[:, None]
        text = axes[:, 0]
    return torch.where(image[:, None], axes, text[:, None])[:, :case["axes"]].to(torch.int32).contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    op, rows, hq, hkv, d, dt = case["op"], case["rows"], case["hq"], case["hkv"], case["d"], _dtype(case)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=dt)  # noqa: E731
    st = {"case": case}
    if own:
        from paper_2608_06146_gb300 import padoc_attn as pa
        st["pa"] = pa
    if op == "copy":
        perm = torch.randperm(case["blocks"], generator=g, device=DEV).to(torch.int32)
        st["src"], st["dst"] = perm[:rows].contiguous(), perm[rows:2 * rows].contiguous()
        shape = (case["layers"], case["blocks"], hkv, BS, d)
        if case["kv"] == "e4m3":
            byte = lambda *s: torch.randint(0, 127, s, generator=g, device=DEV, dtype=torch.uint8)  # noqa: E731
            st["k"], st["v"] = byte(*shape), byte(*shape)
            st["ks"] = torch.rand(shape[:3], generator=g, device=DEV)
            st["vs"] = torch.rand(shape[:3], generator=g, device=DEV)
        else:
            st["k"], st["v"] = randn(*shape), randn(*shape)
        if own and case["kv"] == "e4m3":
            st["pools"] = pa.KvPoolsE4M3([(st["k"][i], st["v"][i], st["ks"][i], st["vs"][i]) for i in range(case["layers"])])
        elif own:
            st["pools"] = pa.KvPools([(st["k"][i], st["v"][i]) for i in range(case["layers"])])
        return st
    inv, axis = _frequencies(case)
    st["inv"] = torch.tensor(inv, dtype=torch.float64, device=DEV)
    st["axis"] = torch.tensor(axis, dtype=torch.int64, device=DEV)
    qkv = randn(rows, hq + 2 * hkv, d)
    st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    st["pos"] = _positions(case, rows, g)
    st["qw"], st["kw"] = ((1 + 0.1 * randn(d), 1 + 0.1 * randn(d)) if case["norm"] else (None, None))
    if op == "rotary_bwd":
        st["dq_out"], st["dk_out"] = randn(rows, hq, d), randn(rows, hkv, d)
    if op in ("append", "append_e4m3"):
        streams, run = -(-rows // case["run"]), case["run"]
        per = run // BS + 2
        blocks = torch.randperm(case["blocks"], generator=g, device=DEV)[:streams * per].reshape(streams, per)
        i = torch.arange(rows, device=DEV)
        first = torch.randint(0, BS, (streams,), generator=g, device=DEV) if run < rows or rows == 1 else torch.zeros(1, dtype=torch.int64, device=DEV)
        at = first[i // run] + i % run
        st["slots"] = (blocks[i // run, at // BS] * BS + at % BS).to(torch.int32)
        # the batch's rows lie in another order than its streams
        st["src_rows"] = torch.randperm(rows, generator=g, device=DEV).to(torch.int32) if run < rows else torch.arange(rows, device=DEV, dtype=torch.int32)
        shape = (case["blocks"], hkv, BS, d)
        if case["kv"] == "e4m3":
            # what the cache holds: codes of values whose largest magnitude is the format's, a scale for each block
            code = lambda: (randn(*shape).float() * 150).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)  # noqa: E731
            scale = lambda: (2.5 + torch.rand(shape[:2], generator=g, device=DEV)) / 448  # noqa: E731
            st["k_codes"], st["v_codes"], st["k_scales"], st["v_scales"] = code(), code(), scale(), scale()
        else:
            st["k_pool"], st["v_pool"] = randn(*shape), randn(*shape)
    if own:
        st["rotary"] = pa.Rotary(inv, axis, case["axes"], d, adjacent=case["adjacent"], q_weight=st["qw"],
                                 k_weight=st["kw"], eps=EPS, device=DEV)
        f32 = dict(dtype=torch.float32, device=DEV)
        st["q_out"] = torch.empty((rows, hq, d), dtype=dt, device=DEV)
        st["k_out"] = torch.empty((rows, hkv, d), dtype=dt, device=DEV)
        if op == "rotary_bwd" and case["norm"]:
            st["dqw"], st["dkw"] = torch.empty(d, **f32), torch.empty(d, **f32)
            ws = pa.padoc_qk_rotary_bwd_workspace_size(st["rotary"], rows)
            st["ws"] = torch.empty(max(ws, 256), dtype=torch.uint8, device=DEV)
        if case["kv"] == "e4m3":
            st["pool"] = pa.E4M3Pool.over(st["k_codes"], st["v_codes"], st["k_scales"], st["v_scales"])
    return st


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------

def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    pa, case = st["pa"], st["case"]
    op = case["op"]
    if op == "copy":
        if case["kv"] == "e4m3":
            pa.padoc_copy_kv_blocks_e4m3(st["pools"], st["src"], st["dst"])
        else:
            pa.padoc_copy_kv_blocks(st["pools"], st["src"], st["dst"])
        return _copied(st)
    rot = st["rotary"]
    if op == "rotary":
        pa.padoc_qk_rotary(rot, st["q"], st["k"], st["pos"], st["q_out"], st["k_out"])
        return {"q": st["q_out"], "k": st["k_out"]}
    if op == "rotary_bwd":
        if not case["norm"]:
            pa.padoc_qk_rotary_bwd(rot, st["dq_out"], st["dk_out"], st["pos"], st["q_out"], st["k_out"])
            return {"dq": st["q_out"], "dk": st["k_out"]}
        pa.padoc_qk_rotary_bwd(rot, st["dq_out"], st["dk_out"], st["pos"], st["q_out"], st["k_out"], st["q"], st["k"],
                               st["dqw"], st["dkw"], st["ws"])
        return {"dq": st["q_out"], "dk": st["k_out"], "dqw": st["dqw"], "dkw": st["dkw"]}
    if op == "append":
        pa.padoc_append_rotary_inputs(rot, st["k_pool"], st["v_pool"], st["k"], st["v"], st["pos"], st["slots"],
                                      st["q"], st["q_out"], st["src_rows"])
        return {"q": st["q_out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"]}
    pa.padoc_append_rotary_inputs_e4m3(rot, st["pool"], st["k"], st["v"], st["pos"], st["slots"], st["q"], st["q_out"],
                                       st["src_rows"])
    return _e4m3_state(st, st["q_out"])


def _copied(st):
    """Copies are compared bit by bit."""
    if st["case"]["kv"] == "e4m3":
        return {"k": st["k"], "v": st["v"], "ks": st["ks"].view(torch.int32), "vs": st["vs"].view(torch.int32)}
    whole = torch.int32 if st["case"]["dtype"] == "f32" else torch.int16
    return {"k": st["k"].view(whole), "v": st["v"].view(whole)}


def _e4m3_state(st, q):
    f8 = torch.float8_e4m3fn
    return {"q": q, "k": st["k_codes"].view(f8), "v": st["v_codes"].view(f8), "ks": st["k_scales"], "vs": st["v_scales"]}


def _cos_sin(st, pos):
    a = pos.double()[:, st["axis"]] * st["inv"]
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _split(st, x):
    """The two members of each rotated pair, and the dims that are not rotated."""
    r, rest = st["case"]["rot"], x[..., st["case"]["rot"]:]
    if st["case"]["adjacent"]:
        return x[..., 0:r:2], x[..., 1:r:2], rest
    return x[..., :r // 2], x[..., r // 2:r], rest


def _join(st, x0, x1, rest):
    if st["case"]["adjacent"]:
        return torch.cat([torch.stack([x0, x1], -1).flatten(-2), rest], -1)
    return torch.cat([x0, x1, rest], -1)


def _forward(st, x, w, c, s):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    x0, x1, rest = _split(st, x)
    return _join(st, x0 * c - x1 * s, x1 * c + x0 * s, rest)


def _backward(st, dz, x, w, c, s):
    d0, d1, rest = _split(st, dz.float())
    g = _join(st, d0 * c + d1 * s, d1 * c - d0 * s, rest)
    if w is None:
        return g.to(dz.dtype), None
    x, wg = x.float(), g * w.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xh = x * r
    dx = r * (wg - xh * (wg * xh).mean(-1, keepdim=True))
    return dx.to(dz.dtype), (g * xh).sum((0, 1), dtype=torch.float64).float()


def _run_plain(st):
    case = st["case"]
    op, dt = case["op"], _dtype(case)
    if op == "copy":
        src, dst = st["src"].long(), st["dst"].long()
        st["k"][:, dst] = st["k"][:, src]
        st["v"][:, dst] = st["v"][:, src]
        if case["kv"] == "e4m3":
            st["ks"][:, dst] = st["ks"][:, src]
            st["vs"][:, dst] = st["vs"][:, src]
        return _copied(st)
    if op in ("rotary", "rotary_bwd"):
        c, s = _cos_sin(st, st["pos"])
        if op == "rotary":
            return {"q": _forward(st, st["q"], st["qw"], c, s).to(dt), "k": _forward(st, st["k"], st["kw"], c, s).to(dt)}
        dq, dqw = _backward(st, st["dq_out"], st["q"], st["qw"], c, s)
        dk, dkw = _backward(st, st["dk_out"], st["k"], st["kw"], c, s)
        return {"dq": dq, "dk": dk, "dqw": dqw, "dkw": dkw} if case["norm"] else {"dq": dq, "dk": dk}
    at, slots = st["src_rows"].long(), st["slots"].long()
    c, s = _cos_sin(st, st["pos"][at])
    q = _forward(st, st["q"][at], st["qw"], c, s).to(dt)
    k, v = _forward(st, st["k"][at], st["kw"], c, s), st["v"][at]
    block, row = slots // BS, slots % BS
    if op == "append":
        st["k_pool"][block, :, row] = k.to(dt)
        st["v_pool"][block, :, row] = v
        return {"q": q, "k_pool": st["k_pool"], "v_pool": st["v_pool"]}
    _append_codes(k, block, row, st["k_codes"], st["k_scales"])
    _append_codes(v.float(), block, row, st["v_codes"], st["v_scales"])
    return _e4m3_state(st, q)


def _append_codes(x, block, row, codes, scales):
    """Rows x [n][heads][d] into their blocks: the block's scale grows to the rows' largest magnitude / 448, and the
    rows before the call's first one are encoded again where it does."""
    first = torch.full((codes.shape[0],), BS, dtype=torch.int64, device=DEV).scatter_reduce(0, block, row, "amin")[block]
    old = torch.where(first[:, None] == 0, 0.0, scales[block])
    heads = block[:, None].expand(-1, scales.shape[1])
    new = torch.zeros_like(scales).scatter_reduce(0, heads, x.abs().amax(-1) / 448, "amax")[block]
    new = torch.maximum(old, new)
    held = codes[block].view(torch.float8_e4m3fn).float() * old[..., None, None]
    again = (new > old) & (old > 0)
    again = again[..., None, None] & (torch.arange(BS, device=DEV)[None, None, :, None] < first[:, None, None, None])
    codes[block] = torch.where(again, _codes(held, new[..., None, None]), codes[block])
    codes[block, :, row] = _codes(x, new[..., None])
    scales[block] = new


def _codes(x, scale):
    y = torch.where(scale > 0, x / scale, 0.0)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


# ------------------------------------------------------------------------------------------------
# The definition in 64 bits
# ------------------------------------------------------------------------------------------------

def _pair_index(case):
    """Dims of the first and of the second member of each pair."""
    i = torch.arange(case["rot"] // 2, device=DEV)
    return (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + case["rot"] // 2)


def _turned(case, x, w, turn):
    """x [n][heads][d] in 64 bits: normed, its pairs as complex numbers times turn [n][1][pairs]."""
    if w is not None:
        x = x / (x.square().sum(-1, keepdim=True) / case["d"] + EPS).sqrt() * w
    i, j = _pair_index(case)
    z = torch.complex(x[..., i], x[..., j]) * turn
    out = x.clone()
    out[..., i] = z.real
    out[..., j] = z.imag
    return out


def exact(case, seed):
    if case["op"] == "copy":
        return None     # moved bits, none computed
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    f64 = lambda t: None if t is None else t.double()  # noqa: E731
    inv, axis = _frequencies(case)
    phase = torch.stack([st["pos"][:, a].double() * f for f, a in zip(inv, axis)], -1)
    turn = torch.polar(torch.ones_like(phase), phase)[:, None]
    q, k, qw, kw = f64(st["q"]), f64(st["k"]), f64(st["qw"]), f64(st["kw"])
    if case["op"] == "rotary":
        return {"q": _turned(case, q, qw, turn), "k": _turned(case, k, kw, turn)}
    if case["op"] == "rotary_bwd":
        out = {}
        for n, x, w, dz in (("q", q, qw, st["dq_out"]), ("k", k, kw, st["dk_out"])):
            leaf = [t.detach().requires_grad_() for t in (x, w) if t is not None]
            z = _turned(case, leaf[0], leaf[1] if w is not None else None, turn)
            grads = torch.autograd.grad(z, leaf, dz.double())
            out.update({"d" + n: grads[0]} if w is None else {"d" + n: grads[0], "d" + n + "w": grads[1]})
        return out
    at = st["src_rows"].long()
    q, k, v = _turned(case, q[at], qw, turn[at]), _turned(case, k[at], kw, turn[at]), st["v"][at].double()
    slots = st["slots"].long()
    if case["op"] == "append":
        out = {"q": q}
        for n, x in (("k_pool", k), ("v_pool", v)):
            pool = st[n].double().transpose(1, 2).flatten(0, 1)     # [slots][heads][d]
            pool[slots] = x
            out[n] = pool.unflatten(0, (-1, BS)).transpose(1, 2)
        return out
    # 8-bit codes have no value in 64 bits, the scales have
    out = {"q": q, "k": None, "v": None}
    for n, x, held in (("ks", k, st["k_scales"]), ("vs", v, st["v_scales"])):
        scales = held.double()
        scales[slots[slots % BS == 0] // BS] = 0
        index = (slots // BS)[:, None].expand(-1, case["hkv"])
        out[n] = scales.scatter_reduce(0, index, x.abs().amax(-1) / 448, "amax")
    return out


def work(case):
    rows, hq, hkv, d = case["rows"], case["hq"], case["hkv"], case["d"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "copy":
        block = 2 * hkv * (BS * d + 4 if case["kv"] == "e4m3" else BS * d * e)
        return {"bytes": rows * (case["layers"] * 2 * block + 8), "flops": 0}
    turned, pos = rows * (hq + hkv) * d, rows * 4 * case["axes"]
    flops = turned * (3 + (5 if case["norm"] else 0))
    if case["op"] == "rotary":
        return {"bytes": 2 * turned * e + pos, "flops": flops}
    if case["op"] == "rotary_bwd":
        return {"bytes": (3 if case["norm"] else 2) * turned * e + pos, "flops": flops + (turned * 6 if case["norm"] else 0)}
    v = rows * hkv * d
    read = (turned + v) * e + pos + 8 * rows
    if case["op"] == "append":
        return {"bytes": read + (turned + v) * e, "flops": flops}
    return {"bytes": read + rows * hq * d * e + 2 * v, "flops": flops + 4 * v}
