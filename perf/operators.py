"""The device-tensor operators as measurable cases: 4-bit microscaled quantisation and the product with such weights,
keys and values appended (rotated) to a paged cache, and attention of one new token over that cache.

A case is a dict of plain values.  `run` makes ONE pass through one operator: in its plain form (elementary torch
operations in fp32) or, where `own` is true, by the calls a user makes.  `exact` gives the same from the definitions in
64 bits.

Definitions
  block of 32 values along a row, a = largest magnitude of the block: scale 2^e, e = floor(log2 a) - 2 within
  [-127, 127]; a value becomes the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (and negatives) times the scale, ties to the
  even code, larger ones 6.  Codes lie two to a byte, the earlier value in the low four bits; a scale is held as e + 127.
  product: y = x W^T, W of codes and scales.
  cache: pages of 16 positions, keys [page][kv head][16][head_dim], values [page][kv head][head_dim][16]; position p of
  sequence s lies on page table[s][p / 16].  Appending rotates the pairs (j, j + head_dim / 2) of queries and keys by
  position * theta^(-2 j / head_dim).
  attention of one token: softmax over the (last `window`) positions of a sequence of q . k / sqrt(head_dim), times the
  values; also the logarithm of the softmax's sum.  A sequence of length 0 gives zeros and -infinity.
"""
import math

import torch

own = False

PAGE = 16
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a fused gate/up-sized matrix of the 8B shape when a model's weights become 4-bit ones
        dict(name="quantize_weight", op="quantize", dtype="bf16", rows=14336, cols=4096),
        # a few hundred fp32 rows whose length ends inside a block
        dict(name="quantize_rows", op="quantize", dtype="f32", rows=777, cols=1000),
        # plain decoding of one sequence: output projection of the 8B shape
        dict(name="project_decode", op="project", dtype="bf16", rows=1, n_in=4096, n_out=4096),
        # verification of a 64-node tree: gate/up projection of the 8B shape
        dict(name="project_tree", op="project", dtype="bf16", rows=65, n_in=4096, n_out=28672),
        # context ingestion: a pass of 2048 rows
        dict(name="project_context", op="project", dtype="bf16", rows=2048, n_in=4096, n_out=14336),
        # fp32 rows, every size odd or ragged
        dict(name="project_odd", op="project", dtype="f32", rows=37, n_in=1001, n_out=1031),
        # one new token for each of eight sequences of the 8B shape
        dict(name="append_step", op="append", dtype="bf16", seqs=8, rows_each=1, longest=4096, q_heads=32, kv_heads=8, head_dim=128, theta=500000.0, spare=0),
        # contexts of five sequences at once, 2040 rows, of the 32B-class shape; some rows of the buffers stay unused
        dict(name="append_context", op="append", dtype="bf16", seqs=5, rows_each=408, longest=1500, q_heads=64, kv_heads=8, head_dim=128, theta=1000000.0, spare=8),
        # the fp32 shape, short rows
        dict(name="append_f32", op="append", dtype="f32", seqs=3, rows_each=13, longest=100, q_heads=4, kv_heads=4, head_dim=64, theta=10000.0, spare=1),
        # one sequence of the 8B shape
        dict(name="attend_one", op="attend", dtype="bf16", seqs=1, longest=8192, q_heads=32, kv_heads=8, head_dim=128, window=0, empty=False),
        # eight ragged sequences up to 32768 tokens, 32B-class shape
        dict(name="attend_long", op="attend", dtype="bf16", seqs=8, longest=32768, q_heads=64, kv_heads=8, head_dim=128, window=0, empty=False),
        # fp32 cache, short ragged sequences, one of them empty, a window over the last positions
        dict(name="attend_f32", op="attend", dtype="f32", seqs=6, longest=700, q_heads=6, kv_heads=2, head_dim=32, window=250, empty=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("quantize", "project", "project", "append", "attend", "attend"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "quantize":
        rows = _log_int(rng, 1, 14336)
        return dict(op=op, dtype=dtype, rows=rows, cols=_log_int(rng, 32, min(14336, (14336 * 2048) // rows)))
    if op == "project":
        rows, n_in = _log_int(rng, 1, 2048), _log_int(rng, 64, 14336)
        n_out = _log_int(rng, 16, min(28672, max(64, 2048 * 4096 * 4096 // (rows * n_in))))
        if rng.random() < 0.5:
            n_in = max(128, n_in // 128 * 128)
        return dict(op=op, dtype=dtype, rows=rows, n_in=n_in, n_out=n_out)
    head_dim = rng.choice((64, 128)) if dtype == "bf16" else rng.choice((16, 32, 64, 128))
    kv_heads = rng.choice((1, 2, 4, 8))
    q_heads = kv_heads * rng.choice((1, 2, 3, 4, 8, 16) if kv_heads <= 4 else (1, 2, 4, 8))
    seqs = _log_int(rng, 1, 64)
    if op == "append":
        each = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(3, 2040 // seqs))
        return dict(op=op, dtype=dtype, seqs=seqs, rows_each=each, longest=_log_int(rng, 1, 4096), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                    theta=rng.choice((10000.0, 500000.0, 1000000.0)), spare=rng.randrange(0, 4))
    longest = _log_int(rng, 1, min(32768, 131072 // seqs))
    window = _log_int(rng, 1, longest) if rng.random() < 0.25 else 0
    return dict(op=op, dtype=dtype, seqs=seqs, longest=longest, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, window=window, empty=rng.random() < 0.25)


def lengths_of(case):
    """Ragged lengths: the first sequence is the longest, the others between 30 % and all of it; `empty`: the last has none."""
    n, top = case["seqs"], case["longest"]
    out = [top] + [max(1, int(top * (0.3 + 0.7 * ((i * 0.6180339887) % 1.0)))) for i in range(1, n)]
    if case.get("empty"):
        out[-1] = 0
    return out


def rows_of(case):
    """New rows of each sequence of an append: as many on average as `rows_each`, alternately fewer and more."""
    e = case["rows_each"]
    return [e + (0 if e == 1 else (e // 4) * (1 if i % 2 else -1)) for i in range(case["seqs"])]


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "quantize":
        n, blocks = case["rows"] * case["cols"], case["rows"] * -(-case["cols"] // 32)
        return {"bytes": 2 * n * es + 17 * blocks, "flops": 3 * n}                 # values in, codes and scales, values out
    if case["op"] == "project":
        r, k, n = case["rows"], case["n_in"], case["n_out"]
        return {"bytes": (r * k + r * n) * es + n * -(-k // 32) * 17, "flops": 2 * r * k * n}
    hd, hq, hkv = case["head_dim"], case["q_heads"], case["kv_heads"]
    if case["op"] == "append":
        r = sum(rows_of(case))
        return {"bytes": 2 * r * (hq + 2 * hkv) * hd * es, "flops": 3 * r * (hq + hkv) * hd}
    seen = sum(min(n, case["window"] or n) for n in lengths_of(case))
    return {"bytes": 2 * seen * hkv * hd * es + case["seqs"] * hq * (2 * hd * es + 4), "flops": 4 * seen * hq * hd}


# ---- inputs ---------------------------------------------------------------------------
def _inputs(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DT[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    if case["op"] == "quantize":
        spread = torch.exp(normal(case["rows"], 1))                                # rows of different magnitudes
        return {"x": (0.02 * spread * normal(case["rows"], case["cols"])).to(dt)}
    if case["op"] == "project":
        x = normal(case["rows"], case["n_in"]) * torch.exp(0.5 * normal(1, case["n_in"]))   # some channels are larger
        codes, scales = _encode(0.02 * normal(case["n_out"], case["n_in"]))
        return {"x": x.to(dt), "codes": codes, "scales": scales}
    hd, hq, hkv, n = case["head_dim"], case["q_heads"], case["kv_heads"], case["seqs"]
    lengths = lengths_of(case)
    new = rows_of(case) if case["op"] == "append" else [0] * n
    need = [-(-(a + b) // PAGE) for a, b in zip(lengths, new)]
    width, total = max(max(need), 1), sum(need)
    pages = total + 3                                                              # some belong to nobody
    order = torch.randperm(pages, generator=g, device=dev)[:total].to(torch.int32)
    starts = torch.tensor([sum(need[:i]) for i in range(n)], device=dev)
    col = torch.arange(width, device=dev)
    held = col[None, :] < torch.tensor(need, device=dev)[:, None]
    table = torch.where(held, order[(starts[:, None] + col[None, :]).clamp(max=max(total - 1, 0))], 0).to(torch.int32) if total else torch.zeros((n, width), dtype=torch.int32, device=dev)
    state = {"k_pages": normal(pages, hkv, PAGE, hd).to(dt), "v_pages": normal(pages, hkv, hd, PAGE).to(dt), "table": table.contiguous(),
             "lengths": torch.tensor(lengths, dtype=torch.int32, device=dev)}
    if case["op"] == "append":
        rows = sum(new)
        # the fused projection's rows: queries, keys and values are slices of one buffer
        state["qkv"] = normal(rows + case["spare"], (hq + 2 * hkv) * hd).to(dt)
        state["offsets"] = torch.tensor([sum(new[:i]) for i in range(n + 1)], dtype=torch.int32, device=dev)
        state["q_out"] = normal(rows + case["spare"], hq * hd).to(dt)               # rows behind the last sequence stay
    else:
        state["q"] = normal(n, hq * hd).to(dt)
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if case["op"] == "append":
        state["rows"] = sum(rows_of(case))
        hq, hkv, hd = case["q_heads"], case["kv_heads"], case["head_dim"]
        state["q"], state["k"], state["v"] = state["qkv"].split((hq * hd, hkv * hd, hkv * hd), 1)
    if case["op"] == "attend":
        state["max_len"] = case["longest"]
    if own:
        from paper_2604_13519_amd import ops
        if case["op"] == "project":              # a program lays its weights out once
            state["packed"] = ops.ts_mx_pack(state["codes"], state["scales"], case["n_in"])
        if case["op"] == "attend":               # and keeps one workspace
            state["workspace"] = ops.ts_kv_attend_workspace(case["seqs"], case["q_heads"], case["kv_heads"], case["head_dim"], case["longest"], case["window"], "cuda")
    return state


# ---- one pass -------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    return {"quantize": _plain_quantize, "project": _plain_project, "append": _plain_append, "attend": _plain_attend}[case["op"]](state, case)


def _own(state, case):
    from paper_2604_13519_amd import ops
    if case["op"] == "quantize":
        codes, scales = ops.ts_mx_quantize(state["x"])
        return ops.ts_mx_dequantize(codes, scales, case["cols"], DT[case["dtype"]])
    if case["op"] == "project":
        return ops.ts_mx_project(state["packed"], case["n_out"], state["x"])
    if case["op"] == "append":
        ops.ts_kv_append(state["k_pages"], state["v_pages"], state["table"], state["lengths"], state["offsets"], state["q"], state["k"], state["v"],
                         case["theta"], state["q_out"])
        return state["q_out"], state["k_pages"], state["v_pages"]
    return ops.ts_kv_attend(state["k_pages"], state["v_pages"], state["table"], state["lengths"], state["q"], state["max_len"], window=case["window"],
                            workspace=state["workspace"])


def _blocks(x):
    """[rows][cols] -> fp32 [rows][blocks][32], zeros behind the last column."""
    x = x.float()
    pad = -x.shape[1] % 32
    if pad:
        x = torch.cat([x, torch.zeros((x.shape[0], pad), device=x.device)], 1)
    return x.view(x.shape[0], -1, 32)


def _scaled(x):
    """Blocks over their scales, rounded to the 4-bit grid, and the exponents of the scales."""
    b = _blocks(x)
    a = b.abs().amax(2, keepdim=True)
    e = torch.where(a > 0, torch.frexp(a).exponent - 3, -127).clamp(-127, 127)
    v = b * torch.exp2(-e.float())
    m = v.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    return torch.copysign((torch.round(m / step) * step).clamp(max=6.0), v), e


def _encode(x):
    v, e = _scaled(x)
    grid = torch.tensor(MAGNITUDES, device=x.device)
    code = torch.bucketize(v.abs(), grid) + torch.where(v < 0, 8, 0)
    code = code.view(x.shape[0], -1).to(torch.uint8)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), (e[..., 0] + 127).to(torch.uint8).contiguous()


def _plain_quantize(state, case):
    x = state["x"]
    v, e = _scaled(x)
    return (v * torch.exp2(e.float())).view(x.shape[0], -1)[:, :x.shape[1]].to(x.dtype)


def _values(codes, scales, cols):
    grid = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    both = torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], -1).int()
    w = grid[both].view(codes.shape[0], -1, 32) * torch.exp2(scales.float() - 127.0)[..., None]
    return w.view(codes.shape[0], -1)[:, :cols]


def _plain_project(state, case):
    x = state["x"]
    return (x.float() @ _values(state["codes"], state["scales"], case["n_in"]).t()).to(x.dtype)


def _turn(x, pos, theta, hd):
    """[rows][heads][hd] rotated by the rows' positions."""
    j = torch.arange(hd // 2, device=x.device, dtype=torch.float64)
    angle = pos[:, None].double() * torch.pow(torch.tensor(theta, dtype=torch.float64, device=x.device), -2.0 * j / hd)
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = x.float().split(hd // 2, 2)
    return torch.cat((a * c - b * s, b * c + a * s), 2)


def _plain_append(state, case):
    hd, n = case["head_dim"], state["rows"]
    row = torch.arange(n, device="cuda", dtype=torch.int32)
    seq = torch.bucketize(row, state["offsets"][1:], right=True)
    pos = (state["lengths"][seq] + row - state["offsets"][seq]).long()
    page, slot = state["table"][seq, pos // PAGE].long(), pos % PAGE
    q, k, v = (state[c][:n].reshape(n, -1, hd) for c in "qkv")
    dt = q.dtype
    state["q_out"][:n] = _turn(q, pos, case["theta"], hd).to(dt).view(n, -1)
    state["k_pages"][page, :, slot] = _turn(k, pos, case["theta"], hd).to(dt)
    state["v_pages"][page, :, :, slot] = v
    return state["q_out"], state["k_pages"], state["v_pages"]


def _plain_attend(state, case):
    hd, hq, hkv, n = case["head_dim"], case["q_heads"], case["kv_heads"], case["seqs"]
    table = state["table"].long()
    keys = state["k_pages"][table].float()                                         # [seq][page][head][slot][dim]
    keys = keys.permute(0, 2, 4, 1, 3).reshape(n, hkv, hd, -1)
    q = state["q"].float().view(n, hkv, hq // hkv, hd)
    s = torch.matmul(q, keys) * (1.0 / math.sqrt(hd))
    del keys
    at = torch.arange(s.shape[-1], device="cuda")
    top = state["lengths"][:, None]
    seen = at[None] < top
    if case["window"]:
        seen = seen & (at[None] >= top - case["window"])
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    l = p.sum(-1, keepdim=True)
    vals = state["v_pages"][table].float().permute(0, 2, 1, 4, 3).reshape(n, hkv, -1, hd)
    vals = vals * seen[:, None, :, None]
    out = torch.matmul(p, vals) / torch.where(l == 0, 1.0, l)
    return out.to(state["q"].dtype).view(n, hq * hd), (m + torch.log(l)).view(n, hq)


# ---- the definitions in 64 bits --------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "quantize":
        return _exact_quantize(s["x"])
    if case["op"] == "project":
        return s["x"].double() @ _exact_weights(s["codes"], s["scales"], case["n_in"]).t().contiguous()
    if case["op"] == "append":
        return _exact_append(case, s)
    return _exact_attend(case, s)


def _exact_quantize(x):
    rows, cols = x.shape
    out = torch.zeros((rows, cols), dtype=torch.float64, device=x.device)
    middles = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device=x.device)
    odd_below = torch.tensor([False, True] * 4, device=x.device)                   # codes 1, 3, 5, 7 give way at a tie above them
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    for c in range(0, cols, 32):
        b = x[:, c:c + 32].double()
        top = b.abs().amax(1)
        e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
        e = torch.where(torch.exp2(e) > top, e - 1, e)
        e = torch.where(torch.exp2(e + 1) <= top, e + 1, e)
        scale = torch.exp2(torch.where(top > 0, e - 2, torch.full_like(e, -127)).clamp(-127, 127))
        v = b.abs() / scale[:, None]
        code = torch.searchsorted(middles, v.contiguous())                         # middles below v
        tie = (code < 7) & (v == middles[code.clamp(max=6)])
        code = torch.where(tie & odd_below[code], code + 1, code)
        out[:, c:c + 32] = torch.sign(b) * grid[code] * scale[:, None]
    return out


def _exact_weights(codes, scales, cols):
    c = codes.long()
    nib = torch.empty((c.shape[0], 2 * c.shape[1]), dtype=torch.int64, device=c.device)
    nib[:, 0::2], nib[:, 1::2] = c % 16, c // 16
    mag, exp = nib % 2, nib // 2 % 4                                               # one fraction bit, two exponent bits
    w = torch.where(exp == 0, 0.5 * mag.double(), (1 + 0.5 * mag.double()) * torch.exp2(exp.double() - 1))
    w = torch.where(nib >= 8, -w, w)
    return (w * torch.exp2(scales.double() - 127).repeat_interleave(32, 1))[:, :cols]


def _exact_append(case, s):
    hd, hq, hkv = case["head_dim"], case["q_heads"], case["kv_heads"]
    qo, kp, vp = (s[c].double() for c in ("q_out", "k_pages", "v_pages"))
    r = 0
    for i, (n, new) in enumerate(zip(lengths_of(case), rows_of(case))):
        pos = torch.arange(n, n + new, device="cuda")
        x = s["qkv"][r:r + new].double()
        j = torch.arange(hd // 2, device="cuda").double()
        turn = torch.polar(torch.ones((new, hd // 2), dtype=torch.float64, device="cuda"), pos[:, None].double() * torch.exp(-2 * j / hd * math.log(case["theta"])))
        qk = x[:, :(hq + hkv) * hd].view(new, hq + hkv, 2, hd // 2)
        z = torch.complex(qk[:, :, 0].contiguous(), qk[:, :, 1].contiguous()) * turn[:, None]
        qk = torch.cat((z.real, z.imag), 2)
        qo[r:r + new] = qk[:, :hq].reshape(new, -1)
        page, slot = s["table"][i].long()[pos // PAGE], pos % PAGE
        kp[page, :, slot] = qk[:, hq:]
        vp[page, :, :, slot] = x[:, (hq + hkv) * hd:].view(new, hkv, hd)
        r += new
    return qo, kp, vp


def _exact_attend(case, s):
    hd, hq, hkv = case["head_dim"], case["q_heads"], case["kv_heads"]
    out = torch.zeros((case["seqs"], hq * hd), dtype=torch.float64, device="cuda")
    lse = torch.full((case["seqs"], hq), -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(lengths_of(case)):
        if n == 0:
            continue
        first = max(0, n - case["window"]) if case["window"] else 0
        pages = s["table"][i, :-(-n // PAGE)].long()
        for h in range(hkv):
            k = s["k_pages"][pages, h].double().reshape(-1, hd)[first:n]
            v = s["v_pages"][pages, h].double().transpose(1, 2).reshape(-1, hd)[first:n]
            q = s["q"][i].double().view(hkv, -1, hd)[h]
            z = q @ k.t().contiguous() / math.sqrt(hd)
            out[i].view(hkv, -1, hd)[h] = torch.softmax(z, 1) @ v
            lse[i].view(hkv, -1)[h] = torch.logsumexp(z, 1)
    return out, lse
