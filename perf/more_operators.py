"""More device-tensor operators as measurable cases, all over the paged cache: rows appended to it with a norm of each head and a
rotation in the same pass, pages of 8-bit values that are written so and read back, and attention of chunks of new rows
(whole prompts, pieces of them, draft trees, single tokens) over pages of any type.

A case is a dict of plain values.  `run` makes ONE pass through one operator: in its plain form (elementary torch
operations in fp32) or, where `own` is true, by the calls a user makes.  `exact` gives the same from the definitions in
64 bits.

Definitions
  cache: pages of 16 positions, keys [page][kv head][16][head_dim], values [page][kv head][head_dim][16]; position p of
  sequence s lies on page table[s][p / 16].  8-bit pages hold e4m3 values and, for each page, head and position, the exponent
  (+ 127) of a power of two that they are multiplied by: the smallest 2^e, e >= -127, with the largest magnitude of the
  head's row at most 448 * 2^e (all zeros: -127); values are rounded to nearest, ties to even.
  append: row i of sequence s goes to position lengths[s] + i.  Queries and keys are divided by sqrt(mean of squares of the head + eps)
  and multiplied by a gain of head_dim values (where there is one), then their first `rope_dim` values are turned in pairs, (j, j + rope_dim / 2)
  or (2 j, 2 j + 1), by angle * frequency[j], and multiplied by a magnitude; the angle's position is the row's, or one that is given.
  frequency[j] = theta^(-2 j / rope_dim) or a table.
  read: positions starts[s] + i of each sequence as rows of keys and of values.
  attention: row i of a sequence with `lengths[s]` earlier positions sees those, and of the chunk's own rows those up to itself;
  with a window only the last `window` positions up to itself; with ancestor sets (64 bits a row) row 0 of the chunk and each row
  j whose bit j - 1 is set.  out = softmax(scale q . k) v, query head h over KV head h / group; also the logarithm of the softmax's sum.
"""
import math
import random

import torch

own = False

PAGE = 16
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
EPS = 1e-6


def listed():
    return [
        # one new token for each of eight sequences of the 8B shape, into 8-bit pages, heads normed
        dict(name="append_step8", op="append", dtype="bf16", cache="e4m3", seqs=8, rows_each=1, longest=4096, q_heads=32, kv_heads=8, head_dim=128,
             norm=True, rope="half", rope_dim=128, theta=500000.0, scaled=False, tree=False, spare=0),
        # contexts of five sequences at once, 2040 rows, of the 32B-class shape, into 8-bit pages; some rows of the buffers stay unused
        dict(name="append_context8", op="append", dtype="bf16", cache="e4m3", seqs=5, rows_each=408, longest=1500, q_heads=64, kv_heads=8, head_dim=128,
             norm=True, rope="half", rope_dim=128, theta=1000000.0, scaled=False, tree=False, spare=8),
        # fp32, short rows, half of the head turned in neighbouring pairs by a table scaled for long contexts
        dict(name="append_partial", op="append", dtype="f32", cache="f32", seqs=3, rows_each=13, longest=100, q_heads=4, kv_heads=4, head_dim=64,
             norm=True, rope="pairs", rope_dim=32, theta=10000.0, scaled=True, tree=False, spare=1),
        # the 8-bit context of four sequences given back as rows, for a program that moves or checks it
        dict(name="read_context8", op="read", dtype="bf16", cache="e4m3", seqs=4, rows_each=4000, longest=8192, kv_heads=8, head_dim=128),
        # a few positions of an fp32 cache
        dict(name="read_few", op="read", dtype="f32", cache="f32", seqs=5, rows_each=9, longest=300, kv_heads=2, head_dim=32),
        # one token of one sequence of the 8B shape over 8-bit pages
        dict(name="attend_one8", op="attend", dtype="bf16", cache="e4m3", seqs=1, rows_each=1, longest=8192, q_heads=32, kv_heads=8, head_dim=128, window=0, tree=False, spare=0),
        # one token for each of eight ragged sequences up to 32768 positions, 32B-class shape, 8-bit pages
        dict(name="attend_long8", op="attend", dtype="bf16", cache="e4m3", seqs=8, rows_each=1, longest=32768, q_heads=64, kv_heads=8, head_dim=128, window=0, tree=False, spare=0),
        # verification of a tree of 64 nodes and its root over 8192 positions of the 8B shape
        dict(name="attend_tree", op="attend", dtype="bf16", cache="bf16", seqs=1, rows_each=65, longest=8192, q_heads=32, kv_heads=8, head_dim=128, window=0, tree=True, spare=0),
        # sixteen requests with a chain of some 33 rows each, ragged contexts
        dict(name="attend_batch", op="attend", dtype="bf16", cache="bf16", seqs=16, rows_each=33, longest=4096, q_heads=32, kv_heads=8, head_dim=128, window=0, tree=False, spare=2),
        # whole prompts of three sequences, packed, nothing in the cache before them
        dict(name="attend_prompts", op="attend", dtype="bf16", cache="bf16", seqs=3, rows_each=3277, longest=0, q_heads=32, kv_heads=8, head_dim=128, window=0, tree=False, spare=0),
        # pieces of long prompts of four sequences, 32B-class shape, 8-bit pages
        dict(name="attend_chunk8", op="attend", dtype="bf16", cache="e4m3", seqs=4, rows_each=512, longest=16384, q_heads=64, kv_heads=8, head_dim=128, window=0, tree=False, spare=0),
        # fp32 cache, short ragged chunks with a window, odd sizes
        dict(name="attend_f32", op="attend", dtype="f32", cache="f32", seqs=3, rows_each=37, longest=700, q_heads=6, kv_heads=2, head_dim=32, window=250, tree=False, spare=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("append", "append", "read", "attend", "attend", "attend"))
    cache = rng.choice(("bf16", "bf16", "e4m3", "e4m3", "f32"))
    dtype = "f32" if cache == "f32" or rng.random() < 0.15 else "bf16"
    hd = rng.choice((16, 32, 64, 128)) if cache == "f32" else rng.choice((64, 128))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 3, 4, 5, 8) if hkv > 1 else (1, 4, 7, 16))
    seqs = _log_int(rng, 1, 64)
    case = dict(op=op, dtype=dtype, cache=cache, seqs=seqs, kv_heads=hkv, head_dim=hd)
    if op == "read":
        longest = _log_int(rng, 1, min(16384, 131072 // seqs))
        return dict(case, rows_each=_log_int(rng, 1, min(longest, max(1, 16384 // seqs))), longest=longest)
    tree = rng.random() < 0.2
    each = rng.choice((1, _log_int(rng, 2, 65), _log_int(rng, 2, max(2, 2040 // seqs))))
    if tree:
        each = rng.randrange(2, 53)                                                # at most 65 rows where they alternate
    if op == "append":
        rope = rng.choice(("half", "half", "pairs"))
        rope_dim = hd if rng.random() < 0.6 else 2 * rng.randrange(1, hd // 2)
        return dict(case, q_heads=hq, rows_each=min(each, max(1, 2040 // seqs)), longest=_log_int(rng, 1, 4096), norm=rng.random() < 0.7, rope=rope, rope_dim=rope_dim,
                    theta=rng.choice((10000.0, 500000.0, 1000000.0)), scaled=rng.random() < 0.3, tree=tree, spare=rng.randrange(0, 4))
    room = 64 << 20                                                                # rows x heads x positions: half of the largest listed case
    if dtype == "f32":
        room >>= 3
    longest = rng.choice((0, _log_int(rng, 1, 32768))) if each > 1 else _log_int(rng, 1, 32768)
    longest = min(longest, 131072 // seqs, 16 * room // (seqs * each * hq))
    window = _log_int(rng, 1, longest + each) if rng.random() < 0.25 and not tree else 0
    return dict(case, q_heads=hq, rows_each=each, longest=longest, window=window, tree=tree, spare=rng.randrange(0, 4))


def lengths_of(case):
    """Positions before the new rows: the first sequence has the most, the others between 30 % and all of it."""
    n, top = case["seqs"], case["longest"]
    return [top] + [min(top, max(1, int(top * (0.3 + 0.7 * ((i * 0.6180339887) % 1.0))))) for i in range(1, n)]


def rows_of(case):
    """New rows of each sequence: as many on average as `rows_each`, alternately fewer and more."""
    e, n = case["rows_each"], case["seqs"]
    new = [e + (0 if n == 1 else (e // 4) * (1 if i % 2 else -1)) for i in range(n)]
    return [min(r, top) for r, top in zip(new, lengths_of(case))] if case["op"] == "read" else new


def starts_of(case):
    """The first position that is read of each sequence: some a little, some far into it."""
    return [(n - r) * (i % 3) // 2 for i, (n, r) in enumerate(zip(lengths_of(case), rows_of(case)))]


def _seen(case):
    """(sum over rows of the positions a row sees, sum over sequences of the positions any of its rows sees)"""
    w, rows, keys = case["window"], 0, 0
    for n, new in zip(lengths_of(case), rows_of(case)):
        full = n + new
        keys += full if not w else min(full, w + new - 1)
        if case["tree"]:
            rows += new * (n + 1) + sum(bin(a).count("1") for a in _tree(case, 0, new)[0])
        else:
            rows += sum(min(n + i + 1, w or n + i + 1) for i in range(new))
    return rows, keys


def work(case):
    es, hd, hkv = (2 if case["dtype"] == "bf16" else 4), case["head_dim"], case["kv_heads"]
    row = hkv * {"bf16": 2 * hd, "f32": 4 * hd, "e4m3": hd + 1}[case["cache"]]     # bytes of a position's keys, or of its values
    r = sum(rows_of(case))
    if case["op"] == "read":
        return {"bytes": 2 * r * (row + hkv * hd * es), "flops": 2 * r * hkv * hd}
    hq = case["q_heads"]
    if case["op"] == "append":
        return {"bytes": 2 * r * hq * hd * es + 2 * r * (row + hkv * hd * es), "flops": 8 * r * (hq + hkv) * hd}
    rows, keys = _seen(case)
    return {"bytes": 2 * keys * row + r * hq * (2 * hd * es + 4), "flops": 4 * rows * hq * hd}


# ---- inputs ---------------------------------------------------------------------------
def _tree(case, seed, rows):
    """A random tree of `rows` rows, the root first: (ancestor sets with the row itself, depths)."""
    rng = random.Random(seed * 1000003 + rows)
    sets, depth = [0], [0]
    for j in range(1, rows):
        up = j - 1 if rng.random() < 0.6 else rng.randrange(0, j)
        sets.append(sets[up] | 1 << (j - 1))
        depth.append(depth[up] + 1)
    return sets, depth


def _frequencies(case):
    """theta^(-2 j / rope_dim); for long contexts the slow ones are divided by 8, those between mixed."""
    j = torch.arange(case["rope_dim"] // 2, dtype=torch.float64)
    f = torch.exp(-2.0 * j / case["rope_dim"] * math.log(case["theta"]))
    turns = f * (4096 / (2 * math.pi))
    keep = ((turns - 1) / 31).clamp(0, 1)
    return (f * keep + f / 8 * (1 - keep)).float()


def _inputs(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    hd, hkv, n, dt = case["head_dim"], case["kv_heads"], case["seqs"], DT[case["dtype"]]
    lengths, new = lengths_of(case), rows_of(case)
    need = [-(-(a + (0 if case["op"] == "read" else b)) // PAGE) for a, b in zip(lengths, new)]
    width, total = max(need), sum(need)
    pages = total + 3                                                              # some belong to nobody
    order = torch.randperm(pages, generator=g, device=dev)[:total].to(torch.int32)
    starts = torch.tensor([sum(need[:i]) for i in range(n)], device=dev)
    col = torch.arange(width, device=dev)
    held = col[None, :] < torch.tensor(need, device=dev)[:, None]
    table = torch.where(held, order[(starts[:, None] + col[None, :]).clamp(max=total - 1)], 0).to(torch.int32)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    state = {"table": table.contiguous(), "lengths": ints(lengths), "offsets": ints([sum(new[:i]) for i in range(n + 1)])}
    k = normal(pages, hkv, PAGE, hd) * torch.exp(0.5 * normal(1, hkv, 1, hd))      # some channels are larger
    v = normal(pages, hkv, PAGE, hd)
    if case["cache"] == "e4m3":
        (kc, ks), (vc, vs) = _encode8(k), _encode8(v)
        state.update(k_pages=kc, v_pages=vc.view(torch.uint8).transpose(2, 3).contiguous().view(DT["e4m3"]), scales=(ks, vs))
    else:
        state.update(k_pages=k.to(DT[case["cache"]]), v_pages=v.to(DT[case["cache"]]).transpose(2, 3).contiguous(), scales=None)
    del k, v
    if case["op"] == "read":
        state["starts"] = ints(starts_of(case))
        return state
    hq, rows = case["q_heads"], sum(new)
    trees = [_tree(case, seed + 7 * i, r) for i, r in enumerate(new)] if case["tree"] else None
    if case["op"] == "append":
        # the fused projection's rows: queries, keys and values are slices of one buffer
        state["qkv"] = (normal(rows + case["spare"], (hq + 2 * hkv) * hd) * torch.exp(0.3 * normal(rows + case["spare"], 1))).to(dt)
        state["q_out"] = normal(rows + case["spare"], hq * hd).to(dt)               # rows behind the last sequence stay
        state["gains"] = ((1 + 0.2 * normal(hd)).to(dt), (1 + 0.2 * normal(hd)).to(dt)) if case["norm"] else (None, None)
        state["freqs"] = _frequencies(case).to(dev) if case["scaled"] else None
        state["positions"] = ints([a + d for a, t in zip(lengths, trees) for d in t[1]] + [0] * case["spare"]) if trees else None
    else:
        state["q"] = normal(rows + case["spare"], hq * hd).to(dt)
        state["out"] = (0.01 * normal(rows + case["spare"], hq * hd)).to(dt)               # rows behind the last sequence stay
        state["lse"] = normal(rows + case["spare"], hq)
        sets = [a if a < 1 << 63 else a - (1 << 64) for t in trees for a in t[0]] + [0] * case["spare"] if trees else None
        state["ancestors"] = torch.tensor(sets, dtype=torch.int64, device=dev) if trees else None
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    state["rows"] = sum(rows_of(case))
    hd, hkv = case["head_dim"], case["kv_heads"]
    if case["op"] == "append":
        state["q"], state["k"], state["v"] = state["qkv"].split((case["q_heads"] * hd, hkv * hd, hkv * hd), 1)
    if case["op"] == "attend":
        state["max_len"] = max(a + b for a, b in zip(lengths_of(case), rows_of(case)))
        state["max_rows"] = max(rows_of(case))
        if own:                                  # a program keeps one workspace
            from paper_2604_13519_amd import ops
            state["workspace"] = ops.ts_kv_attend_rows_workspace(case["seqs"], state["rows"] + case["spare"], case["q_heads"], hkv, hd, state["max_len"], case["window"], "cuda")
    return state


# ---- one pass -------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend}[case["op"]](state, case)


def _own(state, case):
    from paper_2604_13519_amd import ops
    s = state
    if case["op"] == "append":
        ops.ts_kv_append_norm_rope(s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["offsets"], s["q"], s["k"], s["v"], rope_theta=case["theta"],
                                   rope_dim=case["rope_dim"], rope_pairs=case["rope"] == "pairs", rope_freqs=s["freqs"], rope_magnitude=_magnitude(case),
                                   q_norm=s["gains"][0], k_norm=s["gains"][1], norm_eps=EPS, positions=s["positions"], scales=s["scales"], q_out=s["q_out"])
        if case["cache"] != "e4m3":
            return s["q_out"], s["k_pages"], s["v_pages"]
        return (s["q_out"],) + ops.ts_kv_read(s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["offsets"], s["rows"], scales=s["scales"])
    if case["op"] == "read":
        return ops.ts_kv_read(s["k_pages"], s["v_pages"], s["table"], s["starts"], s["offsets"], s["rows"], dtype=DT[case["dtype"]], scales=s["scales"])
    return ops.ts_kv_attend_rows(s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["offsets"], s["q"], s["max_len"], window=case["window"],
                                 ancestors=s["ancestors"], scales=s["scales"], workspace=s["workspace"], out=s["out"], lse=s["lse"])


def _magnitude(case):
    return 1.0 + 0.1 * math.log(8.0) if case["scaled"] else 1.0


def _encode8(x):
    """[...][head_dim] -> (e4m3 values, exponents + 127 of the rows' scales)"""
    a = x.float().abs().amax(-1)
    m, e = torch.frexp(a)
    e = torch.where(a > 0, e - torch.where(m <= 0.875, 9, 8), -127).clamp(min=-127)
    return (x.float() * torch.exp2(-e.float())[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(state, which, pages=None):
    """Pages (all, or those that a tensor names) as fp32."""
    p = state[which + "_pages"]
    if state["scales"] is None:
        return (p if pages is None else p[pages]).float()
    s = state["scales"][0 if which == "k" else 1]
    if pages is not None:
        p, s = p.view(torch.uint8)[pages].view(p.dtype), s[pages]
    s = torch.exp2(s.float() - 127.0)
    return p.float() * (s[..., None] if which == "k" else s[..., None, :])


def _seq_of(state, n):
    row = torch.arange(n, device="cuda", dtype=torch.int32)
    seq = torch.bucketize(row, state["offsets"][1:], right=True)
    return seq, row - state["offsets"][seq]


def _normed(x, gain):
    x = x.float()
    return x if gain is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()


def _turned(x, angle, case):
    """[rows][heads][head_dim], the first rope_dim values turned by [rows][rope_dim / 2] angles"""
    rd, mag = case["rope_dim"], _magnitude(case)
    c, s = (mag * torch.cos(angle)).float()[:, None], (mag * torch.sin(angle)).float()[:, None]
    head, rest = x[..., :rd], x[..., rd:]
    if case["rope"] == "half":
        a, b = head[..., :rd // 2], head[..., rd // 2:]
        return torch.cat((a * c - b * s, b * c + a * s, rest), -1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat((torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2), rest), -1)


def _plain_append(state, case):
    hd, n, rd = case["head_dim"], state["rows"], case["rope_dim"]
    seq, at = _seq_of(state, n)
    pos = (state["lengths"][seq] + at).long()
    page, slot = state["table"][seq, pos // PAGE].long(), pos % PAGE
    if state["freqs"] is not None:
        freq = state["freqs"].double()
    else:
        j = torch.arange(rd // 2, device="cuda", dtype=torch.float64)
        freq = torch.pow(torch.tensor(case["theta"], dtype=torch.float64, device="cuda"), -2.0 * j / rd)
    where = pos if state["positions"] is None else state["positions"][:n]
    angle = where[:, None].double() * freq
    q, k, v = (state[c][:n].reshape(n, -1, hd) for c in "qkv")
    state["q_out"][:n] = _turned(_normed(q, state["gains"][0]), angle, case).to(q.dtype).view(n, -1)
    k = _turned(_normed(k, state["gains"][1]), angle, case)
    kp, vp = state["k_pages"], state["v_pages"]
    if state["scales"] is None:
        kp[page, :, slot] = k.to(kp.dtype)
        vp[page, :, :, slot] = v.to(vp.dtype)
    else:
        (kc, ks), (vc, vs) = _encode8(k), _encode8(v)
        kp.view(torch.uint8)[page, :, slot] = kc.view(torch.uint8)
        vp.view(torch.uint8)[page, :, :, slot] = vc.view(torch.uint8)
        state["scales"][0][page, :, slot] = ks
        state["scales"][1][page, :, slot] = vs
        return (state["q_out"],) + _rows_at(state, pos, seq, torch.bfloat16)       # 8-bit rows come back as the values they stand for
    return state["q_out"], kp, vp


def _rows_at(state, pos, seq, dtype):
    """Keys and values at positions of sequences, as rows."""
    page, slot = state["table"][seq, pos // PAGE].long(), pos % PAGE
    kp, vp, n = state["k_pages"], state["v_pages"], len(pos)
    if state["scales"] is None:
        k, v = kp[page, :, slot].float(), vp[page, :, :, slot].float()
    else:
        k = kp.view(torch.uint8)[page, :, slot].view(kp.dtype).float() * torch.exp2(state["scales"][0][page, :, slot].float() - 127.0)[..., None]
        v = vp.view(torch.uint8)[page, :, :, slot].view(vp.dtype).float() * torch.exp2(state["scales"][1][page, :, slot].float() - 127.0)[..., None]
    return k.to(dtype).view(n, -1), v.to(dtype).view(n, -1)


def _plain_read(state, case):
    seq, at = _seq_of(state, state["rows"])
    return _rows_at(state, (state["starts"][seq] + at).long(), seq, DT[case["dtype"]])


def _plain_attend(state, case):
    hd, hq, hkv, n = case["head_dim"], case["q_heads"], case["kv_heads"], case["seqs"]
    group, most, off = hq // hkv, state["max_rows"], state["offsets"].long()
    table = state["table"].long()
    at = torch.arange(most, device="cuda")
    rows = (off[:-1, None] + at[None]).clamp(max=state["rows"] - 1)                 # [seq][row], too many for the shorter ones
    real = at[None] < (off[1:] - off[:-1])[:, None]
    q = state["q"][rows].float().view(n, most, hkv, group, hd).permute(0, 2, 1, 3, 4).reshape(n, hkv, most * group, hd)
    s = torch.matmul(q, _values(state, "k", table).permute(0, 2, 4, 1, 3).reshape(n, hkv, hd, -1))
    s = s.mul_(1.0 / math.sqrt(hd)).view(n, hkv, most, group, -1)
    key = torch.arange(s.shape[-1], device="cuda")
    first = state["lengths"].long()[:, None, None]
    own_row = key[None, None] - first                                              # [seq][1][key]: row of the chunk
    if state["ancestors"] is not None:
        bits = state["ancestors"][rows][:, :, None] >> (own_row - 1).clamp(0, 63) & 1
        seen = (own_row <= 0) | ((bits == 1) & (own_row < (off[1:] - off[:-1])[:, None, None]))
    else:
        seen = own_row <= at[None, :, None]
    if case["window"]:
        seen = seen & (own_row > at[None, :, None] - case["window"])
    s.masked_fill_(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    vals = _values(state, "v", table).permute(0, 2, 1, 4, 3).reshape(n, hkv, -1, hd)
    out = torch.matmul(p.view(n, hkv, most * group, -1), vals).view(n, hkv, most, group, hd) / l
    out = out.permute(0, 2, 1, 3, 4).reshape(n, most, hq * hd)[real]
    state["out"][:state["rows"]] = out.to(state["q"].dtype)
    state["lse"][:state["rows"]] = (m + torch.log(l)).view(n, hkv, most, group).permute(0, 2, 1, 3).reshape(n, most, hq)[real]
    return state["out"], state["lse"]


# ---- the definitions in 64 bits --------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "read": _exact_read, "attend": _exact_attend}[case["op"]](case, s)


def _decoded(s, which):
    """All pages in 64 bits, positions before dimensions: [page][kv head][16][head_dim]."""
    p = s[which + "_pages"]
    if s["scales"] is None:
        x = p.double()
    else:
        b = p.view(torch.uint8).long()
        mant, exp = b % 8, b // 8 % 16
        x = torch.where(exp == 0, mant.double() / 512, (8 + mant.double()) * torch.exp2(exp.double() - 10))
        x = torch.where(b >= 128, -x, x)
    if which == "v":
        x = x.transpose(2, 3).contiguous()
    return x if s["scales"] is None else x * torch.exp2(s["scales"][which == "v"].double() - 127)[..., None]


def _rounded8(x):
    """[...][head_dim] in 64 bits -> what 8 bits and a scale hold of it"""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 448))
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
    e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e)
    scale = torch.exp2(torch.where(top > 0, e, -127.0).clamp(min=-127))
    y = x / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * scale


def _exact_append(case, s):
    hd, hq, hkv, rd = case["head_dim"], case["q_heads"], case["kv_heads"], case["rope_dim"]
    eight = s["scales"] is not None
    qo, kp, vp = s["q_out"].double(), _decoded(s, "k"), _decoded(s, "v")
    r, read = 0, []
    for i, (n, new) in enumerate(zip(lengths_of(case), rows_of(case))):
        pos = torch.arange(n, n + new, device="cuda")
        x = s["qkv"][r:r + new].double().view(new, hq + 2 * hkv, hd)
        qk = x[:, :hq + hkv].clone()
        if case["norm"]:
            qk /= torch.sqrt((qk * qk).sum(-1, keepdim=True) / hd + EPS)
            qk[:, :hq] *= s["gains"][0].double()
            qk[:, hq:] *= s["gains"][1].double()
        j = torch.arange(rd // 2, device="cuda").double()
        f = s["freqs"].double() if case["scaled"] else torch.exp(-2 * j / rd * math.log(case["theta"]))
        where = pos if s["positions"] is None else s["positions"][r:r + new]
        turn = torch.polar(torch.full((new, rd // 2), _magnitude(case), dtype=torch.float64, device="cuda"), where[:, None].double() * f)
        z = qk[..., :rd]
        z = z.reshape(new, hq + hkv, 2, rd // 2).transpose(2, 3) if case["rope"] == "half" else z.reshape(new, hq + hkv, rd // 2, 2)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None])
        qk[..., :rd] = z.transpose(2, 3).flatten(2) if case["rope"] == "half" else z.flatten(2)
        qo[r:r + new] = qk[:, :hq].reshape(new, -1)
        page, slot = s["table"][i].long()[pos // PAGE], pos % PAGE
        kp[page, :, slot] = qk[:, hq:]
        vp[page, :, slot] = x[:, hq + hkv:]
        read.append(_rounded8(x[:, hq + hkv:]).flatten(1))
        r += new
    if eight:       # a turned key next to a border of 8 bits falls to either side: none is the value
        return qo, None, torch.cat(read)
    return qo, kp, vp.transpose(2, 3).contiguous()


def _exact_read(case, s):
    k, v = _decoded(s, "k"), _decoded(s, "v")
    got = []
    for i, (a, n) in enumerate(zip(starts_of(case), rows_of(case))):
        pos = torch.arange(a, a + n, device="cuda")
        page, slot = s["table"][i].long()[pos // PAGE], pos % PAGE
        got.append((k[page, :, slot].flatten(1), v[page, :, slot].flatten(1)))
    return torch.cat([a for a, _ in got]), torch.cat([b for _, b in got])


def _exact_attend(case, s):
    hd, hq, hkv = case["head_dim"], case["q_heads"], case["kv_heads"]
    g = hq // hkv
    out, lse = s["out"].double(), s["lse"].double()
    keys, vals = _decoded(s, "k"), _decoded(s, "v")
    r = 0
    for i, (n, new) in enumerate(zip(lengths_of(case), rows_of(case))):
        full = n + new
        pages = s["table"][i, :-(-full // PAGE)].long()
        seen = torch.ones((new, full), dtype=torch.bool, device="cuda")
        if case["tree"]:
            sets = s["ancestors"][r:r + new].tolist()
            seen[:, n + 1:] = torch.tensor([[a >> (b - 1) & 1 for b in range(1, new)] for a in sets], device="cuda").reshape(new, -1).bool()
        else:
            seen = seen.tril(n)
        if case["window"]:
            seen = seen.triu(n + 1 - case["window"])
        for h in range(hkv):
            k = keys[pages, h].reshape(-1, hd)[:full].t().contiguous()
            v = vals[pages, h].reshape(-1, hd)[:full].contiguous()
            q = s["q"][r:r + new].double().view(new, hkv, g, hd)[:, h]
            for b in range(0, new, 1024):
                z = (q[b:b + 1024].reshape(-1, hd) @ k / math.sqrt(hd)).view(-1, g, full)
                z.masked_fill_(~seen[b:b + 1024, None], -math.inf)
                norm = torch.logsumexp(z, 2, keepdim=True)
                lse[r:r + new].view(new, hkv, g)[b:b + 1024, h] = norm[..., 0]
                out[r:r + new].view(new, hkv, g, hd)[b:b + 1024, h] = (torch.exp(z - norm).view(-1, full) @ v).view(-1, g, hd)
        r += new
    return out, lse
