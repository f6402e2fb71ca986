"""What a stream of frames that has no end needs beside its paged K/V cache: where a token stands in time and in its
frame, a cache of 4 bits an element, and which of the tokens held so far may go.

Queries and keys are turned by their position along several axes (time, height, width) before the keys go into the
cache, which may hold them as E2M1 codes with a power of two for every 32 channels; the attention that a cached token draws is
added up while chunks pass; and when the cache is full, every head keeps the tokens that drew most.  The kinds of pass:

  rotate  queries and keys of a fused projection, turned by their tokens' positions
  back    the gradients of turned queries and keys, turned back
  store   K and V of new tokens written into a cache of 4 bits, and read back
  attend  the rows of a chunk over the 4-bit keys and values of their sequence
  step    both: K and V of the chunk written first
  weigh   what every cached token of a sequence draws of the rows' attention, given each row's log-sum-exp
  evict   the tokens that drew most (and the first and last ones, whatever they drew), moved to other pages

An axis turns `sections[a]` channels of a head by position * bases[a]^(-i / planes).  Layouts: `halves` pairs channel i of an
axis with channel i + half of the axis's own section, `pairs` its neighbours; `across` pairs over all sections together, with one
ladder of frequencies whose planes are dealt to the axes in turn.  Widths and token counts are the framework's: 16 heads of 64 (the
aggregator) or of 128 (the camera head's trunk), frames of 16 x 16, 28 x 37 and 37 x 37 patches with their 5 special tokens;
shared K/V heads are the usual layouts.
"""
import math

import torch

own = False

LARGEST_FLOPS = 3.3e11  # of a drawn pass; the largest listed one has more
PLAIN_BYTES = 10 << 30  # what the scores of a drawn pass take in 32 bits, at most


def _rotary(op, rows, q_heads, kv_heads, head_dim, layout, sections, dtype="bf16", grid=(28, 37), first_frame=0, name=None):
    c = dict(op=op, rows=rows, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, layout=layout, time=sections[0], height=sections[1],
             width=sections[2], dtype=dtype, grid_h=grid[0], grid_w=grid[1], first_frame=first_frame)
    return c if name is None else dict(c, name=name)


def _over(op, n_seq, rows, keys, q_heads, kv_heads, head_dim, dtype, page_size=64, causal_block=0, ragged=False, name=None):
    c = dict(op=op, n_seq=n_seq, rows=rows, keys=keys, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype,
             page_size=page_size, causal_block=causal_block, ragged=ragged)
    return c if name is None else dict(c, name=name)


def _evict(n_seq, keys, keep, first, last, kv_heads, head_dim, dtype, page_size=64, ragged=False, name=None):
    c = dict(op="evict", n_seq=n_seq, keys=keys, keep=keep, first=first, last=last, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype,
             page_size=page_size, ragged=ragged)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one camera token of a late frame: the smallest call
        _rotary("rotate", 1, 16, 16, 64, "halves", (16, 24, 24), first_frame=90000, name="rotate_token"),
        # the merged tokens of a long scene: bandwidth
        _rotary("rotate", 83280, 16, 16, 64, "across", (16, 24, 24), name="rotate_scene_83280"),
        # gradients of a chunk of frames, shared K/V heads of 128, in 32 bits
        _rotary("back", 10992, 32, 8, 128, "pairs", (32, 48, 48), "fp32", (37, 37), name="back_chunk_hd128_fp32"),
        # a long scene enters the cache at once: bandwidth
        _over("store", 1, 83280, 83280, 16, 16, 64, "e2m1", 128, name="store_scene_83280_e2m1"),
        # one token over all merged tokens of a thousand frames
        _over("attend", 1, 1, 520500, 16, 16, 64, "e2m1", 128, name="token_over_520500_e2m1"),
        # chunks of several token-causal sequences, shared K/V heads of 128
        _over("step", 5, 1741, 4099, 32, 8, 128, "e2m1", 32, causal_block=1, ragged=True, name="chunks_5_hd128_e2m1"),
        # one camera token over a small frame and itself
        _over("weigh", 1, 1, 262, 16, 16, 64, "bf16", name="weigh_token_over_262"),
        # the camera tokens of sixteen scenes, shared K/V heads, 8-bit cache
        _over("weigh", 16, 1, 8328, 32, 4, 128, "e4m3", ragged=True, name="weigh_tokens_16_shared8_e4m3"),
        # four frames at once over forty, each frame blind to the later ones: the largest
        _over("weigh", 1, 4164, 41640, 16, 16, 64, "bf16", 128, causal_block=1041, name="weigh_frames_over_41640"),
        # a short stream halved
        _evict(1, 1044, 522, 5, 261, 16, 64, "bf16", name="evict_1044_to_522"),
        # many scenes of different lengths in 8 bits, read back for a layer that wants them whole
        _evict(24, 5205, 2082, 0, 261, 16, 128, "e4m3", ragged=True, name="evict_24x5205_hd128_e4m3"),
        # the merged tokens of a thousand frames: selection over a long axis
        _evict(1, 520500, 131072, 1041, 4164, 4, 64, "bf16", 128, name="evict_520500_to_131072"),
    ]


def _lengths(case):
    """Rows and lengths of the case's sequences, the first one's being the largest."""
    rows, keys = [], []
    for i in range(case["n_seq"]):
        less = (i * 0.381966) % 1.0 if case["ragged"] else 0.0
        n = max(1, case["keys"] - int(0.75 * less * case["keys"]))
        r = case.get("rows", 0)
        r -= int(0.75 * ((i * 0.618034) % 1.0) * r) if case["ragged"] else 0
        keys.append(n)
        rows.append(min(max(1, r), n))
    return rows, keys


def _kept(case):
    """How many tokens each sequence keeps."""
    return [min(n, max(case["first"] + case["last"], case["keep"] * n // case["keys"])) for n in _lengths(case)[1]]


def _pairs(case):
    """(row, key) pairs that see each other."""
    total = 0
    for r, n in zip(*_lengths(case)):
        c = case["causal_block"]
        total += r * n if c == 0 else r * (n - r) + sum(min(r - b, c) * min(r, b + c) for b in range(0, r, c))
    return total


def draw(rng):
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["rotate", "rotate", "back", "store", "attend", "step", "step", "weigh", "weigh", "weigh", "evict", "evict"])
        head_dim = rng.choice([64, 128])
        q_heads, kv_heads = rng.choice([(16, 16), (16, 16), (32, 8), (16, 2), (8, 1), (12, 4)])
        page_size, dtype, ragged = rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "e4m3", "e2m1"]), rng.random() < 0.6
        if op in ("rotate", "back"):
            rows = between(1, 83280)
            most = head_dim // 2  # planes
            t = rng.randint(1, most - 2)
            h = rng.randint(1, most - t - 1)
            w = rng.choice([most - t - h, rng.randint(1, most - t - h)])
            if rng.random() < 0.7:  # as models have them
                t, h, w = rng.choice([(8, 12, 12), (8, 8, 16), (16, 8, 8), (10, 11, 11)])
                t, h, w = (x * head_dim // 64 for x in (t, h, w))
            c = _rotary(op, rows, q_heads, kv_heads, head_dim, rng.choice(["halves", "pairs", "across"]), (2 * t, 2 * h, 2 * w),
                        rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.choice([(16, 16), (28, 37), (37, 37)]),
                        rng.choice([0, 0, between(1, 10 ** 6)]))
            if work(c)["bytes"] <= 6.8e8:
                return c
        elif op == "evict":
            n_seq, keys = between(1, 24), between(64, 520500)
            keep = max(16, int(keys * rng.uniform(0.05, 1.0)))
            first, last = rng.choice([0, 5, 8]), rng.choice([0, 0, keep // 4])
            c = _evict(n_seq, keys, keep, first, last, kv_heads, head_dim, dtype, page_size, ragged)
            if n_seq * keys * kv_heads * head_dim <= 83280 * 1024:
                return c
        else:
            few = rng.random() < 0.5  # single tokens (and drafts of a few), or chunks
            n_seq = between(1, 48) if few else between(1, 6)
            rows = rng.choice([1, 1, 1, 2, 5]) if few else between(9, 4164)
            if op == "store":
                n_seq, rows = between(1, 24), between(261, 83280)
            keys = between(max(rows, 262), 520500 if few else max(rows, 41640))
            causal = rng.choice([0, 1, 1, 261]) if rows > 1 and op != "store" else 0
            c = _over(op, n_seq, rows, keys, q_heads, kv_heads, head_dim, dtype if op == "weigh" else "e2m1", page_size, causal, ragged)
            scores = 0 if op == "store" else 4 * n_seq * q_heads * rows * keys
            if n_seq * keys * kv_heads * head_dim <= 83280 * 1024 * 6.5 and scores <= PLAIN_BYTES and work(c)["flops"] <= LARGEST_FLOPS:
                return c


def work(case):
    d = case["head_dim"]
    if case["op"] in ("rotate", "back"):
        size = 4 if case["dtype"] == "fp32" else 2
        n = case["rows"] * (case["q_heads"] + case["kv_heads"])
        turned = case["time"] + case["height"] + case["width"]
        return {"bytes": 2 * n * d * size + 12 * case["rows"], "flops": 3 * n * turned}
    rows, keys = _lengths(case)
    h = case["kv_heads"]
    held = {"bf16": 2 * d, "e4m3": d + 1, "e2m1": d // 2 + d // 32}[case["dtype"]]  # bytes of a token's K (or V) of a head
    if case["op"] == "store":
        return {"bytes": sum(rows) * 2 * h * (4 * d + held), "flops": 0}
    if case["op"] in ("attend", "step"):
        n_bytes = sum(keys) * 2 * h * held + sum(rows) * 4 * case["q_heads"] * d
        if case["op"] == "step":  # the new tokens come from outside and go into the cache as well
            n_bytes += sum(rows) * 4 * h * d
        return {"bytes": n_bytes, "flops": 4 * _pairs(case) * case["q_heads"] * d}
    if case["op"] == "weigh":
        qh = case["q_heads"]
        return {"bytes": sum(keys) * h * (held + 4) + sum(rows) * qh * (2 * d + 4), "flops": 2 * _pairs(case) * qh * d}
    kept = sum(_kept(case))
    n_bytes = 4 * h * sum(keys) + kept * h * (4 * held + 4 + 4)
    if case["dtype"] != "bf16":  # read back
        n_bytes += kept * h * 2 * (held + 2 * d)
    return {"bytes": n_bytes, "flops": 0}


# ------------------------------------------------------------------ inputs
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BASES = (10000.0, 100.0, 100.0)  # of time, height and width


def _sections(case):
    return (case["time"], case["height"], case["width"])


def _rotary_inputs(case, seed):
    """A fused projection's queries and keys (or gradients), and where their tokens stand: special tokens at the frame's time and
    at no place, patches from (1, 1) on; of many frames' tokens those that merging left over."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, d, qh, h = case["rows"], case["head_dim"], case["q_heads"], case["kv_heads"]
    qkv = torch.empty(rows, (qh + 2 * h) * d, dtype=_TYPES[case["dtype"]], device="cuda").normal_(generator=g)
    q, k, _ = (t.unflatten(1, (-1, d)) for t in qkv.split([qh * d, h * d, h * d], 1))
    patches = case["grid_h"] * case["grid_w"]
    skip = torch.randint(1, 4, (rows,), generator=g, device="cuda") if rows > patches + 5 else torch.ones(rows, dtype=torch.int64, device="cuda")
    token = torch.cumsum(skip, 0) - skip[0]
    frame, within = token // (patches + 5), token % (patches + 5) - 5
    place = torch.clamp(within, min=0)
    here = (within >= 0).long()
    positions = torch.stack([frame + case["first_frame"], (place // case["grid_w"] + 1) * here, (place % case["grid_w"] + 1) * here])
    return dict(q=q, k=k, positions=positions.int().contiguous())


def _pages(counts, g):
    """Pages of sequences that need so many, in no order; some belong to nobody."""
    n_pages = sum(counts) + sum(counts) // 8 + 1
    order = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    pages, at = [], 0
    for n in counts:
        pages.append(order[at:at + n])
        at += n
    return n_pages, pages


def _cache_inputs(case, seed):
    """The cache's pools, the pages of each sequence, and what has been added up so far."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, keys = _lengths(case)
    h, d, ps = case["kv_heads"], case["head_dim"], case["page_size"]
    n_pages, pages = _pages([-(-n // ps) for n in keys], g)
    into = []
    if case["op"] == "evict":  # the pages that the kept tokens go to lie behind all others
        for m in _kept(case):
            into.append(list(range(n_pages, n_pages - (-m // ps))))
            n_pages += -(-m // ps)
    lean = 2.0 * torch.randn(h, 1, d, generator=g, device="cuda")  # keys lean to one side, in some channels far
    k = torch.empty(n_pages, h, ps, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    k += lean.bfloat16()
    # few tokens draw much, most draw little, and some have come too late to draw anything
    weights = torch.empty(n_pages, h, ps, device="cuda").normal_(generator=g).mul_(2.0).exp_()
    weights *= torch.rand(n_pages, h, ps, generator=g, device="cuda") > 0.1
    s = dict(case=case, rows=rows, keys=keys, pages=pages, into=into, k=k, v=None, k_scale=None, v_scale=None, weights=weights)
    if case["op"] != "weigh":  # (which looks at no values)
        s["v"] = torch.empty(n_pages, h, ps, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    if case["dtype"] != "bf16":
        s["k"], s["k_scale"] = _quantise(s["k"], case["dtype"])
        if s["v"] is not None:
            s["v"], s["v_scale"] = _quantise(s["v"], case["dtype"])
    if case["op"] == "evict":
        s["kept"] = _kept(case)
        return s
    qh = case["q_heads"]
    qkv = torch.empty(sum(rows), (qh + 2 * h) * d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    s["q"], s["k_new"], s["v_new"] = (t.unflatten(1, (-1, d)) for t in qkv.split([qh * d, h * d, h * d], 1))
    s["k_new"] += lean[:, 0].bfloat16()
    if case["op"] == "weigh":
        weights *= max(rows) * qh / (8.0 * h * max(keys))  # of the size of what the rows give out
        s["plan"] = _plan(case, rows, keys, pages)
        scores, _ = _scores(s)
        lse = torch.logsumexp(scores, -1).view(len(rows), h, qh // h, -1)  # an attention pass has left this
        del scores
        lse = lse.permute(0, 3, 1, 2).flatten(2, 3)
        s["lse"] = lse[s["plan"]["seq"], s["plan"]["within"]].contiguous()
    return s


def prepare(case, seed):
    if case["op"] in ("rotate", "back"):
        s = dict(_rotary_inputs(case, seed), case=case)
        if own:
            from paper_2512_04939_b200 import RotaryAxes

            s["rotary"] = RotaryAxes(case["head_dim"], _sections(case), BASES, case["layout"])
        else:
            first, second, axis, power = _planes(case)
            s["first"], s["second"], s["axis"] = (torch.tensor(x, device="cuda") for x in (first, second, axis))
            s["power"] = torch.tensor(power, dtype=torch.float64, device="cuda")
        return s
    s = _cache_inputs(case, seed)
    if own:
        from paper_2512_04939_b200 import KVCache

        v, v_scale = (s["k"], s["k_scale"]) if s["v"] is None else (s["v"], s["v_scale"])
        s["cache"] = KVCache(s["k"], v, s["k_scale"], v_scale, weights=s["weights"] if case["op"] in ("weigh", "evict") else None)
        if case["op"] != "evict":
            s["batch"] = s["cache"].batch(s["rows"], s["keys"], s["pages"], q_heads=case["q_heads"], causal_block=case["causal_block"])
        else:
            s["batch"] = s["cache"].batch([0] * case["n_seq"], s["keys"], s["pages"])
            s["target"] = s["cache"].batch(s["kept"], s["kept"], s["into"])
    elif case["op"] != "evict":
        s["plan"] = _plan(case, s["rows"], s["keys"], s["pages"])
    else:
        s["from"], s["to"] = _plan(case, [0] * len(s["keys"]), s["keys"], s["pages"]), _plan(case, s["kept"], s["kept"], s["into"])
    return s


def run(state):
    case = state["case"]
    if case["op"] in ("rotate", "back"):
        if not own:
            return _plain_rotate(state)
        turn = state["rotary"].rotate if case["op"] == "rotate" else state["rotary"].rotate_back
        return turn(state["positions"], state["q"], state["k"])
    if case["op"] == "weigh":
        if own:  # a tally that begins with these rows
            state["cache"].weigh(state["batch"], state["q"], state["lse"], decay=0.0)
        else:
            _plain_weigh(state)
        return state["weights"]
    if case["op"] != "evict":
        if case["op"] in ("store", "step"):
            if own:
                state["cache"].append(state["batch"], state["k_new"], state["v_new"])
            else:
                _plain_append(state)
        if case["op"] == "store":
            return state["cache"].gather(state["batch"]) if own else _plain_gather(state, state["plan"])
        return state["cache"].attend(state["batch"], state["q"]) if own else _plain_attend(state)
    if own:
        kept = state["cache"].evict(state["batch"], state["target"], first=case["first"], last=case["last"])
    else:
        kept = _plain_evict(state)
    first = state["into"][0][0]
    if case["dtype"] == "bf16":
        return kept, state["weights"][first:], state["k"][first:], state["v"][first:]
    k, v = state["cache"].gather(state["target"]) if own else _plain_gather(state, state["to"])
    return kept, state["weights"][first:], k, v


# ------------------------------------------------------------------ plain form
def _planes(case):
    """First and second channel of every plane, its axis, and what the axis's base is raised to."""
    first, second, axis, power, at = [], [], [], [], 0
    planes = [n // 2 for n in _sections(case)]
    for a, n in enumerate(planes):
        for i in range(n):
            if case["layout"] == "halves":
                first.append(at + i), second.append(at + n + i), power.append(-i / n)
            elif case["layout"] == "pairs":
                first.append(at + 2 * i), second.append(at + 2 * i + 1), power.append(-i / n)
            else:
                j = sum(planes[:a]) + i
                first.append(j), second.append(sum(planes) + j), power.append(-j / sum(planes))
            axis.append(a)
        at += 2 * n
    return first, second, axis, power


def _plain_rotate(s):
    back = s["case"]["op"] == "back"
    base = torch.tensor(BASES, dtype=torch.float64, device="cuda")[s["axis"]]
    angle = s["positions"][s["axis"]].T.double() * base ** s["power"]  # in 64 bits: positions may be far
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if back:
        sin = -sin
    out = []
    for x in (s["q"], s["k"]):
        y = x.float()
        a, b = y[..., s["first"]], y[..., s["second"]]
        y = y.clone()
        y[..., s["first"]] = a * cos - b * sin
        y[..., s["second"]] = a * sin + b * cos
        out.append(y.to(x.dtype))
    return tuple(out)


def _plan(case, rows, keys, pages):
    """Where tokens lie in the pools, and the padded layout that the plain forms work in."""
    ps, c = case["page_size"], case.get("causal_block", 0)
    most = max(len(p) for p in pages)
    table = torch.tensor([p + [p[-1]] * (most - len(p)) for p in pages], device="cuda")
    r, n = torch.tensor(rows, device="cuda"), torch.tensor(keys, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), r)
    within = torch.arange(sum(rows), device="cuda") - (torch.cumsum(r, 0) - r)[seq]
    place = (n - r)[seq] + within
    seen = n[seq] if c == 0 else torch.minimum((n - r)[seq] + (within // c + 1) * c, n[seq])
    # of all tokens: sequence, number, page and place in it
    all_seq = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), n)
    token = torch.arange(sum(keys), device="cuda") - (torch.cumsum(n, 0) - n)[all_seq]
    return dict(table=table, page=table[seq, place // ps], offset=place % ps, seq=seq, within=within, seen=seen, length=n,
                all_seq=all_seq, token=token, token_page=table[all_seq, token // ps], token_offset=token % ps)


_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # of E2M1


def _quantise(x, dtype):
    """Codes of x along its last dimension, and e + 127 of the powers of two 2^e that they are under (255: something in there is not
    finite, and the codes are 0).  E4M3: one for a row, the least e >= -118 with max|x| <= 448 * 2^e.  E2M1: one for every 32, the
    least e >= -126 with max|x| <= 6 * 2^e; the code of an even element is the low half of its byte."""
    y = x if dtype == "e4m3" else x.unflatten(-1, (-1, 32))
    top = y.abs().amax(-1).float()
    bits = top.view(torch.int32)
    if dtype == "e4m3":
        e = ((bits >> 23) + ((bits & 0x7FFFFF) > 0x600000) - 8).clamp_(min=9)
    else:
        e = ((bits >> 23) + ((bits & 0x7FFFFF) > 0x400000) - 2).clamp_(min=1)
    e = torch.where(torch.isfinite(top), e, 255)
    y = y.float() * ((254 - e.clamp(max=253)) << 23).view(torch.float32).unsqueeze(-1)
    y = torch.where((e == 255).unsqueeze(-1), 0.0, y)
    if dtype == "e4m3":
        return y.to(torch.float8_e4m3fn), e.to(torch.uint8)
    code = torch.signbit(y).to(torch.uint8) * 8
    y = y.abs().clamp(max=6.0)
    for i in range(7):  # to the nearest, from the middle to the even code
        middle = (_LEVELS[i] + _LEVELS[i + 1]) / 2
        code += (y > middle if i % 2 == 0 else y >= middle).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, e.to(torch.uint8)


def _values(codes, scale):
    """What pool rows stand for, in 32 bits."""
    if scale is None:
        return codes.float()
    e = scale.to(torch.int32)
    factor = torch.where(e == 255, float("nan"), (e << 23).view(torch.float32)).unsqueeze(-1)
    if scale.dim() < codes.dim():
        return codes.float() * factor
    levels = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device=codes.device)
    x = torch.stack([levels[(codes & 15).long()], levels[(codes >> 4).long()]], -1).flatten(-2)
    return (x.unflatten(-1, (-1, 32)) * factor).flatten(-2)


def _bytes_at(x, at):
    """Indexing, for types that it does not know."""
    return x[at] if x.dtype != torch.float8_e4m3fn else x.view(torch.uint8)[at].view(torch.float8_e4m3fn)


def _whole(s, name):
    """[n_seq, kv_heads, longest, head_dim] in 32 bits, zero beyond a sequence's end."""
    p, scale = s["plan"], s[name + "_scale"]
    x = _values(_bytes_at(s[name], p["table"]), None if scale is None else scale[p["table"]])
    x = x.permute(0, 2, 1, 3, 4).flatten(2, 3)
    return x * (torch.arange(x.shape[2], device="cuda") < p["length"][:, None])[:, None, :, None]


def _scores(s):
    """Scores [n_seq, kv_heads, rows of heads that share K, keys] in 32 bits, minus infinity where a row does not see a key; and
    the rows' numbers of keys seen."""
    p, case = s["plan"], s["case"]
    h, d, qh = case["kv_heads"], case["head_dim"], case["q_heads"]
    k = _whole(s, "k")
    n_seq, most = k.shape[0], max(s["rows"])
    q = torch.zeros(n_seq, most, qh, d, device="cuda")
    q[p["seq"], p["within"]] = s["q"].float() / math.sqrt(d)
    seen = torch.zeros(n_seq, most, dtype=torch.int64, device="cuda")
    seen[p["seq"], p["within"]] = p["seen"]
    q = q.view(n_seq, most, h, qh // h, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
    scores = q @ k.transpose(2, 3)
    hidden = torch.arange(k.shape[2], device="cuda") >= seen[:, :, None]
    scores.view(n_seq, h, qh // h, most, -1).masked_fill_(hidden[:, None, None], float("-inf"))
    return scores, seen


def _plain_append(s):
    at = (s["plan"]["page"], slice(None), s["plan"]["offset"])
    for name in ("k", "v"):
        s[name][at], s[name + "_scale"][at] = _quantise(s[name + "_new"], "e2m1")


def _plain_attend(s):
    p, case = s["plan"], s["case"]
    h, qh = case["kv_heads"], case["q_heads"]
    scores, seen = _scores(s)
    scores -= scores.amax(-1, keepdim=True).clamp_(min=-3e38)
    scores.exp_()
    total = scores.sum(-1, keepdim=True)
    o = (scores @ _whole(s, "v")) / total.clamp_(min=1e-38)
    o = o.view(seen.shape[0], h, qh // h, seen.shape[1], -1).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return o[p["seq"], p["within"]].bfloat16()


def _plain_weigh(s):
    p, case = s["plan"], s["case"]
    h, qh = case["kv_heads"], case["q_heads"]
    scores, seen = _scores(s)
    lse = torch.zeros(seen.shape[0], seen.shape[1], qh, device="cuda")
    lse[p["seq"], p["within"]] = s["lse"]
    scores -= lse.view(*seen.shape, h, qh // h).permute(0, 2, 3, 1).flatten(2, 3).unsqueeze(-1)
    total = scores.exp_().sum(2)  # [n_seq, kv_heads, keys]
    s["weights"][p["token_page"], :, p["token_offset"]] = total[p["all_seq"], :, p["token"]]


def _plain_evict(s):
    a, b, case = s["from"], s["to"], s["case"]
    h = case["kv_heads"]
    w = s["weights"][a["table"]].permute(0, 2, 1, 3).flatten(2, 3)  # [n_seq, kv_heads, keys]
    number = torch.arange(w.shape[2], device="cuda")
    n = a["length"][:, None, None]
    w = torch.where((number < case["first"]) | (number >= n - case["last"]), float("inf"), w.nan_to_num(nan=-math.inf))
    w = torch.where(number < n, w, -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True)[1]  # of equal ones the earlier
    kept = torch.where(number < b["length"][:, None, None], order, w.shape[2]).sort(-1)[0]  # [n_seq, kv_heads, kept ones first]
    chosen = kept[b["seq"], :, b["within"]]  # [tokens kept, kv_heads]
    page = a["table"][b["seq"][:, None], chosen // case["page_size"]]
    heads = torch.arange(h, device="cuda")
    source, target = (page, heads, chosen % case["page_size"]), (b["page"][:, None], heads, b["offset"][:, None])
    for x in (s["k"], s["v"], s["k_scale"], s["v_scale"], s["weights"]):
        if x is not None:
            x = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
            x[target] = x[source]
    return chosen.int()


def _plain_gather(s, plan):
    at = (plan["page"], slice(None), plan["offset"])
    return tuple(_values(_bytes_at(s[n], at), s[n + "_scale"][at]).bfloat16() for n in ("k", "v"))


# ------------------------------------------------------------------ in 64 bits
def _exact_e2m1(x):
    """What the E2M1 codes of x stand for, from the definition, in 64 bits."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 6)).clamp(min=-126)
    e = torch.where(top > 6 * torch.exp2(e), e + 1, e)  # where the logarithm was a hair too small, or too large
    e = torch.where((top <= 6 * torch.exp2(e - 1)) & (e > -126), e - 1, e)
    y = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)
    return (torch.round(y / step) * step * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    d = case["head_dim"]
    if case["op"] in ("rotate", "back"):
        s = _rotary_inputs(case, seed)
        out = [x.double().clone() for x in (s["q"], s["k"])]
        sections = _sections(case)
        at = ladder = 0
        for a, n in enumerate(sections):
            for i in range(n // 2):
                if case["layout"] == "across":
                    one, two, share = ladder + i, sum(sections) // 2 + ladder + i, (ladder + i) / (sum(sections) // 2)
                else:
                    one, two = (at + i, at + i + n // 2) if case["layout"] == "halves" else (at + 2 * i, at + 2 * i + 1)
                    share = i / (n // 2)
                angle = s["positions"][a].double()[:, None] * math.exp(-share * math.log(BASES[a]))
                turn = torch.polar(torch.ones_like(angle), angle if case["op"] == "rotate" else -angle)
                for y in out:
                    z = torch.complex(y[..., one], y[..., two]) * turn
                    y[..., one], y[..., two] = z.real, z.imag
            at += n
            ladder += n // 2
        return tuple(out)
    s = _cache_inputs(case, seed)
    ps, h = case["page_size"], case["kv_heads"]

    def held(name, ids):
        """Tokens of pages, [tokens, kv_heads, head_dim]."""
        x = s[name].view(torch.uint8)[ids].view(s[name].dtype)
        if case["dtype"] == "e2m1":
            x = torch.stack([x % 16, x // 16], -1).flatten(-2).long()
            sign, power, half = x // 8, x // 2 % 4, x % 2
            size = torch.where(power == 0, 0.5 * half, (1 + 0.5 * half) * torch.exp2(power.double() - 1))
            x = (1 - 2 * sign) * size * torch.exp2(s[name + "_scale"][ids].double() - 127).repeat_interleave(32, -1)
        elif case["dtype"] == "e4m3":
            x = x.double() * torch.exp2(s[name + "_scale"][ids].double() - 127).unsqueeze(-1)
        return x.double().transpose(1, 2).reshape(-1, h, d)

    if case["op"] in ("store", "attend", "step"):
        new = [_exact_e2m1(s[n]) for n in ("k_new", "v_new")]
        if case["op"] == "store":
            return tuple(new)
        c, group, row0, out = case["causal_block"], case["q_heads"] // h, 0, []
        for r, n, pages in zip(s["rows"], s["keys"], s["pages"]):
            ids = torch.tensor(pages, device="cuda")
            k, v = held("k", ids)[:n], held("v", ids)[:n]
            if case["op"] == "step":
                k[n - r:], v[n - r:] = (x[row0:row0 + r] for x in new)
            i = torch.arange(r, device="cuda")
            sees = torch.full_like(i, n) if c == 0 else torch.clamp(n - r + (i // c + 1) * c, max=n)
            hidden = torch.arange(n, device="cuda")[None] >= sees[:, None]
            heads = []
            for qh in range(case["q_heads"]):
                x = s["q"][row0:row0 + r, qh].double() @ k[:, qh // group].T * d ** -0.5
                heads.append(torch.softmax(x.masked_fill_(hidden, -math.inf), 1) @ v[:, qh // group])
            out.append(torch.stack(heads, 1))
            row0 += r
        return torch.cat(out)
    weights = s["weights"].double()
    if case["op"] == "weigh":
        c, group, row0 = case["causal_block"], case["q_heads"] // h, 0
        for r, n, pages in zip(s["rows"], s["keys"], s["pages"]):
            ids = torch.tensor(pages, device="cuda")
            k = held("k", ids)[:n]
            i = torch.arange(r, device="cuda")
            sees = torch.full_like(i, n) if c == 0 else torch.clamp(n - r + (i // c + 1) * c, max=n)
            hidden = torch.arange(n, device="cuda")[None] >= sees[:, None]
            drawn = torch.zeros(h, len(pages) * ps, dtype=torch.float64, device="cuda")
            for qh in range(case["q_heads"]):
                x = s["q"][row0:row0 + r, qh].double() @ k[:, qh // group].T * d ** -0.5 - s["lse"][row0:row0 + r, qh].double()[:, None]
                drawn[qh // group, :n] += torch.exp(x).masked_fill_(hidden, 0.0).sum(0)
            before = weights[ids].transpose(0, 1).reshape(h, -1)
            drawn[:, n:] = before[:, n:]
            weights[ids] = drawn.view(h, -1, ps).transpose(0, 1)
            row0 += r
        return weights
    lists, start = [], s["into"][0][0]
    bf16 = case["dtype"] == "bf16"
    moved = {name: (s[name].double() if bf16 else []) for name in ("k", "v")}
    for n, m, pages, into in zip(s["keys"], s["kept"], s["pages"], s["into"]):
        ids, to = torch.tensor(pages, device="cuda"), torch.tensor(into, device="cuda")
        w = weights[ids].transpose(0, 1).reshape(h, -1)[:, :n]
        mine = [torch.arange(n, device="cuda")] * h if m == n else []
        for head in range(h if m < n else 0):
            # the m-th largest of those that may go, and as many of its equals as there is room for, the earlier first
            free = w[head, case["first"]:n - case["last"]]
            room = m - case["first"] - case["last"]
            if room == 0:
                chosen = torch.arange(0, device="cuda")
            else:
                least = torch.kthvalue(free, len(free) - room + 1)[0]
                over = free > least
                equal = (free == least).nonzero()[:room - int(over.sum()), 0]
                chosen = torch.cat([over.nonzero()[:, 0], equal]).sort()[0]
            mine.append(torch.cat([torch.arange(case["first"], device="cuda"), chosen + case["first"],
                                   torch.arange(n - case["last"], n, device="cuda")]))
        index = torch.stack(mine, 1)
        lists.append(index)
        slot = torch.arange(m, device="cuda")
        heads = torch.arange(h, device="cuda")
        weights[to[slot // ps][:, None], heads, (slot % ps)[:, None]] = w.T.gather(0, index)
        for name in ("k", "v"):
            x = held(name, ids).gather(0, index.unsqueeze(-1).expand(-1, -1, d))
            if bf16:
                moved[name][to[slot // ps][:, None], heads, (slot % ps)[:, None]] = x
            else:
                moved[name].append(x)
    k, v = (moved[n][start:] if bf16 else torch.cat(moved[n]) for n in ("k", "v"))
    return torch.cat(lists).int(), weights[start:], k, v
