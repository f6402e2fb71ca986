"""The paged K/V cache and the attention that reads it: what a stream of frames needs next to the global layer.

Frames arrive one after another; the keys and values of their (merged) tokens stay in pages, as bfloat16 or as E4M3
codes with one power of two per token and head, and the tokens of every new chunk attend to all that their sequence
holds.  The pool of a cache is [pages, kv_heads, page_size, head_dim]; a batch names, for each of its sequences, how
many rows belong to it, how many tokens it holds with those rows, and in which pages.  The kinds of pass:

  store   K and V of new tokens written into the cache (quantised where it holds codes), and read back
  load    whole sequences read back as bfloat16
  attend  the rows of a chunk over the cached keys of their sequence
  step    what a layer does with a new chunk: store its K and V, attend over everything

`causal_block` = c: row i of a sequence's chunk sees the tokens before the chunk and those of the chunk's blocks of c
rows up to its own (c = 1: itself and what came before it; c = tokens of a frame: its whole frame); 0: everything.
Widths and token counts are the framework's: 16 heads of 64 (the aggregator) or of 128 (the camera head's trunk), frames of
16 x 16, 28 x 37 and 37 x 37 patches with their 5 special tokens; shared K/V heads are the usual layouts.
"""
import math

import torch

own = False

LARGEST_FLOPS = 4.6e11  # of a drawn pass; the largest listed one has more
PLAIN_BYTES = 10 << 30  # what the scores of a drawn pass take in 32 bits, at most


def _case(op, n_seq, rows, keys, q_heads, kv_heads, head_dim, dtype, page_size=64, causal_block=0, ragged=False, name=None):
    c = dict(op=op, n_seq=n_seq, rows=rows, keys=keys, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype,
             page_size=page_size, causal_block=causal_block, ragged=ragged)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a small frame's K and V go into the cache: launches and latency
        _case("store", 1, 261, 522, 16, 16, 64, "e4m3", name="store_frame_16x16_e4m3"),
        # a long scene enters the cache at once: bandwidth
        _case("store", 1, 83280, 83280, 16, 16, 64, "e4m3", 128, name="store_scene_83280_e4m3"),
        # a few sequences handed to a layer that wants them whole
        _case("load", 3, 1374, 1374, 16, 16, 64, "bf16", 16, ragged=True, name="load_3x1374_bf16"),
        # many scenes read back from 8 bits
        _case("load", 24, 5205, 5205, 16, 16, 128, "e4m3", ragged=True, name="load_24x5205_hd128_e4m3"),
        # one camera token against one small frame: the smallest call
        _case("step", 1, 1, 262, 16, 16, 64, "bf16", name="token_over_262_bf16"),
        # the camera tokens of many scenes of different lengths, each with its own K/V heads
        _case("step", 48, 1, 4164, 16, 16, 128, "bf16", ragged=True, name="tokens_48_hd128_bf16"),
        # single tokens with shared K/V heads, 8-bit cache
        _case("attend", 16, 1, 8328, 32, 4, 128, "e4m3", ragged=True, name="tokens_16_shared8_e4m3"),
        # one token over all merged tokens of a thousand frames, 8-bit cache
        _case("attend", 1, 1, 520500, 16, 16, 64, "e4m3", 128, name="token_over_520500_e4m3"),
        # a new frame over the merged tokens of a hundred frames
        _case("step", 1, 1041, 52050, 16, 16, 64, "bf16", name="frame_over_52050_bf16"),
        # two square frames at once over an 8-bit cache, each frame blind to the later one
        _case("step", 1, 2748, 21984, 16, 16, 64, "e4m3", causal_block=1374, name="frames_over_21984_e4m3"),
        # chunks of several token-causal sequences, shared K/V heads of 128
        _case("attend", 5, 1741, 4099, 32, 8, 128, "bf16", 32, causal_block=1, ragged=True, name="chunks_5_hd128_causal"),
        # four frames at once over forty: the largest
        _case("attend", 1, 4164, 41640, 16, 16, 64, "bf16", 128, causal_block=1041, name="frames_over_41640_bf16"),
    ]


def _lengths(case):
    """Rows and lengths of the case's sequences, the first one's being the largest."""
    rows, keys = [], []
    for i in range(case["n_seq"]):
        less = (i * 0.381966) % 1.0 if case["ragged"] else 0.0
        n = case["keys"] - int(0.75 * less * case["keys"])
        r = case["rows"] if case["op"] != "load" else n
        r -= int(0.75 * ((i * 0.618034) % 1.0) * r) if case["ragged"] and case["op"] != "load" else 0
        keys.append(max(1, n))
        rows.append(max(1, min(r, n)))
    return rows, keys


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
        op = rng.choice(["store", "load", "attend", "attend", "step", "step", "step"])
        head_dim = rng.choice([64, 128])
        q_heads, kv_heads = rng.choice([(16, 16), (16, 16), (32, 8), (16, 2), (8, 1), (12, 4)])
        if op in ("store", "load"):
            n_seq, keys = between(1, 24), between(261, 83280)
            rows = between(261, keys)
        else:
            few = rng.random() < 0.5  # single tokens (and drafts of a few), or chunks
            n_seq = between(1, 48) if few else between(1, 6)
            rows = rng.choice([1, 1, 1, 2, 5]) if few else between(9, 4164)
            keys = between(max(rows, 262), 520500 if few else 52050)
        causal = rng.choice([0, 1, 1, 261]) if op in ("attend", "step") and rows > 1 else 0
        c = _case(op, n_seq, rows, keys, q_heads, kv_heads, head_dim, rng.choice(["bf16", "e4m3"]), rng.choice([16, 32, 64, 128]),
                  causal, rng.random() < 0.6)
        tokens = n_seq * keys * kv_heads * head_dim
        scores = 4 * n_seq * q_heads * rows * keys if op in ("attend", "step") else 0
        if tokens <= 83280 * 1024 * 6.5 and scores <= PLAIN_BYTES and work(c)["flops"] <= LARGEST_FLOPS:
            return c


def work(case):
    rows, keys = _lengths(case)
    h, d, qh = case["kv_heads"], case["head_dim"], case["q_heads"]
    held = 2 * h * (2 * d if case["dtype"] == "bf16" else d + 1)  # bytes of a token's K and V in the cache
    plain = 2 * h * 2 * d
    if case["op"] == "load":
        return {"bytes": sum(rows) * (held + plain), "flops": 0}
    if case["op"] == "store":
        return {"bytes": sum(rows) * (2 * plain + held), "flops": 0}
    n_bytes = sum(keys) * held + sum(rows) * 2 * qh * 2 * d
    if case["op"] == "step":  # the new tokens come from outside and go into the cache as well
        n_bytes += sum(rows) * plain
    return {"bytes": n_bytes, "flops": 4 * _pairs(case) * qh * d}


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    """The cache's pools (or their bfloat16 contents), the fused projection of the new rows, and the pages of each sequence."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, keys = _lengths(case)
    h, d, qh, ps = case["kv_heads"], case["head_dim"], case["q_heads"], case["page_size"]
    counts = [-(-n // ps) for n in keys]
    n_pages = sum(counts) + sum(counts) // 8 + 1  # some belong to nobody
    order = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    pages, at = [], 0
    for n in counts:
        pages.append(order[at:at + n])
        at += n
    lean = 2.0 * torch.randn(h, 1, d, generator=g, device="cuda")  # keys lean to one side, in some channels far
    k = torch.empty(n_pages, h, ps, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    k += lean.bfloat16()
    v = torch.empty(n_pages, h, ps, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    qkv = torch.empty(sum(rows), (qh + 2 * h) * d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    q, k_new, v_new = (t.unflatten(1, (-1, d)) for t in qkv.split([qh * d, h * d, h * d], 1))
    k_new += lean[:, 0].bfloat16()
    if case["dtype"] == "e4m3":
        k, k_scale = _quantise(k)
        v, v_scale = _quantise(v)
    else:
        k_scale = v_scale = None
    return dict(k=k, v=v, k_scale=k_scale, v_scale=v_scale, q=q, k_new=k_new, v_new=v_new, rows=rows, keys=keys, pages=pages)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2512_04939_b200 import KVCache

        s["cache"] = KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["batch"] = s["cache"].batch(s["rows"], s["keys"], s["pages"], q_heads=case["q_heads"], causal_block=case["causal_block"])
    else:
        s["plan"] = _plan(case, s["rows"], s["keys"], s["pages"])
    return s


def run(state):
    op = state["case"]["op"]
    if own:
        cache, batch = state["cache"], state["batch"]
        if op in ("store", "step"):
            cache.append(batch, state["k_new"], state["v_new"])
        if op in ("store", "load"):
            return cache.gather(batch)
        return cache.attend(batch, state["q"])
    if op in ("store", "step"):
        _plain_append(state)
    if op in ("store", "load"):
        return _plain_gather(state)
    return _plain_attend(state)


# ------------------------------------------------------------------ plain form
def _plan(case, rows, keys, pages):
    """Where the rows lie in the pools, and the padded layout that the plain attention works in."""
    ps, c = case["page_size"], case["causal_block"]
    most = max(len(p) for p in pages)
    table = torch.tensor([p + [p[-1]] * (most - len(p)) for p in pages], device="cuda")
    r, n = torch.tensor(rows, device="cuda"), torch.tensor(keys, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), r)
    within = torch.arange(sum(rows), device="cuda") - (torch.cumsum(r, 0) - r)[seq]
    place = (n - r)[seq] + within
    seen = n[seq] if c == 0 else torch.minimum((n - r)[seq] + (within // c + 1) * c, n[seq])
    return dict(table=table, page=table[seq, place // ps], offset=place % ps, seq=seq, within=within, seen=seen, length=n)


def _quantise(x):
    """E4M3 codes of the rows of x along its last dimension, under the least power of two 2^e >= 2^-118 with
    max|x| <= 448 * 2^e, and e + 127; 255 for a row that is not finite."""
    top = x.abs().amax(-1).float()
    bits = top.view(torch.int32)
    e = ((bits >> 23) + ((bits & 0x7FFFFF) > 0x600000) - 8).clamp_(min=9)
    e = torch.where(torch.isfinite(top), e, 255)
    back = ((254 - e.clamp(max=253)) << 23).view(torch.float32)
    codes = (x.float() * back.unsqueeze(-1)).to(torch.float8_e4m3fn)
    codes = torch.where((e == 255).unsqueeze(-1), torch.zeros_like(codes).view(torch.uint8), codes.view(torch.uint8))
    return codes.view(torch.float8_e4m3fn), e.to(torch.uint8)


def _values(codes, scale):
    """What pool rows stand for, in 32 bits."""
    if scale is None:
        return codes.float()
    e = scale.to(torch.int32)
    factor = torch.where(e == 255, torch.full((), float("nan"), device=e.device), (e << 23).view(torch.float32))
    return codes.float() * factor.unsqueeze(-1)


def _plain_append(s):
    at = (s["plan"]["page"], slice(None), s["plan"]["offset"])
    for name, new in (("k", s["k_new"]), ("v", s["v_new"])):
        if s["k_scale"] is None:
            s[name][at] = new
        else:
            codes, scale = _quantise(new)
            s[name].view(torch.uint8)[at] = codes.view(torch.uint8)
            s[name + "_scale"][at] = scale


def _plain_gather(s):
    at = (s["plan"]["page"], slice(None), s["plan"]["offset"])
    out = []
    for name in ("k", "v"):
        scale = s[name + "_scale"]
        rows = s[name][at] if scale is None else s[name].view(torch.uint8)[at].view(torch.float8_e4m3fn)
        out.append(_values(rows, None if scale is None else scale[at]).bfloat16())
    return tuple(out)


def _whole(s, name):
    """[n_seq, kv_heads, longest, head_dim] in 32 bits, zero beyond a sequence's end."""
    p, scale = s["plan"], s[name + "_scale"]
    if scale is None:
        x = _values(s[name][p["table"]], None)
    else:
        x = _values(s[name].view(torch.uint8)[p["table"]].view(torch.float8_e4m3fn), scale[p["table"]])
    x = x.permute(0, 2, 1, 3, 4).flatten(2, 3)
    return x * (torch.arange(x.shape[2], device=x.device) < p["length"][:, None])[:, None, :, None]


def _plain_attend(s):
    p, case = s["plan"], s["case"]
    h, d, qh = case["kv_heads"], case["head_dim"], case["q_heads"]
    k, v = _whole(s, "k"), _whole(s, "v")
    n_seq, most = k.shape[0], max(s["rows"])
    q = torch.zeros(n_seq, most, qh, d, device="cuda")
    q[p["seq"], p["within"]] = s["q"].float() / math.sqrt(d)
    seen = torch.zeros(n_seq, most, dtype=torch.int64, device="cuda")
    seen[p["seq"], p["within"]] = p["seen"]
    q = q.view(n_seq, most, h, qh // h, d).permute(0, 2, 3, 1, 4).flatten(2, 3)  # heads that share K and V under one another
    scores = q @ k.transpose(2, 3)
    del k, q
    hidden = torch.arange(v.shape[2], device="cuda") >= seen[:, :, None]
    scores.view(n_seq, h, qh // h, most, -1).masked_fill_(hidden[:, None, None], float("-inf"))
    scores -= scores.amax(-1, keepdim=True).clamp_(min=-3e38)
    scores.exp_()
    total = scores.sum(-1, keepdim=True)
    o = (scores @ v) / total.clamp_(min=1e-38)
    o = o.view(n_seq, h, qh // h, most, d).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return o[p["seq"], p["within"]].bfloat16()


# ------------------------------------------------------------------ in 64 bits
def _exact_rounded(x):
    """The values that a row's E4M3 codes stand for, from the definition, in 64 bits."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448)).clamp(min=-118)
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)  # where the logarithm was a hair too small, or too large
    e = torch.where((top <= 448 * torch.exp2(e - 1)) & (e > -118), e - 1, e)
    y = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def exact(case, seed):
    s = _inputs(case, seed)
    c, d, ps = case["causal_block"], case["head_dim"], case["page_size"]
    narrow = case["dtype"] == "e4m3"
    group = case["q_heads"] // case["kv_heads"]
    new = {n: (_exact_rounded(s[n]) if narrow else s[n].double()) for n in ("k_new", "v_new")}
    if case["op"] == "store":
        return new["k_new"], new["v_new"]
    out, row0 = [], 0
    for r, n, pages in zip(s["rows"], s["keys"], s["pages"]):
        held = []
        for name in ("k", "v"):
            ids = torch.tensor(pages, device="cuda")
            x = s[name].view(torch.uint8)[ids].view(s[name].dtype).double()
            if narrow:
                x = x * torch.exp2(s[name + "_scale"][ids].double() - 127).unsqueeze(-1)
            x = x.transpose(1, 2).reshape(-1, case["kv_heads"], d)[:n].clone()
            if case["op"] == "step":
                x[n - r:] = new[name + "_new"][row0:row0 + r]
            held.append(x)
        if case["op"] == "load":
            out.append(torch.stack([x[n - r:] for x in held]))
            row0 += r
            continue
        i = torch.arange(r, device="cuda")
        sees = torch.full_like(i, n) if c == 0 else torch.clamp(n - r + (i // c + 1) * c, max=n)
        hidden = torch.arange(n, device="cuda")[None] >= sees[:, None]
        heads = []
        for qh in range(case["q_heads"]):
            a = s["q"][row0:row0 + r, qh].double() @ held[0][:, qh // group].T * d ** -0.5
            a = torch.softmax(a.masked_fill_(hidden, -math.inf), 1)
            heads.append(a @ held[1][:, qh // group])
        out.append(torch.stack(heads, 1))
        row0 += r
    if case["op"] == "load":
        both = torch.cat(out, 1)
        return both[0], both[1]
    return torch.cat(out)
