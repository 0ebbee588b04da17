"""Measured cases of what stands around the attention of the live cache: rows that get their rotary positions on their way
into the cache (rotary_append), the attention weight that each cached token has received (attention_mass), the tokens that
stay when a cache is cut down by it (evict_select), and their rows' way into other pages (cache_gather).

A quantised page is one checkpoint record of `page` tokens: [K codes][K scales][V codes][V scales], codes
[token][head][channel], fp16 scales per `group` channels.  `tag` is the framework's precision tag: 0 = bf16 pool,
1 = K8/V8, 2 = K8/V4, 3 = K4/V4.  Row i of a sequence with `rows` rows and `kv` cached tokens stands at position
kv - rows + i."""
import math

import numpy
import torch

own = False

K_BITS, V_BITS = {0: 16, 1: 8, 2: 8, 3: 4}, {0: 16, 1: 8, 2: 4, 3: 4}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
BASE = 500000.0


def _case(op, tag, heads, q_heads, dim, seqs, kv, rows=1, **more):
    c = {"op": op, "tag": tag, "heads": heads, "q_heads": q_heads, "dim": dim, "group": 32, "page": 16, "seqs": seqs, "kv": kv,
         "rows": rows, "ragged": 0, "type": "bf16",
         "rotary": dim, "interleaved": False, "stretch": 1.0, "factor": 1.0, "far": 0,  # rotary positions
         "window": 0, "sinks": 0, "decay": 1.0,                                         # attention weight
         "keep": 0, "recent": 0, "ties": False}                                         # eviction
    c.update(more)
    return c


def listed():
    return [
        # one decode step's queries and keys of eight requests into the pool that a restore has filled: latency
        _case("rope", 0, 8, 32, 128, 8, 1000, 1, name="rope_step"),
        # a 16k prompt with frequencies scaled for long contexts into 4-bit pages
        _case("rope", 3, 8, 32, 128, 1, 16384, 16384, stretch=8.0, name="rope_prompt"),
        # ragged chunks, half of each head rotated in interleaved pairs, at the far positions of a cache that was cut down before
        _case("rope", 1, 4, 28, 128, 4, 4096, 2000, ragged=777, type="fp16", rotary=64, interleaved=True, factor=1.2, far=100000, name="rope_chunks"),
        # one short request, one token: latency
        _case("mass", 3, 4, 8, 64, 1, 1000, 1, name="mass_step"),
        # a decode step of eight 64k requests of the 70B-shaped geometry
        _case("mass", 3, 8, 64, 128, 8, 65536, 1, decay=0.95, name="mass_decode"),
        # the last 32 rows of a 32k prompt over the pool: what decides which of it stays
        _case("mass", 0, 8, 32, 128, 1, 32768, 32, name="mass_observe"),
        # every row of a prompt over its own quantised cache
        _case("mass", 2, 8, 32, 128, 1, 8192, 8192, decay=0.0, name="mass_prompt"),
        # ragged chunks under a window with sinks, seven query heads for each KV head
        _case("mass", 1, 4, 28, 128, 4, 4096, 2000, ragged=777, window=1024, sinks=4, type="fp16", name="mass_window"),
        # many requests cut down to a quarter after a step
        _case("select", 0, 8, 8, 128, 32, 4096, ragged=2011, keep=1024, recent=64, sinks=4, ties=True, name="select_batch"),
        # eight 128k contexts
        _case("select", 0, 8, 8, 128, 8, 131072, ragged=9973, keep=32768, recent=1024, sinks=4, name="select_long"),
        # a 32k context of 4-bit pages down to 8k
        _case("gather", 3, 8, 8, 128, 1, 32768, keep=8192, recent=64, sinks=4, name="gather_codes"),
        # four 16k contexts of the pool down to half, keys rotated to where they go
        _case("gather", 0, 8, 8, 128, 4, 16384, keep=8192, ragged=5003, recent=256, sinks=4, far=1, name="gather_rotate"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    heads, q_heads, dim = rng.choice([(4, 8, 64), (8, 32, 128), (4, 28, 128), (8, 64, 128), (2, 16, 128), (1, 8, 64), (32, 32, 128)])
    op = rng.choice(["rope", "mass", "mass", "select", "gather"])
    tag = rng.choice([0, 1, 2, 3])
    more = {"type": "bf16" if tag == 0 else rng.choice(["bf16", "fp16"]), "page": rng.choice([16, 16, 32, 64]), "group": rng.choice([32, 32, 64])}
    if op == "rope":
        seqs = _log(rng, 1, 32)
        rows = _log(rng, 1, 16384 // seqs)
        more.update(rotary=rng.choice([dim, dim, dim // 2]), interleaved=rng.random() < 0.4, stretch=rng.choice([1.0, 4.0, 8.0]),
                    factor=rng.choice([1.0, 1.0, 1.1]), far=rng.choice([0, 0, _log(rng, 10, 500000)]), ragged=rng.randrange(rows))
        return _case(op, tag, heads, min(q_heads, 32), dim, seqs, rows + rng.randrange(2000), rows, **more)
    if op == "select" or op == "gather":
        seqs = _log(rng, 1, 32)
        kv = _log(rng, 100, (1048576 if op == "select" else 65536) // max(seqs, 8 if op == "select" else 1))
        more.update(keep=rng.randrange(kv // 10 + 1, kv), sinks=rng.choice([0, 4, 17]), recent=rng.randrange(kv // 4 + 1), ragged=rng.randrange(kv // 2),
                    ties=rng.random() < 0.4, far=int(op == "gather" and tag == 0 and rng.random() < 0.6), interleaved=rng.random() < 0.4,
                    rotary=rng.choice([dim, dim, dim // 2]))
        return _case(op, tag, heads, heads, dim, seqs, kv, **more)
    more.update(decay=rng.choice([0.0, 0.95, 1.0, 1.0]))
    if rng.random() < 0.3:
        more.update(window=_log(rng, 100, 5000), sinks=rng.choice([0, 4, 17]))
    kind = rng.choice(["decode", "decode", "few", "prompt"])
    if kind == "decode":
        seqs = _log(rng, 1, 32)
        kv = _log(rng, 50, 131072 // seqs)
        return _case(op, tag, heads, q_heads, dim, seqs, kv, 1, ragged=rng.randrange(kv // 2), **more)
    if kind == "few":
        seqs = _log(rng, 1, 8)
        kv = _log(rng, 100, 65536 // seqs)
        return _case(op, tag, heads, min(q_heads, 32), dim, seqs, kv, rng.randrange(2, 64), ragged=rng.randrange(20), **more)
    seqs = rng.choice([1, 1, 2, 4])
    kv = _log(rng, 200, 8192 // seqs)
    rows = rng.choice([kv, rng.randrange(kv // 2, kv)])
    return _case(op, tag, heads, min(q_heads, 32), dim, seqs, kv, rows, ragged=rng.randrange(rows // 2), **more)


def _lengths(case):
    """Per sequence: cached tokens and rows.  With `ragged`, later sequences are shorter by up to that much, each by another
    amount; rows stay at one at least and never exceed the tokens."""
    cut = [(b * 7919 * 13) % (case["ragged"] + 1) for b in range(case["seqs"])]
    if case["rows"] == 1:
        return [case["kv"] - c for c in cut], [1] * case["seqs"]
    kv = [case["kv"] - (c if case["kv"] == case["rows"] else c // 3) for c in cut]
    return kv, [max(1, min(case["rows"] - c, t)) for c, t in zip(cut, kv)]


def _kept(case):
    return [min(case["keep"], t) for t in _lengths(case)[0]]


def _row_bytes(case, bits):
    e = case["dim"]
    return case["heads"] * (e * bits // 8 + (0 if bits == 16 else 2 * (e // case["group"])))


def _seen(case, kv, rows):
    """(tokens that some row sees, pairs of row and visible token) of one sequence."""
    w, s = case["window"], case["sinks"]
    pairs, seen, upto = 0, 0, 0
    for p in range(kv - rows, kv):
        low = max(0, p + 1 - w) if w else 0
        low = max(low, min(s, p + 1))
        pairs += p + 1 - low + min(s, p + 1)
        seen += max(0, p + 1 - max(low, upto))
        upto = max(upto, p + 1)
    return min(kv, seen + min(s, kv)), pairs


def work(case):
    kv, rows = _lengths(case)
    n, h, e = sum(rows), case["heads"], case["dim"]
    k, v = _row_bytes(case, K_BITS[case["tag"]]), _row_bytes(case, V_BITS[case["tag"]])
    if case["op"] == "rope":  # rows in; queries and cache rows out (quantised: and what they stand for)
        back = 0 if case["tag"] == 0 else k + v + 4 * h * e
        return {"bytes": n * (4 * case["q_heads"] * e + 4 * h * e + k + v + back), "flops": 3 * n * (case["q_heads"] + h) * case["rotary"]}
    if case["op"] == "mass":
        seen, pairs = (sum(x) for x in zip(*(_seen(case, t, r) for t, r in zip(kv, rows))))
        return {"bytes": seen * k + 2 * n * case["q_heads"] * e + 8 * sum(kv), "flops": 2 * pairs * case["q_heads"] * e}
    kept = sum(_kept(case))
    if case["op"] == "select":
        return {"bytes": 4 * sum(kv) + 8 * kept, "flops": sum(kv)}
    return {"bytes": kept * (2 * (k + v) + 4), "flops": 3 * kept * h * case["rotary"] * case["far"]}


def _values(shape, gen, dev, dtype, outliers):
    x = torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)
    if outliers:  # a few key channels are ten times the others, as in trained models
        x[..., torch.randperm(shape[-1], generator=gen, device=dev)[: shape[-1] // 20]] *= 10.0
    return x.to(dtype)


def _sections(case):
    """Byte sizes of a page's four sections."""
    e = case["page"] * case["heads"] * case["dim"]
    s = 2 * e // case["group"]
    return [e * K_BITS[case["tag"]] // 8, s, e * V_BITS[case["tag"]] // 8, s]


def _inv_freq(case):
    """fp32 frequencies of the rotary pairs; with `stretch` the slow ones that much slower, the fast ones as they were, a ramp between."""
    f = BASE ** (-torch.arange(0, case["rotary"], 2, dtype=torch.float64) / case["rotary"])
    turns = f * 8192 / (2 * math.pi)  # within a training context of 8192
    fast = ((turns - 1) / 31).clamp(0, 1)
    return (f * (fast + (1 - fast) / case["stretch"])).float()


def _random_pages(case, n, gen, dev):
    """Pages of random codes and of scales such as normal rows give."""
    pool = torch.empty((n, sum(_sections(case))), dtype=torch.uint8, device=dev)
    at = 0
    for i, size in enumerate(_sections(case)):
        if i % 2 == 0:
            pool[:, at : at + size] = torch.randint(0, 256, (n, size), generator=gen, device=dev, dtype=torch.uint8)
        else:
            bits = (K_BITS if i == 1 else V_BITS)[case["tag"]]
            s = 2.5 / (2 ** (bits - 1) - 1) * torch.exp(0.3 * torch.randn((n, size // 2), generator=gen, device=dev))
            pool[:, at : at + size] = s.half().view(torch.uint8)
        at += size
    return pool


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dtype, P, H, D = TYPES[case["type"]], case["page"], case["heads"], case["dim"]
    kv, rows = _lengths(case)
    n, most, seqs = sum(rows), -(-max(kv) // P), case["seqs"]
    st = {"case": case, "kv": torch.tensor(kv, device=dev, dtype=torch.int32), "n": n, "max_rows": max(rows), "max_kv": max(kv)}
    if case["op"] in ("mass", "select"):  # accumulated weight has a long tail; tokens that nothing has looked at tie
        st["mass_in"] = torch.exp(2.0 * torch.randn((seqs, max(kv)), generator=gen, device=dev) - 3.0)
        if case["ties"]:
            st["mass_in"] = (st["mass_in"] * 8.0).floor() / 8.0
        st["mass"] = torch.zeros_like(st["mass_in"])
    if case["op"] in ("select", "gather"):
        st["keep"] = torch.full((seqs, case["keep"]), -1, dtype=torch.int32, device=dev)
        st["kept"] = torch.zeros(seqs, dtype=torch.int32, device=dev)
    if case["op"] == "select":
        st["mass"] = torch.zeros((seqs, case["keep"]), device=dev)
    else:
        to = -(-case["keep"] // P)  # pages that the kept rows of a sequence go to
        n_pages = seqs * (most + to) + 3
        pages = torch.randperm(n_pages, generator=gen, device=dev).int()
        st["table"], st["to"] = pages[: seqs * most].view(seqs, most), pages[seqs * most : seqs * (most + to)].view(seqs, to)
        if case["tag"] == 0:
            st["k_pool"] = _values((n_pages, P, H, D), gen, dev, torch.bfloat16, True)
            st["v_pool"] = _values((n_pages, P, H, D), gen, dev, torch.bfloat16, False)
        else:
            st["pool"] = _random_pages(case, n_pages, gen, dev)
        st["inv_freq"] = _inv_freq(case)
    if case["op"] == "gather":  # a choice such as evict_select makes: the first, the last, some of the rest
        for b, (t, k) in enumerate(zip(kv, _kept(case))):
            order = torch.rand(t, generator=gen, device=dev)
            order[: case["sinks"]] = 3.0
            order[t - min(case["recent"], t) :] = 4.0
            st["keep"][b, :k] = order.topk(k).indices.sort().values.int()
            st["kept"][b] = k
    if case["op"] in ("rope", "mass"):
        st["start"] = torch.tensor([sum(rows[:i]) for i in range(seqs + 1)], device=dev, dtype=torch.int32)
        st["q"] = _values((n, case["q_heads"], D), gen, dev, dtype, False)
    if case["op"] == "rope":
        st["k"], st["v"] = _values((n, H, D), gen, dev, dtype, True), _values((n, H, D), gen, dev, dtype, False)
        st["rope_pos"] = (_positions(st) + case["far"]).int() if case["far"] else None
        st["q_out"], st["k_out"], st["v_out"] = (torch.empty_like(st[x]) for x in ("q", "k", "v"))
    if own:  # the handle and the descriptors that a program keeps
        from paper_2609_26219_b200 import binding as pk

        st["ctx"] = pk.Context(device=torch.cuda.current_device())
        if case["op"] != "select":
            style = pk.ROPE_INTERLEAVED if case["interleaved"] else pk.ROPE_HALF
            st["geom"] = pk.make_geom(1, H, D, case["rotary"], style, BASE, P, P, case["group"], st["inv_freq"])
            if case["tag"] == 0:
                st["cache"] = pk.make_pool(st["k_pool"], st["v_pool"], n_pages, (n_pages * P * H * D, P * H * D, H * D, D))
            else:
                st["cache"] = pk.make_qpool(st["pool"], case["tag"], n_pages)
        if case["op"] in ("rope", "mass"):
            st["batch"] = pk.make_batch(row_start=st["start"], kv_len=st["kv"], block_table=st["table"], n_rows=n, max_rows=max(rows), max_kv_len=max(kv))
        if case["op"] == "mass":
            size = pk.attention_mass_workspace_bytes(st["geom"], st["cache"], st["batch"], case["q_heads"], case["window"], case["sinks"])
            st["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device=dev)
    return st


# ---- plain forms


def _sequences(st):
    """Sequence of every packed row, and its place in it."""
    r = torch.arange(st["n"], device=st["kv"].device)
    seq = torch.searchsorted(st["start"][1:].contiguous(), r.int(), right=True)
    return seq, r - st["start"][seq]


def _positions(st):
    seq, at = _sequences(st)
    return st["kv"][seq] - (st["start"][seq + 1] - st["start"][seq]) + at


def _rotated(x, pos, case, inv_freq):
    """x [n, heads, dim], in the type that it comes in, with the rotation of pos [n]; angles in 64 bits."""
    angle = pos.double()[:, None, None] * inv_freq.to(x.device).double()
    c, s = (case["factor"] * angle.cos()).to(x.dtype), (case["factor"] * angle.sin()).to(x.dtype)
    r, rest = x[..., : case["rotary"]], x[..., case["rotary"] :]
    a, b = (r[..., 0::2], r[..., 1::2]) if case["interleaved"] else r.chunk(2, -1)
    a, b = a * c - b * s, a * s + b * c
    r = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((r, rest), -1)


def _to_half(x):
    """float64 >= 0 -> the nearest fp16 in one rounding, ties to even."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), e.clamp_min(-13) - 11)
    return ((x / step).round() * step).half()


def _encode(x, bits, group):
    """float64 [..., dim] -> codes (whole numbers) and fp16 scales."""
    g = x.unflatten(-1, (-1, group))
    top = 2 ** (bits - 1) - 1
    s = _to_half(g.abs().amax(-1) / top)
    q = (g / s.double().unsqueeze(-1)).round().nan_to_num(0.0, 0.0, 0.0).clamp(-top, top)
    return q.flatten(-2), s


def _plain_rope(st):
    case = st["case"]
    seq, _ = _sequences(st)
    at = _positions(st)
    turn = at if st["rope_pos"] is None else st["rope_pos"]
    q = _rotated(st["q"].float(), turn, case, st["inv_freq"]).to(st["q"].dtype)
    page, slot = st["table"][seq, at // case["page"]].long(), (at % case["page"]).long()
    if case["tag"] == 0:
        st["k_pool"][page, slot] = _rotated(st["k"].float(), turn, case, st["inv_freq"]).to(torch.bfloat16)
        st["v_pool"][page, slot] = st["v"]
        return {"q": q, "k": st["k_pool"], "v": st["v_pool"]}
    off, out, sizes = 0, {"q": q}, _sections(case)
    # keys in 64 bits: a value next to the border of two codes differs by a whole step
    for name, x, bits, size, scale in (("k", _rotated(st["k"].double(), turn, case, st["inv_freq"]), K_BITS[case["tag"]], sizes[0], sizes[1]),
                                       ("v", st["v"].double(), V_BITS[case["tag"]], sizes[2], sizes[3])):
        codes, s = _encode(x, bits, case["group"])
        b = codes.to(torch.int16) & (255 if bits == 8 else 15)
        b = (b if bits == 8 else b[..., 0::2] | (b[..., 1::2] << 4)).to(torch.uint8)
        st["pool"][:, off : off + size].unflatten(1, (case["page"], -1))[page, slot] = b.flatten(1)
        off += size
        st["pool"][:, off : off + scale].unflatten(1, (case["page"], -1))[page, slot] = s.view(torch.uint8).flatten(1)
        off += scale
        out[name] = (codes.float().unflatten(-1, (-1, case["group"])) * s.float().unsqueeze(-1)).flatten(-2).to(st["k"].dtype)
    return out


def _plain_keys(st):
    """The keys of the padded sequences, fp32 [seqs, tokens, heads, dim]."""
    case = st["case"]
    t = torch.arange(st["max_kv"], device=st["kv"].device)
    pages, slots = st["table"][:, t // case["page"]].long(), (t % case["page"]).expand(case["seqs"], -1)
    if case["tag"] == 0:
        return st["k_pool"][pages, slots].float()
    codes, scales = _sections(case)[:2]
    b = st["pool"][:, :codes].unflatten(1, (case["page"], case["heads"], -1))[pages, slots]
    s = st["pool"][:, codes : codes + scales].unflatten(1, (case["page"], case["heads"], -1))[pages, slots].contiguous().view(torch.float16)
    if K_BITS[case["tag"]] == 8:
        q = b.view(torch.int8).float()
    else:
        q = torch.stack((b & 15, b >> 4), -1).flatten(-2).to(torch.int8)
        q = (q - 16 * (q >= 8)).float()
    return (q.unflatten(-1, (-1, case["group"])) * s.float().unsqueeze(-1)).flatten(-2)


def _plain_mass(st):
    case = st["case"]
    dev, H, D, seqs, R = st["q"].device, case["heads"], case["dim"], case["seqs"], st["max_rows"]
    t = torch.arange(st["max_kv"], device=dev)
    seq, at = _sequences(st)
    q = torch.zeros((seqs, R, H, case["q_heads"] // H, D), device=dev)
    q[seq, at] = st["q"].float().unflatten(1, (H, -1))
    p = torch.full((seqs, R), -1, device=dev, dtype=torch.int32)
    p[seq, at] = _positions(st).int()
    p = p.unsqueeze(-1)
    see = (t <= p) & (t < st["kv"].view(-1, 1, 1))
    if case["window"]:
        see &= (p - t < case["window"]) | (t < case["sinks"])
    q = q.permute(0, 2, 3, 1, 4).flatten(2, 3) * D**-0.5  # [seq, head, group * row, dim]
    w = (q @ _plain_keys(st).permute(0, 2, 3, 1)).unflatten(2, (-1, R))
    w.masked_fill_(~see[:, None, None], -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    w /= w.sum(-1, keepdim=True).clamp_min(1e-30)
    total = w.flatten(1, 3).sum(1, dtype=torch.float64)
    if case["decay"]:
        total += case["decay"] * st["mass_in"].double()
    return torch.where(t < st["kv"].view(-1, 1), total.float(), st["mass"])


def _plain_select(st):
    case = st["case"]
    n, i = st["kv"].view(-1, 1), torch.arange(st["max_kv"], device=st["kv"].device)
    recent = min(case["recent"], case["keep"])  # where not all fit: the last tokens, then the first, then by weight
    rank = st["mass_in"].clone()
    rank[(i < min(case["sinks"], case["keep"] - recent)).expand_as(rank)] = math.inf
    rank.masked_fill_((i < n) & (i >= n - recent), math.inf)
    rank.masked_fill_(i >= n, -1.0)
    order = rank.sort(dim=1, descending=True, stable=True).indices[:, : case["keep"]]
    count = st["kv"].clamp_max(case["keep"])
    there = torch.arange(order.shape[1], device=order.device) < count.view(-1, 1)
    keep = torch.where(there, order, st["max_kv"]).sort(1).values
    mass = torch.where(there, st["mass_in"].gather(1, keep.clamp_max(st["max_kv"] - 1)), st["mass"][:, : order.shape[1]])
    pad = case["keep"] - order.shape[1]
    keep = torch.nn.functional.pad(torch.where(there, keep, -1).int(), (0, pad), value=-1)
    return {"keep": keep, "kept": count, "mass": torch.cat((mass, st["mass"][:, order.shape[1] :]), 1)}


def _plain_gather(st):
    case = st["case"]
    seq, slot = torch.nonzero(torch.arange(case["keep"], device=st["kv"].device) < st["kept"].view(-1, 1), as_tuple=True)
    old = st["keep"][seq, slot].long()
    page, at = st["table"][seq, old // case["page"]].long(), old % case["page"]
    to, to_at = st["to"][seq, slot // case["page"]].long(), slot % case["page"]
    if case["tag"] == 0:
        k = st["k_pool"][page, at]
        if case["far"]:
            k = _rotated(k.float(), slot - old, case, st["inv_freq"]).to(torch.bfloat16)
        st["k_pool"][to, to_at] = k
        st["v_pool"][to, to_at] = st["v_pool"][page, at]
        return {"k": st["k_pool"], "v": st["v_pool"]}
    a, b, c, d = (x.unflatten(1, (case["page"], -1)) for x in st["pool"].split(_sections(case), 1))
    a[to, to_at], b[to, to_at], c[to, to_at], d[to, to_at] = a[page, at], b[page, at], c[page, at], d[page, at]
    return st["pool"]


def run(st):
    case = st["case"]
    if own:
        ctx = st["ctx"]
        if case["op"] == "rope":
            ctx.rotary_append(st["geom"], st["cache"], 0, st["batch"], st["k"], st["v"], q=st["q"], q_out=st["q_out"], rope_pos=st["rope_pos"], rope_factor=case["factor"])
            if case["tag"] == 0:
                return {"q": st["q_out"], "k": st["k_pool"], "v": st["v_pool"]}
            ctx.cache_read(st["geom"], st["cache"], 0, st["batch"], st["k_out"], st["v_out"])
            return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
        if case["op"] == "mass":
            ctx.attention_mass(st["geom"], st["cache"], 0, st["batch"], st["q"], st["mass"], mass_in=st["mass_in"], decay=case["decay"], scale=case["dim"] ** -0.5,
                               window=case["window"], sinks=case["sinks"], workspace=st["workspace"])
            return st["mass"]
        if case["op"] == "select":
            ctx.evict_select(st["mass_in"], st["kv"], st["keep"], st["kept"], sinks=case["sinks"], recent=case["recent"], mass_out=st["mass"])
            return {"keep": st["keep"], "kept": st["kept"], "mass": st["mass"]}
        ctx.cache_gather(st["geom"], st["cache"], 0, st["keep"], st["kept"], st["kv"], st["table"], st["to"], rotate=bool(case["far"]))
        return {"k": st["k_pool"], "v": st["v_pool"]} if case["tag"] == 0 else st["pool"]
    return {"rope": _plain_rope, "mass": _plain_mass, "select": _plain_select, "gather": _plain_gather}[case["op"]](st)


# ---- the definitions in 64 bits


def _turned64(x, pos, case):
    """x [n, heads, dim] -> rotated, as products of complex numbers."""
    d = case["rotary"]
    f = _inv_freq(case).to(x.device).double()
    phase = torch.polar(torch.full((len(pos), d // 2), case["factor"], dtype=torch.float64, device=x.device), pos.double()[:, None] * f)
    out = x.double().clone()
    first = torch.arange(0, d, 2, device=x.device) if case["interleaved"] else torch.arange(d // 2, device=x.device)
    second = first + (1 if case["interleaved"] else d // 2)
    z = torch.complex(out[..., first], out[..., second]) * phase[:, None, :]
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _keys64(st, case, b, t):
    """Keys of tokens [0, t) of sequence b as float64 [t, heads, dim], a head at a time out of the pages' bytes."""
    P, H, D, G = case["page"], case["heads"], case["dim"], case["group"]
    pages = st["table"][b, : -(-t // P)].long()
    if case["tag"] == 0:
        return st["k_pool"].index_select(0, pages).flatten(0, 1)[:t].double()
    raw = st["pool"].index_select(0, pages).to(torch.int64)
    e = P * H * D
    if K_BITS[case["tag"]] == 8:
        code, at = raw[:, :e], e
    else:
        code, at = torch.empty((len(pages), e), dtype=torch.int64, device=raw.device), e // 2
        code[:, 0::2], code[:, 1::2] = raw[:, :at] % 16, raw[:, :at] // 16
    half = 2 ** (K_BITS[case["tag"]] - 1)
    code = (code + half) % (2 * half) - half
    word = raw[:, at : at + 2 * e // G : 2] + 256 * raw[:, at + 1 : at + 2 * e // G : 2]
    scale = torch.ldexp((word % 1024 + 1024 * (word // 1024 > 0)).double(), (word // 1024).clamp_min(1) - 25)
    return (code.double().unflatten(1, (-1, G)) * scale[..., None]).reshape(-1, H, D)[:t]


def _exact_rope(st, case):
    kv, rows = _lengths(case)
    at = torch.cat([torch.arange(t - r, t) for t, r in zip(kv, rows)]).to(st["q"].device)
    turn = at + case["far"]
    out = {"q": _turned64(st["q"], turn, case), "k": _turned64(st["k"], turn, case), "v": st["v"].double()}
    if case["tag"] == 0:
        seq = torch.repeat_interleave(torch.arange(len(rows)), torch.tensor(rows)).to(at.device)
        place = st["table"][seq, at // case["page"]].long() * case["page"] + at % case["page"]
        for name in ("k", "v"):
            whole = st[name + "_pool"].double()
            whole.flatten(0, 1).index_copy_(0, place, out[name])
            out[name] = whole
        return out
    for name, bits in (("k", K_BITS[case["tag"]]), ("v", V_BITS[case["tag"]])):
        x = out[name].reshape(-1, case["group"])
        top = 2.0 ** (bits - 1) - 1
        want = x.abs().max(1).values / top
        near = want.half().double()  # then the better of it and its neighbours, for one rounding in all
        bits16 = want.half().view(torch.int16).long()
        for d in (-1, 1):
            other = (bits16 + d).clamp_min(0).short().view(torch.float16).double()
            gap, best = (other - want).abs(), (near - want).abs()
            near = torch.where((gap < best) | ((gap == best) & ((bits16 + d) % 2 == 0)), other, near)
        code = torch.where(near[:, None] > 0, torch.round(x / near.clamp_min(1e-30)[:, None]), torch.zeros_like(x)).clamp(-top, top)
        out[name] = (code * near[:, None]).view(out[name].shape)
    return out


def _exact_mass(st, case):
    kv, rows = _lengths(case)
    out, first, share = st["mass"].double(), 0, case["q_heads"] // case["heads"]
    for b, (t, r) in enumerate(zip(kv, rows)):
        keys, token = _keys64(st, case, b, t), torch.arange(t, device=out.device)
        place = torch.arange(t - r, t, device=out.device)[:, None]
        hidden = token > place
        if case["window"]:
            hidden |= (token <= place - case["window"]) & (token >= case["sinks"])
        total = case["decay"] * st["mass_in"][b, :t].double()
        for h in range(case["q_heads"]):
            logits = st["q"][first : first + r, h].double() @ keys[:, h // share].T / math.sqrt(case["dim"])
            total += torch.softmax(logits.masked_fill_(hidden, -math.inf), -1).sum(0)
        out[b, :t] = total
        first += r
    return out


def _exact_select(st, case):
    keep, mass = st["keep"].cpu().numpy().copy(), st["mass"].double().cpu().numpy()
    weight, counts = st["mass_in"].cpu().numpy(), _kept(case)
    for b, (t, k) in enumerate(zip(_lengths(case)[0], counts)):
        last = set(range(max(0, t - min(case["recent"], k)), t))
        first = set(range(min(case["sinks"], t, k - len(last))))
        middle = numpy.array(sorted(set(range(t)) - first - last), dtype=numpy.int64)
        best = middle[numpy.lexsort((middle, -weight[b, middle].astype(numpy.float64)))][: k - len(first | last)]
        chosen = numpy.array(sorted(first | last | set(best.tolist())))
        keep[b, :k], mass[b, :k] = chosen, weight[b, chosen]
    return {"keep": torch.from_numpy(keep), "kept": torch.tensor(counts, dtype=torch.int32), "mass": torch.from_numpy(mass)}


def _exact_gather(st, case):
    P = case["page"]
    froms, tos, moved = [], [], []
    for b, k in enumerate(_kept(case)):
        old, new = st["keep"][b, :k].long(), torch.arange(k, device=st["keep"].device)
        froms.append(st["table"][b].long()[old // P] * P + old % P)
        tos.append(st["to"][b].long()[new // P] * P + new % P)
        moved.append(new - old)
    froms, tos, moved = torch.cat(froms), torch.cat(tos), torch.cat(moved)
    if case["tag"]:
        out = st["pool"].clone()
        at = 0
        for size in _sections(case):
            rows = out[:, at : at + size].reshape(-1, size // P)
            rows[tos] = rows[froms]
            out[:, at : at + size] = rows.view(-1, size)
            at += size
        return out
    k, v = st["k_pool"].double(), st["v_pool"].double()
    rows = k.flatten(0, 1)[froms]
    k.flatten(0, 1)[tos] = _turned64(rows, moved, case) if case["far"] else rows
    v.flatten(0, 1)[tos] = v.flatten(0, 1)[froms]
    return {"k": k, "v": v}


def exact(case, seed):
    return {"rope": _exact_rope, "mass": _exact_mass, "select": _exact_select, "gather": _exact_gather}[case["op"]](prepare(case, seed), case)
