"""Measured cases of the live-cache operators: writing rows into a paged 8- or 4-bit cache and reading them back
(cache_append, cache_read), and attention over such a cache or over the bf16 pool (attention).

A quantised page is one checkpoint record of `page` tokens: [K codes][K scales][V codes][V scales], codes
[token][head][channel], fp16 scales per `group` channels.  `tag` is the framework's precision tag: 0 = bf16 pool,
1 = K8/V8, 2 = K8/V4, 3 = K4/V4.  Row i of a sequence with `rows` rows and `kv` cached tokens stands at position
kv - rows + i, or (scattered) at given ascending positions, as the rows of a repair set do."""
import math

import torch

own = False

K_BITS, V_BITS = {0: 16, 1: 8, 2: 8, 3: 4}, {0: 16, 1: 8, 2: 4, 3: 4}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(op, tag, heads, q_heads, dim, seqs, kv, rows, **more):
    c = {"op": op, "tag": tag, "heads": heads, "q_heads": q_heads, "dim": dim, "group": 32, "page": 16, "seqs": seqs,
         "kv": kv, "rows": rows, "ragged": 0, "window": 0, "sinks": 0, "scattered": False, "type": "bf16"}
    c.update(more)
    return c


def listed():
    return [
        # one decode step's new tokens of eight requests: latency
        _case("write", 3, 8, 8, 128, 8, 1000, 1, name="write_step"),
        # a 16k prompt's rows in the low-bit tier that keeps keys at 8 bits
        _case("write", 2, 8, 8, 128, 1, 16384, 16384, name="write_prompt"),
        # a short odd context of the tiny geometry read back
        _case("read", 1, 4, 4, 64, 1, 1013, 1013, type="fp16", name="read_short"),
        # two 64k contexts read back to bf16
        _case("read", 3, 8, 8, 128, 2, 65536, 65536, name="read_long"),
        # one short request, one token: latency
        _case("attend", 3, 4, 8, 64, 1, 1000, 1, name="decode_short"),
        # one 16k request of the 8B-shaped geometry
        _case("attend", 3, 8, 32, 128, 1, 16384, 1, name="decode_16k"),
        # eight 64k requests of the 70B-shaped geometry
        _case("attend", 3, 8, 64, 128, 8, 65536, 1, name="decode_64k_x8"),
        # many ragged requests under a window with sinks, 4 KV heads, seven query heads each
        _case("attend", 1, 4, 28, 128, 32, 32768, 1, ragged=20011, window=4096, sinks=4, type="fp16", name="decode_window"),
        # decode over the pool that a restore has filled
        _case("attend", 0, 8, 32, 128, 8, 16384, 1, ragged=1001, name="decode_pool"),
        # a whole prompt over its own quantised cache
        _case("attend", 3, 8, 32, 128, 1, 8192, 8192, name="prompt_8k"),
        # the rows of a repair set, 15 % of a 16k suffix, at their positions
        _case("attend", 2, 8, 32, 128, 1, 16384, 2458, scattered=True, name="repair_rows"),
        # ragged prompt chunks over the pool under a window with sinks
        _case("attend", 0, 4, 28, 128, 4, 4096, 2000, ragged=777, window=1024, sinks=4, name="prompt_window"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    heads, q_heads, dim = rng.choice([(4, 8, 64), (8, 32, 128), (4, 28, 128), (8, 64, 128), (2, 16, 128), (1, 8, 64), (32, 32, 128)])
    op = rng.choice(["write", "read", "attend", "attend", "attend"])
    more = {"type": rng.choice(["bf16", "bf16", "fp16"]), "page": rng.choice([16, 16, 32, 64]), "group": rng.choice([32, 32, 64])}
    if op == "write":
        seqs = _log(rng, 1, 32)
        rows = _log(rng, 1, 16384 // seqs)
        kv = rows + rng.randrange(2000)
        return _case(op, rng.choice([1, 2, 3]), heads, heads, dim, seqs, kv, rows, ragged=rng.randrange(rows), **more)
    if op == "read":
        seqs = _log(rng, 1, 8)
        kv = _log(rng, 100, 65536 // seqs)
        return _case(op, rng.choice([1, 2, 3]), heads, heads, dim, seqs, kv, kv, ragged=rng.randrange(kv), **more)
    tag = rng.choice([0, 1, 2, 3, 3])
    if tag == 0:
        more["type"] = "bf16"
    if rng.random() < 0.5:
        more.update(window=_log(rng, 100, 5000), sinks=rng.choice([0, 4, 17]))
    kind = rng.choice(["decode", "decode", "few", "prompt", "repair"])
    if kind == "decode":
        seqs = _log(rng, 1, 32)
        kv = _log(rng, 50, 131072 // seqs)
        return _case(op, tag, heads, q_heads, dim, seqs, kv, 1, ragged=rng.randrange(kv // 2), **more)
    if kind == "few":
        seqs = _log(rng, 1, 8)
        kv = _log(rng, 100, 65536 // seqs)
        return _case(op, tag, heads, q_heads, dim, seqs, kv, rng.randrange(2, 40), ragged=rng.randrange(20), **more)
    if kind == "prompt":
        seqs = rng.choice([1, 1, 2, 4])
        kv = _log(rng, 200, 8192 // seqs)
        rows = rng.choice([kv, rng.randrange(kv // 2, kv)])
        return _case(op, tag, heads, min(q_heads, 32), dim, seqs, kv, rows, ragged=rng.randrange(rows // 2), **more)
    kv = _log(rng, 1000, 16384)
    return _case(op, tag, heads, min(q_heads, 32), dim, 1, kv, rng.randrange(kv // 50, kv // 7), scattered=True, **more)


def _lengths(case):
    """Per sequence: cached tokens and rows.  With `ragged`, later sequences are shorter by up to that much, each by
    another amount; rows stay at one at least and never exceed the tokens."""
    kv, rows = [], []
    for b in range(case["seqs"]):
        cut = (b * 7919 * 13) % (case["ragged"] + 1) if case["ragged"] else 0
        if case["rows"] > 1:
            kv.append(case["kv"] - (cut if case["op"] == "read" or case["kv"] == case["rows"] else cut // 3))
            rows.append(max(1, min(case["rows"] - cut, kv[-1])))
        else:
            kv.append(case["kv"] - cut)
            rows.append(1)
    return kv, rows


def _row_bytes(case):
    e = case["dim"]
    k, v = K_BITS[case["tag"]], V_BITS[case["tag"]]
    scales = 0 if case["tag"] == 0 else 4 * (e // case["group"])
    return case["heads"] * (e * (k + v) // 8 + scales)


def _seen(case, kv, rows):
    """(tokens that some row sees, pairs of row and visible token) of one sequence."""
    w, s = case["window"], case["sinks"]
    if case["scattered"]:
        pos = [(i * kv) // rows for i in range(rows)]
    else:
        pos = range(kv - rows, kv)
    pairs, seen, upto = 0, 0, 0
    for p in pos:
        low = max(0, p + 1 - w) if w else 0
        low = max(low, min(s, p + 1))
        pairs += p + 1 - low + min(s, p + 1)
        seen += max(0, p + 1 - max(low, upto))
        upto = max(upto, p + 1)
    return min(kv, seen + min(s, kv)), pairs


def work(case):
    kv, rows = _lengths(case)
    n, e = sum(rows), case["dim"]
    if case["op"] == "write":  # rows in, record bytes out; the same back again
        return {"bytes": n * 2 * (case["heads"] * e * 4 + _row_bytes(case)), "flops": 8 * n * case["heads"] * e}
    if case["op"] == "read":
        return {"bytes": n * (case["heads"] * e * 4 + _row_bytes(case)), "flops": 2 * n * case["heads"] * e}
    seen, pairs = (sum(x) for x in zip(*(_seen(case, t, r) for t, r in zip(kv, rows))))
    return {"bytes": seen * _row_bytes(case) + 4 * n * case["q_heads"] * e, "flops": 4 * pairs * case["q_heads"] * e}


def _values(shape, gen, dev, dtype, outliers):
    x = torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)
    if outliers:  # a few key channels are ten times the others, as in trained models
        x[..., torch.randperm(shape[-1], generator=gen, device=dev)[: shape[-1] // 20]] *= 10.0
    return x.to(dtype)


def _encode(x, bits, group):
    """fp32 [..., dim] -> codes (whole numbers, fp32) and fp16 scales."""
    g = x.unflatten(-1, (-1, group))
    s = (g.abs().amax(-1) / (2 ** (bits - 1) - 1)).half()
    q = (g / s.float().unsqueeze(-1)).round().nan_to_num(0.0, 0.0, 0.0).clamp(-(2 ** (bits - 1) - 1), 2 ** (bits - 1) - 1)
    return q.flatten(-2), s


def _pack(q, bits):
    """Codes [..., dim] -> the bytes of their section."""
    q = q.to(torch.int16) & (255 if bits == 8 else 15)
    return (q if bits == 8 else q[..., 0::2] | (q[..., 1::2] << 4)).to(torch.uint8)


def _unpack(b, bits):
    if bits == 8:
        return b.view(torch.int8).float()
    n = torch.stack((b & 15, b >> 4), -1).flatten(-2).to(torch.int8)
    return (n - 16 * (n >= 8)).float()


def _sections(case):
    """Byte sizes of a page's four sections."""
    e = case["page"] * case["heads"] * case["dim"]
    s = 2 * e // case["group"]
    return [e * K_BITS[case["tag"]] // 8, s, e * V_BITS[case["tag"]] // 8, s]


def _write_pages(pool, pages, case, k, v):
    """fp32 rows [pages, page, heads, dim] into whole pages of the pool."""
    n = pages.numel()
    parts = []
    for x, bits in ((k, K_BITS[case["tag"]]), (v, V_BITS[case["tag"]])):
        q, s = _encode(x, bits, case["group"])
        parts += [_pack(q, bits).reshape(n, -1), s.reshape(n, -1).view(torch.uint8)]
    pool[pages] = torch.cat(parts, 1)


def _gather(pool, pages, slots, case):
    """The fp32 values of given (page, slot) pairs of the quantised pool: two tensors [..., heads, dim]."""
    out, at = [], 0
    P, H, D, G = case["page"], case["heads"], case["dim"], case["group"]
    sizes = _sections(case)
    for k, bits in ((0, K_BITS[case["tag"]]), (2, V_BITS[case["tag"]])):
        codes = pool[:, at : at + sizes[k]].unflatten(1, (P, H, -1))[pages, slots]
        scales = pool[:, at + sizes[k] : at + sizes[k] + sizes[k + 1]].unflatten(1, (P, H, -1))[pages, slots].contiguous().view(torch.float16)
        at += sizes[k] + sizes[k + 1]
        out.append((_unpack(codes, bits).unflatten(-1, (-1, G)) * scales.float().unsqueeze(-1)).flatten(-2))
    return out


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dtype, P, H, D = TYPES[case["type"]], case["page"], case["heads"], case["dim"]
    kv, rows = _lengths(case)
    n, most = sum(rows), -(-max(kv) // P)
    n_pages = case["seqs"] * most + 3
    table = torch.randperm(n_pages, generator=gen, device=dev)[: case["seqs"] * most].view(case["seqs"], most).int()
    st = {"case": case, "table": table, "kv": torch.tensor(kv, device=dev, dtype=torch.int32), "n": n, "max_rows": max(rows), "max_kv": max(kv),
          "start": torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], device=dev, dtype=torch.int32), "pos": None}
    if case["scattered"]:
        st["pos"] = torch.cat([(torch.arange(r, device=dev) * t) // r for t, r in zip(kv, rows)]).int()
    if case["tag"] == 0:
        st["k_pool"] = _values((n_pages, P, H, D), gen, dev, torch.bfloat16, True)
        st["v_pool"] = _values((n_pages, P, H, D), gen, dev, torch.bfloat16, False)
    else:
        st["pool"] = torch.empty((n_pages, sum(_sections(case))), dtype=torch.uint8, device=dev)
        for i in range(0, n_pages, 2048):
            m = min(2048, n_pages - i)
            _write_pages(st["pool"], torch.arange(i, i + m, device=dev), case, _values((m, P, H, D), gen, dev, torch.float32, True), _values((m, P, H, D), gen, dev, torch.float32, False))
    if case["op"] == "write":
        st["k"], st["v"] = _values((n, H, D), gen, dev, dtype, True), _values((n, H, D), gen, dev, dtype, False)
    if case["op"] in ("write", "read"):
        st["k_out"], st["v_out"] = torch.empty((n, H, D), dtype=dtype, device=dev), torch.empty((n, H, D), dtype=dtype, device=dev)
    else:
        st["q"] = _values((n, case["q_heads"], D), gen, dev, dtype, False)
        st["out"] = torch.empty_like(st["q"])
    if own:  # the handle and the descriptors that a program keeps
        from paper_2609_26219_b200 import binding as pk

        st["ctx"] = pk.Context(device=torch.cuda.current_device())
        st["geom"] = pk.make_geom(1, H, D, D, pk.ROPE_HALF, 10000.0, P, P, case["group"])
        st["batch"] = pk.make_batch(row_start=st["start"], kv_len=st["kv"], block_table=table, n_rows=n, max_rows=max(rows), max_kv_len=max(kv), pos=st["pos"])
        if case["tag"] == 0:
            st["cache"] = pk.make_pool(st["k_pool"], st["v_pool"], n_pages, (n_pages * P * H * D, P * H * D, H * D, D))
        else:
            st["cache"] = pk.make_qpool(st["pool"], case["tag"], n_pages)
        if case["op"] == "attend":
            size = pk.attention_workspace_bytes(st["geom"], st["cache"], st["batch"], case["q_heads"], case["window"], case["sinks"])
            st["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device=dev)
    return st


def _rows(st):
    """Sequence and position of every row."""
    r = torch.arange(st["n"], device=st["kv"].device)
    seq = torch.searchsorted(st["start"][1:].contiguous(), r.int(), right=True)
    at = r - st["start"][seq]
    pos = st["pos"].long() if st["pos"] is not None else st["kv"][seq] - (st["start"][seq + 1] - st["start"][seq]) + at
    return seq, at, pos.long()


def _plain_write(st):
    case = st["case"]
    seq, _, pos = _rows(st)
    page, slot = st["table"][seq, pos // case["page"]].long(), pos % case["page"]
    at, sizes = 0, _sections(case)
    for i, (x, bits) in enumerate(((st["k"], K_BITS[case["tag"]]), (st["v"], V_BITS[case["tag"]]))):
        q, s = _encode(x.float(), bits, case["group"])
        codes = st["pool"][:, at : at + sizes[2 * i]].unflatten(1, (case["page"], -1))
        codes[page, slot] = _pack(q, bits).flatten(1)
        at += sizes[2 * i]
        scales = st["pool"][:, at : at + sizes[2 * i + 1]].unflatten(1, (case["page"], -1))
        scales[page, slot] = s.view(torch.uint8).flatten(1)
        at += sizes[2 * i + 1]
    return _plain_read(st)


def _plain_read(st):
    case = st["case"]
    seq, _, pos = _rows(st)
    k, v = _gather(st["pool"], st["table"][seq, pos // case["page"]].long(), pos % case["page"], case)
    return {"k": k.to(TYPES[case["type"]]), "v": v.to(TYPES[case["type"]])}


def _plain_attend(st):
    case = st["case"]
    dev, H, D = st["q"].device, case["heads"], case["dim"]
    seq, at, pos = _rows(st)
    t = torch.arange(st["max_kv"], device=dev)
    pages, slots = st["table"][:, t // case["page"]].long(), (t % case["page"]).expand(case["seqs"], -1)
    if case["tag"] == 0:
        k, v = st["k_pool"][pages, slots].float(), st["v_pool"][pages, slots].float()
    else:
        k, v = _gather(st["pool"], pages, slots, case)
    q = torch.zeros((case["seqs"], st["max_rows"], H, case["q_heads"] // H, D), device=dev)
    q[seq, at] = st["q"].float().unflatten(1, (H, -1))
    p_row = torch.full((case["seqs"], st["max_rows"]), -1, device=dev)
    p_row[seq, at] = pos
    p_row = p_row.unsqueeze(-1)
    see = (t <= p_row) & (t < st["kv"].view(-1, 1, 1))
    if case["window"]:
        see &= (p_row - t < case["window"]) | (t < case["sinks"])
    q = q.permute(0, 2, 3, 1, 4).flatten(2, 3) * D**-0.5  # [seq, head, group * row, dim]
    s = (q @ k.permute(0, 2, 3, 1)).unflatten(2, (-1, st["max_rows"]))
    s.masked_fill_(~see[:, None, None], -math.inf)
    s = (s - s.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    s /= s.sum(-1, keepdim=True).clamp_min(1e-30)
    o = (s.flatten(2, 3) @ v.permute(0, 2, 1, 3)).unflatten(2, (-1, st["max_rows"]))
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, at].to(st["q"].dtype)


def run(st):
    case = st["case"]
    if own:
        if case["op"] == "attend":
            st["ctx"].attention(st["geom"], st["cache"], 0, st["batch"], st["q"], st["out"], scale=case["dim"] ** -0.5, window=case["window"], sinks=case["sinks"], workspace=st["workspace"])
            return st["out"]
        if case["op"] == "write":
            st["ctx"].cache_append(st["geom"], st["cache"], 0, st["batch"], st["k"], st["v"])
        st["ctx"].cache_read(st["geom"], st["cache"], 0, st["batch"], st["k_out"], st["v_out"])
        return {"k": st["k_out"], "v": st["v_out"]}
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[case["op"]](st)


def _dequantised64(page, which, case):
    """One section pair of a page's bytes, by the layout's definition, as float64 [page, heads, dim]."""
    sizes = _sections(case)
    off = sum(sizes[: 2 * which])
    codes, scales = page[off : off + sizes[2 * which]], page[off + sizes[2 * which] : off + sizes[2 * which] + sizes[2 * which + 1]]
    if (K_BITS, V_BITS)[which][case["tag"]] == 8:
        q = codes.to(torch.int64)
        q = torch.where(q > 127, q - 256, q)
    else:
        q = torch.empty(2 * codes.numel(), dtype=torch.int64, device=codes.device)
        q[0::2], q[1::2] = codes.to(torch.int64) % 16, codes.to(torch.int64) // 16
        q = torch.where(q > 7, q - 16, q)
    s = scales.clone().view(torch.float16).double().repeat_interleave(case["group"])
    return (q.double() * s).view(case["page"], case["heads"], case["dim"])


def exact(case, seed):
    st = prepare(case, seed)
    kv, rows = _lengths(case)
    if case["op"] == "write":
        out = {}
        for name, bits in (("k", K_BITS[case["tag"]]), ("v", V_BITS[case["tag"]])):
            x = st[name].double().reshape(-1, case["group"])
            top = 2.0 ** (bits - 1) - 1
            step = (x.abs().max(1).values / top).to(torch.float16).double()
            code = torch.where(step[:, None] > 0, torch.round(x / step.clamp_min(1e-30)[:, None]), torch.zeros_like(x)).clamp(-top, top)
            out[name] = (code * step[:, None]).view(st[name].shape)
        return out
    if sum(kv) * case["heads"] * case["dim"] > 6e8:
        return None  # minutes of unpacking page by page
    table, P = st["table"].cpu(), case["page"]
    whole = []
    for b, t in enumerate(kv):
        pages = [int(x) for x in table[b, : -(-t // P)]]
        if case["tag"] == 0:
            whole.append([torch.cat([st[x][p].double() for p in pages])[:t] for x in ("k_pool", "v_pool")])
        else:
            whole.append([torch.cat([_dequantised64(st["pool"][p], w, case) for p in pages])[:t] for w in (0, 1)])
    if case["op"] == "read":
        return {"k": torch.cat([w[0] for w in whole]), "v": torch.cat([w[1] for w in whole])}
    out, first, share = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device), 0, case["q_heads"] // case["heads"]
    for b, (t, r) in enumerate(zip(kv, rows)):
        pos = torch.tensor([(i * t) // r if case["scattered"] else t - r + i for i in range(r)], device=out.device)
        key = torch.arange(t, device=out.device)
        hidden = key[None, :] > pos[:, None]
        if case["window"]:
            hidden |= (key[None, :] <= pos[:, None] - case["window"]) & (key[None, :] >= case["sinks"])
        for h in range(case["q_heads"]):
            logits = st["q"][first : first + r, h].double() @ whole[b][0][:, h // share].T / math.sqrt(case["dim"])
            out[first : first + r, h] = torch.softmax(logits.masked_fill(hidden, -math.inf), -1) @ whole[b][1][:, h // share]
        first += r
    return out
