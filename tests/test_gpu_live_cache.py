"""patchkv_cache_append and patchkv_cache_read against a plain 64-bit reference: bytes of whole pools, values, refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from live_common import BF16, BITS, F16, Case, Layout, build_tables, device_batch, random_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pk():
    from paper_2609_26219_b200 import build, binding
    build.build()
    return binding


@pytest.fixture(scope="module")
def ctx(pk):
    c = pk.Context(device=0)
    yield c
    c.close()


def geom_of(pk, lay: Layout, layers=1):
    return pk.make_geom(layers, lay.H, lay.D, lay.D, pk.ROPE_HALF, 1e4, 16, lay.P, lay.G)


def reference_append(lay, pages, case, table, k, v):
    kd, vd = k.double().numpy(), v.double().numpy()
    r = 0
    for b, positions in enumerate(case.positions()):
        for pos in positions:
            lay.put(pages[table[b, pos // lay.P]], pos % lay.P, kd[r], vd[r])
            r += 1


def reference_read(lay, pages, case, table, dtype):
    ks, vs = [], []
    for b, positions in enumerate(case.positions()):
        for pos in positions:
            k, v = lay.values(pages[table[b, pos // lay.P]])
            ks.append(k[pos % lay.P])
            vs.append(v[pos % lay.P])
    # code * scale has 19 significant bits at most: exact in fp32, so one rounding from 64 bits is the rounding meant
    return [torch.from_numpy(np.stack(x)).float().to(dtype) for x in (ks, vs)]


BATCHES = {
    "one_token": Case([1], [1]),
    "one_row_late": Case([1000], [1]),
    "ragged": Case([40, 17, 1, 90], [13, 17, 1, 2]),
    "empty_sequences": Case([5, 0, 33], [0, 0, 33]),
    "scattered": Case([70, 33], [4, 3], [[0, 15, 16, 69], [1, 2, 32]]),
}
GEOMETRIES = [(8, 128, 16, 32), (4, 64, 16, 32), (1, 64, 32, 64), (2, 128, 64, 128), (3, 80, 16, 16), (1, 8, 4, 8),
              (2, 10, 5, 5), (3, 6, 7, 3), (1, 2, 1, 1), (40, 128, 16, 32), (5, 256, 16, 256)]


@pytest.mark.parametrize("tag", [1, 2, 3])
@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("H,D,P,G", GEOMETRIES)
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
def test_append_and_read(pk, ctx, tag, name, H, D, P, G, dtype):
    lay, case = Layout(tag, H, D, P, G), BATCHES[name]
    rng = np.random.default_rng(7)
    table, n_pages = build_tables(case, P, rng)
    batch, keep = device_batch(pk, case, table, DEV)
    n = sum(case.rows)
    k, v = random_rows(rng, n, H, D, dtype), random_rows(rng, n, H, D, dtype, outliers=False)
    if n > 2:
        k[1] = 0                                       # a group of zeros
        v[2] *= 1e-6                                   # subnormal scales
    pages = rng.integers(0, 256, (n_pages, lay.page_bytes()), dtype=np.uint8)
    dev = torch.from_numpy(pages).to(DEV)
    reference_append(lay, pages, case, table, k, v)
    cache = pk.make_qpool(dev, tag, n_pages)
    g = geom_of(pk, lay)
    ctx.cache_append(g, cache, 0, batch, k.to(DEV), v.to(DEV))
    assert ctx.query_status() == 0
    assert np.array_equal(dev.cpu().numpy(), pages)    # every byte of the pool, untouched slots included
    ko, vo = torch.full_like(k, 7.0, device=DEV), torch.full_like(v, 7.0, device=DEV)
    ctx.cache_read(g, cache, 0, batch, ko, vo)
    assert ctx.query_status() == 0
    kw, vw = reference_read(lay, pages, case, table, dtype)
    assert torch.equal(ko.cpu(), kw) and torch.equal(vo.cpu(), vw)
    assert np.array_equal(dev.cpu().numpy(), pages)


@pytest.mark.parametrize("bits_tag", [1, 3])
def test_every_bf16_value_as_group_maximum(pk, ctx, bits_tag):
    """Every positive finite bf16 value whose scale is finite, as the maximum of a group, with neighbours that fall on and
    next to the half-way points of its codes."""
    lay = Layout(bits_tag, 4, 64, 16, 32)
    top = 127 if bits_tag == 1 else 7
    m = torch.arange(1, 0x7F80, dtype=torch.int16).view(BF16)
    m = m[m.double() / top < 65000]
    n = -(-m.numel() // 8)
    m = torch.cat([m, m[:n * 8 - m.numel()]]).view(n, 8, 1)
    s = (m.double() / top).half().double()
    frac = torch.arange(31, dtype=torch.float64) * (top / 31.0)
    half = (torch.floor(frac) + 0.5) * s
    x = torch.cat([m.double(), half], -1).to(BF16).view(n, 4, 64)
    case = Case([n], [n])
    rng = np.random.default_rng(3)
    table, n_pages = build_tables(case, 16, rng)
    batch, keep = device_batch(pk, case, table, DEV)
    pages = np.zeros((n_pages, lay.page_bytes()), np.uint8)
    dev = torch.from_numpy(pages).to(DEV)
    reference_append(lay, pages, case, table, x, x)
    ctx.cache_append(geom_of(pk, lay), pk.make_qpool(dev, bits_tag, n_pages), 0, batch, x.to(DEV), x.to(DEV))
    assert ctx.query_status() == 0
    assert np.array_equal(dev.cpu().numpy(), pages)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
def test_strides_layers_and_rows_behind_the_last_sequence(pk, ctx, dtype):
    """[H][n][D] rows, a padded head stride, an odd row offset, layer 1 of 3, and a packed array longer than the batch."""
    lay, case = Layout(2, 4, 64, 16, 32), Case([50, 20], [7, 20])
    rng = np.random.default_rng(11)
    table, n_pages = build_tables(case, 16, rng)
    n, extra = 27, 5
    batch, keep = device_batch(pk, case, table, DEV, n_rows=n + extra)
    wide = [random_rows(rng, 4, n + extra, 64, dtype) for _ in range(2)]             # [H][n][D]
    padded = [torch.zeros((n + extra, 4, 72), dtype=dtype) for _ in range(2)]
    shifted = [torch.zeros((n + extra) * 256 + 1, dtype=dtype) for _ in range(2)]
    views = {"heads_first": [x.to(DEV).transpose(0, 1) for x in wide], "padded": [x.to(DEV)[..., :64] for x in padded],
             "unaligned": [x.to(DEV)[1:].view(n + extra, 4, 64) for x in shifted]}
    ref_k, ref_v = [x.transpose(0, 1).contiguous() for x in wide]
    g = geom_of(pk, lay, 3)
    for k, v in views.values():
        k.copy_(ref_k.to(DEV))
        v.copy_(ref_v.to(DEV))
        pages = rng.integers(0, 256, (3, n_pages, lay.page_bytes() + 48), dtype=np.uint8)
        dev = torch.from_numpy(pages).to(DEV)
        reference_append(lay, pages[1], case, table, ref_k, ref_v)
        cache = pk.make_qpool(dev, 2, n_pages)
        ctx.cache_append(g, cache, 1, batch, k, v)
        assert np.array_equal(dev.cpu().numpy(), pages)
        k.fill_(3.0)
        v.fill_(3.0)
        ctx.cache_read(g, cache, 1, batch, k, v)
        kw, vw = reference_read(lay, pages[1], case, table, dtype)
        assert torch.equal(k[:n].cpu(), kw) and torch.equal(v[:n].cpu(), vw)
        assert (k[n:] == 3).all() and (v[n:] == 3).all()
    assert ctx.query_status() == 0


@pytest.mark.parametrize("H,D,G", [(4, 64, 32), (2, 10, 5)])
def test_rows_out_of_range_are_skipped_and_latched(pk, ctx, H, D, G):
    lay = Layout(3, H, D, 16, G)
    rng = np.random.default_rng(5)
    good = Case([40, 40], [3, 2], [[0, 5, 39], [1, 2]])
    table, n_pages = build_tables(good, 16, rng)
    k, v = random_rows(rng, 5, H, D, BF16), random_rows(rng, 5, H, D, BF16)
    for what in ("negative", "beyond", "bad_page", "not_ascending", "short_table"):
        pos = [[0, 5, 39], [1, 2]]
        tb = table.copy()
        if what == "negative":
            pos[0][0] = -1
        elif what == "beyond":
            pos[0][2] = 40
        elif what == "bad_page":
            tb[0, 0] = n_pages
            tb[1, 1] = -1                              # not used by the rows: no error of its own
        elif what == "not_ascending":
            pos[0][2] = 5
        else:
            tb = np.ascontiguousarray(table[:, :2])
        skipped = {"negative": [0], "beyond": [2], "bad_page": [0, 1], "not_ascending": [2], "short_table": [2]}[what]
        batch, keep = device_batch(pk, Case(good.kv, good.rows, pos), tb, DEV)
        pages = rng.integers(0, 256, (n_pages, lay.page_bytes()), dtype=np.uint8)
        dev = torch.from_numpy(pages).to(DEV)
        flat = [(b, p) for b, s in enumerate(pos) for p in s]
        for r, (b, p) in enumerate(flat):
            if r not in skipped:
                lay.put(pages[table[b, p // 16]], p % 16, k[r].double().numpy(), v[r].double().numpy())
        cache, g = pk.make_qpool(dev, 3, n_pages), geom_of(pk, lay)
        ctx.cache_append(g, cache, 0, batch, k.to(DEV), v.to(DEV))
        assert ctx.query_status() == pk.E_BOUNDS
        assert np.array_equal(dev.cpu().numpy(), pages), what
        ko, vo = torch.full_like(k, 9.0, device=DEV), torch.full_like(v, 9.0, device=DEV)
        ctx.cache_read(g, cache, 0, batch, ko, vo)
        assert ctx.query_status() == (0 if what == "not_ascending" else pk.E_BOUNDS)
        for r, (b, p) in enumerate(flat):
            if r in skipped and what != "not_ascending":
                assert (ko[r] == 9).all() and (vo[r] == 9).all()
            else:
                kw, vw = lay.values(pages[table[b, p // 16]])
                assert torch.equal(ko[r].cpu(), torch.from_numpy(kw[p % 16]).float().to(BF16))
                assert torch.equal(vo[r].cpu(), torch.from_numpy(vw[p % 16]).float().to(BF16))


def test_infinite_scales_and_overflow(pk, ctx):
    """amax / qmax above 65504: an infinite scale and zero codes; an fp16 read of a value above 65504 is an infinity."""
    lay, case = Layout(3, 4, 64, 16, 32), Case([2], [2])
    rng = np.random.default_rng(5)
    table, n_pages = build_tables(case, 16, rng)
    batch, keep = device_batch(pk, case, table, DEV)
    k = random_rows(rng, 2, 4, 64, BF16)
    k[0, 0, 3], k[1, 1, 40] = 1.0e30, 400000.0
    pages = np.zeros((n_pages, lay.page_bytes()), np.uint8)
    dev = torch.from_numpy(pages).to(DEV)
    reference_append(lay, pages, case, table, k, k)
    cache, g = pk.make_qpool(dev, 3, n_pages), geom_of(pk, lay)
    ctx.cache_append(g, cache, 0, batch, k.to(DEV), k.to(DEV))
    assert np.array_equal(dev.cpu().numpy(), pages)
    ko, vo = torch.zeros((2, 4, 64), dtype=F16, device=DEV), torch.zeros((2, 4, 64), dtype=F16, device=DEV)
    ctx.cache_read(g, cache, 0, batch, ko, vo)
    assert ctx.query_status() == 0
    assert torch.isnan(ko[0, 0, :32]).all()            # 0 * inf
    assert torch.isinf(ko[1, 1, 40]) and torch.isfinite(ko[1, 0]).all()


def test_refusals(pk, ctx):
    lay, case = Layout(3, 4, 64, 16, 32), Case([20], [3])
    rng = np.random.default_rng(5)
    table, n_pages = build_tables(case, 16, rng)
    batch, keep = device_batch(pk, case, table, DEV)
    dev = torch.zeros((n_pages, lay.page_bytes()), dtype=torch.uint8, device=DEV)
    k = torch.ones((3, 4, 64), dtype=BF16, device=DEV)
    cache, g = pk.make_qpool(dev, 3, n_pages), geom_of(pk, lay)

    def refused(code=pk.E_INVALID, geom=g, cache=cache, layer=0, batch=batch, k=k, v=k, read=False):
        f = ctx.cache_read if read else ctx.cache_append
        assert f(geom, cache, layer, batch, k, v, check=False) == code

    for read in (False, True):
        refused(layer=1, read=read)
        refused(layer=-1, read=read)
        refused(cache=pk.make_qpool(dev, 0, n_pages), read=read)
        refused(cache=pk.make_qpool(dev, 4, n_pages), read=read)
        refused(cache=pk.make_qpool(dev, 3, 0), read=read)
        refused(cache=pk.make_qpool(dev, 3, n_pages, stride_page=lay.page_bytes() - 16), read=read)
        refused(cache=pk.make_qpool(dev, 3, n_pages, stride_page=lay.page_bytes() + 8), read=read)
        refused(cache=pk.make_qpool(dev.view(-1)[8:-8].view(1, -1), 3, 1, stride_page=lay.page_bytes()), read=read)
        for field, value in (("n_seqs", -1), ("n_rows", -1), ("row_start", None), ("kv_len", None), ("block_table", None),
                             ("struct_size", 8)):
            bad = pk.Batch.from_buffer_copy(batch)
            setattr(bad, field, value)
            refused(batch=bad, read=read)
        for field, value in (("head_dim", 63), ("group", 24), ("group", 0), ("n_kv_heads", 0), ("page_tokens", 0), ("struct_size", 0)):
            bad = pk.Geom.from_buffer_copy(g)
            setattr(bad, field, value)
            rows = pk.Rows(C.sizeof(pk.Rows), 0, k.data_ptr(), k.data_ptr(), 256, 64)
            f = pk.lib().patchkv_cache_read if read else pk.lib().patchkv_cache_append
            assert f(ctx._h, C.byref(bad), C.byref(cache), 0, C.byref(batch), C.byref(rows), None) == pk.E_INVALID
    wide = pk.make_geom(1, 1 << 14, 256, 256, 0, 1e4, 16, 1 << 10, 32)
    rows = pk.Rows(C.sizeof(pk.Rows), 0, k.data_ptr(), k.data_ptr(), 256, 64)
    assert pk.lib().patchkv_cache_read(ctx._h, C.byref(wide), C.byref(cache), 0, C.byref(batch), C.byref(rows), None) == pk.E_UNSUPPORTED
    # rows of the output that overlap, an unknown type, null rows
    for rows in (pk.Rows(C.sizeof(pk.Rows), 0, k.data_ptr(), k.data_ptr(), 64, 64), pk.Rows(C.sizeof(pk.Rows), 0, k.data_ptr(), k.data_ptr(), 256, 32),
                 pk.Rows(C.sizeof(pk.Rows), 2, k.data_ptr(), k.data_ptr(), 256, 64), pk.Rows(C.sizeof(pk.Rows), 0, None, k.data_ptr(), 256, 64),
                 pk.Rows(C.sizeof(pk.Rows), 0, k.data_ptr() + 1, k.data_ptr(), 256, 64), pk.Rows(C.sizeof(pk.Rows), 0, k.data_ptr(), k.data_ptr(), -1, 64),
                 pk.Rows(4, 0, k.data_ptr(), k.data_ptr(), 256, 64)):
        assert pk.lib().patchkv_cache_read(ctx._h, C.byref(g), C.byref(cache), 0, C.byref(batch), C.byref(rows), None) == pk.E_INVALID
    with pytest.raises(ValueError):
        ctx.cache_append(g, cache, 0, batch, k.float(), k.float())
    with pytest.raises(ValueError):
        ctx.cache_append(g, cache, 0, batch, k[:, :2], k[:, :2])
    empty = pk.Batch.from_buffer_copy(batch)
    empty.n_rows = 0
    assert ctx.cache_append(g, cache, 0, empty, k, k) == 0
    torch.cuda.synchronize()
    assert ctx.query_status() == 0 and (dev == 0).all()


def test_pages_past_4_gib(pk, ctx):
    """Page offsets beyond 32 bits: two pages of a pool whose page stride is 3 GiB apart."""
    lay, case = Layout(3, 4, 64, 16, 32), Case([33], [33])
    stride = 3 << 30
    dev = torch.empty(2 * stride + lay.page_bytes(), dtype=torch.uint8, device=DEV)
    for i in range(3):
        dev[i * stride:i * stride + lay.page_bytes()] = 0
    rng = np.random.default_rng(5)
    table = np.array([[2, 0, 1]], dtype=np.int32)
    batch, keep = device_batch(pk, case, table, DEV)
    k = random_rows(rng, 33, 4, 64, BF16)
    pages = np.zeros((3, lay.page_bytes()), np.uint8)
    reference_append(lay, pages, case, table, k, k)
    cache, g = pk.make_qpool(dev.view(1, -1), 3, 3, stride_page=stride), geom_of(pk, lay)
    ctx.cache_append(g, cache, 0, batch, k.to(DEV), k.to(DEV))
    ko, vo = torch.zeros_like(k, device=DEV), torch.zeros_like(k, device=DEV)
    ctx.cache_read(g, cache, 0, batch, ko, vo)
    assert ctx.query_status() == 0
    for i in range(3):
        assert np.array_equal(dev[i * stride:i * stride + lay.page_bytes()].cpu().numpy(), pages[i])
    kw, vw = reference_read(lay, pages, case, table, BF16)
    assert torch.equal(ko.cpu(), kw) and torch.equal(vo.cpu(), vw)


def test_captured_and_replayed_with_other_contents(pk, ctx):
    lay, case = Layout(3, 4, 64, 16, 32), Case([30, 9], [1, 1])
    rng = np.random.default_rng(5)
    table, n_pages = build_tables(Case([64, 64], [1, 1]), 16, rng)
    batch, keep = device_batch(pk, case, table, DEV, max_kv=64)
    pages = np.zeros((n_pages, lay.page_bytes()), np.uint8)
    dev = torch.from_numpy(pages).to(DEV)
    cache, g = pk.make_qpool(dev, 3, n_pages), geom_of(pk, lay)
    k = random_rows(rng, 2, 4, 64, BF16)
    kd = k.to(DEV)
    ko, vo = torch.zeros_like(kd), torch.zeros_like(kd)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        ctx.cache_append(g, cache, 0, batch, kd, kd)
        ctx.cache_read(g, cache, 0, batch, ko, vo)
    for step in range(3):
        graph.replay()
        reference_append(lay, pages, case, table, k, k)
        torch.cuda.synchronize()
        assert np.array_equal(dev.cpu().numpy(), pages)
        kw, vw = reference_read(lay, pages, case, table, BF16)
        assert torch.equal(ko.cpu(), kw) and torch.equal(vo.cpu(), vw)
        k = random_rows(rng, 2, 4, 64, BF16)           # the next token of each sequence
        kd.copy_(k)
        case = Case([t + 1 for t in case.kv], [1, 1])
        keep["kv"] += 1
    assert ctx.query_status() == 0


@pytest.mark.parametrize("tag", [1, 2, 3])
def test_a_page_restores_as_a_record(pk, ctx, tag):
    """A page written by cache_append is a checkpoint record: patchkv_restore (delta 0) rebuilds it as cache_read reads it."""
    H, D, P, G, n = 4, 64, 16, 32, 64
    lay, case = Layout(tag, H, D, P, G), Case([n], [n])
    rng = np.random.default_rng(5)
    batch, keep = device_batch(pk, case, np.arange(4, dtype=np.int32)[None], DEV)
    dev = torch.zeros((4, lay.page_bytes()), dtype=torch.uint8, device=DEV)
    cache, g = pk.make_qpool(dev, tag, 4), geom_of(pk, lay)
    k, v = random_rows(rng, n, H, D, BF16).to(DEV), random_rows(rng, n, H, D, BF16).to(DEV)
    ctx.cache_append(g, cache, 0, batch, k, v)
    ctx.cache_read(g, cache, 0, batch, k, v)
    kp, vp = torch.zeros((1, 4, P, H, D), dtype=BF16, device=DEV), torch.zeros((1, 4, P, H, D), dtype=BF16, device=DEV)
    pool = pk.make_pool(kp, vp, 4, kp.stride()[:4])
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    keep2 = dict(block_table=i32([0, 1, 2, 3]), tags=torch.full((1, 4), tag, dtype=torch.uint8, device=DEV),
                 blk_off=torch.arange(4, device=DEV).view(1, 4) * lay.page_bytes(), layer_payload=torch.tensor([dev.data_ptr()], device=DEV),
                 layer_bytes=torch.tensor([dev.numel()], device=DEV), reuse_idx=i32([[0, 1, 2, 3]]), reuse_cnt=i32([4]))
    ctx.restore(g, pool, [pk.make_session(n_suffix_tokens=n, delta=0, dst_shift=0, **keep2)])
    assert ctx.query_status() == 0
    assert torch.equal(kp.view(n, H, D), k) and torch.equal(vp.view(n, H, D), v)
