"""patchkv_cache_append and patchkv_cache_read on batches whose row_start entries are out of order, and every fp16 value."""
import numpy as np
import pytest
import torch

from live_common import BF16, F16, Case, Layout, build_tables, device_batch, random_rows
from test_gpu_live_cache import DEV, ctx, geom_of, pk, reference_append  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,D,G", [(4, 64, 32), (2, 10, 5)])
def test_a_sequence_that_starts_below_row_0_is_left_out(pk, ctx, H, D, G):
    """No position in front of the first one is looked at for its rows: they are skipped and latched.  (The array of positions
    has an entry in front of it here, one that would let row 0 pass.)"""
    lay, case = Layout(3, H, D, 16, G), Case([40, 40], [3, 2], [[0, 5, 39], [1, 2]])
    rng = np.random.default_rng(5)
    table, n_pages = build_tables(case, 16, rng)
    batch, keep = device_batch(pk, case, table, DEV)
    padded = torch.cat([torch.tensor([-5], dtype=torch.int32, device=DEV), keep["pos"]])
    batch.pos = padded[1:].data_ptr()
    keep["start"][0] = -1
    pages = rng.integers(0, 256, (n_pages, lay.page_bytes()), dtype=np.uint8)
    dev = torch.from_numpy(pages).to(DEV)
    k, v = random_rows(rng, 5, H, D, BF16), random_rows(rng, 5, H, D, BF16)
    cache, g = pk.make_qpool(dev, 3, n_pages), geom_of(pk, lay)
    ctx.cache_append(g, cache, 0, batch, k.to(DEV), v.to(DEV))
    assert ctx.query_status() == pk.E_BOUNDS
    for r, pos in ((3, 1), (4, 2)):                         # the other sequence's rows
        lay.put(pages[table[1, 0]], pos, k[r].double().numpy(), v[r].double().numpy())
    assert np.array_equal(dev.cpu().numpy(), pages)
    ko, vo = torch.full_like(k, 9.0, device=DEV), torch.full_like(v, 9.0, device=DEV)
    ctx.cache_read(g, cache, 0, batch, ko, vo)
    assert ctx.query_status() == pk.E_BOUNDS
    assert (ko[:3] == 9).all() and (vo[:3] == 9).all() and not (ko[3:] == 9).all(2).any()


@pytest.mark.parametrize("H,D,G", [(4, 64, 32), (2, 10, 5)])
@pytest.mark.parametrize("start", [[0, 3, 0], [0, 3, 2, 5], [0, 2, 9]])
def test_entries_out_of_order_are_latched(pk, ctx, H, D, G, start):
    """row_start that descends or runs past n_rows is an error of both calls; nothing but slots of the batch is written."""
    lay = Layout(3, H, D, 16, G)
    rng = np.random.default_rng(5)
    n_seqs, n = len(start) - 1, 5
    table, n_pages = build_tables(Case([40] * n_seqs, [1] * n_seqs), 16, rng)
    batch, keep = device_batch(pk, Case([40] * n_seqs, [1] * n_seqs), table, DEV, n_rows=n)
    keep["start"].copy_(torch.tensor(start, dtype=torch.int32))
    pages = rng.integers(0, 256, (n_pages, lay.page_bytes()), dtype=np.uint8)
    dev = torch.from_numpy(pages).to(DEV)
    k, v = random_rows(rng, n, H, D, BF16).to(DEV), random_rows(rng, n, H, D, BF16).to(DEV)
    cache, g = pk.make_qpool(dev, 3, n_pages), geom_of(pk, lay)
    ctx.cache_append(g, cache, 0, batch, k, v)
    assert ctx.query_status() == pk.E_BOUNDS
    unused = sorted(set(range(n_pages)) - set(table.reshape(-1).tolist()))
    assert np.array_equal(dev.cpu().numpy()[unused], pages[unused])
    ctx.cache_read(g, cache, 0, batch, k, v)
    assert ctx.query_status() == pk.E_BOUNDS
    keep["start"].copy_(torch.arange(n_seqs + 1, dtype=torch.int32))
    ctx.cache_append(g, cache, 0, batch, k, v)              # in order again: no error
    assert ctx.query_status() == 0


@pytest.mark.parametrize("bits_tag", [1, 3])
def test_every_fp16_value_as_group_maximum(pk, ctx, bits_tag):
    """Every positive finite fp16 value as the maximum of a group, with neighbours that fall on and next to the half-way points
    of its codes."""
    lay = Layout(bits_tag, 4, 64, 16, 32)
    top = 127 if bits_tag == 1 else 7
    m = torch.arange(1, 0x7C00, dtype=torch.int16).view(F16)
    n = -(-m.numel() // 8)
    m = torch.cat([m, m[:n * 8 - m.numel()]]).view(n, 8, 1)
    s = (m.double() / top).half().double()
    half = (torch.floor(torch.arange(31, dtype=torch.float64) * (top / 31.0)) + 0.5) * s
    x = torch.cat([m.double(), torch.minimum(half, m.double())], -1).to(F16).view(n, 4, 64)
    rng = np.random.default_rng(3)
    case = Case([n], [n])
    table, n_pages = build_tables(case, 16, rng)
    batch, keep = device_batch(pk, case, table, DEV)
    pages = np.zeros((n_pages, lay.page_bytes()), np.uint8)
    dev = torch.from_numpy(pages).to(DEV)
    reference_append(lay, pages, case, table, x, x)
    ctx.cache_append(geom_of(pk, lay), pk.make_qpool(dev, bits_tag, n_pages), 0, batch, x.to(DEV), x.to(DEV))
    assert ctx.query_status() == 0
    assert np.array_equal(dev.cpu().numpy(), pages)
