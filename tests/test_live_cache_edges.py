"""CPU checks of the live-cache calls: what their kernels may use, and workspace sizes at the ends of the range."""
import ctypes
import os

import pytest
import torch

from test_live_cache import pk  # noqa: F401  (fixture)

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_26219_b200", "csrc")


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.startswith(("attention", "cache", "live"))))
def test_no_read_only_loads(name):
    """The kernels come onto the SMs while the one in front of them still writes what they will read (dependent launches), so
    loads that ask for memory that does not change while the kernel is there are not theirs to make."""
    text = open(os.path.join(CSRC, name)).read()
    assert "__ldg" not in text and "global.nc" not in text and "__restrict__" not in text


def size(pk, geom, tag, hq, window=0, sinks=0, **batch):
    fields = dict(struct_size=ctypes.sizeof(pk.Batch), n_seqs=1, n_rows=1, max_rows=1, max_kv_len=16384, table_stride=4,
                  row_start=16, kv_len=16, block_table=16)
    b = pk.Batch(**{**fields, **batch})
    return pk.lib().patchkv_attention_workspace_bytes(ctypes.byref(geom), tag, ctypes.byref(b), hq, window, sinks)


@pytest.mark.parametrize("rows", [40, 60])
def test_workspace_of_the_longest_bound(pk, rows):
    """max_kv_len is a bound, and 2^31 - 1 is one: the tokens are split as for any long context."""
    g = pk.make_geom(1, 2, 64, 64, 0, 1e4, 16, 16, 32)
    long = size(pk, g, 3, 4, n_rows=rows, max_rows=rows, max_kv_len=1 << 24)
    assert long > 0
    for kv in (2 ** 31 - 1, 2 ** 31 - 127, 2 ** 31 - 128):
        assert size(pk, g, 3, 4, n_rows=rows, max_rows=rows, max_kv_len=kv) == long


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_workspace_size_needs_no_arrays(pk, rows):
    """The size follows from numbers alone, so it can be asked for before the device arrays exist."""
    g = pk.make_geom(1, 2, 64, 64, 0, 1e4, 16, 16, 32)
    for tag in (0, 3):
        want = size(pk, g, tag, 4, n_rows=rows, max_rows=rows)
        assert want > 0
        assert size(pk, g, tag, 4, n_rows=rows, max_rows=rows, row_start=None, kv_len=None, block_table=None) == want


def test_a_pool_has_no_more_pages_than_its_tensor(pk):
    """With the tensor's own strides; a pool laid out by given strides may have any number."""
    pages = torch.zeros((2, 3, 64), dtype=torch.uint8)
    for t in (pages, pages[0]):
        assert pk.make_qpool(t, 3, 3).n_pages == 3
        with pytest.raises(ValueError):
            pk.make_qpool(t, 3, 4)
    assert pk.make_qpool(pages.view(1, -1), 3, 6, stride_page=64).n_pages == 6


def test_images_where_they_pay(pk):
    """Operands are laid out in the workspace for two CTAs of query vectors over quantised pages, for eight over bf16 pages."""
    g = pk.make_geom(1, 1, 64, 64, 0, 1e4, 16, 16, 32)
    kv, image = 16384, 16384 * 64 * 2
    for tag, tiles in ((0, 8), (1, 2), (2, 2), (3, 2)):
        without, with_ = (size(pk, g, tag, 1, n_rows=n, max_rows=n, max_kv_len=kv) for n in ((tiles - 1) * 256, (tiles - 1) * 256 + 1))
        assert with_ - without > image and without < image * 74
        assert size(pk, g, tag, 1, n_rows=256 * 148, max_rows=256 * 148, max_kv_len=kv) >= 2 * image
