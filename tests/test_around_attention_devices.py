"""The binding of the calls around the attention refuses tensors that are not on the context's GPU before it takes an address.  Needs no
GPU: the library is replaced by one that may not be called, and tensors of a GPU by fake ones."""
import ctypes

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode


@pytest.fixture()
def pk(monkeypatch):
    from paper_2609_26219_b200 import binding

    class Library:
        def __getattr__(self, name):
            raise AssertionError(f"{name} was called")

    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(binding.Context, "close", lambda self: None)
    monkeypatch.setattr(binding.Context, "__del__", lambda self: None)
    return binding


@pytest.fixture()
def ctx(pk):
    c = object.__new__(pk.Context)
    c._h, c.device = ctypes.c_void_p(), 0
    return c


def good(device):
    """The tensors of all calls: 5 rows of 2 sequences, 2 KV heads and 4 query heads of 64 channels."""
    z = lambda *shape, t=torch.int32: torch.zeros(shape, dtype=t, device=device)
    b = torch.bfloat16
    return dict(k=z(5, 2, 64, t=b), v=z(5, 2, 64, t=b), q=z(5, 4, 64, t=b), q_out=z(5, 4, 64, t=b), rope_pos=z(5), mass=z(2, 40, t=torch.float32),
                mass_in=z(2, 40, t=torch.float32), workspace=z(1 << 16, t=torch.uint8), kv_len=z(2), budget=z(2), keep=z(2, 8), kept=z(2),
                mass_out=z(2, 8, t=torch.float32), src_table=z(2, 3), dst_table=z(2, 1))


CALLS = {"rotary_append": ["k", "v", "q", "q_out", "rope_pos"], "attention_mass": ["q", "mass", "mass_in", "workspace"],
         "evict_select": ["mass", "kv_len", "keep", "kept", "budget", "mass_out"], "cache_gather": ["keep", "kept", "kv_len", "src_table", "dst_table"]}


def call(pk, ctx, name, tensors):
    geom, pool = pk.make_geom(1, 2, 64, 64, 0, 1e4, 16, 16, 32), pk.Pool()
    batch = pk.Batch(ctypes.sizeof(pk.Batch), 2, 5, 3, 40, 3, 16, 16, None, 16)
    at = () if name == "evict_select" else (geom, pool, 0) if name == "cache_gather" else (geom, pool, 0, batch)
    getattr(ctx, name)(*at, **{n: tensors[n] for n in CALLS[name]})


@pytest.mark.parametrize("name,tensor", [(c, t) for c in CALLS for t in CALLS[c]])
@pytest.mark.parametrize("where", ["cpu", "cuda:1"])
def test_a_tensor_elsewhere_is_refused(pk, ctx, name, tensor, where):
    with FakeTensorMode():
        tensors = good("cuda:0")
        tensors[tensor] = good(where)[tensor]
        with pytest.raises(ValueError, match=tensor if tensor != "v" else "k and v|v:"):
            call(pk, ctx, name, tensors)


@pytest.mark.parametrize("name", list(CALLS))
def test_all_on_the_context_s_gpu_pass_these_checks(pk, ctx, name, monkeypatch):
    """What is reached behind them is the address of a tensor (fake ones have none) or the library."""
    class Reached(Exception):
        pass

    def reached(self):
        raise Reached

    with FakeTensorMode():
        tensors = good("cuda:0")
        monkeypatch.setattr(torch.Tensor, "data_ptr", reached)
        with pytest.raises(Reached):
            call(pk, ctx, name, tensors)


def test_a_workspace_with_gaps_is_refused(pk, ctx):
    with FakeTensorMode():
        tensors = good("cuda:0")
        tensors["workspace"] = torch.zeros((1, 16), dtype=torch.uint8, device="cuda:0").expand(1 << 16, 16)
        with pytest.raises(ValueError, match="workspace"):
            call(pk, ctx, "attention_mass", tensors)
