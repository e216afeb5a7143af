"""Calls on a stream that is not the current one, without outputs or scratch of the caller's: memory comes from that stream, and results are those of
the current one (needs an MI355X)."""
import pytest
import torch

from paper_2603_06588_amd import binding, workloads as W
from helpers import bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture
def taken(monkeypatch):
    """The streams that were current where memory was taken."""
    streams = []
    for name in ("empty", "empty_like"):
        def noted(*a, make=getattr(torch, name), **kw):
            streams.append(torch.cuda.current_stream())
            return make(*a, **kw)
        monkeypatch.setattr(binding.torch, name, noted)
    return streams


def calls(b):
    heads = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    cu = torch.cat([torch.zeros(1, dtype=torch.int32, device=DEV), b.seq_lens.cumsum(0).int()])
    mass = torch.rand((3, 2, 4, 5), device=DEV)
    return {
        "attn_probe": lambda s: binding.hook_attn_probe_batch(b, s),
        "span_mass": lambda s: (binding.hook_span_mass_batch(b, s),),
        "capture_qk": lambda s: binding.hook_capture_qk(b.q, b.k_cache, b.block_table, b.seq_lens, b.cu_q_lens, b.probe_heads, b.max_sel_q, b.query_sel,
                                                        heads, cu, int(cu[-1]), stream=s),
        "reduce_mass": lambda s: (binding.hook_reduce_mass(mass, binding.REDUCE_SPAN_MEAN, stream=s),),
    }


@pytest.mark.parametrize("name", ["attn_probe", "span_mass", "capture_qk", "reduce_mass"])
def test_a_call_on_another_stream(name, taken):
    b = W.random_batch(91, [300, 700, 90], [300, 1, 1], 8, 2, 128, torch.bfloat16, num_probe_heads=4, max_sel_q=4, max_spans=2).to(DEV)
    call = calls(b)[name]
    want = call(None)
    torch.cuda.synchronize()
    del taken[:]
    side = torch.cuda.Stream()
    got = call(side)
    assert taken and all(s == side for s in taken) and torch.cuda.current_stream() != side
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(got, want))
    got = call(type("Handle", (), {"cuda_stream": side.cuda_stream}))      # a stream known by its handle alone
    assert all(s.cuda_stream == side.cuda_stream for s in taken)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(got, want))
