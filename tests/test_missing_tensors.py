"""Tensors that a call cannot do without are refused where they are missing, before anything is looked at or launched (no GPU)."""
import pytest
import torch

from paper_2603_06588_amd import binding


@pytest.fixture(autouse=True)
def no_launch(monkeypatch):
    launched = []
    binding.load_library()
    monkeypatch.setattr(binding, "_launch", lambda *a: launched.append(a))
    # every tensor is fine and holds what its kind says
    monkeypatch.setattr(binding, "_look", look)
    return launched


def look(where, like, spec, *tensors):
    out = [0]
    for kind, t in zip(spec, tensors):
        sizes = () if t is None else tuple(t.shape)
        n = 0 if t is None else t.numel()
        out += {"i": [n and 4096, n], "f": [n and 4096, n], "c": [n and 4096, sizes], "r": [n and 4096, 0, sizes]}[kind[0]]
    return tuple(out)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("missing", ["src_rows", "block_table_out", "seq_lens_out"])
def test_fork(missing, no_launch):
    """Without source rows the output table of the old one's shape fits, and every count of the old table would be taken down."""
    args = dict(src_rows=ints(2), block_table=ints(2, 3), seq_lens=ints(2), ref_counts=ints(6), block_table_out=ints(2, 3), seq_lens_out=ints(2), status=ints(1))
    binding.hook_pages_fork(**args)
    assert len(no_launch) == 1
    with pytest.raises(binding.HookError) as e:
        binding.hook_pages_fork(**{**args, missing: None})
    assert e.value.status == 1 and len(no_launch) == 1


@pytest.mark.parametrize("missing", ["positions", "inv_freq"])
def test_rope(missing, no_launch):
    """Without frequencies nothing would turn, and the call would report that all is well."""
    args = dict(q=torch.zeros(5, 2, 8), k=None, positions=ints(5), inv_freq=torch.ones(4))
    binding.hook_rope(**args)
    assert len(no_launch) == 1
    with pytest.raises(binding.HookError) as e:
        binding.hook_rope(**{**args, missing: None})
    assert e.value.status == 1 and len(no_launch) == 1
