"""Sizes that the C structs' 32 bits do not hold are refused by the Python calls, where ctypes would take them modulo 2^32: a history of 2^32 + 5 tokens
as one of 5, say.  Sizes are as the look at the tensors reports them; nothing is that large here (no GPU)."""
import pytest
import torch

from paper_2603_06588_amd import binding

WRAPS = 2 ** 32 + 16      # 16 in 32 bits


@pytest.fixture(autouse=True)
def launched(monkeypatch):
    binding.load_library()
    done = []
    monkeypatch.setattr(binding, "_launch", lambda fn, a, *rest: done.append(a))
    return done


class Shape:
    """A tensor of which only the sizes and the type are asked for."""

    def __init__(self, *shape, dtype=torch.int32):
        self.shape, self.dtype = shape, dtype

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return 2 if self.dtype == torch.bfloat16 else 4


def look(where, like, spec, *tensors):
    out = [0]
    for kind, t in zip(spec, tensors):
        sizes = () if t is None else tuple(t.shape)
        n = 0 if t is None else t.numel()
        out += {"i": [n and 4096, n], "f": [n and 4096, n], "c": [n and 4096, sizes], "r": [n and 4096, 0, sizes]}[kind[0]]
    return tuple(out)


def refused(call, launched, monkeypatch):
    monkeypatch.setattr(binding, "_look", look)
    with pytest.raises(binding.HookError) as e:
        call()
    assert e.value.status == 3 and not launched


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("what", [dict(history=Shape(WRAPS), cu_history=Shape(3)), dict(cu_bias=Shape(3), bias_ids=Shape(WRAPS), bias_values=Shape(WRAPS)),
                                  dict(mask=Shape(WRAPS, 2)), dict(logits=Shape(WRAPS, 64, dtype=BF)), dict(logits=Shape(2, WRAPS, dtype=BF))])
def test_logits(what, launched, monkeypatch):
    args = {**dict(logits=Shape(2, 64, dtype=BF)), **what}
    refused(lambda: binding.hook_steer_logits(**args), launched, monkeypatch)


@pytest.mark.parametrize("S,mb,nb,rows", [(WRAPS, 4, 8, 2), (2, WRAPS, 8, 2), (2, 4, WRAPS, 2), (2, 4, 8, WRAPS)])
def test_pages(S, mb, nb, rows, launched, monkeypatch):
    table, lens, refs, status = Shape(S, mb), Shape(S), Shape(nb), Shape(1)
    refused(lambda: binding.hook_pages_fork(Shape(rows), table, lens, refs, Shape(rows, mb), Shape(rows), status), launched, monkeypatch)
    if rows == 2:
        scratch = Shape(256)
        refused(lambda: binding.hook_pages_append(Shape(S + 1), table, lens, refs, [], status, workspace=scratch), launched, monkeypatch)
        refused(lambda: binding.hook_pages_compact(table, lens, refs, [], Shape(nb), Shape(1), status, workspace=scratch), launched, monkeypatch)


def test_heads_of_the_caches(launched, monkeypatch):
    cache = Shape(8, WRAPS, 16, 64, dtype=BF)
    refused(lambda: binding.hook_pages_append(Shape(3), Shape(2, 4), Shape(2), Shape(8), [cache], Shape(1), workspace=Shape(256)), launched, monkeypatch)


@pytest.mark.parametrize("T,hq,hkv,d,pairs", [(WRAPS, 2, 1, 64, 32), (4, WRAPS, 1, 64, 32), (4, 2, WRAPS, 64, 32), (4, 2, 1, WRAPS, 32), (4, 2, 1, 64, WRAPS // 2)])
def test_rope(T, hq, hkv, d, pairs, launched, monkeypatch):
    q, k = Shape(T, hq, d, dtype=BF), Shape(T, hkv, d, dtype=BF)
    refused(lambda: binding.hook_rope(q, k, Shape(T), Shape(pairs, dtype=F32)), launched, monkeypatch)


@pytest.mark.parametrize("S,mb,nb,B", [(WRAPS, 4, 8, 16), (2, WRAPS, 8, 16), (2, 4, WRAPS, 16), (2, 4, 8, WRAPS)])
def test_rope_into_a_cache(S, mb, nb, B, launched, monkeypatch):
    q, k, cache = Shape(4, 2, 64, dtype=BF), Shape(4, 1, 64, dtype=BF), Shape(nb, 1, B, 64, dtype=BF)
    refused(lambda: binding.hook_rope(q, k, Shape(4), Shape(32, dtype=F32), v=k, block_table=Shape(S, mb), seq_lens=Shape(S), cu_q_lens=Shape(S + 1), k_cache=cache,
                                      v_cache=cache), launched, monkeypatch)
