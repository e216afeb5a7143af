"""hook_steer_logits against the 64-bit definition (needs an MI355X)."""
import math
import random

import pytest
import torch

from oracle import generation as G
from paper_2603_06588_amd import binding
from helpers import bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def lists(rows, pad=0):
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + len(r))
    flat = [x for r in rows for x in r] + [0] * pad
    return flat, torch.tensor(cu, dtype=torch.int32, device=DEV)


class Case:
    """Inputs of one call, and what the definition makes of them."""

    def __init__(self, R, V, dtype, seed, hist=40, prompt=True, penalties=True, bias=0, masks=0, own_rows=False):
        r, g = random.Random(seed), torch.Generator().manual_seed(seed)
        self.logits = (torch.randn((R, V), generator=g) * 5).to(dtype)
        some = max(1, V // 3)
        self.history = [[r.choice([r.randrange(V), -1, V, 2 ** 31 - 1, -2 ** 31]) if r.random() < 0.1 else r.randrange(some)
                         for _ in range(r.randint(0, hist))] for _ in range(R)]
        self.prompt = [r.randint(-1, hist) for _ in range(R)] if prompt else None
        u = torch.rand((3, R), generator=g)
        self.rep, self.freq, self.pres = (0.5 + 1.5 * u[0], u[1] - 0.3, u[2] - 0.3) if penalties else (None, None, None)
        if penalties and R > 1:
            self.rep[0], self.freq[0], self.pres[0] = 1.0, 0.0, 0.0
        self.bias = [[(r.choice([r.randrange(V), r.randrange(min(V, 5)), -3, V + 1]), r.uniform(-20, 20)) for _ in range(r.randint(0, bias))] for _ in range(R)] if bias else None
        words = (V + 31) // 32
        self.mask = torch.randint(-(2 ** 31), 2 ** 31, (masks, words), generator=g).int() if masks else None
        if masks > 1:
            self.mask[1] = 0
        self.mask_rows = None if not masks or own_rows else [r.choice([-1, masks] + list(range(masks))) for _ in range(R)]

    def kwargs(self):
        kw = {}
        put = lambda x, dt: torch.tensor(x, dtype=dt, device=DEV)  # noqa: E731
        flat, cu = lists(self.history)
        if flat:
            kw.update(history=put(flat, torch.int32), cu_history=cu)
            if self.prompt is not None:
                kw["prompt_lens"] = put(self.prompt, torch.int32)
        if self.rep is not None:
            kw.update(repetition=self.rep.to(DEV), frequency=self.freq.to(DEV), presence=self.pres.to(DEV))
        if self.bias and any(self.bias):
            flat, cu = lists(self.bias)
            kw.update(cu_bias=cu, bias_ids=put([t for t, _ in flat], torch.int32), bias_values=put([v for _, v in flat], F32))
        if self.mask is not None:
            kw["mask"] = self.mask.to(DEV)
            if self.mask_rows is not None:
                kw["mask_rows"] = put(self.mask_rows, torch.int32)
        return kw

    def want(self):
        bias = [[(t, float(torch.tensor(v, dtype=F32))) for t, v in b] for b in self.bias] if self.bias else None
        prompt = None if self.prompt is None else [max(p, 0) for p in self.prompt]
        return G.steer_logits(self.logits, self.history, prompt, self.rep, self.freq, self.pres, bias, self.mask, self.mask_rows)

    def check(self, got):
        """Five fp32 roundings (division, product, two differences, sum) of values no larger than `size`, and half a step of the type."""
        want, got = self.want(), got.detach().cpu()
        x = self.logits.double().abs()
        most = max((len(h) for h in self.history), default=0)
        size = x * 2 + most * 0.7 + 1 + 20
        fine = torch.isfinite(want)
        assert torch.equal(torch.isneginf(got.double()), torch.isneginf(want))
        slack = 5 * 2.0 ** -24 * size
        over = (got.double() - want).abs() - slack - torch.finfo(got.dtype).eps / 2 * (want.abs() + slack)
        assert not fine.any() or float(over[fine].max()) <= 0, float(over[fine].max())
        # what nothing touches is the input's bits
        same = (want == self.logits.double()) & fine
        assert torch.equal(bits(got)[same], bits(self.logits)[same])


SIZES = [(1, 1), (1, 7), (2, 31), (3, 32), (2, 33), (5, 500), (2, 4095), (2, 4096), (3, 4097), (1, 8192), (2, 9001), (4, 16384), (1, 33000)]


@pytest.mark.parametrize("R,V", SIZES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_everything_at_once(R, V, dtype):
    c = Case(R, V, dtype, seed=R * 100000 + V, bias=12, masks=3)
    out = torch.full((R, V), float("nan"), dtype=dtype, device=DEV)
    x = c.logits.to(DEV)
    binding.hook_steer_logits(x, out=out, **c.kwargs())
    c.check(out)
    assert torch.equal(bits(x), bits(c.logits))
    assert binding.hook_steer_logits(x, **c.kwargs()) is x       # in place
    assert torch.equal(bits(x), bits(out))


@pytest.mark.parametrize("what", [dict(hist=0, penalties=False), dict(penalties=False), dict(prompt=False), dict(hist=3000), dict(hist=0, bias=300),
                                  dict(penalties=False, masks=1), dict(masks=5, own_rows=True), dict(hist=0, penalties=False, bias=5, masks=2)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_parts(what, dtype):
    c = Case(5, 1000, dtype, seed=len(str(what)), **what)
    out = torch.full((5, 1000), float("nan"), dtype=dtype, device=DEV)
    binding.hook_steer_logits(c.logits.to(DEV), out=out, **c.kwargs())
    c.check(out)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("stride,offset", [(1003, 0), (1008, 8), (1000, 1), (1024, 4)])
def test_padded_and_misaligned_rows(dtype, stride, offset):
    c = Case(4, 1000, dtype, seed=stride, bias=4, masks=2)
    wide = torch.full((offset + 4 * stride,), 3.0, dtype=dtype, device=DEV)
    rows = wide[offset:].view(4, stride)[:, :1000]
    rows.copy_(c.logits)
    before = wide.clone()
    binding.hook_steer_logits(rows, **c.kwargs())
    c.check(rows)
    pad = torch.ones_like(wide, dtype=torch.bool)
    pad[offset:].view(4, stride)[:, :1000] = False
    assert torch.equal(bits(wide[pad]), bits(before[pad]))       # what lies between and around the rows


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shift_in,shift_out,stride", [(0, 0, 1003), (3, 3, 1000), (1, 2, 1000), (0, 4, 1008), (5, 5, 1001)])
def test_rows_off_the_borders_of_16_bytes(dtype, shift_in, shift_out, stride):
    """Input and output rows that begin anywhere, alike or not, with masks that begin inside a word for them."""
    c = Case(9, 997, dtype, seed=shift_in + stride, bias=6, masks=4)
    a = torch.zeros(shift_in + 9 * stride, dtype=dtype, device=DEV)
    b = torch.full((shift_out + 9 * stride,), 2.0, dtype=dtype, device=DEV)
    x, y = a[shift_in:].view(9, stride)[:, :997], b[shift_out:].view(9, stride)[:, :997]
    x.copy_(c.logits)
    binding.hook_steer_logits(x, out=y, **c.kwargs())
    c.check(y)
    pad = torch.ones_like(b, dtype=torch.bool)
    pad[shift_out:].view(9, stride)[:, :997] = False
    assert bool((b[pad] == 2.0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_more_touched_tokens_than_are_listed(dtype):
    # nearly every token of a range occurs, and a bias list longer than a workgroup, with tokens named over and over
    c = Case(2, 20000, dtype, seed=4, hist=30000, bias=3000)
    c.history[1] = list(range(0, 20000, 2)) + [3] * 50
    c.prompt[1] = 7000
    out = torch.empty((2, 20000), dtype=dtype, device=DEV)
    binding.hook_steer_logits(c.logits.to(DEV), out=out, **c.kwargs())
    c.check(out)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_counts_beyond_16_bits(dtype):
    # 70000 generated tokens: one of them 40000 times, the rest spread over both halves of the range
    V = 17000
    h = [[5] * 100 + [16500] * 40000 + [t % V for t in range(30000)], [3, 16999]]
    c = Case(2, V, F32, seed=5, bias=40)
    c.logits = c.logits.to(dtype)
    c.history, c.prompt = h, [100, 1]
    c.rep, c.freq, c.pres = torch.tensor([1.5, 1.25]), torch.tensor([2.0 ** -10, 0.5]), torch.tensor([0.25, 0.75])
    out = torch.empty((2, V), dtype=dtype, device=DEV)
    binding.hook_steer_logits(c.logits.to(DEV), out=out, **c.kwargs())
    c.check(out)


def test_long_history_and_counts():
    # one token 20000 times, half of them in the prompt: 10000 * 0.125 is exact
    x = torch.zeros((1, 40000), device=DEV)
    h = torch.full((20000,), 39999, dtype=torch.int32, device=DEV)
    one = lambda v: torch.tensor([v], device=DEV)  # noqa: E731
    cu = torch.tensor([0, 20000], dtype=torch.int32, device=DEV)
    y = binding.hook_steer_logits(x, history=h, cu_history=cu, prompt_lens=torch.tensor([10000], dtype=torch.int32, device=DEV), frequency=one(0.125), presence=one(2.0))
    assert float(y[0, 39999]) == -1252.0 and int((y != 0).sum()) == 1


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinities_and_nan(dtype):
    x = torch.tensor([[math.inf, -math.inf, math.nan, 1.0, math.nan, -math.inf, 0.0, -0.0]] * 2, dtype=dtype, device=DEV)
    h = torch.arange(4, dtype=torch.int32, device=DEV)
    mask = torch.tensor([[0b11001111]], dtype=torch.int32, device=DEV)
    y = binding.hook_steer_logits(x, history=h, cu_history=torch.tensor([0, 4, 4], dtype=torch.int32, device=DEV), repetition=torch.tensor([2.0, 2.0], device=DEV),
                                  presence=torch.tensor([0.5, 0.5], device=DEV), mask=mask, mask_rows=torch.tensor([0, -1], dtype=torch.int32, device=DEV)).cpu()
    assert y[0, 0] == math.inf and y[0, 1] == -math.inf and torch.isnan(y[0, 2]) and y[0, 3] == 0.0
    assert y[0, 4] == -math.inf and y[0, 5] == -math.inf          # barred, whatever they were
    assert torch.isnan(y[1, 2]) and torch.isnan(y[1, 4]) and y[1, 3] == 1.0
    assert torch.signbit(y[0, 7]) and not torch.signbit(y[0, 6])


def test_lists_that_reach_outside_their_arrays():
    # prefix sums that fall, start below 0 or end behind the list are cut to it
    x = torch.ones((3, 64), device=DEV)
    h = torch.tensor([5, 6, 7], dtype=torch.int32, device=DEV)
    cu = torch.tensor([-4, 2, 1, 900], dtype=torch.int32, device=DEV)
    y = binding.hook_steer_logits(x.clone(), history=h, cu_history=cu, presence=torch.ones(3, device=DEV)).cpu()
    assert [r.nonzero()[:, 0].tolist() for r in 1 - y] == [[5, 6], [], [6, 7]]
    y = binding.hook_steer_logits(x.clone(), cu_bias=cu, bias_ids=h, bias_values=torch.ones(3, device=DEV)).cpu()
    assert [r.nonzero()[:, 0].tolist() for r in y - 1] == [[5, 6], [], [6, 7]]


def test_captured_graph_and_other_stream():
    c = Case(6, 5000, BF, seed=77, bias=8, masks=2)
    x, kw = c.logits.to(DEV), c.kwargs()
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.hook_steer_logits(x, out=out, stream=side, **kw)
    side.synchronize()
    c.check(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.hook_steer_logits(x, out=out, **kw)
    for _ in range(3):
        x.mul_(-0.5)
        kw["history"].add_(1).remainder_(5000)
        graph.replay()
        want = binding.hook_steer_logits(x, out=torch.empty_like(x), **kw)
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want))


def test_refusals_of_the_binding():
    x = torch.zeros((2, 64), device=DEV)
    i = torch.zeros(3, dtype=torch.int32, device=DEV)
    for bad in (dict(logits=x.half()), dict(logits=x[0]), dict(out=x[:1]), dict(logits=x.T), dict(history=i, cu_history=i[:2]), dict(history=i.long(), cu_history=i),
                dict(history=i), dict(repetition=i.float()), dict(cu_bias=i, bias_ids=i), dict(mask=i.view(1, 3)), dict(frequency=x[:, 0].double()),
                dict(logits=x[:1].expand(2, 64)), dict(presence=torch.zeros(2))):
        args = {**dict(logits=x), **bad}
        with pytest.raises(binding.HookError):
            binding.hook_steer_logits(args.pop("logits"), **args)
