"""hook_rope against the 64-bit definition, and its cache write against hook_kv_write bit for bit (needs an MI355X)."""
import math

import pytest
import torch

from oracle import generation as G
from paper_2603_06588_amd import binding
from helpers import bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def freqs(r, base=10000.0):
    return (base ** (-torch.arange(r // 2, dtype=torch.float64) * 2 / max(r, 1))).float()


def check(got, x, want, r, magnitude=1.0, neighbours=False, far=0):
    """|error| <= 5e-7 m (|x1| + |x2|) for the fp32 rotation - the angle in fp32 half turns 9.4e-8, a sine 1.2e-7, its magnitude 6e-8,
    product and sum 1.2e-7 - and half a step of the storage type.  Far positions: an angle of that many radians is rounded
    twice by the kernel and once by the definition."""
    half_step = torch.finfo(got.dtype).eps / 2
    got, x = got.detach().cpu().double(), x.detach().cpu().double()
    n = r // 2
    both = torch.zeros_like(x)
    lo, hi = (slice(0, r, 2), slice(1, r, 2)) if neighbours else (slice(0, n), slice(n, r))
    s = x[..., lo].abs() + x[..., hi].abs()
    both[..., lo], both[..., hi] = s, s
    slack = (5e-7 + 3 * 2.0 ** -53 * far) * magnitude * both
    over = (got - want).abs() - slack - half_step * (want.abs() + slack)
    assert float(over.max()) <= 0, f"beyond the bound by {float(over.max()):.3e}"


def inputs(T, hq, hkv, d, dtype, seed=0, far=1000, axes=1):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn((T, h, d), generator=g).to(dtype) for h in (hq, hkv, hkv))
    pos = torch.randint(-5, far, (axes, T), generator=g).int()
    return q, k, v, pos


@pytest.mark.parametrize("T,hq,hkv,d,r", [(1, 1, 1, 64, 64), (3, 32, 8, 128, 128), (17, 6, 2, 128, 64), (5, 5, 1, 80, 80), (2, 3, 3, 80, 48), (9, 2, 1, 72, 36),
                                          (4, 2, 2, 6, 2), (7, 1, 1, 10, 10), (2, 1, 1, 512, 512), (33, 4, 4, 64, 0), (6, 2, 1, 13, 4), (130, 16, 2, 128, 128),
                                          (700, 3, 2, 128, 50), (650, 2, 1, 96, 94), (3, 9, 3, 33, 32), (5, 1, 1, 127, 126), (2, 2, 2, 24, 20)])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_against_the_definition(T, hq, hkv, d, r, neighbours, dtype):
    q, k, _, pos = inputs(T, hq, hkv, d, dtype, seed=T + d + r)
    f = freqs(r)
    q_out = torch.full_like(q, float("nan"), device=DEV)
    k_out = torch.full_like(k, float("nan"), device=DEV)
    binding.hook_rope(q.to(DEV), k.to(DEV), pos.to(DEV), f.to(DEV), layout=int(neighbours), q_out=q_out, k_out=k_out)
    for got, x in ((q_out, q), (k_out, k)):
        check(got, x, G.rope(x, pos, f, neighbours=neighbours), r, neighbours=neighbours)
        assert torch.equal(bits(got[..., r:]), bits(x[..., r:]))
    # the same bits in place
    qi, ki = q.to(DEV), k.to(DEV)
    binding.hook_rope(qi, ki, pos.to(DEV), f.to(DEV), layout=int(neighbours))
    assert torch.equal(bits(qi), bits(q_out)) and torch.equal(bits(ki), bits(k_out))


@pytest.mark.parametrize("axes,sections,cyclic", [(1, (32,), True), (2, (20, 12), False), (3, (12, 10, 10), True), (3, (8, 12, 12), False),
                                                  (4, (8, 8, 8, 8), True), (3, (32, 0, 0), True), (3, (0, 31, 1), False)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_axes(axes, sections, cyclic, dtype):
    q, k, _, pos = inputs(11, 4, 2, 80, dtype, seed=axes, axes=axes, far=60)
    f = freqs(64)
    qo, ko = binding.hook_rope(q.to(DEV), k.to(DEV), pos.to(DEV), f.to(DEV), axis_pairs=sections, axis_order=int(cyclic))
    check(qo, q, G.rope(q, pos, f, sections, cyclic=cyclic), 64)
    check(ko, k, G.rope(k, pos, f, sections, cyclic=cyclic), 64)


@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 1])
def test_far_positions(far):
    q, k, _, pos = inputs(64, 2, 1, 64, F32, seed=5, far=far)
    f = freqs(64)
    qo, _ = binding.hook_rope(q.to(DEV), k.to(DEV), pos.to(DEV), f.to(DEV))
    check(qo, q, G.rope(q, pos, f), 64, far=far)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_inverse_and_magnitude(dtype):
    q, k, _, pos = inputs(9, 4, 4, 64, dtype, seed=8)
    f = freqs(32)
    qo, _ = binding.hook_rope(q.to(DEV), k.to(DEV), pos.to(DEV), f.to(DEV), inverse=True, magnitude=1.25, q_out=torch.empty_like(q, device=DEV),
                              k_out=torch.empty_like(k, device=DEV))
    check(qo, q, G.rope(q, pos, f, inverse=True, magnitude=1.25), 32, magnitude=1.25)
    # there and back again: two roundings
    x = q.to(DEV)
    binding.hook_rope(x, None, pos.to(DEV), f.to(DEV))
    binding.hook_rope(x, None, pos.to(DEV), f.to(DEV), inverse=True)
    pair = torch.cat([(q[..., :16].abs() + q[..., 16:32].abs())] * 2 + [q[..., 32:].abs()], dim=-1).double()
    assert float(((x.cpu().double() - q.double()).abs() - (2 * torch.finfo(dtype).eps + 2e-6) * pair).max()) <= 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shift", [0, 1, 2, 8])
def test_views_alignment_and_untouched_surroundings(dtype, shift):
    """Queries, keys and values side by side in one buffer that starts `shift` elements into its memory; outputs into another."""
    T, hq, hkv, d = 7, 4, 2, 64
    q, k, v, pos = inputs(T, hq, hkv, d, dtype, seed=shift)
    width = (hq + 2 * hkv) * d + shift
    flat = torch.full((shift + T * width,), 7.0, dtype=dtype)
    rows = flat[shift:].view(T, width)
    rows[:, :hq * d], rows[:, hq * d:(hq + hkv) * d], rows[:, (hq + hkv) * d:(hq + 2 * hkv) * d] = q.flatten(1), k.flatten(1), v.flatten(1)
    g = flat.to(DEV)
    part = g[shift:].view(T, width)
    gq, gk = part[:, :hq * d].view(T, hq, d), part[:, hq * d:(hq + hkv) * d].view(T, hkv, d)
    f = freqs(64)
    binding.hook_rope(gq, gk, pos.to(DEV), f.to(DEV))
    check(gq, q, G.rope(q, pos, f), 64)
    check(gk, k, G.rope(k, pos, f), 64)
    assert torch.equal(bits(g[:shift]), bits(flat[:shift])) and torch.equal(bits(part[:, (hq + hkv) * d:]), bits(rows[:, (hq + hkv) * d:]))


@pytest.mark.parametrize("T", [4095, 4096, 5003])
def test_many_tokens(T):
    q, k, _, pos = inputs(T, 3, 1, 64, BF, seed=T)
    f = freqs(64)
    qo, ko = binding.hook_rope(q.to(DEV), k.to(DEV), pos.to(DEV), f.to(DEV))
    check(qo, q, G.rope(q, pos, f), 64)
    check(ko, k, G.rope(k, pos, f), 64)


def batch(new, prior, seed=0, mb_extra=1):
    """Tables of sequences with `new` tokens behind `prior` ones, pages in random order."""
    g = torch.Generator().manual_seed(seed)
    L = [a + b for a, b in zip(new, prior)]
    need = [-(-x // 16) for x in L]
    ids = torch.randperm(sum(need) + 3, generator=g).int()
    table = torch.full((len(new), max(need) + mb_extra), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = ids[at:at + n]
        at += n
    cu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32)
    return table, torch.tensor(L, dtype=torch.int32), cu, sum(need) + 3


def fused_and_apart(q, k, v, pos, f, table, lens, cu, blocks, kv8, **kw):
    """(caches, q, k) of the one call and of hook_rope followed by hook_kv_write."""
    T, hkv, d = k.shape
    g = torch.Generator().manual_seed(1)
    start = torch.randint(0, 100, (2, blocks, hkv, 16, d), generator=g).to(torch.uint8 if kv8 else k.dtype).to(DEV)
    scales = {"k_scale": torch.linspace(0.004, 0.02, hkv).to(DEV), "v_scale": torch.linspace(0.02, 0.01, hkv).to(DEV)} if kv8 else {}
    args = [t.to(DEV) for t in (table, lens, cu)]
    q, k, v, pos, f = (t.to(DEV) for t in (q, k, v, pos, f))
    one, two = start.clone(), start.clone()
    k_before = k.clone()
    q1, k1 = binding.hook_rope(q, k, pos, f, v=v, block_table=args[0], seq_lens=args[1], cu_q_lens=args[2], k_cache=one[0], v_cache=one[1],
                               q_out=torch.empty_like(q), **scales, **kw)
    assert k1 is None and torch.equal(bits(k), bits(k_before))
    k_out = torch.empty_like(k)
    third = start.clone()
    binding.hook_rope(q, k, pos, f, v=v, block_table=args[0], seq_lens=args[1], cu_q_lens=args[2], k_cache=third[0], v_cache=third[1],
                      q_out=torch.empty_like(q), k_out=k_out, **scales, **kw)
    q2, k2 = binding.hook_rope(q, k, pos, f, q_out=torch.empty_like(q), k_out=torch.empty_like(k), **kw)
    binding.hook_kv_write(k2, v, args[0], args[1], args[2], two[0], two[1], **scales)
    same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))  # noqa: E731
    assert torch.equal(bits(q1), bits(q2)) and torch.equal(bits(k_out), bits(k2))
    assert same(one, two) and same(third, two)
    return one, start


@pytest.mark.parametrize("kind", ["bf16", "f32", "kv8"])
@pytest.mark.parametrize("new,prior", [([1], [0]), ([1, 1, 1], [15, 16, 40]), ([5, 0, 33, 1], [3, 20, 15, 0]), ([1] * 70, [9] * 70), ([700, 17], [13, 0])])
def test_cache_write_is_that_of_the_two_calls(kind, new, prior):
    dtype = F32 if kind == "f32" else BF
    table, lens, cu, blocks = batch(new, prior, seed=len(new))
    q, k, v, pos = inputs(sum(new), 8, 2, 128, dtype, seed=3)
    one, start = fused_and_apart(q, k, v, pos, freqs(128), table, lens, cu, blocks, kind == "kv8")
    assert not torch.equal(one, start)


@pytest.mark.parametrize("kind", ["bf16", "kv8"])
@pytest.mark.parametrize("d,r", [(80, 40), (64, 20), (128, 6), (128, 50), (48, 34), (16, 14)])
@pytest.mark.parametrize("layout", [binding.ROPE_HALVES, binding.ROPE_NEIGHBOURS])
def test_cache_write_of_odd_units(kind, d, r, layout):
    table, lens, cu, blocks = batch([4, 9], [14, 7])
    q, k, v, pos = inputs(13, 3, 1, d, BF, seed=d)
    fused_and_apart(q, k, v, pos, freqs(r), table, lens, cu, blocks, kind == "kv8", layout=layout)


@pytest.mark.parametrize("kind", ["bf16", "kv8"])
def test_cache_write_while_keys_turn_in_place(kind):
    """k_out is k: the keys in the cache are those of the two calls, with whole vectors and with parts of one."""
    for d, r in ((64, 64), (64, 38)):
        table, lens, cu, blocks = batch([3, 5], [20, 2])
        q, k, v, pos = (t.to(DEV) for t in inputs(8, 4, 2, d, BF, seed=r))
        f, args = freqs(r).to(DEV), [t.to(DEV) for t in (table, lens, cu)]
        caches = torch.zeros((2, 2, blocks, 2, 16, d), dtype=torch.uint8 if kind == "kv8" else BF, device=DEV)
        scales = {"k_scale": torch.full((2,), 0.01, device=DEV), "v_scale": torch.full((2,), 0.02, device=DEV)} if kind == "kv8" else {}
        want_q, want_k = binding.hook_rope(q, k, pos, f, q_out=torch.empty_like(q), k_out=torch.empty_like(k))
        binding.hook_kv_write(want_k, v, *args, caches[0, 0], caches[0, 1], **scales)
        binding.hook_rope(q, k, pos, f, k_out=k, v=v, block_table=args[0], seq_lens=args[1], cu_q_lens=args[2], k_cache=caches[1, 0], v_cache=caches[1, 1], **scales)
        assert torch.equal(bits(q), bits(want_q)) and torch.equal(bits(k), bits(want_k)) and torch.equal(caches[0].view(torch.uint8), caches[1].view(torch.uint8))


def test_cache_write_drops_what_the_cache_write_drops():
    new, prior = [3, 4, 2, 5, 1], [0, 14, 10, 30, 2]
    table, lens, cu, blocks = batch(new, prior, mb_extra=0)
    table[0, 0] = -7                      # block ids outside the cache
    table[1, 1] = blocks
    lens[2] = 1                           # more new tokens than tokens
    lens[3] = 16 * table.shape[1] + 2     # beyond the table
    lens[4] = -1
    q, k, v, pos = inputs(sum(new), 4, 2, 64, BF, seed=9)
    fused_and_apart(q, k, v, pos, freqs(64), table, lens, cu, blocks, False)


@pytest.mark.parametrize("n", [64, 65, 4097])
def test_sequences_are_found_among_many(n):
    new = [(i * 7) % 3 for i in range(n)]
    table, lens, cu, blocks = batch(new, [i % 20 + 1 for i in range(n)], seed=n)
    q, k, v, pos = inputs(sum(new), 1, 1, 16, BF, seed=n)
    fused_and_apart(q, k, v, pos, freqs(16), table, lens, cu, blocks, False)


def test_nothing_to_turn_and_special_values():
    f = freqs(64).to(DEV)
    empty = torch.empty((0, 2, 64), dtype=BF, device=DEV)
    binding.hook_rope(empty, empty, torch.empty(0, dtype=torch.int32, device=DEV), f)
    x = torch.zeros((1, 1, 64), dtype=F32, device=DEV)
    x[0, 0, 3], x[0, 0, 5] = math.inf, math.nan
    y, _ = binding.hook_rope(x.clone(), None, torch.zeros(1, dtype=torch.int32, device=DEV), f)
    # angle 0: the partner of an infinity is inf * 0
    assert y[0, 0, 3] == math.inf and torch.isnan(y[0, 0, [5, 35, 37]]).all() and int(torch.isfinite(y).sum()) == 60


def test_other_stream_and_captured_graph():
    q, k, _, pos = inputs(40, 4, 2, 128, BF, seed=2)
    gq, gk, gp, f = q.to(DEV), k.to(DEV), pos.to(DEV), freqs(128).to(DEV)
    qo, ko = torch.empty_like(gq), torch.empty_like(gk)
    want = binding.hook_rope(gq, gk, gp, f, q_out=torch.empty_like(gq), k_out=torch.empty_like(gk))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.hook_rope(gq, gk, gp, f, q_out=qo, k_out=ko, stream=side)
    side.synchronize()
    assert torch.equal(bits(qo), bits(want[0])) and torch.equal(bits(ko), bits(want[1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.hook_rope(gq, gk, gp, f, q_out=qo, k_out=ko)
    for step in range(3):
        gp.add_(step)
        gq.mul_(-1)
        graph.replay()
        want = binding.hook_rope(gq, gk, gp, f, q_out=torch.empty_like(gq), k_out=torch.empty_like(gk))
        torch.cuda.synchronize()
        assert torch.equal(bits(qo), bits(want[0])) and torch.equal(bits(ko), bits(want[1]))


def test_refusals_of_the_binding():
    q, k, v, pos = (t.to(DEV) for t in inputs(4, 2, 1, 64, BF))
    f = freqs(64).to(DEV)
    for bad in (dict(q=q.half()), dict(positions=pos.long()), dict(inv_freq=f.double()), dict(positions=pos[:, :3].contiguous()), dict(k=k.float()),
                dict(k=k[:3]), dict(q=q.transpose(0, 1)), dict(q=q[:1].expand(4, 2, 64)), dict(axis_pairs=(16, 16)), dict(axis_pairs=(31,)),
                dict(q_out=torch.empty_like(k)), dict(v=v, k_cache=torch.zeros((2, 1, 16, 64), dtype=BF, device=DEV)),
                dict(inv_freq=torch.ones(40, device=DEV))):
        args = {**dict(q=q.clone(), k=k.clone(), positions=pos, inv_freq=f), **bad}
        with pytest.raises(binding.HookError):
            binding.hook_rope(args.pop("q"), args.pop("k"), args.pop("positions"), args.pop("inv_freq"), **args)


def test_there_and_back_with_a_magnitude():
    """The way back of a scaled rotation takes one over the magnitude.  With s = |x1| + |x2|: the first pass is off by e <= (5e-7 + 2^-24) m s in each
    element, which the second makes 2 e / m at most; its own error is 5e-7 / m of a pair of at most 2 m s, half a step of a result of about s, and
    half a step of 1 / m in fp32: (4 * 5e-7 + 5 * 2^-24) s together."""
    q, _, _, pos = inputs(9, 4, 4, 64, F32, seed=18)
    f, m = freqs(64).to(DEV), 1.25
    x = q.to(DEV)
    binding.hook_rope(x, None, pos.to(DEV), f, magnitude=m)
    binding.hook_rope(x, None, pos.to(DEV), f, inverse=True, magnitude=1 / m)
    s = torch.cat([q[..., :32].abs() + q[..., 32:].abs()] * 2, dim=-1).double()
    assert float(((x.cpu().double() - q.double()).abs() - (4 * 5e-7 + 5 * 2.0 ** -24) * s).max()) <= 0
