"""Steps of sampled generation with the calls together: fork, append, rotation into the cache, hooked attention, adjusted logits, and now
and then a compaction.  Whatever the pages went through, every row reads back the keys and values that were written for it, and
its attention is bit for bit that over a cache of its own (needs an MI355X)."""
import random

import pytest
import torch

from oracle import generation as G
from paper_2603_06588_amd import binding
from helpers import bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HQ, HKV, D, V = 8, 2, 64, 211


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def own_cache(rows, nb_extra=1):
    """A cache and table in which every row has pages of its own, in order."""
    need = [-(-len(r) // 16) for r in rows]
    mb = max(need + [1])
    table = torch.zeros((len(rows), mb), dtype=torch.int32)
    k = torch.zeros((sum(need) + nb_extra, HKV, 16, D), dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    at = 0
    for i, r in enumerate(rows):
        table[i, :need[i]] = torch.arange(at, at + need[i])
        for t, (kr, vr) in enumerate(r):
            k[at + t // 16, :, t % 16], v[at + t // 16, :, t % 16] = kr, vr
        at += need[i]
    return table.to(DEV), k.to(DEV), v.to(DEV)


@pytest.mark.parametrize("seed", [0, 1, 2])
def test_steps(seed):
    r, g = random.Random(seed), torch.Generator().manual_seed(seed)
    layers, nb, mb = 2, 90, 12
    k_caches = [torch.full((nb, HKV, 16, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(layers)]
    v_caches = [torch.full((nb, HKV, 16, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(layers)]
    refs, status = ints([0] * nb), ints([0])
    freq = (1000.0 ** (-torch.arange(D // 2, dtype=torch.float64) * 2 / D)).float().to(DEV)
    S = 3
    table, lens = torch.zeros((S, mb), dtype=torch.int32, device=DEV), ints([0] * S)
    rows = [[[] for _ in range(S)] for _ in range(layers)]      # per layer and row: the (key, value) of each token, on the host
    history = [[] for _ in range(S)]
    for step in range(14):
        # some rows go on, some double, some end, some are cut back
        if step:
            want = r.randint(2, 7)
            src = [r.randrange(S) if r.random() < 0.9 else -1 for _ in range(want)]
            keep = [r.randint(1, 190) if r.random() < 0.3 else 10 ** 6 for _ in range(want)]
            new_table, new_lens = torch.full((want, mb), -9, dtype=torch.int32, device=DEV), ints([0] * want)
            binding.hook_pages_fork(ints(src), table, lens, refs, new_table, new_lens, status, src_lens=ints(keep))
            rows = [[list(layer[p][:k]) if p >= 0 else [] for p, k in zip(src, keep)] for layer in rows]
            history = [list(history[p][:k]) if p >= 0 else [] for p, k in zip(src, keep)]
            table, lens, S = new_table, new_lens, want
        new = [r.choice([0, 1, 1, 1, r.randint(1, 40)]) if len(rows[0][i]) else r.randint(1, 60) for i in range(S)]
        new = [min(n, mb * 16 - len(rows[0][i])) for i, n in enumerate(new)]
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        cu_dev, T = ints(cu), cu[-1]
        binding.hook_pages_append(cu_dev, table, lens, refs, k_caches + v_caches, status)
        assert int(status) == 0
        assert lens.tolist() == [len(x) + n for x, n in zip(rows[0], new)]
        if step % 4 == 3:
            page_map, live = ints([0] * nb), ints([0])
            binding.hook_pages_compact(table, lens, refs, k_caches + v_caches, page_map, live, status)
            held = {p for i, n in enumerate(lens.tolist()) for p in table[i, :-(-n // 16)].tolist()}
            assert held == set(range(int(live))) and int(status) == 0
        # every page is held by as many rows as its count says
        counts = [0] * nb
        for i, n in enumerate(lens.tolist()):
            for p in table[i, :-(-n // 16)].tolist():
                counts[p] += 1
        assert refs.tolist() == counts
        if T == 0:
            continue
        pos = [len(rows[0][i]) + t for i in range(S) for t in range(new[i])]
        for layer in range(layers):
            q, k, v = (torch.randn((T, h, D), generator=g).bfloat16().to(DEV) for h in (HQ, HKV, HKV))
            k_out = torch.empty_like(k)
            binding.hook_rope(q, k, ints(pos), freq, v=v, block_table=table, seq_lens=lens, cu_q_lens=cu_dev, k_cache=k_caches[layer],
                              v_cache=v_caches[layer], k_out=k_out)
            kc, vc = k_out.cpu(), v.cpu()
            for i in range(S):
                rows[layer][i] += [(kc[t], vc[t]) for t in range(cu[i], cu[i + 1])]
            t2, k2, v2 = own_cache(rows[layer])
            a, _ = binding.hook_attn_probe(q, k_caches[layer], v_caches[layer], table, lens, cu_dev)
            b, _ = binding.hook_attn_probe(q, k2, v2, t2, lens, cu_dev)
            assert torch.equal(bits(a), bits(b)), (step, layer)
            gathered = [torch.cat([k_caches[layer][p].transpose(0, 1) for p in table[i, :-(-n // 16)].tolist()])[:n] for i, n in enumerate(lens.tolist()) if n]
            wanted = [torch.stack([x for x, _ in row]) for row in rows[layer] if row]
            assert all(torch.equal(bits(x), bits(y)) for x, y in zip(gathered, wanted))
        # the next token of each row, under penalties
        logits = (torch.randn((S, V), generator=g) * 3).bfloat16()
        for i in range(S):
            history[i] += [r.randrange(V) for _ in range(new[i])]
        cu_h = [0]
        for h in history:
            cu_h.append(cu_h[-1] + len(h))
        rep, pres = torch.full((S,), 1.3), torch.full((S,), 0.7)
        mask = torch.randint(-2 ** 31, 2 ** 31, (S, (V + 31) // 32), generator=g).int()
        y = binding.hook_steer_logits(logits.to(DEV), history=ints([t for h in history for t in h]), cu_history=ints(cu_h), repetition=rep.to(DEV),
                                      presence=pres.to(DEV), mask=mask.to(DEV))
        w = G.steer_logits(logits, history, None, rep, None, pres, None, mask)
        # three fp32 roundings of values below 2 * |x| + 1, half a step of bf16
        slack = 3 * 2.0 ** -24 * (2 * logits.double().abs() + 1)
        fine = torch.isfinite(w)
        assert torch.equal(torch.isneginf(y.cpu().double()), ~fine)
        assert float(((y.cpu().double() - w).abs() - slack - 2.0 ** -8 * (w.abs() + slack))[fine].max()) <= 0


def test_host_threads_on_streams_of_their_own():
    """Three threads make the calls at once, each on its own stream with its own tensors."""
    import threading
    from test_gpu_pages import Pool, check_table, new_caches, run_append
    done, failed = [], []

    def job(seed):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                p = Pool(seed, 40, 12, 150, 200, share=0.8)
                start, status, cu = new_caches(p.nb, 2, 16, torch.bfloat16, 4, seed), ints([0]), list(range(41))
                x = torch.randn((9, 5000), device=DEV, generator=torch.Generator(DEV).manual_seed(seed)).bfloat16()
                h, cu_h = ints([(7 * seed + t) % 5000 for t in range(900)]), ints(list(range(0, 901, 100)))
                for _ in range(20):
                    caches = start.clone()
                    table, lens, refs = run_append(p, cu, caches, True, status)
                    y = binding.hook_steer_logits(x, out=torch.empty_like(x), history=h, cu_history=cu_h, presence=torch.ones(9, device=DEV))
                stream.synchronize()
                rows, L, counts, copies, _ = G.append(cu, p.table(), p.lens, p.refs)
                check_table(table, rows)
                for a, b, n in copies:
                    start[:, b, :, :n] = start[:, a, :, :n]
                assert lens.tolist() == L and refs.tolist() == counts and torch.equal(caches, start)
                want = x.clone()
                at = torch.arange(9, device=DEV).repeat_interleave(100), h.long()
                want[at] = (x[at].float() - 1).bfloat16()
                assert torch.equal(bits(y), bits(want))
            done.append(seed)
        except BaseException as e:      # (pytest does not see other threads' errors)
            failed.append(e)

    threads = [threading.Thread(target=job, args=(k,)) for k in (1, 2, 3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed and sorted(done) == [1, 2, 3], failed
