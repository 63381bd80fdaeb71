"""Gated delta rule and group norm called from several host threads at once, each on a stream of its own."""
import threading

import pytest
import torch

import paper_2405_18425_b200 as vig
from layer_helpers import T, gdr_forward, gdr_gradient, gdr_inputs

pytestmark = pytest.mark.gpu

# pairs of sizes that take the same kernels with very different amounts of shared memory: columns, segments, owners of a walk
PAIRS = [("bf16", (1, 2, 70, 32, 16), (2, 4, 70, 32, 128)), ("bf16", (1, 1, 900, 24, 16), (1, 2, 900, 24, 64)), ("f32", (1, 1, 40, 64, 8), (40, 8, 40, 64, 128))]


def _at_once(jobs, rounds):
    """Every job `rounds` times in a thread and stream of its own; what they raised."""
    raised, start = [], threading.Barrier(len(jobs))

    def work(job):
        try:
            stream = torch.cuda.Stream()
            start.wait()
            with torch.cuda.stream(stream):
                for _ in range(rounds):
                    job()
            stream.synchronize()
        except Exception as e:   # (reported by the test)
            raised.append(e)

    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return raised


@pytest.mark.parametrize("pair", PAIRS, ids=str)
def test_delta_rule(pair):
    dtype, *sizes = pair
    sets = [gdr_inputs(*size, dtype, seed=31, states=True) for size in sizes]
    want = [gdr_forward(d) + tuple(gdr_gradient(d)) for d in sets]
    got = [None, None]
    torch.cuda.synchronize()

    def job(i):
        got[i] = gdr_forward(sets[i]) + tuple(gdr_gradient(sets[i]))

    assert _at_once([lambda i=i: job(i) for i in (0, 1)], 150) == []
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_group_norm(dtype):
    sets = []
    for shape, groups in (((1, 4, 4, 96), 32), ((4, 40, 40, 96), 32)):
        x = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(T[dtype])
        sets.append((x, groups, torch.empty_like(x), torch.empty_like(x), *(torch.empty(shape[0], groups, device="cuda") for _ in range(2))))

    def job(x, groups, out, dx, mean, rstd):
        vig.vig_group_norm(x, None, None, out, groups, act="silu", mean=mean, rstd=rstd)
        vig.vig_group_norm_bwd(x, None, None, mean, rstd, x, dx, None, None, groups, act="silu")

    want = []
    for s in sets:
        job(*s)
        want.append((s[2].clone(), s[3].clone()))
    torch.cuda.synchronize()
    assert _at_once([lambda s=s: job(*s) for s in sets], 300) == []
    torch.cuda.synchronize()
    for s, (out, dx) in zip(sets, want):
        assert torch.equal(s[2], out) and torch.equal(s[3], dx)
