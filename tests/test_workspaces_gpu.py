"""The workspaces that the bindings bring themselves: threads that call on one stream, streams named in the call, and
the memory that is left behind."""
import threading

import pytest
import torch

from paper_2602_06935_amd import binding

pytestmark = pytest.mark.gpu


def programs(seed):
    """Calls of several launches that pass data through a workspace, on inputs of their own."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, device="cuda", generator=gen).to(dtype)

    q, k, v, dO = (normal(2, 2, 700, 64) for _ in range(4))
    g = -torch.rand(2, 2, 700, device="cuda", generator=gen)
    beta = torch.rand(2, 2, 700, device="cuda", generator=gen)
    S0 = normal(2, 2, 64, 64, dtype=torch.float32)
    ids = torch.randint(0, 300, (90, 100), device="cuda", generator=gen)
    dE = normal(90, 100, 32)
    aq, ak, av, ag = (normal(1, 2, 3000, 64) for _ in range(4))

    def segments(**kw):       # states of segments, then outputs
        S1 = torch.empty_like(S0)
        return binding.cotten_delta_fwd(q, k, v, g, beta, None, initial_state=S0, final_state=S1, **kw), S1

    def backward(**kw):       # forwards once more, two walks backwards, gradients
        return binding.cotten_delta_bwd(q, k, v, g, beta, None, dO, initial_state=S0, **kw)

    def table(**kw):          # sort, sums, joined sums
        return (binding.cotten_embed_bwd(ids, dE, 300, **kw),)

    def attention(**kw):      # partial states, then outputs
        O = binding.cotten_attn_fwd(aq, ak, av, None, **kw)
        return (O, *binding.cotten_attn_bwd(aq, ak, av, None, ag, **kw))

    return segments, backward, table, attention


def test_threads_on_one_stream():
    mine = [programs(seed) for seed in range(4)]
    want = [[f() for f in p] for p in mine]
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(len(mine))

    def work(i):
        start.wait()
        got = [[f() for f in mine[i]] for _ in range(20)]
        torch.cuda.synchronize()
        for round_ in got:
            for f, a, b in zip(mine[i], round_, want[i]):
                if not all(torch.equal(x, y) for x, y in zip(a, b)):
                    wrong.append((i, f.__name__))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(mine))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == []


def test_a_stream_named_in_the_call():
    """The workspace belongs to the stream of the call: the current stream's work neither gets it nor gives it."""
    mine = programs(9)
    want = [f() for f in mine]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        for _ in range(5):
            got = [f(stream=stream) for f in mine]
            noise = [torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
            torch.cuda.synchronize()
            del noise
            for a, b in zip(got, want):
                assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_growing_lengths_leave_nothing_behind():
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = 1024
    q = torch.randn(2, 2, n, 64, device="cuda", generator=gen).bfloat16()
    g = -torch.rand(2, 2, n, device="cuda", generator=gen)
    dE = torch.randn(40, n, 32, device="cuda", generator=gen)
    ids = torch.randint(0, 300, (40, n), device="cuda", generator=gen)
    left = []
    for N in range(256, n + 1, 64):
        x, a = q[:, :, :N].contiguous(), g[:, :, :N].contiguous()
        i, e = ids[:, :N].contiguous(), dE[:, :N].contiguous()
        before = torch.cuda.memory_allocated()
        binding.cotten_delta_bwd(x, x, x, a, a.exp(), None, x)
        binding.cotten_embed_bwd(i, e, 300)
        left.append(torch.cuda.memory_allocated() - before)
    assert left == [0] * len(left)
