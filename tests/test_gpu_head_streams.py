"""The operators around a classifier's head on a stream that is not the inputs' own: an input that is dropped after the call keeps its memory until the
stream has read it."""
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

from paper_2509_03110_b200 import binding as G

pytestmark = pytest.mark.gpu
K, R, C, D = 2, 64, 5000, 256


def calls():
    """operator: its call, its inputs by keyword."""
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    label = lambda: torch.randint(0, C, (K, R), generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    l, y = rand(K, R, C), label()
    s = G.lsam_logprob(l, y)
    return {
        "logprob": (lambda t, **k: tuple(v for v in G.lsam_logprob(top_k=3, **t, **k)), dict(logits=l, labels=y)),
        "grad": (lambda t, **k: (G.lsam_logprob_grad(**t, **k),), dict(logits=l, labels=y, lse=s.lse, dlogp=rand(K, R), entropy=s.entropy, dentropy=rand(K, R))),
        "head": (lambda t, **k: G.lsam_head_logprob(**t, **k)[:3], dict(h=rand(K, R, D).bfloat16(), w=rand(K, C, D).bfloat16(), labels=label(), bias=rand(K, C))),
        "dropout": (lambda t, **k: (G.lsam_dropout(p=0.25, seed=3, tick=4, **t, **k),), dict(x=rand(K, R, D), skip=rand(K, R, D))),
    }


@pytest.mark.parametrize("name", ["logprob", "grad", "head", "dropout"])
def test_dropped_inputs_keep_their_memory_until_the_stream_has_read_them(name):
    run, inputs = calls()[name]
    stream = torch.cuda.Stream()
    want, warm = run(inputs), run(inputs, stream=stream)  # the stream has memory for its results from now on: a fresh allocation may wait for the device
    torch.cuda.synchronize()
    del warm
    for dropped in inputs:
        mine = dict(inputs, **{dropped: inputs[dropped].clone()})
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(int(20 * 1.9e6))
        got = run(mine, stream=stream)
        shape, dtype, at = mine[dropped].shape, mine[dropped].dtype, mine[dropped].data_ptr()
        del mine
        other = torch.zeros(shape, dtype=dtype, device="cuda")  # on the current stream, which does not wait for the other one
        assert other.data_ptr() != at
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), dropped


def test_a_dropped_result_buffer_keeps_its_memory():
    for run, inputs, like in ((calls()["grad"][0], calls()["grad"][1], "logits"), (calls()["dropout"][0], calls()["dropout"][1], "x")):
        stream = torch.cuda.Stream()
        out = torch.empty_like(inputs[like])
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(int(20 * 1.9e6))
        run(dict(inputs, out=out), stream=stream)
        shape, at = out.shape, out.data_ptr()
        del out
        other = torch.zeros(shape, device="cuda")
        assert other.data_ptr() != at
        torch.cuda.synchronize()
        assert not other.any()


def test_a_second_stream_inside_a_captured_graph():
    for name, (run, inputs) in calls().items():
        want = run(inputs)
        main, side = torch.cuda.Stream(), torch.cuda.Stream()
        warm = run(inputs, stream=side)
        torch.cuda.synchronize()
        del warm
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=main):
            mine = {k: v.clone() for k, v in inputs.items()}
            side.wait_stream(main)
            got = run(mine, stream=side)
            del mine  # their memory belongs to the graph, and is not used again in it before the side stream has read it
            other = [torch.full_like(v, 9) for v in inputs.values()]
            main.wait_stream(side)
        for _ in range(3):
            for v in got:
                v.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, want)), name
        del other


def test_calls_of_several_threads_at_once():
    table = calls()
    want = {name: run(inputs) for name, (run, inputs) in table.items()}
    torch.cuda.synchronize()

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                for name, (run, inputs) in table.items():
                    got = run(inputs)
                    stream.synchronize()
                    assert all(torch.equal(p, q) for p, q in zip(got, want[name])), name
        return True

    with ThreadPoolExecutor(4) as pool:
        assert all(pool.map(work, range(4)))
