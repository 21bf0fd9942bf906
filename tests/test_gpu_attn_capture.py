"""Captured runs: on another stream than the build's, replayed on a third one,
of an empty batch, on forked streams, and beside calls that cannot be ordered."""
import pytest
import torch

from attn_world import Shared, bf16_rows, compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


def world(salt, ctx, seed=1):
    return Shared(salt, ctx, bf16_rows(300, 2, 64, seed), bf16_rows(300, 2, 64, seed + 1), [2, 1, 3], [260, 17, 100], 8, prompt=40, seed=seed)


def buffers(w):
    return torch.full((w.T, w.heads, w.dim), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((w.T, w.heads), 7.0, device="cuda")


def test_build_capture_and_replay_on_three_streams(salt_lib, ctx):
    w = world(salt_lib, ctx)
    want = w.reference()
    a, b, c = (torch.cuda.Stream() for _ in range(3))
    torch.cuda.synchronize()
    w.build(a)
    w.run(a)
    out, lse = buffers(w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=b):
        salt_lib.salt_attn_run(w.plan, 0, w.q, out, w.scale, lse, b)
    for _ in range(2):
        out.fill_(7.0)
        torch.cuda.synchronize()
        w.build(a)
        c.wait_stream(a)
        with torch.cuda.stream(c):
            graph.replay()
        a.wait_stream(c)                    # the next build and run come after the replay
        got = w.run(a)
        torch.cuda.synchronize()
        compare(out, lse, *want)
        compare(*got, *want)
    assert salt_lib.salt_get_device_error(ctx) == 0


def test_captured_empty_batch(salt_lib, ctx):
    """Replayed for an empty batch it does nothing; for one with tokens it is refused on the device."""
    w = world(salt_lib, ctx)
    out, lse = buffers(w)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    empty = salt_lib.salt_attn_batch([], [], [0], [])
    salt_lib.salt_attn_build(w.plan, empty, st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        salt_lib.salt_attn_run(w.plan, 0, w.q, out, w.scale, lse, st)
    with torch.cuda.stream(st):
        graph.replay()
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0
    w.build(st)
    with torch.cuda.stream(st):
        graph.replay()
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((lse == 7).all())
    assert salt_lib.salt_get_device_error(ctx) == 0x80


def test_forked_streams_of_a_capture(salt_lib, ctx):
    """Two runs of one capture on two streams follow one another."""
    w = world(salt_lib, ctx)
    want = w.reference()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    first, second = buffers(w), buffers(w)
    torch.cuda.synchronize()
    w.build()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=a):
        b.wait_stream(a)
        salt_lib.salt_attn_run(w.plan, 0, w.q, first[0], w.scale, first[1], a)
        salt_lib.salt_attn_run(w.plan, 0, w.q, second[0], w.scale, second[1], b)
        a.wait_stream(b)
    for _ in range(3):
        for t in first + second:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        compare(*first, *want)
        compare(*second, *want)


def test_calls_beside_a_capture(salt_lib, ctx):
    """While the plan's stream is being captured a call on another one cannot be ordered after it: refused,
    and the capture goes on."""
    w = world(salt_lib, ctx)
    want = w.reference()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    out, lse = buffers(w)
    other = buffers(w)
    torch.cuda.synchronize()
    w.build(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=a):
        with pytest.raises(salt_lib.SaltError) as e:
            salt_lib.salt_attn_run(w.plan, 0, w.q, other[0], w.scale, other[1], b)
        assert e.value.name == "SALT_ERR_INVALID_ARG"
        salt_lib.salt_attn_run(w.plan, 0, w.q, out, w.scale, lse, a)
    graph.replay()
    torch.cuda.synchronize()
    compare(out, lse, *want)
    salt_lib.salt_attn_run(w.plan, 0, w.q, other[0], w.scale, other[1], b)
    torch.cuda.synchronize()
    compare(*other, *want)
