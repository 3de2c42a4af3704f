"""Operators around the pass on a stream that is given, and not the current one: whose memory they take."""
import pytest
import torch

from paper_2609_36062_b200 import binding as b

pytestmark = pytest.mark.gpu
LATE = 100_000_000      # clock cycles (some 50 ms) that a kernel waits for before the calls


def flat(out):
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


def calls():
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    x, y, z = rows(2, 600, 384), rows(2, 600, 384), rows(2, 600, 384)
    w, scale = (torch.randn(384, generator=g, device="cuda") for _ in range(2))
    log_a = -torch.rand(2, 600, 384, generator=g, device="cuda") * 0.1
    h0 = torch.randn(2, 384, generator=g, device="cuda")
    q, k = rows(2, 3, 200, 64), rows(2, 2, 200, 64)
    f, _ = b.rotary_frequencies(64)
    plan = b.SmatPlan(1, 2, 512, 64, 64, 2, 64, "f32")
    cache = plan.decode_cache()
    cache.zero_()
    plan.decode_begin(torch.randn(1, 2, 512, 64, generator=g, device="cuda"), torch.randn(1, 2, 512, 64, generator=g, device="cuda"), cache)
    packed = plan.decode_pack(cache)
    return {
        "rotary": lambda s: b.rotary(q, k, f, stream=s),
        "norm_forward": lambda s: b.norm_forward(x, w, residual=y, scale=scale, stream=s),
        "norm_backward": lambda s: b.norm_backward(x, y, w, gate=z, X=z, scale=scale, stream=s),
        "recurrence_forward": lambda s: b.recurrence_forward(x, log_a, h0=h0, stream=s),
        "recurrence_backward": lambda s: b.recurrence_backward(log_a, x, y, h0=h0, stream=s),
        "decode_pack": lambda s: plan.decode_pack(cache, stream=s),
        "decode_unpack": lambda s: plan.decode_unpack(packed, stream=s),
    }


@pytest.mark.parametrize("name", ["rotary", "norm_forward", "norm_backward", "recurrence_forward", "recurrence_backward", "decode_pack", "decode_unpack"])
def test_new_outputs_are_of_the_given_stream(name):
    """Kernels wait behind a long one on the given stream; meanwhile the current stream takes and fills what memory it can get."""
    call = calls()[name]
    want = [t.clone() for t in flat(call(None))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for late, stream in ((0, side), (LATE, side), (LATE, torch.cuda.ExternalStream(side.cuda_stream))):
        with torch.cuda.stream(side):
            torch.cuda._sleep(late)
        given = flat(call(stream))
        at = {t.data_ptr() for t in given}
        sizes = [t.numel() * t.element_size() for t in given]
        filled = [torch.full((n,), 85, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
        assert not late or not side.query()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(p, q) for p, q in zip(given, want))
        assert all(bool((t == 85).all()) for t in filled)
        # given back: the current stream does not get the memory of the other one
        del given, filled
        again = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
        assert not at & {t.data_ptr() for t in again}
        del again
        torch.cuda.synchronize()


@pytest.mark.parametrize("width,rows", [(384, 600), (2048, 700), (128, 4000)])
def test_the_workspace_of_norm_gradients_outlives_its_kernels(width, rows):
    """The call returns before its kernels begin, with its workspace given back; memory that the current stream then takes is not theirs."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x, h, dy = (torch.randn(1, rows, width, generator=g, device="cuda") for _ in range(3))
    w, scale = (torch.randn(width, generator=g, device="cuda") for _ in range(2))
    want = b.norm_backward(dy, h, w, X=x, scale=scale)
    need = b.norm_workspace_bytes(width, scale=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for late in (0, LATE, LATE, LATE):      # (the first time memory comes from the device, which may wait for what runs)
        with torch.cuda.stream(side):
            torch.cuda._sleep(late)
        got = b.norm_backward(dy, h, w, X=x, scale=scale, stream=side)
        filled = [torch.full((need,), 85, dtype=torch.uint8, device="cuda") for _ in range(6)]
        other = b.norm_backward(dy, h, w, X=x, scale=scale)
        assert not late or not side.query()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(p, q) for p, q in zip(got[:4], want)) and all(torch.equal(p, q) for p, q in zip(other[:4], want))
        assert all(bool((t == 85).all()) for t in filled)
        del got, filled, other
        torch.cuda.synchronize()


def test_given_streams_inside_a_graph():
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(2, 500, 256, generator=g, device="cuda") for _ in range(2))
    w = torch.randn(256, generator=g, device="cuda")
    want = b.norm_backward(dy, x, w)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        one = b.norm_backward(dy, x, w, stream=side)
        two = b.norm_backward(dy, x, w)
        torch.cuda.current_stream().wait_stream(side)
        y = b.norm_forward(one[0], w)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for got in (one, two):
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    assert torch.equal(y, b.norm_forward(want[0], w))


@pytest.mark.parametrize("name", ["rotary", "norm_backward", "recurrence_forward", "decode_pack"])
def test_the_default_stream_given_beside_another_current_one(name):
    call = calls()[name]
    want = [t.clone() for t in flat(call(None))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = flat(call(torch.cuda.default_stream()))
        side.wait_stream(torch.cuda.default_stream())
        assert torch.cuda.current_stream() == side
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    torch.cuda.synchronize()
