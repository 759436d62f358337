"""Calls on a stream of the caller's own: the memory that they take belongs to that stream."""
import contextlib
import types

import pytest
import torch

from paper_2609_32420_b200 import carnator as cn

def test_memory_is_taken_on_the_stream_of_the_call(monkeypatch):
    """On a machine without a GPU, with stand-ins for torch's streams: made inside the call's stream, recorded for the current one; without a stream nothing of it."""
    on, log = [], []

    @contextlib.contextmanager
    def inside(stream):
        on.append(stream)
        yield
        on.pop()
    monkeypatch.setattr(torch.cuda, "stream", inside)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: "current")
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: ("external", handle))

    def make():
        log.append(("made", tuple(on)))
        return types.SimpleNamespace(record_stream=lambda s: log.append(("recorded", s)))
    cuda, cpu = torch.device("cuda", 0), torch.device("cpu")
    cn._made(make, cuda, None)
    cn._made(make, cpu, types.SimpleNamespace(cuda_stream=7))
    assert log == [("made", ())] * 2
    cn._made(make, cuda, types.SimpleNamespace(cuda_stream=7))
    assert log[2:] == [("made", (("external", 7),)), ("recorded", "current")]


def _calls():
    """name -> call(stream) with nothing given that it can make itself."""
    g = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *n: torch.randn(n, device="cuda", generator=g)  # noqa: E731
    N, C = 1024, 512
    x, y, w = r(1, N, C).bfloat16(), r(1, N, C).bfloat16(), r(C, C).bfloat16()
    q = r(1, 2, N, 128).bfloat16()
    vec, six = 1 + 0.1 * r(C), 0.1 * r(1, C)
    t = x[:, None]
    ns, ls = cn.make_norm_shape(t, t, vec, six), cn.make_linear_shape(x, w, y, gate=six, Z=y, activation=cn.ACT_GELU)
    mean, rstd = torch.empty((2, 1, 1, N), device="cuda")
    cn.layer_norm(t, ns, weight=vec, shift=six, scale=six, mean=mean, rstd=rstd)
    bs = cn.make_block_norm_shape(x, x, x, x, post_weight=vec, gate=six, scale=six, post=cn.NORM_RMS)
    stats = torch.empty((4, 1, N), device="cuda")
    cn.block_norm(x, x, bs, post_weight=vec, gate=six, shift=six, scale=six, stats=stats)
    qs = cn.make_quantize_shape(x, None, None)
    w8, ws8 = cn.quantize_fp8(w[None], cn.make_quantize_shape(w[None], None, None, block_rows=128))
    fs = cn.make_linear_fp8_shape(x, w8[0], ws8[0], y)
    rs, freq = cn.make_rope_shape(q, None, 64), cn.rope_frequencies(64, device="cuda")[0]
    shape = cn.make_shape(1, 2, N, 128, 0, 1, 1, N, 128, 128, q, q, q)
    p = cn.BuildParams()
    p.mode, p.mass, p.keep_ratio, p.window_frames, p.count_includes_forced = cn.MODE_CUMMASS, 0.8, 0.5, -1, 1
    mask, _ = cn.build_connectivity(q, q, shape, p)
    rec = torch.zeros((1, shape.nqb), dtype=torch.uint8, device="cuda")
    _, lse, _ = cn.sparse_attn(q, q, q, mask, rec, shape)
    seeds = torch.arange(8, dtype=torch.int32, device="cuda")
    return {
        "layer_norm": lambda s: cn.layer_norm(t, ns, weight=vec, shift=six, scale=six, stream=s),
        "layer_norm_backward": lambda s: cn.layer_norm_backward(t, t, mean, rstd, ns, weight=vec, scale=six, stream=s),
        "linear": lambda s: cn.linear(x, w, ls, gate=six, stream=s),
        "linear_backward": lambda s: cn.linear_backward(y, x, w, ls, Z=y, gate=six, stream=s),
        "rope": lambda s: cn.rope(q, freq, rs, stream=s),
        "block_norm": lambda s: cn.block_norm(x, x, bs, post_weight=vec, gate=six, shift=six, scale=six, stream=s),
        "block_norm_backward": lambda s: cn.block_norm_backward(x, x, x, stats, bs, dS=x, post_weight=vec, gate=six, scale=six, stream=s),
        "quantize_fp8": lambda s: cn.quantize_fp8(x, qs, stream=s),
        "linear_fp8": lambda s: cn.linear_fp8(x, w8[0], ws8[0], fs, stream=s),
        "build_connectivity": lambda s: cn.build_connectivity(q, q, shape, p, stream=s),
        "build_connectivity_exact": lambda s: cn.build_connectivity_exact(q, q, lse, shape, p, stream=s),
        "compact_mask": lambda s: cn.compact_mask(mask, rec, shape, stream=s),
        "sparse_attn": lambda s: cn.sparse_attn(q, q, q, mask, rec, shape, stream=s),
        "seed_expansion": lambda s: cn.seed_expansion(q, q, lse, seeds, 4, 4, shape, stream=s),
    }


def _tensors(out):
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


NAMES = ["layer_norm", "layer_norm_backward", "linear", "linear_backward", "rope", "block_norm", "block_norm_backward", "quantize_fp8", "linear_fp8", "build_connectivity",
         "build_connectivity_exact", "compact_mask", "sparse_attn", "seed_expansion"]


@pytest.mark.gpu
@pytest.mark.parametrize("external", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_memory_that_a_call_took_stays_with_its_stream(name, external, monkeypatch):
    """Workspace and results of a call on another stream, all dropped, while the stream is still busy: none of that memory comes back to the current stream, and the results
    are those of a call on the current one."""
    call = _calls()[name]
    want = _tensors(call(None))
    side, taken, made = torch.cuda.Stream(), [], cn._made

    def spy(make, device, stream):
        t = made(make, device, stream)
        taken.append((t.untyped_storage().data_ptr(), t.untyped_storage().nbytes()))
        return t
    monkeypatch.setattr(cn, "_made", spy)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)    # some 10 ms
    out = _tensors(call(torch.cuda.ExternalStream(side.cuda_stream) if external else side))
    copies = []
    with torch.cuda.stream(side):
        for t in out:
            copies.append(t.clone())
    del out, t
    assert taken
    later = []
    for _, size in taken * 4:            # what the current stream takes next, and writes to while the other one still works
        n = torch.empty(size, dtype=torch.uint8, device="cuda")
        assert all(n.data_ptr() + size <= at or at + of <= n.data_ptr() for at, of in taken)
        later.append(n.fill_(255))
    torch.cuda.synchronize()
    for k, (a, b) in enumerate(zip(copies, want)):
        if a.dtype != torch.uint8 or (name.startswith("build") and k == 0):        # a result, not a workspace
            assert torch.equal(a.float(), b.float())


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["block_norm_backward", "linear_backward", "linear_fp8", "rope", "sparse_attn"])
def test_captured_on_a_stream_that_joins_the_capture(name):
    call = _calls()[name]
    want = _tensors(call(None))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = _tensors(call(side))       # drops the workspace that it made
        with torch.cuda.stream(side):
            kept = [t + 0 if t.dtype != torch.uint8 else None for t in out]
        again = _tensors(call(side))
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t in (*out, *again):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c, w in zip(out, kept, again, want):
            if w.dtype != torch.uint8:
                assert torch.equal(a, w) and torch.equal(b, w) and torch.equal(c, w)
