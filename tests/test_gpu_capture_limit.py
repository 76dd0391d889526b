"""A graph takes one call whose workspace it allocates by itself: a second one in the same capture is refused with
nothing recorded, whichever entry points they are; another capture takes one again."""
import contextlib
import gc

import pytest

import paper_2208_05419_amd as afno
from gpu_util import dev_weights, to_dev
from paper_2208_05419_amd import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def data():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    wl = synth.Workload("capture", 1, 16, 32, 128, 4, "bf16", 0.01, 1.0)
    w = dev_weights(synth.make_weights(wl, seed=0), "bf16")
    p = {k: to_dev(v, "bf16") for k, v in synth.make_block_params(wl, seed=0).items()}
    return to_dev(synth.make_x(wl, seed=0), "bf16"), (w["w1"], w["b1"], w["w2"], w["b2"], 4, 0.01), p


def _calls(data):
    """Every entry point that allocates, into tensors of its own."""
    x, args, p = data
    return {
        "forward": lambda: [afno.filter_forward(x, *args)],
        "backward": lambda: list(afno.filter_backward(x, *args[:4], x, *args[4:]).values()),
        "block": lambda: [afno.block_forward(x, p, *args[4:])],
        "stage": lambda: [afno.filter_stage(x, *args, 1.0, afno.AFNO_STAGE_SPECTRUM)],
    }


@contextlib.contextmanager
def _capture():
    """A capture during which nothing is collected: an old graph that the collector destroys in the middle of
    another's capture synchronizes the device in its destructor, which ends the process."""
    graph = torch.cuda.CUDAGraph()
    gc.collect()
    gc.disable()
    try:
        with torch.cuda.graph(graph):
            yield graph
    finally:
        gc.enable()


def _refusal(call):
    """The code and text of the error that a call raises, without the exception, whose traceback would hold the
    graph in a cycle."""
    try:
        call()
    except afno.AfnoError as e:
        return e.code, str(e)
    return None


@pytest.mark.parametrize("second", ["forward", "backward", "block", "stage"])
@pytest.mark.parametrize("first", ["forward", "backward", "block", "stage"])
def test_second_allocating_call_is_refused(data, first, second):
    calls = _calls(data)
    calls[first](), calls[second]()
    torch.cuda.synchronize()
    for _ in range(2):  # another capture takes one again
        with _capture():
            ok = _refusal(calls[first])
            again = [_refusal(calls[second]) for _ in range(2)]
        assert ok is None
        assert all(code == afno.AFNO_ERR_UNSUPPORTED and "a graph takes one call" in text for code, text in again)
    calls[second]()  # outside of a capture as ever
    torch.cuda.synchronize()


def test_the_recorded_call_replays_after_a_refusal(data):
    calls = _calls(data)
    want = calls["forward"]()[0]
    with _capture() as graph:
        held = calls["forward"]()[0]
        again = _refusal(calls["forward"])
    assert again is not None
    for _ in range(3):
        held.zero_()
        torch.cuda.synchronize()
        graph.replay()
        calls["forward"]()
        torch.cuda.synchronize()
        assert torch.equal(held, want)


def test_a_captured_step_without_allocations(data):
    """Several filter calls through the entry point without an allocation, and the products, LayerNorm and dropout
    with workspaces of torch's, in one graph."""
    x, args, p = data
    bufs = [torch.empty_like(x) for _ in range(2)]
    z = torch.empty(*x.shape[:-1], 4 * x.shape[-1], dtype=x.dtype, device="cuda")

    def step():
        t = afno.layer_norm_forward(x, p["ln1_g"], p["ln1_b"])
        u = afno.filter_forward_noalloc(t, *args, 1.0, bufs[0])
        h = afno.linear_forward(u, p["wa"], p["ba"], activation="gelu", pre=z, p=0.1, seed=2)
        y = afno.linear_forward(h, p["wb"], p["bb"], residual=u)
        v = afno.filter_forward_noalloc(y, *args, 1.0, bufs[1])
        d = afno.linear_backward(v, h, p["wb"])
        d1 = afno.linear_backward(d["dx"], u, p["wa"], pre=z, activation="gelu", p=0.1, seed=2)
        return [v, d["dw"], d["db"], *d1.values()]

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    with _capture() as graph:
        held = step()
    for _ in range(4):
        [b.zero_() for b in bufs]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        step()
        torch.cuda.synchronize()


@pytest.mark.parametrize("stage", [afno.AFNO_STAGE_SPECTRUM, afno.AFNO_STAGE_MIXED, afno.AFNO_STAGE_DELTA])
def test_a_captured_stage_of_nothing_kept(data, stage):
    """No mode passes: the stage is 0, in every replay whatever its memory held before."""
    x, args, _ = data
    call = lambda: afno.filter_stage(x, *args, 0.01, stage)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    assert not want.any()
    with _capture() as graph:
        held = call()
    for rep in range(4):
        held.fill_(float(rep + 1))
        torch.cuda.synchronize()
        graph.replay()
        call()
        torch.cuda.synchronize()
        assert not held.any()
