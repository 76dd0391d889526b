"""Workspaces of the linear products and LayerNorm's gradient where they hold something: splits' sums, copies of
rows that are no 16-byte units, dz, column sums, row statistics.  Each call gets exactly the bytes that its
query names, between fences and full of NaN; the same sizes run in graphs, on two streams and in two threads."""
import threading

import numpy as np
import pytest

import linear_paths
import paper_2208_05419_amd as afno
from gpu_util import say, to_dev
from paper_2208_05419_amd import synth

torch = pytest.importorskip("torch")

CODE = {"fp32": 0, "bf16": 1}
FENCE = 272  # bytes: the workspace begins at a multiple of 16 that is none of 32
SEED = 0xFEDCBA9876543210

# dtype, M, K, N, aligned arrays, what the rules make of it (checked below on the CPU): the products that are split
LINEAR = [
    ("bf16", 2100, 72, 2104, True, {"dx", "dw"}),
    ("bf16", 136, 2056, 2056, True, {"forward", "dx"}),
    ("bf16", 4200, 1032, 4104, True, {"dx", "dw"}),    # 256 tiles
    ("bf16", 2100, 77, 2099, True, {"dx", "dw"}),      # x, w and dz copied to whole units
    ("bf16", 2100, 72, 2104, False, {"dx", "dw"}),     # copied for their addresses
    ("bf16", 300, 4099, 333, True, {"forward"}),
    ("bf16", 300, 9, 269, False, {"dx", "dw"}),        # not copied
    ("fp32", 2100, 72, 520, True, {"dx", "dw"}),
    ("fp32", 200, 4096, 264, True, {"forward"}),
    ("fp32", 131, 2051, 2053, True, {"forward", "dx"}),
    ("fp32", 8200, 261, 521, True, {"dw"}),            # copied, in 128 tiles
    ("fp32", 1400, 260, 2952, False, {"dx"}),          # copied for their addresses
]
NORM = [("fp32", 1500, 333), ("bf16", 1500, 333), ("bf16", 900, 2056), ("fp32", 300, 9001), ("bf16", 300, 9001)]


def test_the_sizes_do_what_their_comments_say(tmp_path):
    exe = linear_paths.build(str(tmp_path))
    calls = [({"bf16": 2, "fp32": 4}[d], M, K, N, a, a, a, 1) for d, M, K, N, a, _ in LINEAR]
    for case, products in zip(LINEAR, linear_paths.walk(exe, calls)):
        assert {layout for layout, _, splits in products if splits > 1} >= case[5], (case, products)


def _put(a, dtype, aligned=True):
    t = to_dev(synth.quantize(a, dtype), dtype)
    if aligned:
        return t
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    flat[1:] = t.reshape(-1)
    return flat[1:].reshape(t.shape)


def _bits(ts):
    return [t.view(torch.int16 if t.element_size() == 2 else torch.int32).clone() for t in ts]


def _same(a, b):
    return all(torch.equal(u, v) for u, v in zip(a, b))


class Fenced:
    """`need` bytes at .ptr, all NaN in either type, between fences."""

    def __init__(self, need):
        assert need > 0
        self.need = need
        self.all = torch.full((need + 2 * FENCE,), 0xFF, dtype=torch.uint8, device="cuda")
        self.all[:FENCE] = 9
        self.all[-FENCE:] = 9
        self.ptr = self.all.data_ptr() + FENCE
        assert self.ptr % 32 == 16

    def whole(self):
        return bool((self.all[:FENCE] == 9).all() and (self.all[-FENCE:] == 9).all())


def _linear_data(dtype, M, K, N, aligned, seed=0):
    r = np.random.default_rng(seed)
    put = lambda s, sd=1.0: _put(sd * r.standard_normal(s), dtype, aligned)  # noqa: E731
    return {"x": put((M, K)), "w": put((K, N), K ** -0.5), "b": put(N), "g": put((M, N)), "residual": put((M, N))}


@pytest.mark.gpu
@pytest.mark.parametrize("case", LINEAR, ids=lambda c: "{}_{}x{}x{}{}".format(*c[:4], "" if c[4] else "_odd"))
def test_linear_in_exactly_its_bytes(case):
    dtype, M, K, N, aligned, _ = case
    v, code, st = _linear_data(dtype, M, K, N, aligned), CODE[dtype], torch.cuda.current_stream().cuda_stream
    pre = torch.empty_like(v["g"])
    want = afno.linear_forward(v["x"], v["w"], v["b"], activation="gelu", residual=v["residual"], pre=pre, p=0.1, seed=SEED)
    grads = afno.linear_backward(v["g"], v["x"], v["w"], pre=pre, activation="gelu", p=0.1, seed=SEED)
    assert all(torch.isfinite(t).all() for t in (want, *grads.values()))
    p = {k: t.data_ptr() for k, t in v.items()}
    need = afno.afno_linear_forward_workspace(M, K, N, code, int(aligned))
    say(f"[forward] {case} {need} bytes")
    if "forward" in case[5]:
        assert need > 0
    if need > 0:
        ws, out, z = Fenced(need), torch.empty_like(want), torch.empty_like(want)
        call = lambda have: afno.afno_linear_forward(  # noqa: E731
            p["x"], p["w"], p["b"], p["residual"], M, K, N, afno.AFNO_ACT_GELU, 0.1, SEED, 0, None, code, out.data_ptr(),
            z.data_ptr(), ws.ptr, have, st)
        assert call(need) == afno.AFNO_OK
        torch.cuda.synchronize()
        assert ws.whole() and _same(_bits([out, z]), _bits([want, pre]))
    need = afno.afno_linear_backward_workspace(M, K, N, code, int(aligned))
    say(f"[backward] {case} {need} bytes")
    ws, outs = Fenced(need), [torch.empty_like(t) for t in grads.values()]
    call = lambda have: afno.afno_linear_backward(  # noqa: E731
        p["g"], p["x"], p["w"], pre.data_ptr(), M, K, N, afno.AFNO_ACT_GELU, 0.1, SEED, 0, None, code,
        *(o.data_ptr() for o in outs), ws.ptr, have, st)
    assert call(need) == afno.AFNO_OK
    torch.cuda.synchronize()
    assert ws.whole() and _same(_bits(outs), _bits(grads.values()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,C", NORM)
def test_layer_norm_gradient_in_exactly_its_bytes(dtype, M, C):
    r = np.random.default_rng(C)
    x, g, ga = (_put(r.standard_normal(s), dtype) for s in ((M, C), (M, C), C))
    want = afno.layer_norm_backward(g, x, ga)
    need = afno.afno_layer_norm_backward_workspace(M, C, CODE[dtype])
    say(f"[norm] {dtype} {M} {C} {need} bytes")
    assert need >= 2 * 2 * C * 4  # more than one chunk of sums
    ws, outs = Fenced(need), [torch.empty_like(t) for t in want.values()]
    assert afno.afno_layer_norm_backward(g.data_ptr(), x.data_ptr(), ga.data_ptr(), None, M, C, 1e-6, CODE[dtype],
                                         *(o.data_ptr() for o in outs), ws.ptr, need,
                                         torch.cuda.current_stream().cuda_stream) == afno.AFNO_OK
    torch.cuda.synchronize()
    assert ws.whole() and _same(_bits(outs), _bits(want.values()))


# ---------------------------------------------------------------- graphs, streams and threads

def _step(v, counter, stream=None):
    """Forward and gradients of a call whose dx and dw are both split, and LayerNorm's gradient of what comes out."""
    rng = dict(p=0.2, seed=SEED, offset=7, counter=counter, stream=stream)
    pre = torch.empty_like(v["g"])
    out = afno.linear_forward(v["x"], v["w"], v["b"], activation="gelu", residual=v["residual"], pre=pre, **rng)
    d = afno.linear_backward(v["g"], v["x"], v["w"], pre=pre, activation="gelu", **rng)
    n = afno.layer_norm_backward(v["g"], out, v["b"], stream=stream)
    return [out, pre, d["dx"], d["dw"], d["db"], n["dx"], n["dgamma"], n["dbeta"]]


SHARED = [c for c in LINEAR if c[5] >= {"dx", "dw"}]


@pytest.mark.gpu
@pytest.mark.parametrize("case", SHARED, ids=lambda c: "{}_{}x{}x{}{}".format(*c[:4], "" if c[4] else "_odd"))
def test_two_graphs_with_eager_calls_between(case):
    """Two graphs of the same step on different data, replayed in turn with eager work of the program between
    the replays: every replay gives the eager bits, and the counter draws another mask."""
    data = [_linear_data(*case[:5], seed=s) for s in (1, 2)]
    step = torch.tensor([1], dtype=torch.int64, device="cuda")
    eager = {}
    for s in (1, 2, 3):
        step.fill_(s)
        eager[s] = [_bits(_step(v, step)) for v in data]
    torch.cuda.synchronize()
    assert not torch.equal(eager[1][0][0], eager[2][0][0])
    graphs, held = [torch.cuda.CUDAGraph() for _ in data], []
    for graph, v in zip(graphs, data):
        with torch.cuda.graph(graph):
            held.append(_step(v, step))
    for s in (3, 1, 2, 1, 3):
        step.fill_(s)
        for i in (0, 1):
            graphs[i].replay()
            _step(data[1 - i], step)
        torch.cuda.synchronize()
        for i in (0, 1):
            assert _same(_bits(held[i]), eager[s][i]), (s, i)


@pytest.mark.gpu
@pytest.mark.parametrize("case", SHARED, ids=lambda c: "{}_{}x{}x{}{}".format(*c[:4], "" if c[4] else "_odd"))
def test_two_threads_with_split_products(case):
    data = [_linear_data(*case[:5], seed=s) for s in (3, 4)]
    want = [_bits(_step(v, None)) for v in data]
    torch.cuda.synchronize()
    ok = [False, False]

    def work(i):
        st = torch.cuda.Stream()
        for _ in range(10):
            got = _step(data[i], None, stream=st)
            st.synchronize()
            with torch.cuda.stream(st):
                if not _same(_bits(got), want[i]):
                    return
        ok[i] = True

    ts = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in ts]
    [t.join() for t in ts]
    assert ok == [True, True]
