"""bf16 products grouped by expert, all three directions, against the 64-bit definition, and a training step of a layer whose
experts have a frozen 4-bit weight and a trained adapter each."""
import numpy as np
import pytest
import torch

from paper_2505_14742_amd import binding as q
from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf16, f32 = torch.bfloat16, torch.float32


def _rand(*shape, seed, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(bf16).to(DEV)


def _offsets(lens, start=0):
    return torch.tensor([start] + list(lens), dtype=torch.int64).cumsum(0).to(DEV)


def _ws(t, c_in, c_out, n):
    return torch.empty(q.grouped_linear_workspace_bytes(t, c_in, c_out, n), dtype=torch.int8, device=DEV)


def _run(op, P, Q, offsets, scale, out, accumulate=False, ws=None):
    """op fwd: P = X, Q = W; dx: P = dY, Q = W; dw: P = X, Q = dY."""
    n = offsets.numel() - 1
    c_in, c_out = (P.shape[1], Q.shape[1]) if op == "dw" else Q.shape[1:]
    ws = _ws(P.shape[0], c_in, c_out, n) if ws is None else ws
    if op == "dw":
        q.grouped_linear_bwd_dw(P, Q, offsets, scale, out, ws)
    else:
        fn = q.grouped_linear_fwd if op == "fwd" else q.grouped_linear_bwd_dx
        fn(P, offsets, Q, scale, out, ws, bf16_out=out.dtype == bf16, accumulate=accumulate)


def _check(op, P, Q, offsets, out, scale=0.5, accumulate=False):
    t = P.shape[0]
    p, w = P.double().cpu().numpy(), Q.double().cpu().numpy()
    want, bound = out.double().cpu().numpy().copy(), np.zeros(out.shape)
    for g, (a, b) in enumerate(ref.spans(offsets.tolist(), t)):
        if op == "dw":
            want[g] = scale * p[a:b].T @ w[a:b]
            bound[g] = ref.sum_bound(b - a, 16, abs(scale) * np.abs(p[a:b]).T @ np.abs(w[a:b]))
            continue
        m = w[g] if op == "fwd" else w[g].T
        y = scale * p[a:b] @ m
        bd = ref.sum_bound(p.shape[1], 16, abs(scale) * np.abs(p[a:b]) @ np.abs(m))
        if accumulate:
            bd = bd + 2.0 ** -23 * (np.abs(want[a:b]) + np.abs(y))
            y = y + want[a:b]
        want[a:b], bound[a:b] = y, ref.bf16_bound(bd, y) if out.dtype == bf16 else bd
    _run(op, P, Q, offsets, scale, out, accumulate)
    got = out.double().cpu().numpy()
    worst = np.abs(got - want) - bound
    assert worst.max(initial=-1.0) <= 0, "worst excess %.3e at %s" % (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


CASES = [([1], 0, 16, 16), ([0, 2, 0], 3, 48, 16), ([1, 0, 1, 1, 0, 0, 2], 0, 512, 528), ([0, 0], 4, 64, 64), ([130, 1, 0, 257], 0, 320, 400),
         ([40, 0, 300, 17, 5], 21, 1040, 144), ([3] * 70, 1, 256, 16), ([700, 900], 0, 528, 784), ([2100, 0, 33], 5, 16, 272), ([64, 128, 63, 65], 0, 64, 128),
         ([5, 6], 0, 4096, 32), ([31, 1, 40], 0, 2064, 1040), ([513], 0, 272, 48)]


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("op", ["fwd", "dx"])
@pytest.mark.parametrize("lens,behind,c_in,c_out", CASES)
def test_rows_of_a_group_meet_its_weight(op, lens, behind, c_in, c_out, dtype):
    t = sum(lens) + behind + 1
    k, n = (c_in, c_out) if op == "fwd" else (c_out, c_in)
    P, W = _rand(t, k, seed=t), _rand(len(lens), c_in, c_out, seed=c_in, scale=0.1)
    P[0] = float("nan")                                          # rows of no group
    if behind:
        P[-behind:] = float("inf")
    _check(op, P, W, _offsets(lens, 1), torch.full((t, n), 3.0, dtype=dtype, device=DEV))


@pytest.mark.parametrize("lens,behind,c_in,c_out", CASES + [
    ([5000, 3], 0, 208, 16), ([9000], 0, 16, 400), ([0, 1, 3000, 17], 9, 64, 2064), ([3000, 0, 40], 2, 400, 272), ([2900, 256, 257], 0, 272, 64),
    ([50, 39], 0, 64, 400), ([9, 0, 80], 0, 16, 400)])
def test_weight_gradient_sums_the_rows_of_its_group(lens, behind, c_in, c_out):
    t = sum(lens) + behind + 1
    X, G = _rand(t, c_in, seed=t), _rand(t, c_out, seed=t + 1, scale=0.02)
    for M in (X, G):
        M[0] = float("nan")
        if behind:
            M[-behind:] = float("inf")
    _check("dw", X, G, _offsets(lens, 1), torch.full((len(lens), c_in, c_out), 7.0, device=DEV))


def test_strides():
    off = _offsets([50, 40, 0])
    X, G = _rand(90, 360, seed=1), _rand(90, 504, seed=2)
    W = _rand(3, 272, 400, seed=3, scale=0.1)
    out = torch.full((90, 424), -2.0, device=DEV)
    keep = out.clone()
    _check("fwd", X[:, 40:312], W, off, out[:, 8:408])
    assert torch.equal(out[:, :8], keep[:, :8]) and torch.equal(out[:, 408:], keep[:, 408:])
    _check("dx", G[:, 48:448], W, off, torch.full((90, 288), -2.0, dtype=bf16, device=DEV)[:, 8:280])
    _check("dw", X[:, 40:312], G[:, 48:448], off, torch.empty(3, 272, 400, device=DEV))


@pytest.mark.parametrize("op", ["fwd", "dx"])
@pytest.mark.parametrize("lens", [[3, 0, 2], [200, 0, 70]])
def test_accumulate_adds_to_the_rows_of_groups_only(op, lens):
    t = sum(lens) + 3
    W = _rand(3, 272, 208, seed=3, scale=0.1)
    k, n = (272, 208) if op == "fwd" else (208, 272)
    _check(op, _rand(t, k, seed=4), W, _offsets(lens, 2), torch.randn(t, n, device=DEV), accumulate=True)


@pytest.mark.parametrize("op,lens,c_in,c_out", [("fwd", [2000, 0, 2101], 80, 4112), ("dx", [520, 900], 4112, 80), ("dx", [500, 77], 1040, 528)])
def test_accumulate_with_whole_tiles(op, lens, c_in, c_out):
    t = sum(lens) + 5
    k, n = (c_in, c_out) if op == "fwd" else (c_out, c_in)
    _check(op, _rand(t, k, seed=4), _rand(len(lens), c_in, c_out, seed=3, scale=0.1), _offsets(lens, 2), torch.randn(t, n, device=DEV),
           accumulate=True)


def test_offsets_outside_the_batch_are_clamped_and_checked():
    W = _rand(3, 64, 48, seed=3, scale=0.1)
    _check("fwd", _rand(20, 64, seed=4), W, torch.tensor([-5, 7, 7, 1 << 40], device=DEV), torch.full((20, 48), 3.0, device=DEV))
    res = torch.full((1,), -7, dtype=torch.int32, device=DEV)
    for values, want in (([0, 7, 7, 20], 0), ([3, 3], 0), ([0, 21], 2), ([-1, 4], 1), ([0, 5, 4, 20], 3), (list(range(700)) + [698, 800], 701)):
        q.check_group_offsets(torch.tensor(values, dtype=torch.int64, device=DEV), 900 if len(values) > 10 else 20, res)
        assert int(res.item()) == want, values


def test_many_groups():
    lens = [(i * 7) % 4 for i in range(1024)]
    t = sum(lens)
    X, W = _rand(t, 32, seed=1), _rand(1024, 32, 16, seed=2)
    _check("fwd", X, W, _offsets(lens), torch.zeros(t, 16, device=DEV))
    _check("dw", X, _rand(t, 16, seed=3), _offsets(lens), torch.zeros(1024, 32, 16, device=DEV))


def test_no_rows():
    off = _offsets([0, 0])
    W = _rand(2, 64, 48, seed=1)
    empty = lambda c, dt=bf16: torch.empty(0, c, dtype=dt, device=DEV)
    _run("fwd", empty(64), W, off, 1.0, empty(48, f32))
    _run("dx", empty(48), W, off, 1.0, empty(64, f32))
    dW = torch.full((2, 64, 48), 3.0, device=DEV)
    _run("dw", empty(64), empty(48), off, 1.0, dW)
    assert not dW.any()


def test_offsets_past_32_bits():
    """The third group's weight starts 4.3 GB into the array; the last rows of the result 2.3 G elements into theirs."""
    n = 32768
    W = torch.zeros(3, n, n, dtype=bf16, device=DEV)
    W[2, :48, :] = _rand(48, n, seed=1, scale=0.1)
    X = torch.zeros(3, n, dtype=bf16, device=DEV)
    X[:, :48] = _rand(3, 48, seed=2)
    Y = torch.zeros(3, n, device=DEV)
    _run("fwd", X, W, torch.tensor([0, 0, 1, 3], device=DEV), 1.0, Y)
    want = X[1:, :48].double() @ W[2, :48].double()
    assert float((Y[1:].double() - want).abs().max()) <= 1e-4 and not Y[0].any()
    del W, Y
    t = 70000
    X, W = _rand(t, 16, seed=3), _rand(1, 16, n, seed=4)
    Y = torch.empty(t, n, dtype=bf16, device=DEV)
    _run("fwd", X, W, torch.tensor([0, t], device=DEV), 1.0, Y)
    want = X[-300:].double() @ W[0].double()
    assert bool(((Y[-300:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())


def test_directions_are_adjoint():
    """<G, fwd(X; W)> = <dx(G; W), X> = <dw(X, G), W>: gradients against the forward product itself (it is linear in both)."""
    lens, c_in, c_out = [33, 0, 150, 4], 272, 208
    t, off = sum(lens), _offsets(lens)
    X, G, W = _rand(t, c_in, seed=1), _rand(t, c_out, seed=2), _rand(4, c_in, c_out, seed=3)
    Y, D, dW = torch.zeros(t, c_out, device=DEV), torch.zeros(t, c_in, device=DEV), torch.zeros(4, c_in, c_out, device=DEV)
    _run("fwd", X, W, off, 0.75, Y)
    _run("dx", G, W, off, 0.75, D)
    _run("dw", X, G, off, 0.75, dW)
    a, b, c = (G.double() * Y.double()).sum(), (X.double() * D.double()).sum(), (W.double() * dW.double()).sum()
    # every sum has t c_in c_out products of magnitude about 1, each off by at most 300 roundings of 2^-23 of its own partial sums
    tol = 300 * 2.0 ** -23 * 0.75 * float(sum((G[s:e].double().abs() @ W[g].double().abs().t() * X[s:e].double().abs()).sum()
                                               for g, (s, e) in enumerate(ref.spans(off.tolist(), t))))
    assert abs(float(a - b)) <= tol and abs(float(a - c)) <= tol
    # a difference quotient of the forward in one weight and one input (linear: exact up to the sums)
    W2 = W.clone()
    W2[2, 5, 7] += 1.0
    Y2 = torch.zeros_like(Y)
    _run("fwd", X, W2, off, 0.75, Y2)
    step = float(W2[2, 5, 7].double() - W[2, 5, 7].double())
    quotient = float(((Y2 - Y).double() * G.double()).sum()) / step
    assert abs(quotient - float(dW[2, 5, 7])) <= 300 * 2.0 ** -23 * float((Y.double().abs() * G.double().abs()).sum()) / step


def test_equal_calls_give_equal_bits_and_captured_calls_follow_their_offsets():
    lens = [300, 0, 41, 3]
    t = sum(lens)
    off = _offsets(lens)
    X, G, W = _rand(t, 528, seed=1), _rand(t, 272, seed=2), _rand(4, 528, 272, seed=3)
    Y, D, dW = torch.zeros(t, 272, dtype=bf16, device=DEV), torch.zeros(t, 528, device=DEV), torch.zeros(4, 528, 272, device=DEV)
    ws = _ws(t, 528, 272, 4)

    def step():
        _run("fwd", X, W, off, 0.5, Y, ws=ws)
        _run("dx", G, W, off, 0.5, D, ws=ws)
        _run("dw", X, G, off, 0.5, dW, ws=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, other in enumerate((lens, lens[::-1], [0, t, 0, 0], [0, 0, 0, 0])):
        off.copy_(_offsets(other))
        X.copy_(_rand(t, 528, seed=20 + i))
        for M in (Y, D, dW):
            M.fill_(5.0)
        step()
        want = [M.clone() for M in (Y, D, dW)]
        for M in (Y, D, dW):
            M.fill_(5.0)
        ws.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((Y, D, dW), want)), i


@pytest.mark.parametrize("r", [16, 64])
def test_a_training_step_of_experts_with_frozen_weights_and_adapters(r):
    """The layer forward and input gradient, and the adapters' gradients from grouped products on its inner activations, against
    the 64-bit formulas and differences of the layer's own forward."""
    from tests.test_gpu_mx4 import Layer
    lens, c_in, c_out, scale = [90, 0, 37, 130], 528, 784, 0.5
    t, off, n = sum(lens), _offsets(lens), 4
    L = Layer(n, c_in, c_out, r, 11)
    X, G = _rand(t, c_in, seed=5), _rand(t, c_out, seed=6, scale=0.1)
    Y, D = torch.zeros(t, c_out, device=DEV), torch.zeros(t, c_in, device=DEV)
    L.check(False, X, off, Y)
    L.check(True, G, off, D)
    T, U = torch.zeros(t, r, dtype=bf16, device=DEV), torch.zeros(t, r, dtype=bf16, device=DEV)
    dA, dB = torch.zeros(n, c_in, r, device=DEV), torch.zeros(n, r, c_out, device=DEV)
    _check("fwd", X, L.A, off, T, 1.0)
    _check("dx", G, L.B, off, U, 1.0)
    _check("dw", X, U, off, dA, scale)
    _check("dw", T, G, off, dB, scale)
    # one entry of A raised: the change of <G, Y> over the step is its gradient, up to the roundings of U to bf16 and of Y's sums
    before, entry = Y.double().clone(), L.A[2, 7, 3].double()
    L.A[2, 7, 3] += 0.5
    L.run(False, X, off, Y)
    step = float(L.A[2, 7, 3].double() - entry)
    quotient = float(((Y.double() - before) * G.double()).sum()) / step
    x, g = X[90:127].double(), G[90:127].double()
    u = scale * (x[:, 7].abs() @ (g.abs() @ L.B[2, 3].double().abs()))
    tol = float(2.0 ** -8 * u) + 200 * 2.0 ** -23 * float((before.abs() * G.double().abs()).sum()) / step
    assert abs(quotient - float(dA[2, 7, 3])) <= tol


def test_adapters_on_top_of_the_int8_layer():
    """A batch whose sequences use different adapters on one frozen int8 layer: its product without adapter, then the grouped
    products of the adapters added to it, equal the layer's own low-rank branch group by group."""
    from tests.gpu_harness import Layer as Int8Layer, bf16_dev
    from paper_2505_14742_amd import synth
    ec = synth.EdgeCase("adapters", 96, 512, 384, [3, 64, 65, 500], 16)
    Xn, _dY, W, O, A, B = synth.edge_case_inputs(ec, 7)
    X = bf16_dev(Xn)
    whole, base = Int8Layer(W, O, A, B, 0.5, ec.t), Int8Layer(W, O, None, None, 0.5, ec.t)
    whole.fwd_step(X, 0.2)
    base.fwd_step(X, 0.2)
    X, A1, B1, off = X.view(bf16), whole.A.view(bf16), whole.B.view(bf16), _offsets([40, 0, 56])
    As, Bs = (M.unsqueeze(0).repeat(3, 1, 1).contiguous() for M in (A1, B1))
    T = torch.zeros(96, 16, dtype=bf16, device=DEV)
    _run("fwd", X, As, off, 1.0, T)
    _run("fwd", T, Bs, off, 0.5, base.Y, accumulate=True)
    mag = 0.5 * (X.double().abs() @ A1.double().abs()) @ B1.double().abs()
    # T is rounded to bf16 here (half a step, 2^-8 of it), the rest is fp32 sums
    tol = 2.0 ** -8 * mag + 600 * 2.0 ** -23 * (mag + whole.Y.double().abs())
    assert bool(((base.Y.double() - whole.Y.double()).abs() <= tol).all())


@pytest.mark.parametrize("op,lens,c_in,c_out,dtype", [
    ("fwd", [2000, 0, 2101], 80, 4112, f32), ("fwd", [2000, 2101], 592, 4112, bf16), ("dx", [2000, 0, 2101], 4112, 144, bf16),
    ("dx", [4101], 4112, 528, f32), ("dw", [70, 0, 130, 1], 2064, 2064, f32), ("dw", [64] * 16, 1040, 1040, f32)])
def test_large_tiles(op, lens, c_in, c_out, dtype):
    t = sum(lens) + 5
    off = _offsets(lens, 2)
    if op == "dw":
        _check(op, _rand(t, c_in, seed=1), _rand(t, c_out, seed=2), off, torch.full((len(lens), c_in, c_out), 7.0, device=DEV))
    else:
        k, n = (c_in, c_out) if op == "fwd" else (c_out, c_in)
        _check(op, _rand(t, k, seed=1), _rand(len(lens), c_in, c_out, seed=2, scale=0.1), off, torch.full((t, n), 3.0, dtype=dtype, device=DEV))


@pytest.mark.parametrize("dtype,accumulate", [(f32, False), (f32, True), (bf16, False)])
@pytest.mark.parametrize("op,lens,c_in,c_out", [("fwd", [100, 0, 700, 33], 4112, 16), ("dx", [100, 0, 700, 33], 48, 4112), ("fwd", [150], 2064, 272),
                                                ("dx", [64, 70], 400, 16400), ("fwd", [1000, 37], 2048, 64),
                                                ("fwd", [210, 0, 190], 8400, 2064), ("dx", [500, 90], 784, 8208)])
def test_few_columns_of_a_long_contraction(op, lens, c_in, c_out, dtype, accumulate):
    """Sizes at which several workgroups share a contraction and a second launch joins their sums."""
    t = sum(lens) + 9
    k, n = (c_in, c_out) if op == "fwd" else (c_out, c_in)
    assert q.grouped_linear_workspace_bytes(t, c_in, c_out, len(lens)) > 2 * t * n * 4
    P = _rand(t, k, seed=t)
    P[:4] = float("nan")
    P[-5:] = float("nan")
    _check(op, P, _rand(len(lens), c_in, c_out, seed=2, scale=0.1), _offsets(lens, 4), torch.full((t, n), 3.0, dtype=dtype, device=DEV),
           accumulate=accumulate)


@pytest.mark.parametrize("op,c_in,c_out,dtype", [("fwd", 80, 1040, f32), ("fwd", 528, 1168, bf16), ("dx", 1040, 144, bf16), ("dx", 1168, 592, f32)])
def test_medium_tiles(op, c_in, c_out, dtype):
    """Many groups of about a hundred rows, odd widths."""
    lens = [(i * 37) % 201 for i in range(40)]
    t = sum(lens) + 3
    k, n = (c_in, c_out) if op == "fwd" else (c_out, c_in)
    P = _rand(t, k, seed=1)
    P[0] = P[-2:] = float("nan")
    _check(op, P, _rand(40, c_in, c_out, seed=2, scale=0.1), _offsets(lens, 1), torch.full((t, n), 3.0, dtype=dtype, device=DEV))
