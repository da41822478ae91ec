"""Every form of the orthogonalised update (muon_cases.py) on the GPU against the recipe in 64 bits: wavefronts with one chunk of columns
and with several, wide and tall matrices, one launch, one a pass and two.

Tolerance.  An error made in X_k grows by at most a per remaining step, so |dX| <= e sum_k a^(steps - k) |X_k|_F, with e the error of
a pass relative to its operands, in the sums of G, G^2 and P X.  A product of two fp32 values held as two fp16 each is off by at most
2^-21 of itself (2^-23 for each value, 2^-22 for the product of the lower parts, which is left out): 8 * 2^-24.  n products in a row
round n times, 2^-25 each at random signs on sums that grow to the whole: below sqrt(n) / 2 * 2^-24.  The longest such row
is a wavefront's columns, 32 a chunk, or the blocks' shares, or the shorter side.  e = 3 (8 + sqrt(n) / 2) 2^-24."""
import numpy as np
import pytest
import torch

from helpers import record
from muon_cases import FORMS, chunks
from test_gpu_muon import A, B, C, gradient, up

pytestmark = pytest.mark.gpu

EVERY = sorted(FORMS)


def recipe(u, steps, eps, in_a_row, abc=(A, B, C)):
    a, b, c = abc
    tall = u.shape[0] > u.shape[1]
    X = u.T if tall else u
    n = max(32 * in_a_row, 256, X.shape[0])
    e = 3 * (8 + np.sqrt(n) / 2) * 2.0 ** -24
    X = X / (np.sqrt((X * X).sum()) + eps)
    bound = 0.0
    for k in range(steps):
        bound += abs(a) ** (steps - k) * np.sqrt((X * X).sum())
        G = X @ X.T
        X = a * X + (b * G + c * (G @ G)) @ X
    bound += np.sqrt((X * X).sum())
    return (X.T if tall else X), e * bound


def form(name):
    (tiles, alone, _, in_a_row), shapes = FORMS[name]
    return shapes, in_a_row if not alone else -(-max(chunks(s) for s in shapes) // 8)


def zeros(shapes):
    return up([np.zeros(s, np.float32) for s in shapes])


def distance(got, ref):
    return np.linalg.norm(got.cpu().numpy().astype(np.float64) - ref)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("name", EVERY)
def test_direction(gpu_api, name, nesterov):
    rng = np.random.default_rng(21)
    shapes, row = form(name)
    g = [gradient(rng, *s, kind=("mixed", "noise", "one")[i % 3]) for i, s in enumerate(shapes)]
    m = [gradient(rng, *s, kind="noise") for s in shapes]
    hp = gpu_api.Muon(lr=1.0, momentum=0.9, nesterov=nesterov, scale_mode=gpu_api.MUON_SCALE_NONE)
    dp, dg, dm = zeros(shapes), up(g), up(m)
    gpu_api.muon_step(hp, dp, dg, dm)
    mu, worst = float(hp.momentum), 0.0
    for i, s in enumerate(shapes):
        assert np.array_equal(dg[i].cpu().numpy(), g[i])
        m64 = mu * m[i].astype(np.float64) + g[i]
        got_m = dm[i].cpu().numpy().astype(np.float64)
        assert np.abs(got_m - m64).max() <= 2.0 ** -24 * np.abs(m64).max()
        ref, bound = recipe(g[i] + mu * got_m if nesterov else got_m, hp.steps, float(hp.eps), row)
        off = distance(-dp[i], ref)
        worst = max(worst, off / bound)
        assert off <= bound, (s, off, bound)
    record(f"muon {name} nesterov={nesterov}", of_bound=worst)


@pytest.mark.parametrize("steps,abc", [(1, (A, B, C)), (2, (A, B, C)), (9, (1.5, -0.5, 0.0)), (16, (1.5, -0.5, 0.0))])
@pytest.mark.parametrize("name", EVERY)
def test_steps_and_coefficients(gpu_api, name, steps, abc):
    rng = np.random.default_rng(22)
    shapes, row = form(name)
    g = [gradient(rng, *s, kind="noise") for s in shapes]
    hp = gpu_api.Muon(lr=1.0, momentum=0.0, a=abc[0], b=abc[1], c=abc[2], steps=steps, nesterov=False, scale_mode=0)
    dp = zeros(shapes)
    gpu_api.muon_step(hp, dp, up(g), zeros(shapes))
    for i, s in enumerate(shapes):
        ref, bound = recipe(g[i].astype(np.float64), steps, float(hp.eps), row, abc)
        assert distance(-dp[i], ref) <= bound, s


@pytest.mark.parametrize("name", EVERY)
def test_decay_scale_and_consumed_gradients(gpu_api, name):
    rng = np.random.default_rng(23)
    shapes, row = form(name)
    g = [gradient(rng, *s) for s in shapes]
    p = [rng.standard_normal(s).astype(np.float32) for s in shapes]
    hp = gpu_api.Muon(lr=0.02, momentum=0.95, weight_decay=0.1, scale_mode=gpu_api.MUON_SCALE_RMS)
    dp, dg, dm = up(p), up(g), zeros(shapes)
    gpu_api.muon_step(hp, dp, dg, dm, zero_grads=True)
    lr, wd, mu = float(hp.lr), float(hp.weight_decay), float(hp.momentum)
    for i, s in enumerate(shapes):
        assert not dg[i].any() and torch.equal(dm[i].cpu(), torch.from_numpy(g[i]))
        X, bound = recipe(g[i] * (1 + mu), 5, float(hp.eps), row)
        step = lr * 0.2 * max(s) ** 0.5
        ref = p[i].astype(np.float64) * (1 - lr * wd) - step * X
        # the decay, the step size, u and the result are rounded once each
        tol = 2.0 ** -24 * (2 * np.linalg.norm(p[i]) + 2 * step * np.linalg.norm(X) + np.linalg.norm(ref))
        assert distance(dp[i], ref) <= step * bound + tol, s


@pytest.mark.parametrize("name", EVERY)
def test_what_one_matrix_holds_stays_in_it(gpu_api, name):
    """A NaN, an infinity or nothing at all in one matrix: the others come out as they do without, bit for bit; reruns on
    workspaces of zeros and of NaN likewise."""
    rng = np.random.default_rng(24)
    shapes, _ = form(name)
    g = [gradient(rng, *s) for s in shapes]
    p = [rng.standard_normal(s).astype(np.float32) for s in shapes]
    hp = gpu_api.Muon(lr=0.1, momentum=0.5)

    def step(g, fill):
        dp, dm = up(p), zeros(shapes)
        ws = torch.full((gpu_api.muon_workspace_bytes(dp),), fill, dtype=torch.uint8, device="cuda")
        gpu_api.muon_step(hp, dp, up(g), dm, ws=ws)
        return dp, dm

    clean = step(g, 0)
    assert all(torch.equal(a, b) for x, y in zip(step(g, 255), clean) for a, b in zip(x, y))
    for i in {0, len(shapes) - 1}:
        for value in (np.nan, np.inf, 0.0):
            h = [a.copy() for a in g]
            if value == 0.0:
                h[i][:] = 0.0
            else:
                h[i][-1, -1] = value
            dp, dm = step(h, 255)
            for k in range(len(shapes)):
                if k != i:
                    assert torch.equal(dp[k], clean[0][k]) and torch.equal(dm[k], clean[1][k]), (shapes[i], value, shapes[k])
            assert torch.equal(dp[i].cpu(), torch.from_numpy(p[i])) if value == 0.0 else bool(torch.isnan(dp[i]).all())


@pytest.mark.parametrize("name", EVERY)
def test_captured_replays(gpu_api, name):
    """A captured step, replayed with new gradients in its buffers and eager steps of other matrices between."""
    rng = np.random.default_rng(25)
    shapes, _ = form(name)
    p0 = [rng.standard_normal(s).astype(np.float32) for s in shapes]
    hp = gpu_api.Muon(lr=0.05, weight_decay=0.01)
    g = up([gradient(rng, *s) for s in shapes])
    ep, em, cp, cm = up(p0), zeros(shapes), up(p0), zeros(shapes)
    ws = torch.empty(gpu_api.muon_workspace_bytes(cp), dtype=torch.uint8, device="cuda")
    gpu_api.muon_step(hp, up(p0), g, zeros(shapes), ws=ws)   # the first use of a kernel sets its LDS attribute
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        gpu_api.muon_step(hp, cp, g, cm, ws=ws)
    for k in range(3):
        for t in g:
            t.mul_(1.5 + k)
        graph.replay()
        gpu_api.muon_step(hp, ep, g, em)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(cp + cm, ep + em)), k


@pytest.mark.parametrize("name", EVERY)
@pytest.mark.parametrize("eps", [1e-30, 1e-37])
def test_norms_that_squares_lose(gpu_api, name, eps):
    """Gradients whose squares are lost in fp32: X0 is their multiple by 2^47, far below one, and every pass multiplies it by a.
    The first pass splits X0 at a scale for a norm of one, 2^14: off by half a step of an fp16 subnormal, 2^-25 / 2^14 an element."""
    rng = np.random.default_rng(26)
    shapes, row = form(name)
    g = [gradient(rng, *s, kind="noise") * np.float32(1e-20 * (2000 / max(2000, s[0] * s[1])) ** 0.5) for s in shapes]
    hp = gpu_api.Muon(lr=1.0, momentum=0.0, eps=eps, nesterov=False, scale_mode=0)
    dp = zeros(shapes)
    gpu_api.muon_step(hp, dp, up(g), zeros(shapes))
    for i, s in enumerate(shapes):
        X0 = 2.0 ** 47 * g[i].astype(np.float64)
        e = 3 * (8 + np.sqrt(max(32 * row, 256)) / 2) * 2.0 ** -24
        assert np.linalg.norm(-dp[i].cpu().numpy().astype(np.float64) - A ** 5 * X0) <= A ** 5 * (
            2.0 ** -39 * X0.size ** 0.5 + 5 * e * np.linalg.norm(X0)), s


@pytest.mark.parametrize("name", ["alone1", "alone2", "direct1", "direct2", "sums1", "sums2", "sums4", "sums4_two"])
def test_a_product_by_itself(gpu_api, name):
    """With b = c = 0 the one step is X = a X0, element by element one product of split operands: 2^-21 (8 half steps of fp32).  X0's
    element, a's square in |P|_F (which only sets a scale: none), y's scale back (a power of two: none), the step size and the
    parameter are rounded once each (3), and the norm, common to all elements, in its squares' products and sums (half of 8 + sqrt(n) / 2), its
    root, eps, and reciprocal (3)."""
    rng = np.random.default_rng(27)
    shapes, row = form(name)
    g = [(rng.uniform(0.5, 1, s) * rng.choice([-1, 1], s)).astype(np.float32) for s in shapes]
    a = float(np.float32(1.7))
    hp = gpu_api.Muon(lr=1.0, momentum=0.0, a=a, b=0.0, c=0.0, steps=1, nesterov=False, scale_mode=0)
    dp = zeros(shapes)
    gpu_api.muon_step(hp, dp, up(g), zeros(shapes))
    worst = 0.0
    for i, s in enumerate(shapes):
        ref = -a * g[i].astype(np.float64) / (np.linalg.norm(g[i].astype(np.float64)) + float(hp.eps))
        off = (np.abs(dp[i].cpu().numpy() - ref) / np.abs(ref)).max()
        limit = (8 + 3 + 4 + np.sqrt(max(32 * row, 256)) / 4 + 3) * 2.0 ** -24
        worst = max(worst, off / 2.0 ** -24)
        assert off <= limit, s
    record(f"muon product {name}", half_steps=worst)


@pytest.mark.parametrize("shape", [(64, 1408), (40, 64), (128, 64)], ids=str)
def test_the_published_factor_of_matrices_stored_in_out(gpu_api, shape):
    """f = sqrt(max(1, out / in)) by way of lr f and weight_decay / f: p = p (1 - lr wd) - lr f X."""
    rng = np.random.default_rng(28)
    lr, wd, f = 0.02, 0.1, max(1.0, shape[1] / shape[0]) ** 0.5
    g, p = [gradient(rng, *shape)], [rng.standard_normal(shape).astype(np.float32)]
    hp = gpu_api.Muon(lr=lr * f, momentum=0.0, weight_decay=wd / f, scale_mode=gpu_api.MUON_SCALE_NONE, nesterov=False)
    dp = up(p)
    gpu_api.muon_step(hp, dp, up(g), zeros([shape]))
    X, bound = recipe(g[0].astype(np.float64), 5, float(hp.eps), 1)
    ref = p[0] * (1 - lr * wd) - lr * f * X
    # lr f, weight_decay / f, the decay, the step size and the result are rounded once each
    tol = 2.0 ** -24 * (4 * np.linalg.norm(p[0]) + 2 * lr * f * np.linalg.norm(X) + np.linalg.norm(ref))
    assert distance(dp[0], ref) <= lr * f * bound + tol


def test_two_calls_at_once(gpu_api):
    """Steps on two streams, and a linear with its epilogue and the backward of that beside them: as one after the other."""
    rng = np.random.default_rng(29)
    names = ("sums4_two", "direct2_two")
    hp = gpu_api.Muon(lr=0.05)
    start = {n: ([rng.standard_normal(s).astype(np.float32) for s in FORMS[n][1]], [gradient(rng, *s) for s in FORMS[n][1]]) for n in names}
    desc = gpu_api.make_desc(512, 1032, 4, 32, 16, 0.25)
    gen = torch.Generator("cuda").manual_seed(6)
    codes = torch.randint(0, 16, (512, 1032), generator=gen, device="cuda", dtype=torch.uint8)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    weights = (gpu_api.pack(desc, codes), 0.01 * draw(16, 1032), 0.01 * draw(16, 1032), draw(16, 16), draw(16, 1032))
    x, mul = draw(700, 512).to(torch.bfloat16), draw(700, 1032).to(torch.bfloat16)

    def block():
        y, z, _ = gpu_api.forward_epilogue(desc, x, *weights, act="gelu", mul=mul, keep_z=True, out_dtype=torch.bfloat16)
        return [y, z, *gpu_api.epilogue_backward(y, z, "gelu", mul=mul, want_dbias=True)]

    def steps(n, state):
        for _ in range(3):
            gpu_api.muon_step(hp, state[0], state[1], state[2])

    state = {n: (up(p), up(g), zeros(FORMS[n][1])) for n, (p, g) in start.items()}
    for n in names:
        steps(n, state[n])
    alone = block()
    torch.cuda.synchronize()
    again = {n: (up(p), up(g), zeros(FORMS[n][1])) for n, (p, g) in start.items()}
    torch.cuda.synchronize()
    streams, beside = [torch.cuda.Stream() for _ in range(3)], []
    for s, n in zip(streams, names):
        with torch.cuda.stream(s):
            steps(n, again[n])
    with torch.cuda.stream(streams[2]):
        for _ in range(3):
            beside.append(block())
    torch.cuda.synchronize()
    for n in names:
        assert all(torch.equal(a, b) for x, y in zip(state[n], again[n]) for a, b in zip(x, y))
    assert all(torch.equal(a, b) for got in beside for a, b in zip(got, alone))
