"""The orthogonalised update (qalora_muon_step) on the GPU against the same recipe in 64 bits.

The step is read off parameters that start at zero, so that the matrix X itself is compared and not a parameter
that it moves a little.  Tolerance: an error made in X_k grows by at most a per remaining step, so
|dX| <= e * sum_k a^(steps - k) |X_k|_F, with e the error of one pass relative to its operands.  A pass sums at most
a few hundred products in a row (the shares of the blocks are added afterwards): their roundings, 2^-25 each at random
signs, add up to under sqrt(512) / 2 * 2^-24 of the sum, for G, G^2 and P X: e = 32 * 2^-24."""
import numpy as np
import pytest
import torch

from helpers import record

pytestmark = pytest.mark.gpu

A, B, C = (float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315))


def gradient(rng, rows, cols, kind="mixed"):
    """Kinds: noise; a few strong directions over weak noise; rank one."""
    g = rng.standard_normal((rows, cols)) * 1e-3
    if kind == "mixed":
        k = max(1, min(rows, cols) // 4)
        g += (rng.standard_normal((rows, k)) * 0.5 ** np.arange(k)) @ rng.standard_normal((k, cols))
    if kind == "one":
        g = np.outer(rng.standard_normal(rows), rng.standard_normal(cols))
    return g.astype(np.float32)


def orthogonal(u, steps, eps, abc=(A, B, C)):
    """X of the recipe in 64 bits, and the tolerance of its distance in the 2-norm over the elements."""
    a, b, c = abc
    X = u.T if u.shape[0] > u.shape[1] else u
    X = X / (np.sqrt((X * X).sum()) + eps)
    bound = 0.0
    for k in range(steps):
        bound += abs(a) ** (steps - k) * np.sqrt((X * X).sum())
        G = X @ X.T
        X = a * X + (b * G + c * (G @ G)) @ X
    bound += np.sqrt((X * X).sum())
    return (X.T if u.shape[0] > u.shape[1] else X), 32 * 2.0 ** -24 * bound


def up(arrays):
    return [torch.from_numpy(a.copy()).cuda() for a in arrays]


LISTS = {
    "adapter": [(32, 16), (16, 1024)],
    "odd": [(1, 1), (1, 7), (7, 1), (3, 5), (17, 63), (65, 33), (64, 64), (15, 64), (16, 65), (63, 64)],
    "wide": [(128, 128), (127, 1000), (128, 4096), (688, 128), (129, 100)],
    "mixed": [(5, 300), (128, 500), (40, 40), (1, 3000), (2000, 90)],
    "layer": [s for i, o in [(512, 512)] * 4 + [(512, 1408)] * 2 + [(1408, 512)] for s in ((i // 32, 64), (64, o))],
    "many": [(8 + k, 40 * k + 1) for k in range(32)],
    "long": [(64, 22016), (48, 20001)],
    # at the longest sides that one launch takes, that one launch a pass takes, and one beyond
    "one32": [(32, 768), (768, 31), (1, 1)],
    "one64": [(64, 384), (384, 33), (50, 383), (64, 1)],
    "each32": [(32, 769), (12288, 32), (9, 40), (31, 12287)],
    "each64": [(64, 385), (4096, 64), (33, 4095), (1, 1)],
    "sums32": [(32, 12289), (9, 40)],
    "sums64": [(4097, 64), (7, 9)],
    "alone32": [(32, 1024), (1024, 32), (31, 1023), (1, 1), (9, 40)],
    "alone64": [(64, 512), (512, 33), (50, 511), (64, 1)],
    "beyond32": [(1025, 32), (9, 40), (1, 1)],
    "beyond64": [(64, 513), (7, 9)],
}
KINDS = {  # of launches: by the largest matrix
    "alone": (1, 1),
    "alone64": (40, 500),
    "beyond32": (20, 1100),
    "beyond64": (44, 700),
    "beyond128": (80, 90),
    "sums32": (8, 12300),
    "sums64": (36, 4100),
}


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_direction_matches_the_recipe(gpu_api, name, nesterov):
    rng = np.random.default_rng(7)
    shapes = LISTS[name]
    g = [gradient(rng, *s, kind=("mixed", "noise", "one")[i % 3]) for i, s in enumerate(shapes)]
    m = [gradient(rng, *s, kind="noise") for s in shapes]
    hp = gpu_api.Muon(lr=1.0, momentum=0.9, nesterov=nesterov, scale_mode=gpu_api.MUON_SCALE_NONE)
    dp, dg, dm = up([np.zeros(s, np.float32) for s in shapes]), up(g), up(m)
    gpu_api.muon_step(hp, dp, dg, dm)
    mu, worst = float(hp.momentum), 0.0
    for i in range(len(shapes)):
        assert np.array_equal(dg[i].cpu().numpy(), g[i])
        m64 = mu * m[i].astype(np.float64) + g[i]
        got_m = dm[i].cpu().numpy()
        assert np.abs(got_m - m64).max() <= 2.0 ** -24 * np.abs(m64).max()
        u = g[i] + mu * got_m.astype(np.float64) if nesterov else got_m.astype(np.float64)
        ref, bound = orthogonal(u, hp.steps, float(hp.eps))
        off = np.sqrt(((-dp[i].cpu().numpy().astype(np.float64) - ref) ** 2).sum())
        worst = max(worst, off / bound)
        assert off <= bound, (shapes[i], off, bound)
    record(f"muon {name} nesterov={nesterov}", of_bound=worst)


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("steps,abc", [(1, (A, B, C)), (2, (A, B, C)), (9, (1.5, -0.5, 0.0)), (16, (1.5, -0.5, 0.0))])
def test_steps_and_coefficients(gpu_api, steps, abc, kind):
    rng = np.random.default_rng(8)
    shapes = [(16, 200), (300, 24), KINDS[kind]]
    g = [gradient(rng, *s, kind="noise") for s in shapes]
    hp = gpu_api.Muon(lr=1.0, momentum=0.0, a=abc[0], b=abc[1], c=abc[2], steps=steps, nesterov=False, scale_mode=0)
    dp, dg, dm = up([np.zeros(s, np.float32) for s in shapes]), up(g), up([np.zeros(s, np.float32) for s in shapes])
    gpu_api.muon_step(hp, dp, dg, dm)
    for i in range(len(shapes)):
        ref, bound = orthogonal(g[i].astype(np.float64), steps, float(hp.eps), abc)
        assert np.sqrt(((-dp[i].cpu().numpy() - ref) ** 2).sum()) <= bound
        if steps == 16 and i < 2:   # singular values of noise are near each other: they have all come to one
            assert np.abs(np.linalg.svd(dp[i].cpu().numpy().astype(np.float64), compute_uv=False) - 1).max() <= 1e-4


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("mode,scale", [(0, lambda r, c: 1.0), (1, lambda r, c: max(1.0, r / c) ** 0.5),
                                        (2, lambda r, c: 0.2 * max(r, c) ** 0.5)])
def test_parameters_decay_and_scale(gpu_api, mode, scale, kind):
    rng = np.random.default_rng(9)
    shapes = [(24, 500), (500, 24), KINDS[kind]]
    g = [gradient(rng, *s) for s in shapes]
    p = [rng.standard_normal(s).astype(np.float32) for s in shapes]
    hp = gpu_api.Muon(lr=0.02, momentum=0.95, weight_decay=0.1, scale_mode=mode)
    dp, dg, dm = up(p), up(g), up([np.zeros(s, np.float32) for s in shapes])
    gpu_api.muon_step(hp, dp, dg, dm, zero_grads=True)
    lr, wd, mu = float(hp.lr), float(hp.weight_decay), float(hp.momentum)
    for i, s in enumerate(shapes):
        assert not dg[i].any()      # consumed: ready for an accumulating backward
        X, bound = orthogonal(g[i] * (1 + mu), 5, float(hp.eps))
        step = lr * scale(*s)
        ref = p[i].astype(np.float64) * (1 - lr * wd) - step * X
        off = np.sqrt(((dp[i].cpu().numpy() - ref) ** 2).sum())
        # the decay, the step size and the result are rounded once each
        assert off <= step * bound + 2.0 ** -24 * (2 * np.linalg.norm(p[i]) + step * np.linalg.norm(X) + np.linalg.norm(ref))


def test_several_steps_and_reruns(gpu_api):
    """Five steps with the state carried on the device, twice: bit-identical, and each as the recipe says."""
    rng = np.random.default_rng(10)
    shapes = LISTS["layer"]
    p0 = [rng.standard_normal(s).astype(np.float32) * 0.02 for s in shapes]
    gs = [[gradient(rng, *s) for s in shapes] for _ in range(5)]
    hp = gpu_api.Muon(lr=0.02, momentum=0.95, weight_decay=0.01)
    runs = []
    for _ in range(2):
        dp, dm = up(p0), up([np.zeros(s, np.float32) for s in shapes])
        for g in gs:
            before = [x.cpu().numpy().astype(np.float64) for x in dp]
            gpu_api.muon_step(hp, dp, up(g), dm)
            for i, s in enumerate(shapes):
                m64 = dm[i].cpu().numpy().astype(np.float64)
                X, bound = orthogonal(g[i] + float(hp.momentum) * m64, 5, float(hp.eps))
                step = float(hp.lr) * 0.2 * max(s) ** 0.5
                ref = before[i] * (1 - float(hp.lr) * float(hp.weight_decay)) - step * X
                off = np.sqrt(((dp[i].cpu().numpy() - ref) ** 2).sum())
                assert off <= step * bound + 2.0 ** -22 * (np.linalg.norm(ref) + step * np.linalg.norm(X))
        runs.append([x.cpu() for x in dp + dm])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("long", [600, 1000, 3000, 13000])  # one launch, one a pass, and two
def test_zero_infinite_and_tiny_gradients(gpu_api, long):
    """A zero matrix moves nothing (a fresh adapter's A has the gradient zero); a NaN stays in its own matrix; gradients far
    below eps do not blow up."""
    rng = np.random.default_rng(11)
    shapes = [(16, 100), (100, 16), (16, 100), (8, long), (16, 100)]
    g = [gradient(rng, *s) for s in shapes]
    g[0][:] = 0
    g[1][50, 3] = np.nan
    g[2] *= 1e-30
    g[4][3, 7] = np.inf
    dp, dg, dm = up([np.ones(s, np.float32) for s in shapes]), up(g), up([np.zeros(s, np.float32) for s in shapes])
    hp = gpu_api.Muon(lr=1.0, momentum=0.5, scale_mode=0)
    gpu_api.muon_step(hp, dp, dg, dm)
    p = [x.cpu().numpy() for x in dp]
    assert (p[0] == 1).all()
    assert np.isnan(p[1]).all() and np.isnan(p[4]).all()
    assert np.abs(p[2] - 1).max() <= 1e-6
    X, bound = orthogonal(g[3] * 1.5, 5, float(hp.eps))
    assert np.sqrt(((1 - p[3].astype(np.float64) - X) ** 2).sum()) <= bound + 2.0 ** -24 * np.sqrt(p[3].size)


@pytest.mark.parametrize("name", ["mixed", "alone64", "one64", "each32", "sums32"])
def test_workspace_contents_do_not_matter(gpu_api, name):
    rng = np.random.default_rng(12)
    shapes = LISTS[name]
    g = [gradient(rng, *s) for s in shapes]
    out = []
    for fill in (0, 255):   # 255: every float of the workspace a NaN
        dp, dm = up([np.ones(s, np.float32) for s in shapes]), up([np.zeros(s, np.float32) for s in shapes])
        ws = torch.full((gpu_api.muon_workspace_bytes(dp),), fill, dtype=torch.uint8, device="cuda")
        gpu_api.muon_step(gpu_api.Muon(lr=0.1), dp, up(g), dm, ws=ws)
        out.append([x.cpu() for x in dp + dm])
    assert all(torch.equal(a, b) for a, b in zip(*out))
    with pytest.raises(gpu_api.QaloraError) as e:
        gpu_api.muon_step(gpu_api.Muon(lr=0.1), dp, up(g), dm, ws=ws[:-256])
    assert e.value.status == gpu_api.EWORKSPACE


@pytest.mark.parametrize("long", [600, 1000, 3000, 13000])
def test_captured_step_replays(gpu_api, long):
    """A captured step replayed with eager steps of other matrices between: state moves as by eager steps."""
    rng = np.random.default_rng(13)
    shapes = [(32, 64), (64, 512) if long == 3000 else (24, 512), (16, long)]
    g = up([gradient(rng, *s) for s in shapes])
    p0, z = [rng.standard_normal(s).astype(np.float32) for s in shapes], [np.zeros(s, np.float32) for s in shapes]
    hp = gpu_api.Muon(lr=0.05)
    ep, em = up(p0), up(z)
    cp, cm = up(p0), up(z)
    ws = torch.empty(gpu_api.muon_workspace_bytes(cp), dtype=torch.uint8, device="cuda")
    gpu_api.muon_step(hp, up(p0), g, up(z), ws=ws)    # the first use of a kernel sets its LDS attribute
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        gpu_api.muon_step(hp, cp, g, cm, ws=ws)
    for _ in range(4):
        graph.replay()
        gpu_api.muon_step(hp, ep, g, em)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(cp + cm, ep + em))


def test_refusals(gpu_api):
    ok = [torch.zeros((8, 40), device="cuda")]
    hp = gpu_api.Muon(lr=0.1)

    def status(hp, p, g=None, m=None):
        with pytest.raises(gpu_api.QaloraError) as e:
            gpu_api.muon_step(hp, p, g or [torch.zeros_like(t) for t in p], m or [torch.zeros_like(t) for t in p])
        return e.value.status

    assert status(hp, [torch.zeros((129, 130), device="cuda")]) == gpu_api.EUNSUPPORTED
    assert status(hp, ok * 33) == gpu_api.EINVAL
    assert status(gpu_api.Muon(lr=0.1, steps=0), ok) == gpu_api.EINVAL
    assert status(gpu_api.Muon(lr=0.1, eps=0.0), ok) == gpu_api.EINVAL
    with pytest.raises(ValueError):
        gpu_api.muon_step(hp, [torch.zeros(40, device="cuda")], [torch.zeros(40, device="cuda")], [torch.zeros(40, device="cuda")])
    with pytest.raises(ValueError):
        gpu_api.muon_step(hp, [torch.zeros((40, 8), device="cuda").T], ok, ok)
    with pytest.raises(ValueError):
        gpu_api.muon_step(hp, ok, [torch.zeros((8, 40))], ok)
    with pytest.raises(ValueError):
        gpu_api.muon_step(hp, ok, [torch.zeros((8, 40), device="cuda", dtype=torch.bfloat16)], ok)
    with pytest.raises(ValueError):
        gpu_api.muon_step(hp, ok, [], ok)
    with pytest.raises(ValueError):
        gpu_api.muon_step(hp, [], [], [])
    assert not ok[0].any()


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("eps", [1e-30, 1e-37])
def test_lost_norms_with_a_tiny_eps(gpu_api, eps, kind):
    """Zeros, and gradients whose squares are lost in fp32: X0 is their multiple by 2^47 at most, far below one, and every pass
    multiplies it by a: the update is a^steps X0.  Tolerance: the first pass takes X0 for a matrix of norm one, times 2^14 in two fp16
    whose lower one has steps of 2^-24: off by half of that, 2^-39 an element, at most; and 32 * 2^-24 a pass, as above."""
    rng = np.random.default_rng(15)
    shapes = [(16, 300), (300, 20), KINDS[kind], (12, 40)]
    g = [gradient(rng, *s, kind="noise") * np.float32(1e-20) for s in shapes]
    g[3][:] = 0
    hp = gpu_api.Muon(lr=1.0, momentum=0.0, eps=eps, nesterov=False, scale_mode=0)
    dp, dg, dm = up([np.zeros(s, np.float32) for s in shapes]), up(g), up([np.zeros(s, np.float32) for s in shapes])
    gpu_api.muon_step(hp, dp, dg, dm)
    for i in range(len(shapes)):
        X0 = 2.0 ** 47 * g[i].astype(np.float64)
        off = np.linalg.norm(-dp[i].cpu().numpy().astype(np.float64) - A ** 5 * X0)
        assert off <= A ** 5 * (2.0 ** -39 * X0.size ** 0.5 + 5 * 32 * 2.0 ** -24 * np.linalg.norm(X0))


@pytest.mark.parametrize("size", [1e-15, 1e-8, 1.0, 1e8, 1e15])
def test_gradients_of_any_size(gpu_api, size):
    """The direction does not depend on the gradients' size (eps far below them)."""
    rng = np.random.default_rng(14)
    shapes = [(16, 300), (100, 700), (513, 40)]
    g = [gradient(rng, *s) * np.float32(size) for s in shapes]
    hp = gpu_api.Muon(lr=1.0, momentum=0.0, eps=1e-20, nesterov=False, scale_mode=0)
    dp, dg, dm = up([np.zeros(s, np.float32) for s in shapes]), up(g), up([np.zeros(s, np.float32) for s in shapes])
    gpu_api.muon_step(hp, dp, dg, dm)
    for i in range(len(shapes)):
        ref, bound = orthogonal(g[i].astype(np.float64), hp.steps, float(hp.eps))
        assert np.sqrt(((-dp[i].cpu().numpy().astype(np.float64) - ref) ** 2).sum()) <= bound
