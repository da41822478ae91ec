"""The operators together, as a fine-tuning step and the serving after it use them: a gated MLP block forward with epilogues, its
backward, the orthogonalised step on the six adapters, merge, deployment and single tokens.

Every stage is compared in 64 bits at the tensors that the stage before it left on the GPU: a linear to TOL of its largest value, as
everywhere here, and half a bf16 step of the value where the result is bf16.  The gradients of the whole block are then
compared with differences of the whole block in 64 bits, along the gradient: up to eight bf16 roundings lie on a path (2^-8 each)
and three linears (TOL of the largest value, at most four times the root mean square: 4 TOL), 8 * 2^-8 + 3 * 4 * TOL = 0.055."""
import ctypes

import pytest
import torch

import epilogue_cases as ec
from helpers import TOL, record

pytestmark = pytest.mark.gpu

S = 0.25
BF16 = torch.bfloat16
NAMES = ("gate", "up", "down")


class Block:
    """x + down(silu(gate x) * up x), d wide with ff between."""

    def __init__(self, api, T, d, ff, bits, group, rank):
        self.api, self.group, self.bits, self.rank = api, group, bits, rank
        self.host, self.desc, self.triple, self.p = {}, {}, {}, {}
        for k, n in enumerate(NAMES):
            i, o = (ff, d) if n == "down" else (d, ff)
            codes, alpha, beta, x, A, B = ec.drawn_layer(20 + k, T, i, o, bits, group, rank)
            self.host[n] = (codes, alpha, beta)
            self.desc[n] = api.make_desc(i, o, bits, group, rank, S)
            self.triple[n] = (api.pack(self.desc[n], codes.cuda()), alpha.cuda(), beta.cuda())
            self.p[n] = [A.cuda(), B.cuda()]
            if n == "gate":
                self.x = x.cuda()
        self.dy = torch.randn((T, d), generator=torch.Generator().manual_seed(30)).to(BF16).cuda()
        self.m = {n: [torch.zeros_like(t) for t in self.p[n]] for n in NAMES}
        self.hp = api.Muon(lr=0.02, momentum=0.9, weight_decay=0.1)

    def step(self):
        """Forward, backward and update; everything it made."""
        api, d, t, p = self.api, self.desc, self.triple, self.p
        v = {}
        v["up"], _, kept_u = api.forward_epilogue(d["up"], self.x, *t["up"], *p["up"], keep=True, out_dtype=BF16)
        v["h"], v["z"], kept_g = api.forward_epilogue(d["gate"], self.x, *t["gate"], *p["gate"], act="silu", mul=v["up"], keep_z=True,
                                                      keep=True, out_dtype=BF16)
        v["y"], _, kept_d = api.forward_epilogue(d["down"], v["h"], *t["down"], *p["down"], residual=self.x, keep=True, out_dtype=BF16)
        g = {}
        v["dh"], *g["down"] = api.backward_kept(d["down"], self.dy, kept_d, *t["down"], *p["down"])
        v["dz"], v["dup"], _ = api.epilogue_backward(v["dh"], v["z"], "silu", mul=v["up"])
        v["dx_gate"], *g["gate"] = api.backward_kept(d["gate"], v["dz"], kept_g, *t["gate"], *p["gate"])
        v["dx_up"], *g["up"] = api.backward_kept(d["up"], v["dup"], kept_u, *t["up"], *p["up"])
        v["before"] = {n: [a.clone() for a in p[n]] for n in NAMES}
        api.muon_step(self.hp, *([t for n in NAMES for t in of[n]] for of in (p, g, self.m)))
        v["g"] = g
        return v

    def linear64(self, n, x, A, B):
        return ec.linear64(*self.host[n], x.cpu(), self.group, A.cpu(), B.cpu(), S)

    def loss64(self, p):
        """<y, dy> of the whole block in 64 bits."""
        x = self.x.cpu().double()
        h = ec.act64(self.linear64("gate", x, *p["gate"]), "silu")[0] * self.linear64("up", x, *p["up"])
        return float(((x + self.linear64("down", h, *p["down"])) * self.dy.cpu().double()).sum())

    def gradients64(self, n, x, dy, A, B):
        codes, alpha, beta = self.host[n]
        rows = lambda t: t.double().repeat_interleave(self.group, 0)  # noqa: E731
        x, dy, A, B = (t.cpu().double() for t in (x, dy, A, B))
        pooled = x.view(x.shape[0], -1, self.group).mean(2)
        dq = dy @ B.T
        dx = dy @ (codes.double() * rows(alpha) + rows(beta)).T + S / self.group * (dq @ A.T).repeat_interleave(self.group, 1)
        return dx, S * pooled.T @ dq, S * (pooled @ A).T @ dy


def near(got, ref, tol=0.0, what=""):
    got = got.cpu()
    bound = tol + (2.0 ** -8 * (ref.abs() + tol) if got.dtype == BF16 else 0.0)
    worst = float(((got.double() - ref).abs() / bound).max())
    assert worst <= 1, (what, worst)     # (a NaN is not)
    return worst


@pytest.mark.parametrize("T,d,ff,bits,group,rank", [(77, 256, 704, 4, 32, 16), (300, 512, 1408, 4, 64, 48), (1, 256, 704, 4, 32, 8),
                                                    (130, 384, 1152, 3, 64, 24), (40, 512, 1024, 2, 128, 4)])
def test_mlp_step_and_serving(gpu_api, T, d, ff, bits, group, rank):
    b = Block(gpu_api, T, d, ff, bits, group, rank)
    v = b.step()
    old, worst = v["before"], {}
    lin = lambda n, x: b.linear64(n, x, *old[n])  # noqa: E731
    bar = lambda t: TOL * float(t.abs().max())  # noqa: E731

    up = lin("up", b.x)
    worst["up"] = near(v["up"], up, bar(up))
    z = lin("gate", b.x)
    worst["z"] = near(v["z"], z, bar(z))
    mul = v["up"].cpu().double()
    worst["h"] = near(v["h"], ec.act64(z, "silu")[0] * mul, 1.1 * bar(z) * mul.abs() + 1e-30)   # silu's slope is at most 1.1
    y = lin("down", v["h"])
    worst["y"] = near(v["y"], y + b.x.cpu().double(), bar(y))

    for n, x, dy, dx in (("down", v["h"], b.dy, "dh"), ("gate", b.x, v["dz"], "dx_gate"), ("up", b.x, v["dup"], "dx_up")):
        for got, ref, what in zip((v[dx], *v["g"][n]), b.gradients64(n, x, dy, *old[n]), ("x", "A", "B")):
            worst[f"d{what} {n}"] = near(got, ref, bar(ref), f"{n} d{what}")
    dh, zk = v["dh"].cpu().double(), v["z"].cpu().double()
    value, slope, _ = ec.act64(zk, "silu")
    # fp32 at z: exp's argument is rounded by 2^-24 |z|, and eight half steps more
    worst["dz"] = near(v["dz"], dh * mul * slope, 2.0 ** -24 * (8 + 4 * zk.abs()) * (dh * mul).abs() * (1 + zk.abs()) + 1e-30)
    worst["dup"] = near(v["dup"], dh * value, 2.0 ** -24 * (8 + 4 * zk.abs()) * (dh * value).abs() + 1e-30)

    for n in NAMES:                      # against differences
        for k in range(2):
            g64 = v["g"][n][k].cpu().double()
            if not float(g64.norm()) > 0:
                continue
            D = g64 / g64.norm()
            e = 1e-4
            at = lambda sign: b.loss64({m: [a.cpu().double() + (sign * e * D if (m, j) == (n, k) else 0) for j, a in enumerate(old[m])]  # noqa: E731
                                        for m in NAMES})
            slope = (at(1) - at(-1)) / (2 * e)
            off = abs(float(g64.norm()) - slope) / abs(slope)
            worst[f"slope {n}{k}"] = off
            assert off <= 0.055, (n, k, off)

    # the step moved every adapter by lr 0.2 sqrt(longer side) X, X's singular values near one
    for n in NAMES:
        for new, was in zip(b.p[n], old[n]):
            r = min(new.shape)
            X = (was.double() * (1 - 0.02 * 0.1) - new.double()) / (0.02 * 0.2 * max(new.shape) ** 0.5)
            assert 0.3 * r ** 0.5 < float(X.norm()) < 1.3 * r ** 0.5 or T < r

    # serving: adapters merged, the block on one and on three tokens
    flat = {n: gpu_api.make_desc(b.desc[n].d_in, b.desc[n].d_out, bits, group) for n in NAMES}
    beta = {n: gpu_api.merge(b.desc[n], b.triple[n][2], *b.p[n]) for n in NAMES}
    for tokens in {1, min(T, 3)}:
        x = b.x[:tokens].contiguous()

        def linear(n, x, **kw):
            packed, alpha = b.triple[n][:2]
            if gpu_api.load().qalora_deployed_bytes(ctypes.byref(flat[n])):   # 4 bits and its shapes
                return gpu_api.forward_deployed_epilogue(flat[n], x, gpu_api.deploy(flat[n], packed, alpha, beta[n]), packed,
                                                         out_dtype=BF16, **kw)
            return gpu_api.forward_epilogue(flat[n], x, packed, alpha, beta[n], out_dtype=BF16, **kw)

        ups = linear("up", x)
        h = linear("gate", x, act="silu", mul=ups)
        stream = x.clone()
        y = linear("down", h, residual=stream, y=stream)
        assert y is stream
        now = lambda n, x: b.linear64(n, x, *b.p[n])  # noqa: E731
        u64, z64, y64 = now("up", x), now("gate", x), now("down", h)
        worst[f"serve up {tokens}"] = near(ups, u64, bar(u64))
        mul = ups.cpu().double()
        worst[f"serve h {tokens}"] = near(h, ec.act64(z64, "silu")[0] * mul, 1.1 * bar(z64) * mul.abs() + 1e-30)
        worst[f"serve y {tokens}"] = near(y, y64 + x.cpu().double(), bar(y64))
    record(f"mlp step {T}x{d}x{ff} bits {bits}", **{k.replace(" ", "_"): w for k, w in worst.items()})


def test_captured_step_follows_the_eager_one(gpu_api):
    """The whole step in one graph, replayed with eager steps of a second block between."""
    shape = (130, 256, 704, 4, 32, 16)
    eager, caught = Block(gpu_api, *shape), Block(gpu_api, *shape)
    Block(gpu_api, *shape).step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        w = caught.step()
    for _ in range(4):
        graph.replay()
        v = eager.step()
        torch.cuda.synchronize()
        for n in NAMES:
            assert all(torch.equal(a, b) for a, b in zip(eager.p[n] + eager.m[n], caught.p[n] + caught.m[n]))
        assert all(torch.equal(v[k], w[k]) for k in ("up", "h", "z", "y", "dh", "dz", "dup", "dx_gate", "dx_up"))
