"""The operators around the linear layers run together, as a training step of an MLP block uses them: norm, up-projection with
bias and GELU, down-projection with bias, gate and residual sum with the next norm; every gradient; the global norm and clipping.
The gradients are compared with 64-bit arithmetic and, through it, with differences of the loss."""
import numpy as np
import pytest
import torch

import paper_2105_14450_amd as c3
from oracle import block, mlp
from oracle.layout import Cube
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


class Step:
    """x -> n0 = N0(x); z = n0 W1 + b1, h = gelu(z); u = h W2 + b2; r = x + scale g u, n = N1(r); loss = <dr, r> + <dn, n>"""

    def __init__(self, q, M, K, N, dtype, seed=3):
        self.q, self.M, self.K, self.N, self.dtype, self.scale = q, M, K, N, dtype, 0.5
        g = np.random.default_rng(seed)
        code, n3 = gu.CODE[dtype], q ** 3
        # the residual stream lies as the X shards of the first layer (input in y), that is as the Y shards of the second (input in z)
        self.c1, self.c2 = Cube(q, M, K, N, "y"), Cube(q, M, N, K, "z")
        self.d1 = c3.make_desc(q, M, K, N, in_dtype=code, shard_dtype=code, in_axis=c3.AXIS_Y)
        self.d2 = c3.make_desc(q, M, N, K, in_dtype=code, shard_dtype=code, in_axis=c3.AXIS_Z)
        self.m = c3.make_matrix(q, M, K, c3.AXIS_X, c3.AXIS_Z, c3.SPLIT_ROWS, code)
        f = lambda s, sigma, mean=0.0: g.normal(mean, sigma, size=s).astype(np.float32)
        self.v = {"x": f((M, K), 1.0), "W1": f((K, N), K ** -0.5), "b1": f(N, 0.3), "W2": f((N, K), N ** -0.5), "b2": f(K, 0.3),
                  "g0": f(K, 0.2, 1.0), "beta0": f(K, 0.2), "gate": f(K, 0.2, 1.0), "g1": f(K, 0.2, 1.0), "dr": f((M, K), 1.0), "dn": f((M, K), 1.0)}
        T = torch.bfloat16 if dtype == "bf16" else torch.float32
        if dtype == "bf16":
            for k in ("x", "W1", "W2", "dr", "dn"):
                self.v[k] = torch.from_numpy(self.v[k]).to(T).float().numpy()
        up = lambda s: torch.from_numpy(np.ascontiguousarray(s.reshape((n3,) + s.shape[3:]))).cuda()
        put = lambda s: up(s).to(T)
        t = self.t = {"x": put(self.c1.shard_x(self.v["x"])), "W1": put(self.c1.shard_w(self.v["W1"])), "W2": put(self.c2.shard_w(self.v["W2"])),
                      "dr": put(self.c2.shard_y(self.v["dr"])), "dn": put(self.c2.shard_y(self.v["dn"]))}
        np.testing.assert_array_equal(self.c1.shard_x(self.v["x"]), self.c2.shard_y(self.v["x"]))
        for k, cube in (("b1", self.c1), ("b2", self.c2), ("g0", self.c2), ("beta0", self.c2), ("gate", self.c2), ("g1", self.c2)):
            t[k] = up(cube.shard_bias(self.v[k]).astype(np.float32))
        like = lambda k: torch.full_like(t[k], float("nan"))
        wide = torch.full((n3, self.c1.Ms, self.c1.Nb), float("nan"), dtype=T, device="cuda")
        for k in ("n0", "u", "r", "n", "du", "dx1", "dn0", "dx"):
            t[k] = like("x")
        for k in ("z", "h", "dh", "dz"):
            t[k] = wide.clone()
        for k in ("W1", "W2", "b1", "b2", "g0", "beta0", "gate", "g1"):
            t["d" + k] = like(k)
        t["s0"], t["s1"] = (torch.full((M, 4), float("nan"), device="cuda") for _ in range(2))
        self.nd0 = c3.make_norm(pre=c3.NORM_LAYER, block_dtype=code)
        self.nd1 = c3.make_norm(pre=c3.NORM_RMS, block_dtype=code, scale=self.scale)
        P = c3.make_norm_params
        self.p0, self.p1 = P(pre_gamma=t["g0"], pre_beta=t["beta0"]), P(gate=t["gate"], pre_gamma=t["g1"])
        self.dp0, self.dp1 = P(pre_gamma=t["dg0"], pre_beta=t["dbeta0"]), P(gate=t["dgate"], pre_gamma=t["dg1"])
        self.e1 = c3.make_epilogue(c3.ACT_GELU, bias=t["b1"], z=t["z"], z_dtype=code)
        self.e2 = c3.make_epilogue(c3.ACT_NONE, bias=t["b2"])
        scratch = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        eb = c3.cube3d_epilogue_workspace_bytes
        self.ws = scratch(max(eb(self.d1, c3.OP_FWD), eb(self.d2, c3.OP_FWD), eb(self.d1, c3.OP_BIAS_BWD),
                              c3.cube3d_workspace_bytes(self.d2, c3.OP_BIAS_BWD, True), c3.cube3d_norm_workspace_bytes(self.m, self.nd0)))
        self.names = ("dW1", "db1", "dW2", "db2", "dg0", "dbeta0", "dgate", "dg1")
        self.grads = c3.make_tensor_list([t[k] for k in self.names])
        self.clipped = [torch.full(t[k].shape, float("nan"), device="cuda") for k in self.names]
        self.out = c3.make_tensor_list(self.clipped)
        self.sumsq, self.norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
        self.gws = scratch(c3.cube3d_grad_norm_workspace_bytes(self.grads))

    def run(self):
        t, code, ws = self.t, gu.CODE[self.dtype], self.ws
        c3.virtual_cube_norm_fwd(self.m, self.nd0, self.p0, t["x"], None, None, t["n0"], t["s0"])
        c3.virtual_cube_linear_fwd_fused(self.d1, self.e1, t["n0"], t["W1"], t["h"], ws)
        c3.virtual_cube_linear_fwd_fused(self.d2, self.e2, t["h"], t["W2"], t["u"], ws)
        c3.virtual_cube_norm_fwd(self.m, self.nd1, self.p1, t["x"], t["u"], t["r"], t["n"], t["s1"])
        c3.virtual_cube_norm_bwd(self.m, self.nd1, self.p1, t["s1"], t["dr"], t["dn"], t["r"], t["u"], t["dx1"], t["du"], self.dp1, ws)
        c3.virtual_cube_bias_bwd(self.d2, t["du"], t["db2"], ws)
        c3.virtual_cube_linear_bwd_dw(self.d2, t["h"], t["du"], t["dW2"])
        c3.virtual_cube_linear_bwd_dx(self.d2, t["du"], t["W2"], t["dh"])
        c3.virtual_cube_linear_epilogue_bwd(self.d1, c3.ACT_GELU, code, code, code, t["z"], t["dh"], t["dz"], t["db1"], ws)
        c3.virtual_cube_linear_bwd_dw(self.d1, t["n0"], t["dz"], t["dW1"])
        c3.virtual_cube_linear_bwd_dx(self.d1, t["dz"], t["W1"], t["dn0"])
        c3.virtual_cube_norm_bwd(self.m, self.nd0, self.p0, t["s0"], t["dx1"], t["dn0"], t["x"], None, t["dx"], None, self.dp0, ws)
        c3.cube3d_grad_norm(self.grads, self.sumsq, self.norm, self.gws)
        c3.cube3d_grad_clip(self.grads, self.out, self.sumsq, 1.0)

    def forward(self, v):
        o = block.norm_forward(v["x"], None, "none", "layer", 1e-5, 1e-5, 1.0, {"pre_gamma": v["g0"], "pre_beta": v["beta0"]})
        z = o["n"] @ v["W1"] + v["b1"]
        u = mlp.act(z, "gelu") @ v["W2"] + v["b2"]
        o1 = block.norm_forward(v["x"], u, "none", "rms", 1e-5, 1e-5, self.scale, {"gate": v["gate"], "pre_gamma": v["g1"]})
        return o, z, u, o1

    def loss(self, v):
        o1 = self.forward(v)[3]
        return (v["dr"] * o1["r"]).sum() + (v["dn"] * o1["n"]).sum()

    def reference(self):
        v = {k: a.astype(np.float64) for k, a in self.v.items()}
        o, z, u, o1 = self.forward(v)
        g1 = block.norm_backward(v["dr"], v["dn"], o1["r"], u, o1["stats"], "none", "rms", self.scale, {"gate": v["gate"], "pre_gamma": v["g1"]})
        h, dh = mlp.act(z, "gelu"), g1["du"] @ v["W2"].T
        dz = dh * mlp.act_grad(z, "gelu")
        g0 = block.norm_backward(g1["dx"], dz @ v["W1"].T, v["x"], None, o["stats"], "none", "layer", 1.0,
                                 {"pre_gamma": v["g0"], "pre_beta": v["beta0"]})
        return v, {"r": o1["r"], "n": o1["n"], "dx": g0["dx"], "dW1": o["n"].T @ dz, "db1": dz.sum(0), "dW2": h.T @ g1["du"], "db2": g1["du"].sum(0),
                   "dg0": g0["pre_gamma"], "dbeta0": g0["pre_beta"], "dgate": g1["gate"], "dg1": g1["pre_gamma"]}

    def results(self):
        host = lambda t: t.float().cpu().numpy().astype(np.float64).reshape((self.q,) * 3 + tuple(t.shape[1:]))
        cut = {"r": self.c2.unshard_y, "n": self.c2.unshard_y, "dx": self.c2.unshard_y, "dW1": self.c1.unshard_w, "dW2": self.c2.unshard_w,
               "db1": self.c1.unshard_bias}
        return {k: cut.get(k, self.c2.unshard_bias)(host(self.t[k])) for k in ("r", "n", "dx") + self.names}


@pytest.mark.parametrize("q,M,K,N,dtype", [(2, 64, 64, 256, "f32"), (3, 45, 36, 144, "f32"), (1, 7, 24, 96, "f32"), (2, 512, 256, 1024, "bf16"),
                                           (1, 33, 128, 512, "bf16")])
def test_training_step(q, M, K, N, dtype):
    s = Step(q, M, K, N, dtype)
    s.run()
    torch.cuda.synchronize()
    v, want = s.reference()
    got = s.results()
    # fp32: a few dozen fp32 operations deep.  bf16: about ten roundings of 2^-8 lie on the longest way (n0, h, u, du, dh, dz, dn0,
    # dx and the two weights' products), independent of each other: sqrt(10) 2^-8 = 1.2 % of the largest entry, 3 % allowed.
    tol = 2e-5 if dtype == "f32" else 0.03
    for k in want:
        err = np.abs(got[k] - want[k]).max() / np.abs(want[k]).max()
        assert err <= tol, "%s: %g" % (k, err)
    norm = block.gradient_norm([got[k] for k in s.names])
    assert abs(s.norm.item() - norm) <= 2.0 ** -23 * norm
    f = min(1.0, 1.0 / norm)
    for k, c in zip(s.names, s.clipped):
        np.testing.assert_allclose(c.cpu().numpy(), s.t[k].float().cpu().numpy().astype(np.float64) * f, rtol=4 * 2.0 ** -24, atol=1e-40)
    if M * K <= 4096:       # the oracle's gradients against differences of the loss, along random directions
        g = np.random.default_rng(1)
        for k in ("x", "W1", "b1", "W2", "b2", "g0", "beta0", "gate", "g1"):
            direction = g.normal(size=v[k].shape)
            h = 1e-5
            diff = (s.loss({**v, k: v[k] + h * direction}) - s.loss({**v, k: v[k] - h * direction})) / (2 * h)
            along = (want["d" + k] * direction).sum()
            assert abs(diff - along) <= 1e-6 * (abs(diff) + np.abs(want["d" + k]).max())


def test_training_step_as_a_graph():
    s = Step(2, 512, 256, 1024, "bf16")
    c3.cube3d_init()
    s.run()
    torch.cuda.synchronize()
    keys = ("r", "n", "dx") + s.names
    state = lambda: [s.t[k].float().cpu().numpy() for k in keys] + [c.cpu().numpy() for c in s.clipped] + [s.norm.cpu().numpy()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for turn in range(3):
        s.t["x"].mul_(0.5 + turn)
        for k in keys:
            s.t[k].fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = state()
        s.run()
        torch.cuda.synchronize()
        for a, e in zip(replayed, state()):
            np.testing.assert_array_equal(a, e)
            assert np.isfinite(a).all()
