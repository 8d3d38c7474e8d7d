"""Digital operators beside the crossbar layers, without a GPU: their definitions against differences, the library's refusals, the
binding's checks, the plan of the launches."""
import ctypes as C

import numpy as np
import pytest

from oracle import digital


@pytest.fixture(scope="module")
def xb():
    import os
    from paper_2002_11151_amd import xbar
    if not os.path.exists(xbar.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    xbar.lib()
    return xbar


def differences(f, at, h=1e-5):
    """Gradient of the scalar f at the array `at` by central differences."""
    out = np.zeros_like(at)
    flat, grad = at.reshape(-1), out.reshape(-1)
    for i in range(flat.size):
        keep = flat[i]
        flat[i] = keep + h
        up = f()
        flat[i] = keep - h
        grad[i] = (up - f()) / (2 * h)
        flat[i] = keep
    return out


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_group_norm_gradient_is_that_of_the_formula(kind):
    rng = np.random.default_rng(3)
    x, skip, dy = (rng.normal(size=(2, 2, 3, 6)) for _ in range(3))
    gamma, beta = rng.uniform(0.5, 1.5, 6), rng.normal(size=6)

    def loss():
        mean, invstd = digital.gn_stats(x, 3, 1e-5)
        return float((digital.act(digital.gn_z(x, gamma, beta, mean, invstd, skip)[1], kind) * dy).sum())
    mean, invstd = digital.gn_stats(x, 3, 1e-5)
    got = digital.gn_bwd(x, dy, gamma, beta, mean, invstd, kind, skip)
    for g, at in zip(got, (x, gamma, beta, skip)):
        # truncation h^2 f''' / 6 and rounding 1e-16 |loss| / h
        assert np.abs(g - differences(loss, at)).max() < 1e-6


def test_adapter_gradients_are_those_of_the_formula():
    rng = np.random.default_rng(4)
    rows = np.array([1, -1, 0, 1, 5, 1])
    X, dY = rng.normal(size=(6, 4)), rng.normal(size=(6, 5))
    A, B, scale = rng.normal(size=(2, 3, 4)), rng.normal(size=(2, 3, 5)), rng.uniform(0.5, 2, 2)
    base, back = rng.normal(size=(6, 5)), np.zeros((6, 4))
    loss = lambda: float((digital.adapter_fwd(rows, base, X, A, B, scale)[0] * dY).sum())
    T = digital.adapter_fwd(rows, base, X, A, B, scale)[1]
    dX, dA, dB, _ = digital.adapter_bwd(rows, back, dY, X, T, A, B, scale)
    for g, at in ((dX, X), (dA, A), (dB, B)):
        assert np.abs(g - differences(loss, at)).max() < 1e-6
    assert not dX[1].any() and not dX[4].any()                   # rows without an adapter


P = 0x10000                                                      # an address that is never looked at: every call below is refused


def test_group_norm_refusals(xb):
    lib = xb.lib()
    big = 1 << 40
    ok = dict(x=P, gamma=P, beta=P, skip=None, y=2 * big, mean=P, invstd=P, batch=2, positions=9, channels=12, groups=3, eps=1e-5, act=0, ws=P, n=big)

    def fwd(**kw):
        a = dict(ok, **kw)
        return lib.xbar_gn_fwd(a["x"], a["gamma"], a["beta"], a["skip"], a["y"], a["mean"], a["invstd"], a["batch"], a["positions"], a["channels"],
                               a["groups"], a["eps"], a["act"], a["ws"], a["n"], None)
    assert fwd(batch=0) == fwd(positions=0) == fwd(channels=0) == fwd(groups=0) == fwd(groups=5) == fwd(groups=24) == -2
    assert fwd(batch=1 << 24, groups=1) == fwd(batch=1 << 20, positions=1 << 18) == fwd(batch=1 << 22, positions=2048) == fwd(channels=(1 << 20) + 3) == -2
    assert fwd(x=None) == fwd(gamma=P + 4) == fwd(skip=P + 8) == fwd(y=None) == fwd(mean=None) == fwd(ws=P + 1) == -3
    assert fwd(eps=-1.0) == fwd(eps=float("nan")) == fwd(act=3) == fwd(act=-1) == -1
    assert fwd(y=P) == fwd(y=P + 16) == fwd(skip=2 * big + 16) == -1
    assert fwd(n=lib.xbar_gn_workspace_bytes(2, 9, 12, 3) - 1) == -4
    assert lib.xbar_gn_workspace_bytes(2, 9, 12, 5) == 0 and lib.xbar_gn_workspace_bytes(2, 9, 12, 3) > 0

    bok = dict(x=P, dy=P, gamma=P, beta=P, skip=None, mean=P, invstd=P, dx=2 * big, dgamma=P, dbeta=P, dskip=None, groups=3, act=0, ws=P, n=big)

    def bwd(**kw):
        a = dict(bok, **kw)
        return lib.xbar_gn_bwd(a["x"], a["dy"], a["gamma"], a["beta"], a["skip"], a["mean"], a["invstd"], a["dx"], a["dgamma"], a["dbeta"], a["dskip"],
                               2, 9, 12, a["groups"], a["act"], a["ws"], a["n"], None)
    assert bwd(groups=7) == -2
    assert bwd(dy=None) == bwd(dx=P + 4) == bwd(dgamma=None) == bwd(dbeta=P + 8) == bwd(dskip=P + 4, skip=P) == bwd(invstd=None) == -3
    assert bwd(dskip=P) == bwd(act=7) == bwd(dx=P) == bwd(skip=P, dskip=P) == bwd(skip=P, dskip=2 * big) == -1
    assert bwd(n=0) == -4


def test_adapter_refusals(xb):
    lib = xb.lib()
    size = lambda M=8, K=16, N=24, rank=4, n=3, op=xb.OP_FWD: lib.xbar_adapter_workspace_bytes(op, M, K, N, rank, n)
    assert size(M=0) == size(K=0) == size(N=0) == size(rank=0) == size(rank=129) == size(n=0) == size(n=65537) == size(K=1 << 24) == 0
    assert size(op=xb.OP_UPDATE) == 0 and size() > 0 and size(op=xb.OP_BWD) > size()
    assert lib.xbar_adapter_plan_bytes(0, 1) == lib.xbar_adapter_plan_bytes((1 << 24) + 1, 1) == lib.xbar_adapter_plan_bytes(1, 0) == 0
    plan = lib.xbar_adapter_plan_bytes(8, 3)
    assert lib.xbar_adapter_plan(P, 0, 3, P, plan, None) == -2
    assert lib.xbar_adapter_plan(None, 8, 3, P, plan, None) == lib.xbar_adapter_plan(P, 8, 3, P + 4, plan, None) == -3
    assert lib.xbar_adapter_plan(P, 8, 3, P, plan - 1, None) == -4
    far = [(i + 1) << 32 for i in range(12)]
    ok = dict(plan=far[0], plan_bytes=plan, base=far[1], X=far[2], A=far[3], B=far[4], type=0, scale=far[5], Y=far[6], T=far[7], M=8, K=16, N=24, rank=4,
              n=3, ws=far[8], ws_bytes=size())

    def fwd(**kw):
        a = dict(ok, **kw)
        return lib.xbar_adapter_fwd(a["plan"], a["plan_bytes"], a["base"], a["X"], a["A"], a["B"], a["type"], a["scale"], a["Y"], a["T"], a["M"], a["K"],
                                    a["N"], a["rank"], a["n"], a["ws"], a["ws_bytes"], None)
    assert fwd(M=0) == fwd(rank=129) == fwd(n=0) == -2
    assert fwd(type=2) == fwd(Y=far[2]) == fwd(Y=far[1] + 16) == fwd(T=far[6]) == fwd(T=far[2]) == fwd(Y=far[3]) == -1
    assert fwd(plan=None) == fwd(base=None) == fwd(X=far[2] + 4) == fwd(A=None) == fwd(scale=None) == fwd(Y=None) == fwd(T=far[7] + 4) == fwd(ws=None) == -3
    assert fwd(plan_bytes=plan - 1) == fwd(ws_bytes=size() - 1) == -4
    bok = dict(ok, dY=far[6], T=far[7], dX=far[9], dA=far[10], dB=far[11], base=far[1], ws_bytes=size(op=xb.OP_BWD))

    def bwd(**kw):
        a = dict(bok, **kw)
        return lib.xbar_adapter_bwd(a["plan"], a["plan_bytes"], a["base"], a["dY"], a["X"], a["T"], a["A"], a["B"], a["type"], a["scale"], a["dX"], a["dA"],
                                    a["dB"], a["M"], a["K"], a["N"], a["rank"], a["n"], a["ws"], a["ws_bytes"], None)
    assert bwd(K=0) == -2
    assert bwd(type=-1) == bwd(dX=far[2]) == bwd(dA=far[3]) == bwd(dB=far[10]) == bwd(dX=far[1] + 64) == -1
    assert bwd(base=None) == bwd(T=None) == bwd(dA=None) == bwd(dB=None) == bwd(dX=far[9] + 4) == -3
    assert bwd(ws_bytes=size(op=xb.OP_BWD) - 1) == -4


def test_gradient_list_refusals(xb):
    lib = xb.lib()

    def lists(*tensors):
        return (C.c_void_p * len(tensors))(*[t[0] for t in tensors]), (C.c_size_t * len(tensors))(*[t[1] for t in tensors])
    far, n = 1 << 40, lib.xbar_grads_workspace_bytes(2)
    g, sizes = lists((P, 4), (2 * P, 5))
    p, _ = lists((3 * P, 4), (4 * P, 5))
    norm = lambda g=g, sizes=sizes, k=2, out=far, ws=2 * far, n=n: lib.xbar_grad_norm(g, sizes, k, out, ws, n, None)
    clip = lambda g=g, sizes=sizes, k=2, most=1.0, out=far, ws=2 * far, n=n: lib.xbar_grad_clip(g, sizes, k, most, out, ws, n, None)
    step = lambda p=p, g=g, sizes=sizes, k=2, lr=0.1, most=1.0, out=far, ws=2 * far, n=n: lib.xbar_clip_sgd(p, g, sizes, k, lr, most, out, ws, n, None)
    assert norm(k=0) == norm(k=2049) == lib.xbar_grads_workspace_bytes(0) - 2 == lib.xbar_grads_workspace_bytes(2049) - 2 == -2
    assert norm(sizes=lists((0, 4), (0, 1 << 38))[1]) == -2
    assert norm(g=None) == norm(sizes=None) == step(p=None) == -1
    assert norm(out=None) == norm(ws=None) == norm(ws=2 * far + 4) == norm(g=lists((P, 0), (None, 0))[0]) == norm(g=lists((P + 4, 0), (P, 0))[0]) == -3
    assert step(p=lists((3 * P, 0), (4 * P + 8, 0))[0]) == -3
    assert norm(n=n - 1) == clip(n=0) == step(n=n - 1) == -4
    assert clip(most=0.0) == clip(most=float("nan")) == clip(most=-1.0) == step(most=0.0) == step(lr=float("inf")) == step(lr=float("nan")) == -1
    assert norm(out=P) == norm(ws=2 * P - 16) == norm(out=2 * far) == -1
    # the same memory twice: among the gradients that are scaled, the parameters, parameters and gradients, results and workspace
    assert clip(g=lists((P, 0), (P, 0))[0]) == clip(g=lists((P, 0), (P - 16, 0))[0]) == clip(out=P) == clip(ws=P) == -1
    assert step(p=lists((3 * P, 0), (3 * P, 0))[0]) == step(p=lists((3 * P, 0), (2 * P + 16, 0))[0]) == step(out=3 * P) == step(ws=P) == -1


def test_binding_checks_lists_and_devices(xb):
    torch = pytest.importorskip("torch")
    with pytest.raises((AssertionError, RuntimeError)):
        xb.TensorList([])
    with pytest.raises((AssertionError, RuntimeError)):          # host tensors
        xb.grad_norm([torch.zeros(4)])
    with pytest.raises((AssertionError, RuntimeError)):
        xb.gn_fwd(torch.zeros(2, 4), torch.ones(4), torch.zeros(4), 2)
    with pytest.raises((AssertionError, RuntimeError)):
        xb.adapter_plan(torch.zeros(4, dtype=torch.int32), 2)


# ---- networks --------------------------------------------------------------------------------------
def _stand_in(xb):
    torch = pytest.importorskip("torch")
    from test_network_host import StandIn

    class Ops(StandIn):
        """With the digital operators, from their definitions."""

        def tile(self, cfg, W, w_max, step=0, profile=None, planes=None):
            self.programmed = getattr(self, "programmed", {})
            self.programmed[planes.data_ptr()] = W.clone()
            return super().tile(cfg, W, w_max, step, profile, planes)

        def fwd(self, cfg, planes, x, N, w_max, x_scale, ws=None):
            self.W = self.programmed[planes.data_ptr()]
            return super().fwd(cfg, planes, x, N, w_max, x_scale, ws)

        def bwd(self, cfg, planes, dy, K, w_max, g_scale, ws=None):
            self.W = self.programmed[planes.data_ptr()]
            return super().bwd(cfg, planes, dy, K, w_max, g_scale, ws)

        def adapter_plan(self, rows, n):
            self._log("adapter_plan", n=n)
            return rows

        def adapter_fwd(self, plan, base, X, A, B, scale, out=None, ws=None):
            self._log("adapter_fwd", in_place=out is base)
            Y, T = digital.adapter_fwd(plan.numpy(), base.numpy(), X.numpy(), A.numpy(), B.numpy(), scale.numpy())
            out.copy_(torch.from_numpy(Y))
            return out, torch.from_numpy(T).float()

        def adapter_bwd(self, plan, base, dY, X, T, A, B, scale, out=None, ws=None):
            self._log("adapter_bwd", wants_dx=base is not None)
            f = lambda t: t.numpy()
            dX, dA, dB, _ = digital.adapter_bwd(f(plan), np.zeros(X.shape) if base is None else f(base), f(dY), f(X), f(T), f(A), f(B), f(scale))
            if out is not None:
                out.copy_(torch.from_numpy(dX))
            return out, torch.from_numpy(dA).float(), torch.from_numpy(dB).float()

        def gn_fwd(self, x, gamma, beta, groups, eps, act, skip=None, ws=None):
            self._log("gn_fwd", groups=groups, act=act)
            mean, invstd = digital.gn_stats(x.numpy(), groups, eps)
            z = digital.gn_z(x.numpy(), gamma.numpy(), beta.numpy(), mean, invstd)[1]
            return (torch.from_numpy(digital.act(z, ("none", "relu", "silu")[act])).float(), torch.from_numpy(mean).float(),
                    torch.from_numpy(invstd).float())

        def gn_bwd(self, x, dy, gamma, beta, mean, invstd, act, skip=None, ws=None):
            self._log("gn_bwd", act=act)
            got = digital.gn_bwd(*(t.numpy() for t in (x, dy, gamma, beta, mean, invstd)), ("none", "relu", "silu")[act])
            return tuple(torch.from_numpy(t).float() for t in got[:3])

        def sgd(self, p, g, lr):
            self._log("sgd", size=p.numel())
            p.sub_(lr * g)

        def clip_sgd(self, params, grads, lr, max_norm):
            norm = digital.grad_norm([g.numpy() for g in grads])
            self._log("clip_sgd", tensors=len(params), max_norm=max_norm)
            c = digital.clip_factor(norm, max_norm)
            for p, g in zip(params, grads):
                p.sub_(lr * c * g)
            return torch.tensor([norm])
    return Ops(xb)


def _network(xb, spec, flags=0):
    import workloads
    from paper_2002_11151_amd import resnet_cifar, sequential
    ops = _stand_in(xb)
    resnet_cifar.Network.ops = ops
    try:
        net = sequential.Sequential(workloads.config_kwargs("mlp"), spec, batch=6, in_shape=(12,), signed_input=False, seed=1, device="cpu")
    finally:
        resnet_cifar.Network.ops = xb
    net.ops = ops
    return net, ops


def _batch():
    torch = pytest.importorskip("torch")
    g = torch.Generator().manual_seed(0)
    return torch.rand((6, 12), generator=g), (torch.arange(6) % 5).to(torch.int32)


SPEC = [("flatten",), ("fc", 20), ("groupnorm", 4, "silu"), ("fc", 5)]


def test_frozen_network_trains_its_digital_parameters(xb):
    """The crossbars are programmed once and not written; adapters and normalisation step together, clipped."""
    import torch
    net, ops = _network(xb, SPEC)
    x, labels = _batch()
    net.calibrate(x, labels)
    net.frozen, net.max_grad_norm = True, 0.25
    net.add_adapters(2, 3, scale=2.0)
    net.set_requests(torch.tensor([0, 1, -1, 1, 0, 0], dtype=torch.int32))
    weights = [L.W.clone() for L in net.layers]
    gamma = net.stack[2][1][0].gamma.clone()
    ops.calls.clear()
    for _ in range(2):
        net.train_step(x, labels, 0.1)
    names = [c[0] for c in ops.calls]
    once = ["fwd", "adapter_fwd", "gn_fwd", "fwd", "adapter_fwd", "bwd", "adapter_bwd", "gn_bwd", "adapter_bwd", "clip_sgd"]
    assert names == ["tile"] + once[:3] + ["tile"] + once[3:] + once
    assert [c[1]["tensors"] for c in ops.calls if c[0] == "clip_sgd"] == [6, 6]
    assert [c[1]["wants_dx"] for c in ops.calls if c[0] == "adapter_bwd"][:2] == [True, False]
    assert all(torch.equal(L.W, w) for L, w in zip(net.layers, weights))
    assert not torch.equal(net.stack[2][1][0].gamma, gamma) and all(L.adapters.B.any() for L in net.layers) and float(net.grad_norm) > 0
    # unfrozen again, the devices are written and programmed anew
    net.frozen = False
    ops.calls.clear()
    net.train_step(x, labels, 0.1)
    assert [c[0] for c in ops.calls].count("tile") == 2 and [c[0] for c in ops.calls].count("update") == 2


def test_digital_parameters_step_one_by_one_without_a_limit(xb):
    import torch
    net, ops = _network(xb, SPEC)
    x, labels = _batch()
    net.calibrate(x, labels)
    assert not [c for c in ops.calls if c[0] in ("sgd", "clip_sgd", "update")]
    net.add_adapters(2, 3)
    net.set_requests(torch.zeros(6, dtype=torch.int32))
    ops.calls.clear()
    net.train_step(x, labels, 0.1)
    assert [c[1]["size"] for c in ops.calls if c[0] == "sgd"] == [2 * 3 * 20, 2 * 3 * 5, 20, 20, 2 * 3 * 12, 2 * 3 * 20]
    net.set_requests(None)
    ops.calls.clear()
    net.train_step(x, labels, 0.1)
    assert not [c for c in ops.calls if c[0].startswith("adapter")]
    # a step that an error cut short leaves nothing behind
    net.max_grad_norm = 1.0
    net._pending = ((x, x),)
    ops.calls.clear()
    net.train_step(x, labels, 0.1)
    assert [c[1]["tensors"] for c in ops.calls if c[0] == "clip_sgd"] == [2]


def test_normalisations_of_the_residual_networks(xb):
    import workloads
    from paper_2002_11151_amd import resnet_cifar, resnet_imagenet
    ops = _stand_in(xb)
    resnet_cifar.Network.ops = ops
    try:
        kw = workloads.config_kwargs("resnet20")
        net = resnet_cifar.ResNetCifar(kw, batch=1, n_blocks=1, image=8, widths=(12, 16, 32), device="cpu", norm="group", groups=8)
        assert [net.stem_bn.groups] + [b["bn_b"].groups for b in net.blocks] == [4, 4, 8, 8] and net.norm_bytes > 0
        deep = resnet_imagenet.ResNetBottleneck(kw, batch=1, image=32, classes=10, blocks=(1, 1), widths=(16, 32), stem=16, device="cpu", norm="group")
        assert deep.blocks[0]["bn_c"].groups == 32 and deep.blocks[1]["bn_down"].groups == 32
        with pytest.raises(ValueError):
            resnet_cifar.ResNetCifar(kw, batch=1, n_blocks=1, image=8, device="cpu", norm="layer")
        with pytest.raises(ValueError):
            _network(xb, [("flatten",), ("fc", 20), ("groupnorm", 3, "relu"), ("fc", 5)])
    finally:
        resnet_cifar.Network.ops = xb


# ---- captured steps --------------------------------------------------------------------------------
@pytest.fixture()
def no_graphs(monkeypatch):
    """capture() and replay() without a GPU: the two passes of a capture run one after another, a replay launches nothing."""
    import contextlib
    import torch

    class Nothing:
        def __init__(self, *a, **k):
            pass

        def wait_stream(self, other):
            pass

        def replay(self):
            pass
    from paper_2002_11151_amd import xbar
    for name in ("Stream", "CUDAGraph"):
        monkeypatch.setattr(torch.cuda, name, Nothing)
    for name in ("stream", "graph"):
        monkeypatch.setattr(torch.cuda, name, lambda *a, **k: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Nothing())
    monkeypatch.setattr(xbar, "set_step_source", lambda counter: None)


def _adapted(xb, spec=None, requests=(0, 1, -1, 1, 0, 0)):
    """A frozen network with adapters whose plans lie in buffers, as the binding's."""
    import torch
    net, ops = _network(xb, SPEC if spec is None else spec)

    class Planned(type(ops)):
        def adapter_plan(self, rows, n, buffer=None):
            self._log("adapter_plan", n=n)
            buffer = rows.clone() if buffer is None else buffer.copy_(rows)
            return xb.AdapterPlan(buffer, rows.shape[0], n)

        def adapter_fwd(self, plan, *args, **kw):
            self.planned = plan.buffer.data_ptr()
            return super().adapter_fwd(plan.buffer, *args, **kw)

        def adapter_bwd(self, plan, *args, **kw):
            return super().adapter_bwd(plan.buffer, *args, **kw)

        def step_advance(self, counter):
            counter += 1
    ops.__class__ = Planned
    x, labels = _batch()
    net.calibrate(x, labels)
    net.frozen, net.max_grad_norm = True, 0.25
    net.add_adapters(2, 3)
    if requests is not None:
        net.set_requests(torch.tensor(requests, dtype=torch.int32))
    ops.calls.clear()
    return net, ops, x, labels


def test_requests_of_a_captured_step_are_planned_where_it_reads_them(xb, no_graphs):
    import torch
    net, ops, x, labels = _adapted(xb)
    net.capture(x, labels, 0.1)
    read = ops.planned
    for rows in ([1] * 6, [-1, 0, 1, 0, 1, -1]):
        net.set_requests(torch.tensor(rows, dtype=torch.int32))
        assert net.requests.buffer.data_ptr() == read and net.requests.buffer.tolist() == rows
        net.replay(x, labels)
    # what a captured step cannot follow is refused, and its plan and adapters stay in memory
    net.set_requests(None)
    with pytest.raises(ValueError):
        net.replay(x, labels)
    net.set_requests(torch.tensor([0, 1], dtype=torch.int32))
    assert net.requests.buffer.data_ptr() != read
    with pytest.raises(ValueError):
        net.replay(x, labels)
    net.set_requests(torch.tensor([0, 0, 0, 0, 1, 1], dtype=torch.int32))       # the captured number again: back in its buffer
    assert net.requests.buffer.data_ptr() == read
    net.replay(x, labels)
    net.add_adapters(2, 3)
    with pytest.raises(ValueError):
        net.replay(x, labels)
    net.capture(x, labels, 0.1)
    net.replay(x, labels)
    for L in net.layers:
        L.adapters.compact()
    with pytest.raises(ValueError):
        net.replay(x, labels)


def test_requests_after_a_capture_without_them_are_refused(xb, no_graphs):
    import torch
    net, ops, x, labels = _adapted(xb, requests=None)
    net.capture(x, labels, 0.1)
    net.replay(x, labels)
    net.set_requests(torch.tensor([0, 1, -1, 1, 0, 0], dtype=torch.int32))
    with pytest.raises(ValueError):
        net.replay(x, labels)
    net.set_requests(None)
    net.replay(x, labels)


def test_norm_of_a_captured_step_is_that_of_the_last_step(xb, no_graphs):
    """capture() leaves the norm of the step that it ran, a replay the captured step's own, whatever eager steps came between."""
    net, ops, x, labels = _adapted(xb)
    norms, clip = [], ops.clip_sgd
    ops.clip_sgd = lambda *a: norms.append(clip(*a)) or norms[-1]
    net.capture(x, labels, 0.1)
    assert len(norms) == 2 and net.grad_norm is norms[0]        # of the real step; the other one is the graph's, not yet computed
    net.replay(x, labels)
    assert net.grad_norm is norms[1]
    net.train_step(x, labels, 0.1)
    assert net.grad_norm is norms[2]
    net.replay(x, labels)
    assert net.grad_norm is norms[1]


def test_capture_leaves_out_what_a_broken_step_left(xb, no_graphs):
    net, ops, x, labels = _adapted(xb)
    net._pending = ((x, x),)
    net.capture(x, labels, 0.1)
    assert [c[1]["tensors"] for c in ops.calls if c[0] == "clip_sgd"] == [6, 6]


# ---- frozen networks -------------------------------------------------------------------------------
def test_weights_written_while_frozen_are_programmed(xb):
    import torch
    net, ops, x, labels = _adapted(xb)
    first, second = net.layers

    def tiles():
        ops.calls.clear()
        got = net.forward(x, 7)
        return [c[1]["step"] for c in ops.calls if c[0] == "tile"], got
    assert tiles()[0] == [7, 7] and tiles()[0] == []
    before = tiles()[1]
    first.W.mul_(0.5)                                             # in place
    steps, after = tiles()
    assert steps == [7] and not torch.equal(before, after) and tiles()[0] == []
    second.W = second.W * 2                                       # another tensor
    assert tiles()[0] == [7] and tiles()[0] == []
    first.W.data.mul_(0.5)                                        # a write that torch does not count
    net.reprogram()
    assert tiles()[0] == [7, 7] and tiles()[0] == []
    assert torch.equal(ops.programmed[first.planes.data_ptr()], first.W)
    net.frozen = False
    net.train_step(x, labels, 0.1)                                # the library writes W, which torch does not count either
    net.frozen = True
    assert tiles()[0] == [7, 7] and tiles()[0] == []


def test_weights_without_a_count_of_writes(xb):
    """A network made in inference mode: its tensors have no such count; programmed once, anew on demand."""
    import torch
    with torch.inference_mode():
        net, ops, x, labels = _adapted(xb)
        for _ in range(2):
            net.forward(x, 0)
        assert [c[0] for c in ops.calls].count("tile") == 2
        net.reprogram()
        net.forward(x, 0)
        assert [c[0] for c in ops.calls].count("tile") == 4


def test_replays_program_weights_written_while_frozen(xb, no_graphs):
    net, ops, x, labels = _adapted(xb)
    net.capture(x, labels, 0.1)
    ops.calls.clear()
    net.replay(x, labels)
    assert not ops.calls
    net.layers[1].W.mul_(0.5)
    net.replay(x, labels)
    assert [(c[0], c[1]["step"]) for c in ops.calls] == [("tile", 2)]
    net.replay(x, labels)
    assert len(ops.calls) == 1


def test_replays_that_write_the_devices_leave_no_plane_valid(xb, no_graphs):
    net, ops, x, labels = _adapted(xb)
    net.frozen = False
    net.capture(x, labels, 0.1)
    net.frozen = True
    net.forward(x, 0)
    net.frozen = False
    net.replay(x, labels)
    net.frozen = True
    ops.calls.clear()
    net.forward(x, 0)
    assert [c[0] for c in ops.calls].count("tile") == 2


def test_replays_with_other_settings_are_refused(xb, no_graphs):
    net, ops, x, labels = _adapted(xb)
    net.capture(x, labels, 0.1)
    for name, value in (("frozen", False), ("max_grad_norm", None), ("max_grad_norm", 1.0)):
        kept = getattr(net, name)
        setattr(net, name, value)
        with pytest.raises(ValueError):
            net.replay(x, labels)
        setattr(net, name, kept)
        net.replay(x, labels)


def test_frozen_network_with_a_stored_profile_is_captured(xb, no_graphs):
    """It refreshes the profile only when it programs, which a captured step does not; the schedule is that of eager steps."""
    import workloads
    kw = workloads.config_kwargs("mlp")
    flags = (kw["flags"] & ~workloads.NI_WIRE_AAM) | workloads.NI_WIRE_PROFILE

    def steps(captured):
        net, ops, x, labels = _adapted(xb)
        for L in net.layers:
            L.cfg.flags |= flags & workloads.NI_WIRE_PROFILE
            L.cfg.flags &= ~workloads.NI_WIRE_AAM
        net.ws = net.ws.new_empty(max(L.workspace_bytes(6) for L in net.layers))
        net.fcm_every, net.step_no = 3, 3
        net.frozen = False
        net.train_step(x, labels, 0.1)
        net.frozen = True
        ops.calls.clear()
        net.capture(x, labels, 0.1) if captured else net.train_step(x, labels, 0.1)          # step 4: no refresh
        net.layers[0].W.mul_(0.5)
        net.replay(x, labels) if captured else net.train_step(x, labels, 0.1)                # step 5: programmed again, no refresh
        net.layers[0].W.mul_(0.5)
        net.replay(x, labels) if captured else net.train_step(x, labels, 0.1)                # step 6: programmed again and refreshed
        return [c[0] + str(c[1]["step"]) for c in ops.calls if c[0] in ("tile", "fcm_profile")], net, x, labels
    assert steps(False)[0] == ["tile4", "tile4", "tile5", "fcm_profile6", "tile6"]
    got, net, x, labels = steps(True)
    assert got == ["tile4", "tile4", "tile5", "fcm_profile6", "tile6"]
    net.frozen = False
    with pytest.raises(ValueError):                               # steps that write the devices refresh on some of them only, as before
        net.capture(x, labels, 0.1)


@pytest.mark.parametrize("clipped", [False, True])
def test_a_normalisation_before_the_first_weight_layer_learns(xb, clipped):
    """Errors go back as far as something learns, no further."""
    import torch
    net, ops = _network(xb, [("flatten",), ("groupnorm", 3, "none"), ("flatten",), ("fc", 20), ("relu",), ("fc", 5)])
    x, labels = _batch()
    net.calibrate(x, labels)
    net.max_grad_norm = 0.5 if clipped else None
    norm = net.stack[1][1][0]
    norm.gamma.copy_(torch.linspace(0.5, 1.5, 12))
    before = norm.gamma.clone(), norm.beta.clone()
    ops.calls.clear()
    net.train_step(x, labels, 0.1)
    names = [c[0] for c in ops.calls]
    assert names == ["gn_fwd", "tile", "fwd", "tile", "fwd", "bwd", "update", "bwd", "update", "gn_bwd"] + (["clip_sgd"] if clipped else ["sgd"] * 2)
    assert not torch.equal(norm.gamma, before[0]) and not torch.equal(norm.beta, before[1])


# ---- limits ----------------------------------------------------------------------------------------
def test_group_norm_limits(xb):
    """Both sides of every limit: 0 bytes and XBAR_ESHAPE beyond, a size and a refusal for the size alone (-4) inside."""
    lib = xb.lib()
    far = 1 << 45

    def sizes(*shape):
        nbytes = lib.xbar_gn_workspace_bytes(*shape)
        assert nbytes < 1 << 44
        codes = [lib.xbar_gn_fwd(P, P, P, None, far, P, P, *shape, 1e-5, 0, P, max(nbytes, 1) - 1, None),
                 lib.xbar_gn_bwd(P, P, P, P, None, P, P, far, P, P, None, *shape, 0, P, max(nbytes, 1) - 1, None)]
        assert codes == ([-4, -4] if nbytes else [-2, -2]), (shape, nbytes, codes)
        return nbytes > 0
    most = 2 ** 31 - 512
    assert sizes(1, most, 1, 1) and not sizes(1, most + 1, 1, 1) and not sizes(1, 2 ** 31 - 1, 1, 1) and not sizes(1, 2 ** 31 - 1, 127, 1)
    assert sizes(1, most, 127, 127) and not sizes(1, most, 129, 129)                           # 2^38 elements
    assert sizes(4, most, 8, 1) and not sizes(5, most, 8, 1)                                   # batch ceil(positions / 512) below 2^24
    assert sizes((1 << 23) - 8, 513, 8, 1) and not sizes((1 << 23) - 8, 1025, 8, 1)
    assert sizes(1, 1, 1 << 20, 1) and not sizes(1, 1, (1 << 20) + 1, 1)
    for values in (1, 64, 255, 256):                                                           # batch groups below 2^25 for short groups,
        assert sizes((1 << 22) - 1, 1, 8 * values, 8) and not sizes(1 << 22, 1, 8 * values, 8)
    for values in (257, 1024, 4096, 4100, 16384):                                              # up to 2^23 - 8 for all
        assert sizes((1 << 20) - 1, 1, 8 * values, 8)
    assert not sizes(1 << 20, 1, 8 * 16384, 8)


def test_adapter_outputs_over_plans_scales_and_workspaces_are_refused(xb):
    """An output over an input, the plan, another output or the workspace, or a workspace or plan over an input, by its first or last bytes."""
    lib = xb.lib()
    M, K, N, rank, n = 8, 16, 24, 4, 3
    plan, fwd_ws, bwd_ws = lib.xbar_adapter_plan_bytes(M, n), *(lib.xbar_adapter_workspace_bytes(op, M, K, N, rank, n) for op in (xb.OP_FWD, xb.OP_BWD))
    at = {name: (i + 1) << 32 for i, name in enumerate("plan base X A B scale Y T ws dY dX dA dB".split())}
    fwd = lambda **kw: (lambda a: lib.xbar_adapter_fwd(a["plan"], plan, a["base"], a["X"], a["A"], a["B"], 0, a["scale"], a["Y"], a["T"], M, K, N, rank, n,
                                                       a["ws"], fwd_ws, None))(dict(at, **kw))
    bwd = lambda **kw: (lambda a: lib.xbar_adapter_bwd(a["plan"], plan, a["base"], a["dY"], a["X"], a["T"], a["A"], a["B"], 0, a["scale"], a["dX"], a["dA"],
                                                       a["dB"], M, K, N, rank, n, a["ws"], bwd_ws, None))(dict(at, **kw))
    bytes_of = dict(plan=plan, base=4 * M * N, X=4 * M * K, A=4 * n * rank * K, B=4 * n * rank * N, scale=4 * n, Y=4 * M * N, T=4 * M * rank, dY=4 * M * N,
                    dX=4 * M * K, dA=4 * n * rank * K, dB=4 * n * rank * N)
    last = lambda name: at[name] + (bytes_of[name] - 1) // 16 * 16
    for out, others in (("Y", "X A B scale plan T"), ("T", "X A B scale plan base Y")):
        for other in others.split():
            assert fwd(**{out: at[other]}) == fwd(**{out: last(other)}) == -1, (out, other)
        assert fwd(**{out: at["ws"]}) == fwd(**{out: at["ws"] + fwd_ws - 16}) == -1
    for out in ("dX", "dA", "dB"):
        for other in "dY X T A B scale plan dX dA dB".split():
            if other != out:
                assert bwd(**{out: at[other]}) == bwd(**{out: last(other)}) == -1, (out, other)
        assert bwd(**{out: at["ws"]}) == bwd(**{out: at["ws"] + bwd_ws - 16}) == -1
    for call, size, others in ((fwd, fwd_ws, "base X A B scale plan"), (bwd, bwd_ws, "base dY X T A B scale plan")):
        bytes_of["base"] = 4 * M * (N if call is fwd else K)
        for other in others.split():
            assert call(ws=last(other)) == call(ws=at[other] - (size - 1) // 16 * 16) == -1, other
    assert fwd(ws=at["base"], Y=at["base"]) == bwd(ws=at["base"], dX=at["base"]) == -1
    assert lib.xbar_adapter_plan(at["X"], M, n, at["X"] + 16, plan, None) == lib.xbar_adapter_plan(at["X"], M, n, at["X"] - plan + 16, plan, None) == -1


def test_group_norm_outputs_over_parameters_statistics_and_workspaces_are_refused(xb):
    lib = xb.lib()
    at = {name: (i + 1) << 32 for i, name in enumerate("x dy gamma beta skip mean invstd y dgamma dbeta dskip dx ws".split())}
    bytes_of = dict(gamma=48, beta=48, mean=24, invstd=24, dgamma=48, dbeta=48)
    last = lambda name: at[name] + (bytes_of[name] - 1) // 16 * 16
    ws = lib.xbar_gn_workspace_bytes(2, 9, 12, 3)
    gn_fwd = lambda **kw: (lambda a: lib.xbar_gn_fwd(a["x"], a["gamma"], a["beta"], a["skip"], a["y"], a["mean"], a["invstd"], 2, 9, 12, 3, 1e-5, 0, a["ws"], ws,
                                                     None))(dict(at, **kw))
    gn_bwd = lambda **kw: (lambda a: lib.xbar_gn_bwd(a["x"], a["dy"], a["gamma"], a["beta"], a["skip"], a["mean"], a["invstd"], a["dx"], a["dgamma"], a["dbeta"],
                                                     a["dskip"], 2, 9, 12, 3, 0, a["ws"], ws, None))(dict(at, **kw))
    for other in "gamma beta mean invstd".split():
        assert gn_fwd(y=at[other]) == gn_fwd(y=last(other)) == -1, other
    assert gn_fwd(y=at["ws"]) == gn_fwd(y=at["ws"] + ws - 16) == -1
    for out in ("dx", "dskip"):
        for other in "gamma beta mean invstd dgamma dbeta".split():
            assert gn_bwd(**{out: at[other]}) == gn_bwd(**{out: last(other)}) == -1, (out, other)
        assert gn_bwd(**{out: at["ws"]}) == gn_bwd(**{out: at["ws"] + ws - 16}) == -1


def test_adapter_limits(xb):
    """Shapes just inside the stated limits have a workspace, those beyond the exact ones do not."""
    size = lambda M=8, K=16, N=24, rank=4, n=3: xb.lib().xbar_adapter_workspace_bytes(xb.OP_FWD, M, K, N, rank, n) > 0
    top = (1 << 24) - 1
    assert size(M=1 << 24, K=1, N=1, n=65536) and not size(M=(1 << 24) + 1, K=1, N=1)
    assert size(K=top, rank=1) and not size(K=1 << 24, rank=1) and size(N=top, rank=1) and not size(N=1 << 24, rank=1)
    assert size(K=top, rank=64, n=1) and not size(K=top, rank=65, n=1)                         # rank max(K, N) below 2^30
    assert size(M=1, K=(1 << 17) - 1, N=1, rank=32, n=65536) and not size(M=1, K=1 << 17, N=1, rank=32, n=65536)    # adapters rank max(K, N) below 2^38
    cost = lambda M, K, N, n: (M / 32 + n + 8) * (K + N + 126) / 64
    for M, K, N, n in ((1 << 18, 8000, 2000, 65536), (1 << 24, 1000, 690, 65536), (28, 13_000_000, 13_000_000, 28), (65537, 7850, 7850, 65536),
                       (1, 29, 1, 1), (300, 5000, 11000, 60000), (16, 16_000_000, 16_000_000, 16)):
        assert cost(M, K, N, n) < 1 << 24 and size(M, K, N, 1, n), (M, K, N, n)
    assert not size(M=65536, K=10000, N=10000, rank=1, n=65536) and not size(M=40, K=top, N=top, rank=1, n=40)


def test_replays_count_the_eager_steps_between_them(xb, no_graphs):
    net, ops, x, labels = _adapted(xb)
    net.capture(x, labels, 0.1)
    net.train_step(x, labels, 0.1)
    net.train_step(x, labels, 0.1)
    net.replay(x, labels)                                         # (it advances nothing here)
    assert int(net._graph_counter) == 3 and net.step_no == 4
