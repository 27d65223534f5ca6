"""Nets with group normalisation: plans, the oracle's gradient against differences, the HIP path against the oracle, and the calls that promise each other's bits."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from paper_1312_6186_amd import binding as B
from paper_1312_6186_amd import workloads as wl

DEV = "cuda:0"
TDT = {B.F32: torch.float32, B.BF16: torch.bfloat16}


def _gn(cout, k, stride, pad, groups, relu=True):
    return [("conv", cout, k, stride, pad), ("groupnorm", groups)] + [("relu",)] * relu


# channels that are padded (12, 20); with and without a ReLU; under a convolution, a pool, a pool of a pool, a fully-connected layer
RAGGED = dict(name="gn ragged", in_shape=(3, 37, 29), classes=10,
              layers=_gn(12, 5, 2, 1, 4) + _gn(20, 3, 2, 1, 5) + _gn(12, 3, 1, 1, 3) + [("maxpool", 3, 2), ("fc", 24), ("relu",), ("dropout", 0.3, 1.5), ("fc", 10), ("softmax_ce",)])
BARE = dict(name="gn bare", in_shape=(3, 19, 17), classes=10,
            layers=_gn(16, 3, 1, 1, 2, relu=False) + _gn(24, 3, 1, 1, 8) + [("maxpool", 2, 2), ("maxpool", 2, 1)] + _gn(8, 3, 1, 0, 1)
            + [("fc", 16), ("relu",), ("fc", 10), ("softmax_ce",)])
# enough parameters for the side stream
FORKED = dict(name="gn forked", in_shape=(3, 24, 24), classes=10,
              layers=_gn(32, 5, 1, 2, 8) + [("maxpool", 3, 2)] + _gn(48, 3, 1, 1, 12) + [("fc", 1024), ("relu",), ("fc", 10), ("softmax_ce",)])
NETS = [(RAGGED, 5), (RAGGED, 1), (BARE, 7), (FORKED, 6), (wl.SMALL_GN, 16)]
IDS = ["ragged5", "ragged1", "bare7", "forked6", "small16"]


def test_layout_shapes_and_refusals():
    layers = RAGGED["layers"]
    net = B.asgd_net_create(layers, 5, RAGGED["in_shape"], B.BF16)
    ref = wl.param_shapes(layers, RAGGED["in_shape"])
    lay = B.asgd_param_layout(net)
    off = 0
    for t, (li, wshape, blen, _) in zip(lay, ref):
        assert t["layer"] == li and t["w_offset"] == off and t["w_shape"][:len(wshape)] == tuple(wshape) and t["b_count"] == blen
        off += t["w_count"] + t["b_count"]
    assert len(lay) == len(ref) and off == B.asgd_param_count(net) == wl.param_count(layers, RAGGED["in_shape"]) == oracle.OracleNet(layers, RAGGED["in_shape"]).param_count
    assert lay[1]["kind"] == B.LAYER_GROUP_NORM and lay[1]["w_shape"] == (12, 1, 1, 1)
    assert B.asgd_layer_shape(net, 1) == B.asgd_layer_shape(net, 2) == B.asgd_layer_shape(net, 0)
    B.asgd_net_destroy(net)
    p = wl.make_params(layers, RAGGED["in_shape"], 1)
    assert (p[lay[1]["w_offset"]:][:12] == 1).all() and (p[lay[1]["b_offset"]:][:12] == 0).all()

    def rc(layers):
        arr, h = B.layer_descs(layers), ctypes.c_void_p(0)
        code = B.lib().asgd_net_create(arr, len(arr), 2, 3, 16, 16, B.F32, ctypes.byref(h))
        if code == 0:
            B.asgd_net_destroy(h)
        return code

    tail = [("maxpool", 2, 2), ("fc", 10), ("softmax_ce",)]
    conv, relu, pool = ("conv", 16, 3, 1, 1), ("relu",), ("maxpool", 2, 2)
    assert rc([conv, ("groupnorm", 4), relu] + tail) == B.OK and rc([conv, ("groupnorm", 4, 1e-3)] + tail) == B.OK
    for bad in ([("groupnorm", 1)], [conv, relu, ("groupnorm", 4)], [conv, pool, ("groupnorm", 4)], [conv, ("groupnorm", 3)], [conv, ("groupnorm", 0)],
                [conv, ("groupnorm", 32)], [conv, ("groupnorm", 4, -1.0)], [conv, ("groupnorm", 4, float("nan"))], [conv, ("groupnorm", 4, float("inf"))],
                [conv, ("groupnorm", 4), ("groupnorm", 4)], [conv, ("groupnorm", 4), relu, ("lrn", 5, 1e-4, 0.75, 2.0)]):
        assert rc(bad + tail) == B.ESHAPE, bad
    assert rc([conv] + tail[:2] + [("groupnorm", 2)] + tail[2:]) == B.ESHAPE       # behind a fully-connected layer


def test_oracle_gradient_by_central_differences():
    cfg = dict(in_shape=(2, 7, 6), classes=3, layers=_gn(6, 3, 1, 1, 2) + _gn(4, 3, 2, 1, 4, relu=False) + [("maxpool", 2, 1), ("fc", 3), ("softmax_ce",)])
    net = oracle.OracleNet(cfg["layers"], cfg["in_shape"])
    rng = np.random.default_rng(3)
    params = wl.make_params(cfg["layers"], cfg["in_shape"], 4).astype(np.float64)
    params += 0.1 * rng.standard_normal(params.size)
    images, labels = wl.make_batch(cfg["in_shape"], 3, 3, 5)
    _, grads, _ = net.fwd_bwd(params, images, labels)
    h, fd = 1e-5, np.empty_like(params)
    for i in range(params.size):
        hi, lo = params.copy(), params.copy()
        hi[i] += h; lo[i] -= h
        fd[i] = (net.fwd_bwd(hi, images, labels, want_grads=False)[0] - net.fwd_bwd(lo, images, labels, want_grads=False)[0]) / (2 * h)
    err = np.abs(fd - grads)   # a ReLU or pooling kink inside [-h, h] would show as an error of order one on that entry
    assert np.median(err) < 1e-9 and (err < 1e-6 * (1 + np.abs(grads))).mean() > 0.99 and np.linalg.norm(fd - grads) / np.linalg.norm(grads) < 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("cfg,batch", NETS, ids=IDS)
def test_minibatch_gradient_matches_oracle(cfg, batch, dtype):
    from gpu_harness import TOL, grad_errors, rel_l2
    from test_gpu_parity import _net_case
    g, onet, (loss, grads), (ref_loss, ref, trace), _ = _net_case(cfg, batch, dtype, seed=3002, step=4, worker=1)
    try:
        tol, layers = TOL[dtype], cfg["layers"]
        assert abs(loss - ref_loss) <= tol * abs(ref_loss)
        errs = dict(grad_errors(onet, grads, ref))
        for li, (_, _, b_off, b_len) in onet.param_slices.items():
            assert errs[" layer%d.dW" % li] < tol, (li, errs)
            if layers[li + 1][0] != "groupnorm":
                assert errs[" layer%d.db" % li] < tol, (li, errs)
                continue
            # A bias under a normalisation: what its channel's gradients do not cancel.  Each of them is stored with a relative error of its own (bf16: half
            # a step of 2^-8, and as much again from the layers above), which add up as their squares do.
            d = np.sqrt((trace["dx"][li + 1] ** 2).sum(axis=(0, 2, 3)))
            off = np.abs(grads[b_off:b_off + b_len] - ref[b_off:b_off + b_len])
            assert (off <= tol * np.abs(ref[b_off:b_off + b_len]).max() + (2.0 ** -6 if dtype == B.BF16 else 2.0 ** -16) * d).all(), li
        for li, l in enumerate(layers[:-1]):
            end = l[0] in ("maxpool", "dropout") or (l[0] == "relu" and layers[li + 1][0] != "dropout") or (l[0] in ("conv", "groupnorm", "fc") and layers[li + 1][0] != "relu")
            if end:
                assert rel_l2(g.debug(B.DEBUG_OUTPUT, li), trace[li]["out"]) < tol, ("output of layer", li)
    finally:
        g.close()


def _state(cfg, batch, dtype, seed=7):
    params = torch.from_numpy(wl.make_params(cfg["layers"], cfg["in_shape"], seed)).to(DEV)
    params += 0.05 * torch.randn(params.numel(), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
    images, labels = wl.make_batch(cfg["in_shape"], batch, cfg["classes"], seed + 1)
    P = params.numel()
    return dict(w=params, v=torch.zeros(P, device=DEV), copy=torch.empty(P, dtype=TDT[dtype], device=DEV), grads=torch.zeros(P, device=DEV), loss=torch.zeros(1, device=DEV),
                images=torch.from_numpy(images).to(DEV).to(TDT[dtype]), labels=torch.from_numpy(labels).to(DEV))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("cfg,batch", NETS, ids=IDS)
def test_steps_serial_and_static_calls_give_the_same_bits(cfg, batch, dtype):
    net = B.asgd_net_create(cfg["layers"], batch, cfg["in_shape"], dtype)
    try:
        got = {}
        for how in ("calls", "serial", "static", "by layer", "fused"):
            s = _state(cfg, batch, dtype)
            B.asgd_net_set_serial(net, how == "serial")
            B.asgd_snapshot(s["w"], s["copy"], dtype)
            for step in range(2):
                if how in ("by layer", "fused"):
                    f = B.asgd_train_step if how == "by layer" else B.asgd_train_step_fused
                    f(net, s["w"], s["v"], s["copy"], s["images"], s["labels"], 3, step, 0, s["loss"], s["grads"], 0.01, 0.9, 5e-4)
                else:
                    f = B.asgd_fwd_bwd_static if how == "static" else B.asgd_fwd_bwd
                    f(net, s["copy"], s["images"], s["labels"], 3, step, 0, s["loss"], s["grads"])
                    B.asgd_apply_update_snapshot(s["w"], s["v"], s["grads"], 0.01, 0.9, 5e-4, s["copy"], dtype)
            torch.cuda.synchronize()
            got[how] = s
        for how, s in got.items():
            for k in ("w", "v", "copy", "loss") + (("grads",) if how != "fused" else ()):
                assert torch.equal(s[k], got["calls"][k]), (how, k)
    finally:
        torch.cuda.synchronize()
        B.asgd_net_destroy(net)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_replay_of_normalised_replicas_equals_calls_in_order(dtype):
    """Three replicas, staleness up to two, against their snapshots, gradients and updates one after the other."""
    cfg, batch, W, T = wl.SMALL_GN, 8, 3, 7
    nets = [B.asgd_net_create(cfg["layers"], batch, cfg["in_shape"], dtype) for _ in range(W)]
    try:
        s = _state(cfg, batch * T, dtype)
        worker, rv = B.asgd_schedule_generate(T, 4005, W, W - 1)
        P = s["w"].numel()
        w, v = s["w"].clone(), s["v"].clone()
        copies, grads = [torch.empty_like(s["copy"]) for _ in range(W)], [torch.empty_like(s["grads"]) for _ in range(W)]
        losses, log = torch.zeros(T, device=DEV), torch.zeros(3 * T, dtype=torch.int32, device=DEV)
        B.asgd_replay_run(nets, w, v, copies, grads, s["images"], s["labels"], worker, rv, 0.01, 0.9, 5e-4, 9, losses, log)
        versions, ref = [s["w"].clone()], torch.zeros(T, device=DEV)
        mom, g = torch.zeros(P, device=DEV), torch.empty(P, device=DEV)
        for a in range(T):
            B.asgd_snapshot(versions[rv[a]], s["copy"], dtype)
            B.asgd_fwd_bwd(nets[0], s["copy"], s["images"][a * batch:], s["labels"][a * batch:], 9, a, int(worker[a]), ref[a:], g)
            nxt = versions[-1].clone()
            B.asgd_apply_update(nxt, mom, g, 0.01, 0.9, 5e-4)
            versions.append(nxt)
        torch.cuda.synchronize()
        assert torch.equal(w, versions[-1]) and torch.equal(v, mom) and torch.equal(losses, ref)
    finally:
        torch.cuda.synchronize()
        for n in nets:
            B.asgd_net_destroy(n)


@pytest.mark.gpu
def test_normalised_nets_train_with_clipped_pushes():
    """The two together, as a replica uses them: steps of a normalised net whose pushes are clipped, against gradient, clipping by tensors and update."""
    cfg, batch, dtype, max_norm = wl.SMALL_GN, 8, B.BF16, 0.25
    net = B.asgd_net_create(cfg["layers"], batch, cfg["in_shape"], dtype)
    try:
        a, b = _state(cfg, batch, dtype), _state(cfg, batch, dtype)
        norm, norm2 = torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
        ws = torch.empty(B.asgd_grad_norm_workspace_bytes(1), dtype=torch.uint8, device=DEV)
        for s in (a, b):
            B.asgd_snapshot(s["w"], s["copy"], dtype)
        for step in range(4):
            B.asgd_train_step_clipped(net, a["w"], a["v"], a["copy"], a["images"], a["labels"], 3, step, 0, a["loss"], a["grads"], 0.05, 0.9, 5e-4, max_norm, norm, ws)
            B.asgd_fwd_bwd(net, b["copy"], b["images"], b["labels"], 3, step, 0, b["loss"], b["grads"])
            assert torch.equal(a["grads"], b["grads"])
            B.asgd_clip_grads([b["grads"]], [b["grads"]], B.F32, max_norm, norm2, ws)
            B.asgd_apply_update_snapshot(b["w"], b["v"], b["grads"], 0.05, 0.9, 5e-4, b["copy"], dtype)
            assert norm.item() == norm2.item() and norm.item() > max_norm
            clipped = b["grads"].double().norm().item()
            assert abs(clipped - max_norm) <= 2.0 ** -23 * max_norm
            for k in ("w", "v", "copy", "loss"):
                assert torch.equal(a[k], b[k]), k
    finally:
        torch.cuda.synchronize()
        B.asgd_net_destroy(net)
