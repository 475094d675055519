"""Training nets whose backward passes run from activations in 8 bits, and the gradient of a net's input: every way that the passes
take, against the plain form in 64 bits on the values that were kept; and a run of nets, norms and checkpoints together."""
import numpy as np
import pytest
import torch

from paper_2104_11805_amd import sdnn, workloads as wl
from tests import blocks, pan_nets
from tests.blocks import close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def host(t):
    return t.cpu().numpy()


def caps(net, activation, cap):
    return [0.0] + [1.0 if activation == "sigmoid" else cap] * net.n_layers


def kept_blocks(net, ckpt, b, activation, cap):
    """The values of X_0 .. X_L that a checkpoint holds, by sdnn_unpack8 of its parts."""
    widths, at, out = [net.shapes[0][1]] + [s[0] for s in net.shapes], 0, []
    for n, c in zip(widths, caps(net, activation, cap)):
        size = sdnn.sdnn_pack8_bytes(n, b)
        out.append(sdnn.sdnn_unpack8(sdnn.Packed8(ckpt[at:at + size], n, b, c)))
        at += size
    assert at == ckpt.numel()
    return out


# widths, entries of the rows, samples, samples that the net is made for, activation, cap, options: the ways through the backward pass
NETS = {
    "one sample": ((300, 200, 250), (7, 40), 1, 1, "relu", 2.0, {}),
    "one sample, sigmoid": ((300, 200, 250), (7, 40), 1, 1, "sigmoid", 1.0, {}),
    "one sample of many": ((300, 200, 250), (7, 40), 1, 50, "relu", 2.0, {}),
    "one sample, long rows": ((400, 400, 300), (200, 150), 1, 1, "relu", 2.0, {}),
    "one sample, wide": ((2500, 2600, 2300), (9, 3), 1, 20, "sigmoid", 1.0, {}),
    "small": ((31, 45, 17), (3, 0, 9), 5, 5, "relu", 1.0, {}),
    "launch per pass": ((300, 260, 310, 64, 290), (16, 5), 24, 40, "relu", 2.0, {}),
    "launch per pass, sigmoid": ((300, 260, 310, 64, 290), (16, 5), 33, 33, "sigmoid", 1.0, {}),
    "launch per pass off": ((300, 260, 310, 64, 290), (16, 5), 24, 40, "relu", 2.0, dict(lds_forward=-1)),
    "fused, few rows": ((500, 700, 600), (20, 33), 64, 64, "relu", 2.0, dict(fuse_gradient=1)),
    "fused, few rows, ragged": ((500, 700, 600), (20, 33), 37, 64, "sigmoid", 1.0, dict(fuse_gradient=1)),
    "fused, several rows": ((6300, 6200, 40), (5, 21), 50, 64, "relu", 2.0, dict(fuse_gradient=1)),
    "fused, 99": ((700, 600, 650), (20, 33), 99, 99, "relu", 2.0, dict(fuse_gradient=1)),
    "fused, two windows": ((700, 600, 650), (20, 33), 128, 128, "relu", 2.0, dict(fuse_gradient=1)),
    "fused, long rows": ((1100, 1000, 900), (300, 150), 200, 200, "relu", float("inf"), dict(fuse_gradient=1)),
    "fused, long rows, ragged": ((1100, 1000, 900), (300, 150), 201, 256, "relu", 2.0, dict(fuse_gradient=1)),
    "fused, too many samples": ((500, 600, 400), (20,), 300, 300, "relu", 2.0, dict(fuse_gradient=1)),
    "separate": ((500, 600, 400), (20, 64), 130, 130, "relu", 2.0, dict(fuse_gradient=-1)),
    "separate, ragged": ((500, 600, 400), (20, 64), 131, 200, "sigmoid", 1.0, dict(fuse_gradient=-1)),
    "separate, long rows": ((600, 500, 400), (300,), 70, 70, "relu", 2.0, dict(fuse_gradient=-1)),
    "separate, uneven rows": ((600, 500, 400), (5, 5, 0, 40, 300, 31, 33), 29, 64, "relu", 2.0, dict(fuse_gradient=-1)),
    "separate, uneven rows, two windows": ((609, 500, 609), (5, 64, 400, 5, 65), 133, 133, "relu", 2.0, dict(fuse_gradient=-1)),
    "separate, many rows": ((900, 17000, 700), (33, 1, 90), 20, 20, "relu", 2.0, dict(fuse_gradient=-1)),
    "panels": ((3000, 2900, 2800), (32, 40), 64, 64, "relu", 2.0, dict(fuse_gradient=-1, panel_cols=512)),
    "panels, ragged": ((3000, 2900, 2800), (32, 40), 77, 90, "relu", 2.0, dict(fuse_gradient=-1, panel_cols=512)),
    "clustered": ((1024, 1024, 1024), (32,), 48, 48, "relu", 2.0, dict(reorder_rows=True)),
    "a layer without entries": ((40, 50, 60), (0,), 9, 9, "relu", 2.0, {}),
    "a layer without entries, fused": ((40, 50, 60), (0,), 9, 9, "relu", 2.0, dict(fuse_gradient=1)),
}


def make(name, **more):
    widths, lengths, b, max_b, activation, cap, options = NETS[name]
    layers = pan_nets.layers(widths, lengths, seed=9000 + len(name))
    net = sdnn.Net(layers, cap, max_b, training=True, activation=activation, **{**options, **more})
    x = wl.normal_inputs(9100, widths[0], b)
    dloss = wl.normal_inputs(9101, widths[-1], b)
    return layers, net, x, dloss, b, activation, cap


def results(net, b):
    L = net.n_layers
    return [net.sdnn_get_delta(k, b) for k in range(1, L + 1)] + [t for k in range(1, L + 1) for t in net.sdnn_weight_grad(k)]


@pytest.mark.parametrize("name", NETS)
def test_backward_from_a_checkpoint(name):
    layers, net, x, dloss, b, activation, cap = make(name)
    net.sdnn_forward(dev(x))
    forward = [net.sdnn_get_activation(k, b) for k in range(net.n_layers + 1)]
    ckpt = net.sdnn_checkpoint_save(b)
    # what is kept is what the plain form keeps of the pass's activations
    kept = kept_blocks(net, ckpt, b, activation, cap)
    for k, (f, v, c) in enumerate(zip(forward, kept, caps(net, activation, cap))):
        np.testing.assert_array_equal(host(v).astype(np.float64), blocks.pack8(host(f), c)[2], err_msg=f"X_{k}")
    net.sdnn_forward(dev(-3 * x))  # another batch, while the first one is away
    net.sdnn_checkpoint_load(ckpt, b)
    for k, v in enumerate(kept):
        assert torch.equal(net.sdnn_get_activation(k, b), v), f"X_{k}"
    again = kept_blocks(net, net.sdnn_checkpoint_save(b), b, activation, cap)
    assert all(np.array_equal(host(u), blocks.pack8(host(v), c)[2]) for u, v, c in zip(again, kept, caps(net, activation, cap)))
    dx0 = net.sdnn_backward_input(dev(dloss))
    grads, (want, bound) = blocks.backward(layers, [host(v).astype(np.float64) for v in kept], dloss, cap, activation)
    close(host(dx0), want, bound, "dX_0")
    for k, pair in enumerate(grads):
        for got, (g, limit), what in zip(net.sdnn_weight_grad(k + 1), pair, ("entries", "biases")):
            close(host(got), g, limit, f"layer {k + 1}, {what}")
    if "entries" not in name and "small" not in name:
        assert all(np.abs(g[0][0]).max() > 0 for g in grads) and np.abs(want).max() > 0
    net.close()


@pytest.mark.parametrize("name", NETS)
def test_the_gradient_of_the_input_changes_nothing_else(name):
    """sdnn_backward and sdnn_backward_input: the same bits of everything; and dX_0 against the plain form on the pass's own activations."""
    layers, net, x, dloss, b, activation, cap = make(name)
    net.sdnn_forward(dev(x))
    net.sdnn_backward(dev(dloss))
    want = results(net, b)
    net.sdnn_forward(dev(x))
    whole = torch.full((x.size + 8,), 777.0, device=DEV)
    dx0 = net.sdnn_backward_input(dev(dloss), whole[1:1 + x.size].view(x.shape))  # not aligned to more than 4 bytes
    assert all(torch.equal(u, v) for u, v in zip(results(net, b), want))
    assert float(whole[0]) == 777 and bool((whole[1 + x.size:] == 777).all())
    net.sdnn_forward(dev(x))
    torch.testing.assert_close(net.sdnn_backward_input(dev(dloss)), dx0, rtol=4 * blocks.HALF, atol=1e-9)
    xs = [host(net.sdnn_get_activation(k, b)).astype(np.float64) for k in range(net.n_layers + 1)]
    _, (ref, bound) = blocks.backward(layers, xs, dloss, cap, activation)
    close(host(dx0), ref, bound, "dX_0")
    net.sdnn_sgd_step(0.01)
    net.close()


@pytest.mark.parametrize("name", ["launch per pass", "one sample", "fused, 99", "separate, ragged"])
def test_a_step_from_a_checkpoint_moves_the_weights_by_its_gradient(name):
    layers, net, x, dloss, b, activation, cap = make(name)
    lr = 0.25
    for _ in range(2):  # the second step's passes read copies that have followed the first one's
        before = [net.sdnn_get_weights(k) for k in range(1, net.n_layers + 1)]
        net.sdnn_forward(dev(x))
        ckpt = net.sdnn_checkpoint_save(b)
        net.sdnn_forward(dev(x[:, ::-1].copy()))
        net.sdnn_checkpoint_load(ckpt, b)
        net.sdnn_backward(dev(dloss))
        grads = [net.sdnn_weight_grad(k) for k in range(1, net.n_layers + 1)]
        net.sdnn_sgd_step(lr)
        for k in range(net.n_layers):
            for new, old, g in zip(net.sdnn_get_weights(k + 1), before[k], grads[k]):
                want = old.double() - lr * g.double()
                # the gradient and the result are rounded once each
                assert bool(((new.double() - want).abs() <= 2 * blocks.HALF * (old.abs() + lr * g.abs()).double() + 1e-40).all())
    net.close()


@pytest.mark.parametrize("name", ["launch per pass", "one sample", "fused, 99", "fused, long rows", "separate, ragged"])
def test_captured_and_replayed(name):
    layers, net, x, dloss, b, activation, cap = make(name)
    xd, d, dx0 = dev(x), dev(dloss), torch.empty(x.shape, device=DEV)
    ckpt = torch.zeros(net.sdnn_checkpoint_bytes(b), dtype=torch.uint8, device=DEV)
    grads = [torch.empty(s[2], device=DEV) for s in net.shapes]

    def step():
        net.sdnn_forward(xd)
        net.sdnn_checkpoint_save(b, ckpt)
        net.sdnn_forward(d0)
        net.sdnn_checkpoint_load(ckpt, b)
        net.sdnn_backward_input(d, dx0)
        for k, g in enumerate(grads):
            sdnn._check(sdnn.lib().sdnn_weight_grad(net._handle, k + 1, g.data_ptr(), None, torch.cuda.current_stream().cuda_stream), net._handle)

    d0 = dev(2 * x)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        xd.mul_(0.8)
        d.mul_(1.1)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (ckpt, dx0, *grads)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, (ckpt, dx0, *grads)))
    net.close()


@pytest.mark.parametrize("widths,b,options", [((400, 300, 350), 40, {}), ((900, 800, 850), 96, dict(fuse_gradient=1)), ((64, 50, 60), 1, {})])
def test_nets_norms_and_micro_batches_together(widths, b, options):
    """norm, net, norm, net over three micro-batches that are all forward before the first goes back: gradients of all parts against the
    plain forms on the kept values."""
    first = pan_nets.layers(widths, (16, 9), seed=9300)
    second = pan_nets.layers((widths[-1], widths[0], widths[1]), (12,), seed=9301)
    nets = [sdnn.Net(layers, 2.0, b, training=True, **options) for layers in (first, second)]
    rng = np.random.default_rng(9302)
    gammas = [(1 + 0.2 * rng.normal(size=n)).astype(np.float32) for n in (widths[0], widths[-1])]
    betas = [(0.2 * rng.normal(size=n)).astype(np.float32) for n in (widths[0], widths[-1])]
    batches = [(rng.normal(size=(widths[0], b)) + k).astype(np.float32) for k in range(3)]
    dlosses = [rng.normal(size=(widths[1], b)).astype(np.float32) for _ in range(3)]
    away = []
    for x in batches:
        x = dev(x)
        keep = dict(x=sdnn.sdnn_pack8(x))
        y, keep["stats0"] = sdnn.sdnn_layernorm(x, dev(gammas[0]), dev(betas[0]))
        mid = torch.empty(widths[-1], b, device=DEV)
        nets[0].sdnn_forward(y, mid)
        keep["ckpt0"] = nets[0].sdnn_checkpoint_save(b)
        z, keep["stats1"] = sdnn.sdnn_layernorm(mid, dev(gammas[1]), dev(betas[1]))
        nets[1].sdnn_forward(z)
        keep["ckpt1"] = nets[1].sdnn_checkpoint_save(b)
        away.append(keep)
    for keep, dloss in zip(away, dlosses):
        # the second norm's input is the last block of the first net's checkpoint
        at = nets[0].sdnn_checkpoint_bytes(b) - sdnn.sdnn_pack8_bytes(widths[-1], b)
        mid = sdnn.Packed8(keep["ckpt0"][at:], widths[-1], b, 2.0)
        nets[1].sdnn_checkpoint_load(keep["ckpt1"], b)
        dz = nets[1].sdnn_backward_input(dev(dloss))
        dmid, dg1, db1 = sdnn.sdnn_layernorm_backward(dz, mid, keep["stats1"], dev(gammas[1]))
        nets[0].sdnn_checkpoint_load(keep["ckpt0"], b)
        dy = nets[0].sdnn_backward_input(dmid)
        dx, dg0, db0 = sdnn.sdnn_layernorm_backward(dy, keep["x"], keep["stats0"], dev(gammas[0]))
        # plain: each part from what the part above handed down, so that every bound is that part's own
        for net, layers, ckpt, back, below in ((nets[1], second, "ckpt1", dloss, dz), (nets[0], first, "ckpt0", host(dmid), dy)):
            kept = [host(v).astype(np.float64) for v in kept_blocks(net, keep[ckpt], b, "relu", 2.0)]
            grads, (want, bound) = blocks.backward(layers, kept, back, 2.0, "relu")
            close(host(below), want, bound, ckpt)
            net.sdnn_checkpoint_load(keep[ckpt], b)
            net.sdnn_backward(dev(back))
            for k, pair in enumerate(grads):
                for got, (g, limit) in zip(net.sdnn_weight_grad(k + 1), pair):
                    close(host(got), g, limit, f"{ckpt}, layer {k + 1}")
        for block, stats, gamma, up, got in ((mid, "stats1", gammas[1], dz, (dmid, dg1, db1)), (keep["x"], "stats0", gammas[0], dy, (dx, dg0, db0))):
            x, st = host(sdnn.sdnn_unpack8(block)).astype(np.float64), host(keep[stats])
            want = blocks.norm_backward(host(up), x, st, gamma)
            h = (np.abs(x) + np.abs(st[0])) * st[1]
            for v, w, terms in zip(got, want, (st[1] * np.abs(gamma[:, None] * host(up)) * (1 + h * h), (np.abs(host(up)) * h).sum(1), np.abs(host(up)).sum(1))):
                bound = blocks.HALF * np.abs(w) + 1e-12 * (terms + terms.max()) + blocks.TINY
                close(host(v), w, bound, stats)
    for net in nets:
        net.close()


def test_samples_other_than_those_of_the_pass_are_refused():
    layers, net, x, dloss, b, activation, cap = make("launch per pass")
    xd, d = dev(x), dev(dloss)
    net.sdnn_forward(xd)
    ckpt = net.sdnn_checkpoint_save(b)
    for other in (b - 1, b + 1):
        with pytest.raises(sdnn.SdnnError, match="samples"):
            net.sdnn_checkpoint_save(other)
        with pytest.raises(sdnn.SdnnError, match="dloss"):
            net.sdnn_backward_input(torch.zeros(dloss.shape[0], other, device=DEV))
    with pytest.raises(sdnn.SdnnError):
        net.sdnn_forward(dev(wl.normal_inputs(9103, x.shape[0], net.cfg.max_batch + 1)))  # refused: the pass before it is still the last
    want = net.sdnn_backward_input(d)
    net.sdnn_forward(dev(wl.normal_inputs(9102, x.shape[0], 3)))
    with pytest.raises(sdnn.SdnnError, match="needed"):
        net.sdnn_checkpoint_load(ckpt, b + 16)
    net.sdnn_checkpoint_load(ckpt, b)
    assert net.sdnn_backward_input(d).shape == want.shape
    net.close()


@pytest.mark.parametrize("widths,lengths,b", [((70,) * 71, (3, 0, 64, 33), 40), ((130,) * 65, (1, 120, 2), 21), ((40, 300, 40, 300, 40), (40, 2, 2, 2, 300), 200)])
def test_steps_of_few_rows_in_many_layers(widths, lengths, b):
    """The separate update where several wavefronts share a row's chunks, of many layers at once and of one: the step takes the gradient
    that sdnn_weight_grad hands out, and that is the plain form's on the pass's own blocks."""
    layers = pan_nets.layers(widths, lengths, seed=9400)
    net = sdnn.Net(layers, 1.0, b, training=True, activation="sigmoid", fuse_gradient=-1, lds_forward=-1)
    net.sdnn_forward(dev(wl.normal_inputs(9401, widths[0], b)))
    net.sdnn_backward(dev(wl.normal_inputs(9402, widths[-1], b)))
    before = [net.sdnn_get_weights(k) for k in range(1, net.n_layers + 1)]
    grads = [net.sdnn_weight_grad(k) for k in range(1, net.n_layers + 1)]
    for k, (layer, (g, gb)) in enumerate(zip(layers, grads)):
        x, delta = (host(t).astype(np.float64) for t in (net.sdnn_get_activation(k, b), net.sdnn_get_delta(k + 1, b)))
        rows = np.repeat(np.arange(layer.n_out), np.diff(layer.row_ptr))
        terms = delta[rows] * x[layer.col_idx]
        close(host(g), terms.sum(1), blocks.HALF * np.abs(terms.sum(1)) + 1e-12 * np.abs(terms).sum(1) + blocks.TINY, f"layer {k + 1}, entries")
        close(host(gb), delta.sum(1), blocks.HALF * np.abs(delta.sum(1)) + 1e-12 * np.abs(delta).sum(1) + blocks.TINY, f"layer {k + 1}, biases")
    net.sdnn_sgd_step(0.25)
    for k in range(net.n_layers):
        for new, old, g in zip(net.sdnn_get_weights(k + 1), before[k], grads[k]):
            want = old.double() - 0.25 * g.double()
            assert bool(((new.double() - want).abs() <= blocks.HALF * want.abs() + 1e-40).all())
    net.close()
