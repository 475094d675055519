"""Layer norm over the neurons of each sample, activations kept in 8 bits, and training passes that run from them, as cases that
can be timed and compared.

Blocks are those of the nets: [neurons][samples], the samples of one neuron contiguous, fp32.

  norm     a block before it goes into a net (or between two nets): y and what the backward pass needs of the statistics
  grad     the norm's backward pass: gradients of the block, of the scale and of the shift; the block as it is, or from 8 bits
  keep     a block put away in 8 bits and taken out again
  replay   the backward pass of a net whose activations were put away: the gradients of all its weights and biases and of
           its input

With `own` the framework's operators run, without it the same in elementary torch operations.
"""
import math

import torch

own = False  # set by the tools

DEV = "cuda:0"
EPS = 1e-5
GROUP = 128  # values that share a scale


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # configuration 1's width and minibatch: the smallest block, where latency counts
        dict(name="norm-n1024-b64", kind="norm", n=1024, batch=64),
        # sizes that are multiples of nothing
        dict(name="norm-n3001-b777", kind="norm", n=3001, batch=777),
        # configuration 4's training step: a few samples of many neurons
        dict(name="norm-n65536-b64", kind="norm", n=65536, batch=64),
        # configuration 3's bulk inference: a block larger than any cache
        dict(name="norm-n16384-b4096", kind="norm", n=16384, batch=4096),
        # the smallest backward pass
        dict(name="grad-n1024-b64", kind="grad", n=1024, batch=64, packed=False),
        # a minibatch that fits no tile on a width that fits none either
        dict(name="grad-n10007-b99", kind="grad", n=10007, batch=99, packed=False),
        # configuration 4's training step, the block as it was put away
        dict(name="grad-packed-n65536-b64", kind="grad", n=65536, batch=64, packed=True),
        # a large batch on configuration 5's width, as it was put away
        dict(name="grad-packed-n8192-b2048", kind="grad", n=8192, batch=2048, packed=True),
        # inputs of both signs and of ragged sizes
        dict(name="keep-n3001-b777", kind="keep", n=3001, batch=777, signed=True),
        # configuration 4's width, the activations of a bulk block
        dict(name="keep-n65536-b1024", kind="keep", n=65536, batch=1024, signed=False),
        # configuration 2's minibatch, a stretch of its layers
        dict(name="replay-n4096-b128", kind="replay", topo="even", act="relu", n=4096, layers=8, batch=128),
        # configuration 5: irregular rows
        dict(name="replay-pruned-n8192-b256", kind="replay", topo="pruned", act="relu", n=8192, layers=2, batch=256),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: widths from 256 to 65536 neurons (nets: to 16384, pruned ones to 8192), batches from one sample to 4096
    (nets: 256), both spread over their logarithm, half of the widths odd."""
    kind = rng.choice(["norm", "grad", "grad", "keep", "replay", "replay"])
    topo = rng.choice(["even", "even", "pruned"])
    n = _log_uniform(rng, 256, 65536 if kind != "replay" else 16384 if topo == "even" else 8192)
    n = n | 1 if rng.random() < 0.5 else n // 32 * 32
    if kind == "replay":
        return dict(kind=kind, topo=topo, act=rng.choice(["relu", "relu", "sigmoid"]), n=n, layers=2, batch=_log_uniform(rng, 1, 256))
    case = dict(kind=kind, n=n, batch=_log_uniform(rng, 1, min(4096, (1 << 24 if kind == "grad" else 1 << 26) // n)))
    if kind == "grad":
        case["packed"] = rng.random() < 0.5
    if kind == "keep":
        case["signed"] = rng.random() < 0.5
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------

class _Layer:
    """What sdnn.Net takes: CSR arrays on the host."""

    def __init__(self, layer, n):
        self.n_out = self.n_in = n
        self.row_ptr = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), layer["count"].cumsum(0)]).to(torch.int32).cpu().numpy()
        self.col_idx = layer["col"].to(torch.int32).cpu().numpy()
        self.values = layer["value"].cpu().numpy()
        self.bias = layer["bias"].cpu().numpy()


def _degrees(n):
    """Links per neuron of a pruned layer: the n quantiles of a Pareto tail of shape 1.2, scaled to a mean of about n/10 and
    clipped to 1 .. n/4."""
    tail = ((torch.arange(n, dtype=torch.float64, device=DEV) + 0.5) / n).pow(-1.0 / 1.2)
    return (tail * (0.1 * n / 3.3)).round().clamp(1, max(1, n // 4)).to(torch.int64)


def _layer(gen, case):
    """One layer's entries, row by row and ascending in a row: `row`, `col`, `value` of each, `count` per row, biases."""
    n = case["n"]
    if case["topo"] == "even":  # 32 links per neuron to distinct, uniformly random sources
        count = torch.full((n,), min(32, n), dtype=torch.int64, device=DEV)
    else:
        count = _degrees(n)[torch.randperm(n, generator=gen, device=DEV)]
    pieces = []
    for first in range(0, n, 4096):  # a row keeps the links with the smallest keys
        some = count[first:first + 4096]
        key = torch.rand(some.numel(), n, generator=gen, device=DEV)
        order = key.topk(int(some.max()), dim=1, largest=False, sorted=True).indices
        keep = torch.arange(order.shape[1], device=DEV)[None, :] < some[:, None]
        order = torch.where(keep, order, n).sort(dim=1).values
        pieces.append(order[order < n])
    col = torch.cat(pieces)
    row = torch.repeat_interleave(torch.arange(n, device=DEV), count)
    sd = 0.25 if case["topo"] == "even" else count[row].float().rsqrt()
    value = torch.randn(col.numel(), generator=gen, device=DEV) * sd * (4.0 if case["act"] == "sigmoid" else 1.0)
    return dict(row=row, col=col, value=value, count=count, bias=0.1 * torch.randn(n, generator=gen, device=DEV))


def _cap(case):
    """The bound of the activations that are put away: 1 for the sigmoid; 32 or none for the clamped ReLU."""
    return 1.0 if case["act"] == "sigmoid" else 32.0 if case["topo"] == "even" else math.inf


def _activations(case, layers, x):
    """X_0 .. X_L, every sum in 64 bits."""
    blocks = [x]
    for y in layers:
        dense = torch.zeros(case["n"], case["n"], device=DEV, dtype=torch.float64)
        dense[y["row"], y["col"]] = y["value"].double()
        z = dense @ blocks[-1].double() + y["bias"].double()[:, None]
        blocks.append((torch.sigmoid(z) if case["act"] == "sigmoid" else z.clamp(0, _cap(case))).float())
    return blocks


def _inputs(case, seed):
    """What a case's passes work on, from the seed alone."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, batch = case["n"], case["batch"]
    rand = lambda *shape: torch.rand(*shape, generator=gen, device=DEV)  # noqa: E731
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)  # noqa: E731
    if case["kind"] == "replay":
        layers = [_layer(gen, case) for _ in range(case["layers"])]
        x = randn(n, batch) if case["topo"] == "pruned" else (rand(n, batch) < 0.19).float()
        return dict(layers=layers, blocks=_activations(case, layers, x), dloss=randn(n, batch) / batch)
    # what a layer of a net leaves: half of the values zero, every sample and every neuron with a level of its own, a few at the cap
    x = (randn(n, batch) + 0.5 * randn(n, 1)) * (1.0 + rand(1, batch))
    if case["kind"] == "keep" and case["signed"]:
        return dict(x=x)
    x = torch.where(rand(n, batch) < 0.001, 32.0, x.clamp(0, 32))
    if case["kind"] == "keep":
        return dict(x=x)
    g = dict(x=x, gamma=1.0 + 0.2 * randn(n), beta=0.2 * randn(n))
    if case["kind"] == "grad":
        g["dy"] = randn(n, batch) / batch
        g["stats"] = _statistics(x)  # left by the forward pass
    return g


def prepare(case, seed):
    state = dict(case=case, **_inputs(case, seed))
    n, batch, kind = case["n"], case["batch"], case["kind"]
    if kind == "grad" and case["packed"]:
        state["packed"] = _pack(state.pop("x"), 32.0)
    if kind == "replay":
        caps = [0.0] + [_cap(case)] * case["layers"]
        state["kept"] = torch.cat([_pack(x, cap) for x, cap in zip(state.pop("blocks"), caps)])
        if own:
            from paper_2104_11805_amd import sdnn
            state["net"] = sdnn.Net([_Layer(y, n) for y in state.pop("layers")], 1.0 if case["act"] == "sigmoid" else _cap(case), batch,
                                    activation=case["act"])
        else:
            state["by_column"] = [_by_column(y, n) for y in state["layers"]]
    if own:
        from paper_2104_11805_amd import sdnn
        state["sdnn"] = sdnn
        if kind in ("norm", "grad"):
            state["work"] = torch.empty(sdnn.sdnn_layernorm_workspace_bytes(n, batch), dtype=torch.uint8, device=DEV)
        if kind == "keep":
            state["packed"] = torch.empty(sdnn.sdnn_pack8_bytes(n, batch), dtype=torch.uint8, device=DEV)
        state["out"] = torch.empty(n, batch, device=DEV)
    return state


# ---- 8 bits -----------------------------------------------------------------------------------------------------------
# A packed block: a byte for every value of the block in its order, filled up to whole groups of 128; then a scale of 16 bits (the
# upper half of a float) for every group; filled up to a multiple of 256 bytes.  With a cap of 0 the values have both signs: the
# byte is a signed number of scales, -128 stands for what is not finite.  With a cap they are 0 to cap: 0 for zero, 255 for the cap,
# 254 for NaN, else 1 to 253 scales.  The scale is the smallest for which the largest value fits.

def _pack(x, cap):
    flat = x.reshape(-1)
    v = torch.nn.functional.pad(flat, (0, -flat.numel() % GROUP)).view(-1, GROUP)
    live = (v > 0) & (v < cap) if cap > 0 else v.isfinite()
    most = 253 if cap > 0 else 127
    size = torch.where(live, v.abs(), 0.0)
    largest = size.amax(dim=1, keepdim=True).double()
    down = ((largest / most).float().view(torch.int32) >> 16)
    scale = torch.where((down << 16).view(torch.float32).double() * most >= largest, down, down + 1)
    step = (scale << 16).view(torch.float32)
    times = torch.where(live, (size.double() / step.double() + 0.5).floor(), 0.0).int()
    if cap > 0:
        code = torch.where(live, times.clamp(1, 253), torch.where(v >= cap, 255, torch.where(v.isnan(), 254, 0)))
    else:
        code = torch.where(live, torch.where(v < 0, -times, times), -128) & 255
    packed = torch.cat([code.to(torch.uint8).view(-1), scale.to(torch.int16).view(-1).view(torch.uint8)])
    return torch.nn.functional.pad(packed, (0, -packed.numel() % 256))


def _unpack(packed, n, batch, cap):
    groups = -(-n * batch // GROUP)
    code = packed[:groups * GROUP].view(groups, GROUP)
    scale = packed[groups * GROUP:groups * (GROUP + 2)].view(torch.int16).int()
    step = (scale << 16).view(torch.float32)[:, None]
    if cap > 0:
        below = torch.nextafter(torch.tensor(cap), torch.tensor(0.0)).item()
        v = torch.minimum(code.float() * step, torch.full((), below, device=DEV))
        v = torch.where(code == 255, cap, torch.where(code == 254, math.nan, v))
    else:
        v = code.view(torch.int8).float() * step
        v = torch.where(code == 128, math.nan, v)
    return v.view(-1)[:n * batch].view(n, batch)


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _statistics(x):
    """[2][samples] in 64 bits (long sums, and a variance next to a large mean): the mean of each sample and 1/sqrt(variance + eps)."""
    x = x.double()
    mean = x.mean(dim=0)
    var = (x - mean).square().mean(dim=0)
    return torch.stack([mean, (var + EPS).rsqrt()])


def _norm(s):
    stats = _statistics(s["x"])
    hat = (s["x"].double() - stats[0]).float() * stats[1].float()
    return hat * s["gamma"][:, None] + s["beta"][:, None], stats


def _norm_grad(s):
    case = s["case"]
    x = _unpack(s["packed"], case["n"], case["batch"], 32.0) if case["packed"] else s["x"]
    mean, rstd = s["stats"]
    hat = (x.double() - mean).float() * rstd.float()
    dy = s["dy"]
    d = dy * s["gamma"][:, None]
    dx = (d - d.mean(dim=0) - hat * (d * hat).mean(dim=0)) * rstd.float()
    return dx, (dy * hat).sum(dim=1), dy.sum(dim=1)


def _by_column(y, n):
    """The entries of each column side by side, filled up with a row n of weight 0."""
    order = torch.argsort(y["col"], stable=True)
    count = torch.bincount(y["col"], minlength=n)
    place = torch.arange(order.numel(), device=DEV) - (count.cumsum(0) - count)[y["col"][order]]
    rows = torch.full((n, int(count.max())), n, device=DEV)
    values = torch.zeros(rows.shape, device=DEV)
    rows[y["col"][order], place] = y["row"][order]
    values[y["col"][order], place] = y["value"][order]
    return rows, values


def _slope(x, case):
    return x * (1.0 - x) if case["act"] == "sigmoid" else ((x > 0) & (x < _cap(case))).float()


def _replay(s):
    case = s["case"]
    n, batch = case["n"], case["batch"]
    kept = s["kept"].view(case["layers"] + 1, -1)
    x = _unpack(kept[case["layers"]], n, batch, _cap(case))
    back, grads = s["dloss"], []
    for l in reversed(range(case["layers"])):
        y, (rows, values) = s["layers"][l], s["by_column"][l]
        delta = back * _slope(x, case)
        x = _unpack(kept[l], n, batch, _cap(case) if l else 0.0)
        grads.append(((delta[y["row"]] * x[y["col"]]).sum(dim=1), delta.sum(dim=1)))
        some = torch.nn.functional.pad(delta, (0, 0, 0, 1))[rows]
        back = some.mul_(values[:, :, None]).sum(dim=1)
    return grads[::-1], back


# ---- one pass -----------------------------------------------------------------------------------------------------------

def _run_own(s):
    sdnn, case = s["sdnn"], s["case"]
    if case["kind"] == "norm":
        return sdnn.sdnn_layernorm(s["x"], s["gamma"], s["beta"], eps=EPS, y=s["out"], work=s["work"])
    if case["kind"] == "grad":
        x = sdnn.Packed8(s["packed"], case["n"], case["batch"], 32.0) if case["packed"] else s["x"]
        return sdnn.sdnn_layernorm_backward(s["dy"], x, s["stats"], s["gamma"], dx=s["out"], work=s["work"])
    if case["kind"] == "keep":
        packed = sdnn.sdnn_pack8(s["x"], cap=0.0 if case["signed"] else 32.0, packed=s["packed"])
        return sdnn.sdnn_unpack8(packed, x=s["out"])
    net = s["net"]
    net.sdnn_checkpoint_load(s["kept"], case["batch"])
    dx0 = net.sdnn_backward_input(s["dloss"], s["out"])
    return [net.sdnn_weight_grad(l + 1) for l in range(case["layers"])], dx0


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["kind"] == "norm":
        return _norm(state)
    if case["kind"] == "grad":
        return _norm_grad(state)
    if case["kind"] == "keep":
        cap = 0.0 if case["signed"] else 32.0
        return _unpack(_pack(state["x"], cap), case["n"], case["batch"], cap)
    return _replay(state)


# ---- what it cannot do without, and the values in 64 bits -----------------------------------------------------------------

def work(case):
    """A norm reads the block once and writes one; its backward pass reads two (one of them, where it was put away, in a byte a
    value and 2 bytes a group) and writes one.  The backward pass of a net reads its kept blocks, index and value of every entry and
    the loss gradient, and writes the gradients and that of the input; two operations per entry and sample and product."""
    n, batch = case["n"], case["batch"]
    count = n * batch
    byte = (1 + 2 / GROUP) * count
    if case["kind"] == "norm":
        return {"bytes": 8 * count + 8 * n + 16 * batch, "flops": 8 * count}
    if case["kind"] == "grad":
        return {"bytes": 8 * count + (byte if case["packed"] else 4 * count) + 12 * n + 16 * batch, "flops": 14 * count}
    if case["kind"] == "keep":
        return {"bytes": 8 * count + 2 * byte, "flops": 6 * count}
    entries = n * (min(32, n) if case["topo"] == "even" else 0.1 * n)
    layers = case["layers"]
    return {"bytes": layers * (12 * entries + byte + 4 * n) + byte + 8 * count, "flops": layers * 4 * entries * batch}


def _as_kept(x, cap):
    """The values that come back of a block, by the rule that scales have 8 significant bits and values go to the nearest multiple."""
    v = torch.nn.functional.pad(x.double().flatten(), (0, -x.numel() % GROUP)).reshape(-1, GROUP)
    inside = (v > 0) & (v < cap) if cap > 0 else torch.ones_like(v, dtype=torch.bool)
    top = 253.0 if cap > 0 else 127.0
    mantissa, exponent = torch.frexp((v * inside).abs().max(dim=1, keepdim=True).values / top)
    step = torch.ldexp(torch.ceil(mantissa * 256.0), exponent - 8)
    count = torch.floor(torch.where(step > 0, v.abs() / step, 0.0) + 0.5)
    if cap > 0:
        below = float(torch.nextafter(torch.tensor(cap, dtype=torch.float32), torch.tensor(0.0)))
        near = (count.clamp(min=1.0) * step).clamp(max=below)
        back = near * inside + torch.where(v >= cap, v, 0.0)
    else:
        back = torch.copysign(count * step, v)
    return back.flatten()[:x.numel()].reshape(x.shape)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "keep":
        return _as_kept(s["x"], 0.0 if case["signed"] else 32.0)
    if kind in ("norm", "grad"):
        x = s["x"].double()
        n = case["n"]
        mean = x.sum(0) / n
        rstd = 1.0 / torch.sqrt(((x - mean) ** 2).sum(0) / n + EPS)
        if kind == "norm":
            return (x - mean) * rstd * s["gamma"].double()[:, None] + s["beta"].double()[:, None], torch.stack([mean, rstd])
        hat = ((_as_kept(s["x"], 32.0) if case["packed"] else x) - mean) * rstd
        dy, gamma = s["dy"].double(), s["gamma"].double()
        p, q = (gamma @ dy) / n, (gamma[:, None] * dy * hat).sum(0) / n
        return rstd * (gamma[:, None] * dy - p - hat * q), (dy * hat).sum(1), dy.sum(1)
    caps = [0.0] + [_cap(case)] * case["layers"]
    kept = [_as_kept(x, cap) for x, cap in zip(s["blocks"], caps)]
    back, grads = s["dloss"].double(), []
    for y, below, above in zip(s["layers"][::-1], kept[-2::-1], kept[:0:-1]):
        slope = above * (1 - above) if case["act"] == "sigmoid" else torch.where((above <= 0) | (above >= _cap(case)), 0.0, 1.0).double()
        delta = back * slope
        grads.insert(0, ((delta @ below.T)[y["row"], y["col"]], delta.sum(1)))
        weights = torch.zeros(case["n"], case["n"], dtype=torch.float64, device=DEV)
        weights[y["row"], y["col"]] = y["value"].double()
        back = weights.T.contiguous() @ delta
    return grads, back
