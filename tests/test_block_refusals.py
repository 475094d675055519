"""What the operators on blocks and the checkpoints refuse, and what they launch, without a GPU (see tests/routes.py); and the plain
forms of the tests against differences."""
import numpy as np
import pytest

from paper_2104_11805_amd import sdnn
from tests import blocks, routes

PTR = """
        A = [k << 41 for k in range(1, 9)]
        size = C.c_size_t()
        def call(name, *args):
            stub.stub_clear()
            rc = getattr(lib, name)(*[C.c_void_p(a) if isinstance(a, int) and a >= 1 << 41 else a for a in args])
            return rc, [l for l in stub.stub_log().decode().split("\\n") if l]
        def refused(code, text, name, *args):
            rc, log = call(name, *args)
            assert rc == code and not log and text in sdnn.last_error(), (rc, log, sdnn.last_error())
"""


def test_layer_norm_refusals():
    routes.run(PTR + """
        lib.sdnn_layernorm_workspace_bytes(100, 7, C.byref(size))
        w = size.value
        ok = [A[0], A[1], A[2], 100, 7, 1e-5, A[3], A[4], A[5], w, None]
        def fwd(**kw):
            a = list(ok)
            for k, v in kw.items():
                a[int(k[1:])] = v
            return ("sdnn_layernorm", *a)
        rc, log = call(*fwd())
        assert rc == 0 and log, sdnn.last_error()
        assert call(*fwd(a1=None, a2=None, a7=None))[0] == 0
        for k, v in [(3, 0), (3, -1), (4, 0), (4, -3), (3, (1 << 30) + 1), (4, (1 << 30) + 1)]:
            refused(-1, "block of", *fwd(**{f"a{k}": v}))
        refused(-1, "block of", *fwd(a3=1 << 25, a4=1 << 15))
        for v in (0.0, -1e-5, float("nan"), float("inf")):
            refused(-1, "eps", *fwd(a5=v))
        refused(-1, "d_X", *fwd(a0=None))
        refused(-1, "d_Y", *fwd(a6=None))
        refused(-1, "d_work", *fwd(a8=None))
        refused(-1, "aligned", *fwd(a8=A[5] + 8))
        refused(-3, "workspace", *fwd(a9=w - 1))
        refused(-1, "block of", "sdnn_layernorm_workspace_bytes", 0, 5, C.byref(size))
        refused(-1, "bytes", "sdnn_layernorm_workspace_bytes", 5, 5, None)

        okb = [A[0], A[1], A[2], A[3], 100, 7, A[4], A[5], A[6], A[7], w, None]
        def bwd(**kw):
            a = list(okb)
            for k, v in kw.items():
                a[int(k[1:])] = v
            return ("sdnn_layernorm_backward", *a)
        assert call(*bwd())[0] == 0
        assert call(*bwd(a6=None))[0] == call(*bwd(a7=None, a8=None))[0] == call(*bwd(a3=None))[0] == 0
        refused(-1, "no result", *bwd(a6=None, a7=None, a8=None))
        refused(-1, "d_dY", *bwd(a0=None))
        refused(-1, "d_X", *bwd(a1=None))
        refused(-1, "d_stats", *bwd(a2=None))
        refused(-3, "workspace", *bwd(a10=w - 1))
        refused(-1, "block of", *bwd(a4=0))

        lib.sdnn_pack8_bytes(100, 7, C.byref(size))
        p = size.value
        okp = [A[0], A[1], p, 0.0, A[2], A[3], 100, 7, A[4], A[5], A[6], A[7], w, None]
        def bwp(**kw):
            a = list(okp)
            for k, v in kw.items():
                a[int(k[1:])] = v
            return ("sdnn_layernorm_backward_packed", *a)
        assert call(*bwp())[0] == call(*bwp(a3=float("inf")))[0] == 0
        refused(-1, "cap", *bwp(a3=-1.0))
        refused(-1, "cap", *bwp(a3=float("nan")))
        refused(-3, "packed", *bwp(a2=p - 1))
        refused(-1, "aligned", *bwp(a1=A[1] + 4))
        refused(-1, "d_packed", *bwp(a1=None))
    """)


def test_sizes_at_the_ends_of_what_is_taken():
    """Every launch holds less than 2^32 threads and has room in its grid (the stand-in refuses what the runtime does)."""
    routes.run(PTR + """
        M = 1 << 30
        for n, b in [(1, 1), (1, M), (M, 1), (M, 1023), (1023, M), (1000, 1 << 27), (1000, 1 << 26), (1000, (1 << 26) + 1), (2000, 1 << 23), (2100, 1 << 26), (2100, (1 << 26) + 5),
                     (4, 1 << 28), (300, 1 << 25), (1 << 20, 1 << 19), (1 << 25, 128), (1 << 25, 3), (1 << 24, 17)]:
            assert lib.sdnn_layernorm_workspace_bytes(n, b, C.byref(size)) == 0
            w = size.value
            assert call("sdnn_layernorm", A[0], A[1], A[2], n, b, 1e-5, A[3], A[4], A[5], w, None)[0] == 0, (n, b, sdnn.last_error())
            assert call("sdnn_layernorm_backward", A[0], A[1], A[2], A[3], n, b, A[4], A[5], A[6], A[7], w, None)[0] == 0, (n, b, sdnn.last_error())
            assert lib.sdnn_pack8_bytes(n, b, C.byref(size)) == 0
            assert call("sdnn_layernorm_backward_packed", A[0], A[1], size.value, 2.0, A[2], A[3], n, b, None, A[5], A[6], A[7], w, None)[0] == 0, (n, b, sdnn.last_error())
            assert call("sdnn_pack8", A[0], n, b, 0.0, A[1], size.value, None)[0] == 0 and call("sdnn_unpack8", A[1], size.value, n, b, 2.0, A[0], None)[0] == 0, (n, b)
    """)


def test_packed_block_sizes_and_refusals():
    for n, b in [(0, 3), (1, 1), (127, 1), (128, 1), (129, 1), (3, 1000), (65536, 65536)]:
        assert sdnn.sdnn_pack8_bytes(n, b) == blocks.packed_bytes(n, b)
    routes.run(PTR + """
        lib.sdnn_pack8_bytes(100, 7, C.byref(size))
        p = size.value
        for name, x in (("sdnn_pack8", 0), ("sdnn_unpack8", 5)):
            def args(X=A[0], n=100, B=7, cap=0.0, packed=A[1], bytes=p):
                return (name, *((X, n, B, cap, packed, bytes, None) if x == 0 else (packed, bytes, n, B, cap, X, None)))
            assert call(*args())[0] == call(*args(cap=32.0))[0] == call(*args(cap=float("inf")))[0] == 0
            assert call(*args(n=0, X=None, packed=None, bytes=0)) == (0, [])
            refused(-1, "block of", *args(n=-1))
            refused(-1, "block of", *args(B=0))
            refused(-1, "block of", *args(n=1 << 30, B=1 << 10))
            refused(-1, "cap", *args(cap=-0.5))
            refused(-1, "cap", *args(cap=float("nan")))
            refused(-1, "d_X", *args(X=None))
            refused(-1, "d_packed", *args(packed=None))
            refused(-1, "aligned", *args(packed=A[1] + 8))
            refused(-3, "needed", *args(bytes=p - 1))
        refused(-1, "bytes", "sdnn_pack8_bytes", 4, 4, None)
        refused(-1, "block of", "sdnn_pack8_bytes", 4, 0, C.byref(size))
    """)


def test_checkpoint_refusals_and_order_of_calls():
    routes.run("""
        CK = 5 << 40
        net = Net([layer(300, 200, (8,)), layer(100, 300, (8,))], 20, training=True)
        size = C.c_size_t()
        def need(b):
            rc = lib.sdnn_checkpoint_bytes(net.h, b, C.byref(size))
            return rc, size.value
        block = lambda n, b: -(-130 * -(-n * b // 128) // 256) * 256
        assert need(7) == (0, block(200, 7) + block(300, 7) + block(100, 7))
        assert need(0)[0] == need(21)[0] == -1 and lib.sdnn_checkpoint_bytes(net.h, 5, None) == -1 and lib.sdnn_checkpoint_bytes(None, 5, C.byref(size)) == -1
        n7 = need(7)[1]

        def refused(code, text, name, *args):
            rc, log = net(name, *args)
            assert rc == code and not log and text in sdnn.last_error(net.h), (rc, log, sdnn.last_error(net.h))
        refused(-2, "sdnn_forward", "sdnn_checkpoint_save", CK, n7, None)
        refused(-2, "sdnn_forward", "sdnn_backward_input", DL, XL, None)
        refused(-1, "d_ckpt", "sdnn_checkpoint_load", None, n7, 7, None)
        refused(-1, "aligned", "sdnn_checkpoint_load", CK + 8, n7, 7, None)
        refused(-3, "needed", "sdnn_checkpoint_load", CK, n7 - 1, 7, None)
        refused(-1, "B = 0", "sdnn_checkpoint_load", CK, n7, 0, None)
        refused(-1, "B = 21", "sdnn_checkpoint_load", CK, 1 << 20, 21, None)
        assert net("sdnn_forward", X0, 7, XL, None)[0] == 0
        refused(-3, "needed", "sdnn_checkpoint_save", CK, n7 - 1, None)
        refused(-1, "d_ckpt", "sdnn_checkpoint_save", None, n7, None)
        refused(-1, "d_dX0", "sdnn_backward_input", DL, None, None)
        rc, log = net("sdnn_checkpoint_save", CK, n7, None)
        assert rc == 0 and len(log) == 1, log
        assert net("sdnn_backward", DL, None)[0] == 0           # the net is as it was
        refused(-2, "sdnn_forward", "sdnn_checkpoint_save", CK, n7, None)
        rc, log = net("sdnn_checkpoint_load", CK, n7, 7, None)
        assert rc == 0 and len(log) == 1, log
        assert net("sdnn_checkpoint_save", CK, n7, None)[0] == 0
        refused(-2, "sdnn_backward", "sdnn_sgd_step", C.c_float(0.1), None)
        assert net("sdnn_backward_input", DL, XL, None)[0] == 0 and net("sdnn_weight_grad", 1, XL, None, None)[0] == 0
        assert net("sdnn_sgd_step", C.c_float(0.1), None)[0] == 0
        refused(-2, "sdnn_forward", "sdnn_checkpoint_save", CK, n7, None)

        net = Net([layer(300, 200, (8,))], 20)                     # inference
        refused(-2, "training", "sdnn_checkpoint_load", CK, 1 << 20, 7, None)
        refused(-2, "training", "sdnn_checkpoint_save", CK, 1 << 20, None)
        refused(-2, "training", "sdnn_backward_input", DL, XL, None)
        assert lib.sdnn_checkpoint_bytes(net.h, 7, C.byref(size)) == -2
        for name, args in (("sdnn_checkpoint_save", (None, 0, None)), ("sdnn_checkpoint_load", (None, 0, 1, None)), ("sdnn_backward_input", (None, None, None))):
            assert getattr(lib, name)(None, *args) == -1
    """)


def test_a_checkpoint_of_a_block_that_the_passes_refuse():
    routes.run("""
        net = Net([layer(40, 1 << 20, (8,)), layer(3, 40, (8,))], 1200, training=True)
        size = C.c_size_t()
        for B, rc in ((1000, 0), (1024, -1), (1100, -1)):
            assert lib.sdnn_checkpoint_bytes(net.h, B, C.byref(size)) == 0
            assert net("sdnn_checkpoint_load", 5 << 40, size.value, B, None)[0] == rc
            assert net("sdnn_forward", X0, B, XL, None)[0] == rc
    """)


def test_backward_input_adds_one_product_or_none():
    """A sweep that gathers Delta_1 for the gradient forms dJ/dX_0 too; else it takes a launch more."""
    routes.run("""
        for options, layers, B, more in [
                (dict(fuse_gradient=1), [layer(9000, 9000, (32,))] * 2, 64, 0), (dict(fuse_gradient=1), [layer(300, 200, (8,))], 20, 0),
                (dict(fuse_gradient=1), [layer(4096, 4096, (400,))] * 2, 200, 0), (dict(fuse_gradient=-1), [layer(300, 200, (8,))] * 1, 20, 1),
                (dict(fuse_gradient=-1), [layer(300, 300, (8,))] * 5, 64, 1), (dict(), [layer(300, 300, (8,))] * 2, 1, 1),
                (dict(fuse_gradient=1), [layer(300, 300, (8,))] * 2, 300, 1)]:
            net = Net(layers, B, training=True, **options)
            n = []
            for name, args in (("sdnn_backward", (DL, None)), ("sdnn_backward_input", (DL, 6 << 40, None))):
                assert net("sdnn_forward", X0, B, XL, None)[0] == 0
                rc, log = net(name, *args)
                assert rc == 0, sdnn.last_error(net.h)
                n.append(len(log))
            assert n[1] == n[0] + more, (options, B, n)
    """)


def test_tensors_that_the_binding_refuses():
    torch = pytest.importorskip("torch")
    x = torch.zeros(3, 4)
    for call in (lambda: sdnn.sdnn_layernorm(x), lambda: sdnn.sdnn_pack8(x), lambda: sdnn.sdnn_layernorm_backward(x, x, torch.zeros(2, 4)),
                 lambda: sdnn.sdnn_layernorm(None)):
        with pytest.raises(sdnn.SdnnError) as e:
            call()
        assert e.value.code == sdnn.SDNN_EINVAL


# ---- the plain forms themselves ------------------------------------------------------------------------------------

def test_plain_norm_gradients_against_differences():
    rng = np.random.default_rng(1)
    n, b, eps = 6, 3, 1e-2
    x, gamma, beta, c = rng.normal(size=(n, b)), rng.normal(size=n), rng.normal(size=n), rng.normal(size=(n, b))
    loss = lambda x, gamma, beta: (c * blocks.norm(x, gamma, beta, eps)[0]).sum()
    grads = blocks.norm_backward(c, x, blocks.norm(x, gamma, beta, eps)[1], gamma)
    for k, v in enumerate((x, gamma, beta)):
        for i in np.ndindex(v.shape):
            args = [[a.copy() for a in (x, gamma, beta)] for _ in range(2)]
            args[0][k][i] += 1e-5
            args[1][k][i] -= 1e-5
            diff = (loss(*args[0]) - loss(*args[1])) / 2e-5
            assert abs(diff - grads[k][i]) < 1e-8 * max(1.0, abs(diff)), (k, i)  # h^2 of the third derivative and 1e-16 / h


def test_plain_backward_against_differences():
    from paper_2104_11805_amd import workloads as wl
    rng = np.random.default_rng(2)
    for activation, cap in (("sigmoid", 1.0), ("relu", 0.7)):
        layers = [wl.random_layer(40 + k, o, i, 0.6) for k, (o, i) in enumerate([(5, 4), (6, 5)])]
        x, c = rng.normal(size=(4, 3)), rng.normal(size=(6, 3))
        loss = lambda x: (c * blocks.forward(layers, x, cap, activation)[-1]).sum()
        _, (dx0, _) = blocks.backward(layers, blocks.forward(layers, x, cap, activation), c, cap, activation)
        for i in np.ndindex(x.shape):
            up, down = x.copy(), x.copy()
            up[i] += 1e-6
            down[i] -= 1e-6
            diff = (loss(up) - loss(down)) / 2e-6
            assert abs(diff - dx0[i]) < 1e-6, (activation, i)


@pytest.mark.parametrize("cap", [0.0, 32.0, float("inf")])
def test_plain_packing_moves_values_by_half_a_scale(cap):
    rng = np.random.default_rng(3)
    x = (rng.normal(size=(37, 61)) * np.exp(rng.normal(size=(37, 1)))).astype(np.float32)
    x[5, 7:20] = [0, -0.0, 1e-38, 1e-44, 2.0 ** -149, 3e38, -3e38, 32, 31.99, 33, 1e-3, 5, 6]
    codes, scales, value = blocks.pack8(x, cap)
    t = np.repeat((scales.astype(np.uint32) << 16).view(np.float32).astype(np.float64), 128)[:x.size].reshape(x.shape)
    v = np.clip(x.astype(np.float64), 0, cap) if cap > 0 else x.astype(np.float64)
    low = (v > 0) & (v < t / 2) if cap > 0 else np.zeros(x.shape, bool)
    assert np.all(np.abs(value - v) <= np.where(low, t, t / 2))
    if cap > 0:
        assert np.array_equal(value > 0, v > 0) and np.array_equal(value >= cap, v >= cap)
    big = np.repeat(np.pad(np.where((v < cap) | (cap == 0), np.abs(v), 0).ravel(), (0, -x.size % 128)).reshape(-1, 128).max(1), 128)[:x.size].reshape(x.shape)
    most = 253 if cap > 0 else 127
    assert np.all(t * most >= big) and np.all((t <= big / most * (1 + 2.0 ** -7)) | (t == 2.0 ** -133))
