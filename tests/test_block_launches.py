"""What the layer norm launches at the ends of the sizes that it takes, without a GPU (see tests/routes.py)."""
from tests import routes
from tests.test_block_refusals import PTR

WIDE = """
        M = 1 << 30
        sizes = [(n, b) for b in ((1 << 26) + 1, (1 << 29) - 3, 1 << 29, (1 << 29) + 1, (1 << 29) + 2, 600000000, M - 128, M - 127, M - 1, M)
                 for n in (1, 2, 3, 700, 1023)] + [(M, 1), (M, 1023), (1 << 20, 1 << 19), (1000, 1 << 26), (2047, 1 << 29)]
        def launches(n, b):
            assert lib.sdnn_layernorm_workspace_bytes(n, b, C.byref(size)) == 0
            w = size.value
            assert lib.sdnn_pack8_bytes(n, b, C.byref(size)) == 0
            yield "forward", call("sdnn_layernorm", A[0], A[1], A[2], n, b, 1e-5, A[3], A[4], A[5], w, None)
            yield "back", call("sdnn_layernorm_backward", A[0], A[1], A[2], A[3], n, b, A[4], A[5], A[6], A[7], w, None)
            yield "back from 8 bits", call("sdnn_layernorm_backward_packed", A[0], A[1], size.value, 0.0, A[2], A[3], n, b, A[4], A[5], A[6], A[7], w, None)
"""


def test_every_size_that_is_taken_is_launched():
    """(A launch that the runtime refuses is in no log.)"""
    routes.run(PTR + WIDE + """
        for n, b in sizes:
            for what, (rc, log) in launches(n, b):
                assert rc == 0, (what, n, b, sdnn.last_error())
                names = [l.split("<")[0].split()[0] for l in log]
                if what == "forward":
                    assert names in (["k_norm_whole"], ["k_norm_sums", "k_norm_apply"]), (what, n, b, log)
                else:
                    assert [k for k in names if k != "k_norm_finish"] == ["k_norm_grad_sums", "k_norm_grad_apply"], (what, n, b, log)
    """)


def test_every_packed_block_that_is_taken_is_launched():
    routes.run(PTR + """
        M = 1 << 30
        for n, b in [(1, 1), (1, M), (M, 1), (M, 1023), (1023, M), ((1 << 31) - 1, 511), (1, (1 << 31) - 1), (1 << 20, (1 << 20) - 1)]:
            assert lib.sdnn_pack8_bytes(n, b, C.byref(size)) == 0, (n, b)
            for cap in (0.0, 2.0):
                rc, log = call("sdnn_pack8", A[0], n, b, cap, A[1], size.value, None)
                assert rc == 0 and len(log) == 1 and log[0].startswith("k_pack8<"), (n, b, rc, log)
                rc, log = call("sdnn_unpack8", A[1], size.value, n, b, cap, A[0], None)
                groups = sum(int(l.split()[-3]) for l in log)
                assert rc == 0 and all(l.startswith("k_unpack8<") for l in log) and groups == -(-n * b // 1024), (n, b, rc, log)
    """)


def test_the_stand_in_remembers_a_launch_that_it_refuses():
    """As the runtime does: hipGetLastError returns it, once."""
    routes.run("""
        class dim3(C.Structure):
            _fields_ = [("x", C.c_uint32), ("y", C.c_uint32), ("z", C.c_uint32)]
        stub.hipLaunchKernel.argtypes = [C.c_void_p, dim3, dim3, C.c_void_p, C.c_size_t, C.c_void_p]
        stub.stub_clear()
        launch = lambda x, threads: stub.hipLaunchKernel(None, dim3(x, 1, 1), dim3(threads, 1, 1), None, 0, None)
        assert launch(1 << 23, 512) != 0 and launch(5, 256) == 0
        assert stub.hipGetLastError() != 0 and stub.hipGetLastError() == 0
        assert stub.stub_log().decode().split() == ["5", "1", "1"]
    """)


def test_a_lane_finds_its_columns_by_32_bits():
    """A wavefront of a kernel with CL lanes across a tile has 64 / CL rows at a time; the bytes from its first row's start to a lane's four
    columns are a number of 32 bits, and the columns of all rows an int."""
    routes.run(PTR + WIDE + """
        import re
        for n, b in sizes:
            for what, (rc, log) in launches(n, b):
                for line in log:
                    if m := re.match(r"k_norm_(?:grad_)?(?:sums|apply)<(\\d+),", line):
                        columns = (64 // int(m[1]) - 1) * b + b - 4
                        assert columns < 1 << 31 and 4 * columns < 1 << 32, (what, n, b, line)
    """)


def test_which_blocks_are_read_past_the_caches():
    """The backward pass over 48 2^20 values and more with tiles of 256 columns; narrower tiles (also where a quarter of the lanes of wide ones would be idle) never."""
    routes.run(PTR + WIDE + """
        for n, b, past in [(16384, 4096, True), (2101, 24001, True), (960, 52430, True), (3 << 14, 1 << 10, True), ((3 << 14) - 1, 1 << 10, False), (8192, 2048, False),
                           (786433, 64, False), (50331648, 1, False), (393217, 128, False), (60000, 1030, True), (200000, 300, False)]:
            (_, (rc, log)), (_, (rc8, log8)) = list(launches(n, b))[1:]
            assert rc == rc8 == 0
            for line in log + log8:
                if "k_norm_grad" in line:
                    assert line.split(", ")[2].startswith("true") == past, (n, b, line)
    """)
