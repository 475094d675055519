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
