"""The largest sizes that the expert router and the MXFP4 operators take, and the texts of errors, checked on the CPU: every call below is refused."""
import ctypes as C

import pytest
import torch

import paper_2601_23278_amd as pk
from test_mx_refusals import P, lib, refused, router
from paper_2601_23278_amd import binding


@pytest.mark.parametrize("rows", [2 ** 26 - 1, 2 ** 26 - 2, 2 ** 26 - 3])
def test_route_refuses_rows_that_make_a_launch_too_large(rows):
    """Four rows a workgroup of 256 threads: 2^24 workgroups are 2^32 threads, one more than a launch may have."""
    refused(lib.focus_route(C.byref(router()), None, rows, 0, P, 16, None, P, P), "n_rows")


@pytest.mark.parametrize("rows,cols", [(2 ** 30 - 1, 1), (2 ** 30 - 63, 32), (17, 32 * 63161283), ((2 ** 30 - 1) // 3, 65)])
def test_conversions_refuse_blocks_that_make_a_launch_too_large(rows, cols):
    """Four threads a block: the last 63 counts of blocks below 2^30 make 2^24 workgroups of 256."""
    mx = binding.focus_mx(P, P)
    for dtype in (0, 1):
        refused(lib.focus_mx_quantize(None, dtype, rows, cols, P, cols, P, P), "large")
        refused(lib.focus_mx_dequantize(None, dtype, rows, cols, C.byref(mx), P, cols), "large")


@pytest.mark.parametrize("at,scales", [(binding.FOCUS_BF16, None), (binding.FOCUS_MX4, P)])
@pytest.mark.parametrize("tiles", [2 ** 24 - 1, 2 ** 24 - 7])
def test_gemm_refuses_tiles_that_make_a_launch_too_large(at, scales, tiles):
    """A launch of tiles is rounded up to the eight XCDs."""
    mx, n = binding.focus_mx(P, P), C.c_size_t()
    for m, cols in ((128 * tiles - 5, 100), (77, 128 * tiles - 100)):
        refused(lib.focus_mx_gemm(None, m, cols, 32, at, P, scales, 32, C.byref(mx), 0, P, cols, None, 0), "large")
        refused(lib.focus_mx_gemm_bytes(m, cols, 32, at, C.byref(n)), "large")
    assert lib.focus_mx_gemm_bytes(128 * (2 ** 24 - 8), 100, 32, at, C.byref(n)) == 0


def test_python_refuses_sizes_that_do_not_fit_32_bits():
    """The C entries take 32-bit sizes: a longer one must not arrive as its lower half."""
    for call in (lambda: pk.focus_mx_gemm_bytes(2 ** 32 + 5, 8, 64, 1), lambda: pk.focus_mx_gemm_bytes(5, 2 ** 32 + 8, 64, 1), lambda: pk.focus_mx_gemm_bytes(5, 8, 2 ** 32 + 64, 2),
                 lambda: pk.focus_mx_gemm_bytes(-2 ** 32 + 5, 8, 64, 1), lambda: pk.focus_mx_experts_bytes(8, 64, 32, 2 ** 32 + 4, 2),
                 lambda: pk.focus_mx_experts_bytes(2 ** 32 + 8, 64, 32, 4, 2), lambda: pk.focus_mx_experts_bytes(8, 64, 32, 4, 2 ** 32 + 2)):
        with pytest.raises(pk.FocusError):
            call()
    for shape in ((2 ** 32 + 5, 1), (2 ** 31, 32), (3, 2 ** 32 + 32)):
        with pytest.raises(pk.FocusError):
            binding._rows_of(torch.empty(shape, dtype=torch.bfloat16, device="meta"), "x")
    assert binding._rows_of(torch.empty(2 ** 31 - 1, 32, dtype=torch.bfloat16, device="meta"), "x")[0] == 2 ** 31 - 1
    long = torch.empty((1, 2 ** 31), dtype=torch.uint8, device="meta"), torch.empty((1, 2 ** 27), dtype=torch.uint8, device="meta")
    with pytest.raises(pk.FocusError):
        binding._mx_of(long, "w", 1)


def test_errors_of_other_threads():
    """A thread that had no failed call reads the last one of any thread, as a program does that opens contexts on one thread and reports from another; a thread
    that had one reads its own."""
    import threading

    def on_a_thread(f):
        got = []
        t = threading.Thread(target=lambda: got.append(f()))
        t.start()
        t.join()
        return got[0]

    def fail_then_wait():
        rc = lib.focus_workspace_bytes(None, None)
        on_a_thread(lambda: lib.focus_route(None, None, 1, 0, P, 16, None, P, P))
        return rc, lib.focus_last_error(None).decode()
    rc, own = on_a_thread(fail_then_wait)
    assert rc == binding.FOCUS_EINVAL and own == "null argument"
    assert on_a_thread(lambda: lib.focus_last_error(None).decode()) == "null router"
