"""CPU-only checks of what sizes the layer operators take: what no launch or no address of a kernel reaches is refused before any GPU work."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2403_12983_amd as pkg
    if not os.path.exists(pkg.lib_path()):
        from paper_2403_12983_amd import build
        build.build()
    return pkg.load_library()


P = C.c_void_p(1 << 20)      # an address that no refused call may touch


def _desc(n, d, f, dtype, rows_out):
    from paper_2403_12983_amd.binding import _GatedDesc
    return _GatedDesc(n, d, f, d, d if rows_out else f, f, dtype, 0, rows_out, 0)


def _refused(lib, q, backward):
    """of the workspace query and of the call"""
    size = 1 << 50
    if backward:
        kept = (P, P) if backward == 1 else (None, None)
        return (lib.osscar_gated_workspace_bytes(C.byref(q), backward) == 0 and
                lib.osscar_gated_backward(C.byref(q), P, P, P, P, *kept, P, q.d, P, P, max(q.d, q.f), q.dtype, P, size, None) == 1)
    return lib.osscar_gated_workspace_bytes(C.byref(q), 0) == 0 and lib.osscar_gated_forward(C.byref(q), P, P, P, P, None, None, P, size, None) == 1


def test_products_of_more_threads_than_a_launch_takes_are_refused(lib):
    # few rows: a workgroup of 512 threads per 16 columns (f x d, or 8-bit channels), one of 256 per 64 (float32, d x f)
    for n in (1, 16):
        assert _refused(lib, _desc(n, 9, 1 << 27, 1, 1), 0)
        assert lib.osscar_gated_workspace_bytes(C.byref(_desc(n, 9, (1 << 27) - 16, 1, 1)), 0) > 0
        assert _refused(lib, _desc(n, 9, 1 << 30, 0, 0), 0)
        assert lib.osscar_gated_workspace_bytes(C.byref(_desc(n, 9, (1 << 30) - 64, 0, 0)), 0) > 0
    for n, m in ((1, 1 << 27), (2, 1 << 28)):      # (two rows and more: 32 channels)
        assert lib.osscar_int_workspace_bytes(n, 16, m) == 0 and lib.osscar_int_workspace_bytes(n, 16, m - 32) > 0
        assert lib.osscar_int_product(P, n, 16, 16, 1, None, P, 16, P, m, None, P, m, 1, P, 1 << 50, None) == 1
        assert b"too large" in lib.osscar_last_error(None)
    # no rows: nothing to do, whatever the rest
    assert lib.osscar_gated_forward(C.byref(_desc(0, 9, 1 << 27, 1, 1)), P, P, P, P, None, None, P, 1 << 50, None) == 0
    assert lib.osscar_int_product(P, 0, 16, 16, 1, None, P, 16, P, 1 << 27, None, P, 1 << 27, 1, P, 1 << 50, None) == 0


def test_rows_that_the_bf16_tiles_cannot_address_are_refused(lib):
    long, longest = 4194296, 16777208      # a tile's 256 rows of `long`, a stage's 64 of `longest`, just below 2^31 bytes
    query = lambda *a, backward=0: lib.osscar_gated_workspace_bytes(C.byref(_desc(*a)), backward)  # noqa: E731
    for rows_out in (0, 1):
        for n in (17, 300):
            assert query(n, long, 8, 1, rows_out) > 0 and _refused(lib, _desc(n, long + 1, 8, 1, rows_out), 0) and _refused(lib, _desc(n, 1 << 25, 8, 1, rows_out), 0)
            assert _refused(lib, _desc(n, long + 1, 8, 1, rows_out), 2) and query(n, long + 1, 8, 1, rows_out, backward=1) > 0 and _refused(lib, _desc(n, longest + 1, 8, 1, rows_out), 1)
            for backward in (1, 2):
                assert query(n, 8, long, 1, rows_out, backward=backward) > 0 and _refused(lib, _desc(n, 8, long + 1, 1, rows_out), backward)
            # float32 has pointers of its own
            assert query(n, 1 << 25, 8, 0, rows_out) > 0 and query(n, 8, 1 << 25, 0, rows_out, backward=2) > 0
        assert _refused(lib, _desc(17, 8, longest + 1, 1, 0), 0) and query(17, 8, longest, 1, 0) > 0 and query(17, 8, 1 << 25, 1, 1) > 0
    assert query(16, 1 << 25, 9, 1, 1) > 0 and query(16, 1 << 25, 9, 1, 0) == 0      # few rows of f x d weights do not go through tiles
    assert query(0, 1 << 25, 8, 1, 0) > 0


def test_calls_without_rows_do_not_touch_the_gpu(lib):
    assert lib.osscar_logprobs(None, 0, 100, 100, 1, None, 1.0, 0, None, None, None, None, None, None, 0, None) == 0
    assert lib.osscar_logprobs_backward(None, 0, 100, 100, 1, None, 1.0, None, None, None, None, 0, None, None, None, 100, None) == 0
    assert lib.osscar_int_rows(None, 0, 16, 16, 1, None, 16, None, None) == 0
    assert lib.osscar_gated_forward(C.byref(_desc(0, 16, 16, 1, 0)), None, P, P, None, None, None, None, 0, None) == 0


def test_scales_whose_product_with_log2_e_is_no_float_are_refused(lib):
    for scale, refused in ((2.4e38, True), (3.4e38, True), (2.3e38, False), (1e-45, False)):
        # (without rows nothing is done with a scale that is taken)
        assert lib.osscar_logprobs(P, 0, 100, 100, 1, P, scale, 0, P, P, P, None, None, None, 0, None) == int(refused)
        assert lib.osscar_logprobs_backward(P, 0, 100, 100, 1, P, scale, P, P, None, None, 0, None, None, P, 100, None) == int(refused)
