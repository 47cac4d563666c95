"""What the 8-bit products and the layer of a few tokens ask of HIP, recorded on the host in place of a GPU."""
import pytest

from test_expert_launches import record  # noqa: F401  (a fixture)


def _matmul(N, R, E, O, I, t=0, offsets="p"):
    return ["do_expert_matmul_fp8", "pppppplliiiipp",
            ["p", "p", "p", "p", offsets, "p", N, R, E, O, I, t, "p", None]]


def _swiglu(N, R, E, H, F):
    return ["do_expert_swiglu_fp8", "pppppipplliiippppp",
            ["p", "p", "p", "p", "p", 0, "p", "p", N, R, E, H, F, "p", "p", "p", "p", None]]


def _grad(N, E, k, H, F):
    return ["do_expert_swiglu_grad_fp8", "pppppippppliiiipppppplp",
            ["p", "p", "p", "p", "p", 0, "p", "p", "p", "p", N, E, k, H, F, "p", "p", "p", "p", "p", "p", 1 << 40, None]]


def _layer(N, E, k, H, F, dtype=1, w8=True):
    e = "p" if w8 else None
    return ["do_expert_layer", "pipipippppliiiipplp",
            ["p", dtype, "p", 0, "p", 0, "p", e, "p", e, N, E, k, H, F, "p", "p", 1 << 40, None]]


def _launched(record, call):  # noqa: F811
    """(threads, whether most of a CU's shared memory) of each launch."""
    return [(r[4], r[2] > 100 << 10) for r in record([call]) if r[1] < 0]


def test_the_gpu_tests_shapes_reach_their_tiles(record):  # noqa: F811
    import test_gpu_expert_fp8 as t

    whole = lambda *w: all(v % 16 == 0 for v in w)  # noqa: E731
    seen = {(*_launched(record, _matmul(N, N * k, E, O, I, tr))[0], whole(O, I), tr)
            for N, E, k, O, I in t.SHAPES for tr in (0, 1)}
    for tr in (0, 1):
        for pieces in (True, False):  # 128 x 64 and 256 x 256
            assert {(256, False, pieces, tr), (512, True, pieces, tr)} <= seen
        assert (128, False, True, tr) in seen  # 128 x 32
    seen = {(*_launched(record, _swiglu(N, N * k, E, H, F))[0], whole(H)) for N, E, k, H, F in t.GATED}
    # 256 x 32, through registers 256 x 64, and 256 x 256
    assert seen == {(256, False, True), (512, False, False), (512, True, True), (512, True, False)}
    seen = {tuple(n for n, _ in _launched(record, _grad(N, E, k, H, F))) for N, E, k, H, F in t.GATED}
    assert seen == {(256, 256)}  # 128 x 64 and 128 x 128; then the sums of p's gradient


def test_shared_memory_stays_within_its_limit(record):  # noqa: F811
    calls = []
    for E in (1, 1024):
        for N in (1, 3000, 400000):
            calls += [_matmul(N, N * 4, E, 256, 256, t) for t in (0, 1)] + [_swiglu(N, N * 4, E, 256, 256)]
            calls += [_matmul(N, N * 4, E, 255, 255, t) for t in (0, 1)] + [_swiglu(N, N * 4, E, 255, 255)]
            calls += [_grad(N, E, 1, 256, 256), _grad(N, E, 1, 255, 255)]
    limits = {}
    for func, limit, shared, blocks, threads in record(calls):
        if limit >= 0:
            assert limit <= 160 << 10
            limits[func] = max(limit, limits.get(func, 0))
        else:
            assert shared <= limits.get(func, 64 << 10)  # what a kernel has without asking
            assert blocks * threads < 1 << 32


@pytest.mark.parametrize("N,E,k,H,F", [(1, 128, 8, 2048, 768), (64, 1024, 1024, 65536, 65536), (64, 1, 1, 1, 1)])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("w8", [False, True])
def test_a_layer_is_two_kernels(record, N, E, k, H, F, dtype, w8):  # noqa: F811
    launches = [r for r in record([_layer(N, E, k, H, F, dtype, w8)]) if r[1] < 0]
    assert len(launches) == 2
    for _, _, shared, blocks, threads in launches:
        assert threads == 256 and 1 <= blocks and blocks * threads < 1 << 32 and shared <= 24 << 10


def test_one_matrix_needs_no_offsets(record):  # noqa: F811
    assert len(_launched(record, _matmul(100, 100, 1, 64, 64, 0, None))) == 1
    record([_matmul(100, 100, 2, 64, 64, 0, None)], expect=[1])


def test_rows_whose_sums_pass_int32_are_refused(record):  # noqa: F811
    most = (1 << 31) - 1024
    record([_matmul(50, most, 8, 1, 1), _swiglu(50, most, 8, 1, 1), _grad(most // 2, 8, 2, 1, 1)])
    assert record([_matmul(50, most + 2, 8, 1, 1), _swiglu(50, most + 2, 8, 1, 1), _grad(most // 2 + 1, 8, 2, 1, 1)],
                  expect=[4, 4, 4]) == []
