"""Refusals of the experts' entry points: on the host, before any GPU work."""
import pytest
import torch

FAKE = 0x10000  # a non-null, well-aligned address: validation fails before it is ever dereferenced


@pytest.fixture(scope="module")
def dl():
    import os

    import paper_2609_32398_amd as p

    if not os.path.exists(p.LIB_PATH):
        p.build()
    return p


def _rejects(dl, name, good, changes):
    f = getattr(dl.lib(), name)
    for at, value, status in changes:
        args = list(good)
        for i, v in zip(at, value) if isinstance(at, tuple) else [(at, value)]:
            args[i] = v
        assert f(*args) == status, (name, at, value)
        assert dl.lib().do_last_error()


def test_rows(dl):
    good = [FAKE, 1000, 8, 2, FAKE, FAKE, FAKE, FAKE, FAKE, 64, None]
    _rejects(dl, "do_expert_rows", good, [
        (0, None, 1), (0, FAKE + 4, 1), (1, 0, 1), (1, -1, 1), (1, 1 << 30, 4), (2, 0, 1), (2, 1025, 1), (3, 0, 1),
        (3, 9, 1), (4, None, 1), (5, FAKE + 2, 1), (6, None, 1), (7, None, 1), (8, None, 1), (9, 63, 1)])
    L = dl.lib()
    assert L.do_expert_rows_workspace(512, 8) == 0
    assert L.do_expert_rows_workspace(1000, 8) == 2 * 8 * 4
    assert L.do_expert_rows_workspace(1 << 30, 1024) == 512 * 1024 * 4
    assert L.do_expert_rows_workspace(0, 8) == 0 and L.do_expert_rows_workspace(5000, 1025) == 0


def test_combine(dl):
    good = [FAKE, 1, FAKE, 100, 2, 64, FAKE, None]
    _rejects(dl, "do_expert_combine", good, [
        (0, None, 1), (0, FAKE + 1, 1), (1, 3, 2), (2, None, 1), (3, 0, 1), (3, 1 << 30, 4), (4, 0, 1), (5, 0, 1),
        (5, 65537, 1), (6, None, 1)])


def test_matmul(dl):
    good = [FAKE, FAKE, 1, FAKE, None, 50, 100, 8, 64, 32, 0, FAKE, None]
    _rejects(dl, "do_expert_matmul", good, [
        (0, None, 1), (1, FAKE + 1, 1), (2, 2, 2), (3, None, 1), (4, FAKE + 1, 1), (5, 0, 1), (6, 0, 1),
        (6, 1 << 31, 4), (7, 0, 1), (7, 1025, 1), (8, 0, 1), (9, 1 << 17, 1), (11, None, 1),
        ((6, 8), ((1 << 31) - 1, 65536), 4)])


def test_weight_grad(dl):
    good = [FAKE, FAKE, 1, FAKE, None, None, 50, 100, 8, 64, 32, 0, FAKE, None]
    _rejects(dl, "do_expert_weight_grad", good, [
        (0, None, 1), (1, None, 1), (2, 5, 2), (3, FAKE + 2, 1), (4, FAKE + 2, 1), (5, FAKE + 1, 1), (6, 0, 1),
        (7, -3, 1), (8, 0, 1), (9, 0, 1), (10, 65537, 1), (12, None, 1), (12, FAKE + 2, 1)])


def test_swiglu(dl):
    good = [FAKE, FAKE, 1, FAKE, 0, FAKE, FAKE, 50, 100, 8, 64, 32, FAKE, FAKE, FAKE, None]
    _rejects(dl, "do_expert_swiglu", good, [
        (0, None, 1), (1, None, 1), (2, 7, 2), (3, FAKE + 2, 1), (4, 9, 2), (5, None, 1), (6, None, 1), (7, 0, 1),
        (8, 0, 1), (9, 0, 1), (10, 0, 1), (11, 0, 1), (12, None, 1), (13, None, 1), (14, None, 1)])


def test_swiglu_grad(dl):
    need = dl.lib().do_expert_swiglu_grad_workspace(100, 65)
    assert need == 100 * 2 * 4
    good = [FAKE, FAKE, 1, FAKE, 0, FAKE, FAKE, FAKE, FAKE, 50, 8, 2, 64, 65, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
            need, None]
    _rejects(dl, "do_expert_swiglu_grad", good, [
        (0, None, 1), (1, FAKE + 1, 1), (2, 7, 2), (3, None, 1), (4, 9, 2), (5, None, 1), (6, None, 1), (7, None, 1),
        (8, None, 1), (9, 0, 1), (9, 1 << 31, 4), (10, 0, 1), (11, 9, 1), (12, 0, 1), (13, 0, 1), (14, None, 1),
        (15, None, 1), (16, None, 1), (17, None, 1), (18, FAKE + 2, 1), (19, None, 1), (20, need - 1, 1)])


def test_act8(dl):
    _rejects(dl, "do_act8_pack", [FAKE, 0, 10, 64, FAKE, FAKE, None], [
        (0, None, 1), (0, FAKE + 2, 1), (1, 4, 2), (2, 0, 1), (2, 1 << 31, 4), (3, 0, 1), (3, 65537, 1), (4, None, 1),
        (5, None, 1)])
    _rejects(dl, "do_act8_unpack", [FAKE, FAKE, 10, 64, FAKE, 1, None], [
        (0, None, 1), (1, None, 1), (2, 0, 1), (3, 0, 1), (4, None, 1), (4, FAKE + 1, 1), (5, 9, 2)])


def _rows(dl, N=4, E=3, k=2):
    return dl.ExpertRows(torch.zeros(E + 1, dtype=torch.int32), torch.zeros(N * k, dtype=torch.int32),
                         torch.zeros((N, k), dtype=torch.int32), torch.zeros((N, k), dtype=torch.int32))


def test_binding_takes_device_tensors_of_matching_shapes(dl):
    rows = _rows(dl)
    w, x = torch.zeros(3, 8, 16), torch.zeros(8, 16)
    calls = [
        lambda: dl.do_expert_rows(torch.zeros(2, 3, 8, dtype=torch.int64), 4, 2),       # units of another N
        lambda: dl.do_expert_rows(torch.zeros(2, 1, 3, 8, dtype=torch.int64), 4, 2),    # two layers
        lambda: dl.do_expert_rows(torch.zeros(1, 3, 8, dtype=torch.int64), 4, 2),       # host memory
        lambda: dl.do_expert_combine(torch.zeros(8, 16), tuple(rows)),                  # not an ExpertRows
        lambda: dl.do_expert_combine(torch.zeros(8, 16), rows),                         # host memory
        lambda: dl.do_expert_matmul(x, w, rows),
        lambda: dl.do_expert_weight_grad(torch.zeros(8, 8), x, rows),
        lambda: dl.do_expert_swiglu(torch.zeros(4, 16), w, rows),
        lambda: dl.do_expert_swiglu_grad(torch.zeros(4, 8), w, rows, dl.Act8(None, None)),
        lambda: dl.do_act8_pack(x),
        lambda: dl.do_act8_pack(torch.zeros(0, 16)),
        lambda: dl.do_act8_unpack(dl.Act8(torch.zeros(2, 8, dtype=torch.int8), torch.zeros(2, 1, dtype=torch.uint8)),
                                  torch.float32),
        lambda: dl.do_act8_unpack(dl.Act8(torch.zeros(2, 8, dtype=torch.int8), torch.zeros(2, 1, dtype=torch.uint8)),
                                  torch.float16),
        lambda: dl.do_act8_unpack((x, x), torch.float32),
    ]
    for c in calls:
        with pytest.raises(ValueError):
            c()
