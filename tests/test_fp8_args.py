"""Refusals of the 8-bit floating point entry points: on the host, before any GPU work."""
import os

import pytest
import torch

from test_expert_args import FAKE, _rejects

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def dl():
    import paper_2609_32398_amd as p

    if not os.path.exists(p.LIB_PATH):
        p.build()
    return p


def test_pack_and_unpack(dl):
    _rejects(dl, "do_fp8_pack", [FAKE, 0, 10, 64, FAKE, FAKE, None], [
        (0, None, 1), (0, FAKE + 2, 1), (1, 2, 2), (2, 0, 1), (2, 1 << 31, 4), (3, 0, 1), (3, 65537, 1), (4, None, 1),
        (5, None, 1)])
    _rejects(dl, "do_fp8_unpack", [FAKE, FAKE, 10, 64, FAKE, 1, None], [
        (0, None, 1), (1, None, 1), (2, -1, 1), (2, 1 << 31, 4), (3, 0, 1), (4, None, 1), (4, FAKE + 1, 1), (5, 7, 2)])
    changes = [(2, 0, 1), (2, 1 << 31, 4), (3, 0, 1), (3, 131073, 1), (4, 0, 1), (4, 65537, 1),
               ((2, 3, 4), (1 << 30, 129, 128), 4)]
    _rejects(dl, "do_fp8_pack_weights", [FAKE, 1, 2, 64, 64, FAKE, FAKE, None],
             changes + [(0, None, 1), (0, FAKE + 1, 1), (1, 9, 2), (5, None, 1), (6, None, 1)])
    _rejects(dl, "do_fp8_unpack_weights", [FAKE, FAKE, 2, 64, 64, FAKE, 0, None],
             changes + [(0, None, 1), (1, None, 1), (5, None, 1), (5, FAKE + 2, 1), (6, 9, 2)])


def test_products(dl):
    _rejects(dl, "do_expert_matmul_fp8", [FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 10, 20, 4, 64, 64, 0, FAKE, None], [
        (0, None, 1), (1, None, 1), (2, None, 1), (3, None, 1), (4, None, 1), (4, FAKE + 2, 1), (5, FAKE + 1, 1),
        (6, 0, 1), (6, 1 << 31, 4), (7, 0, 1), (7, (1 << 31) - 1000, 4), (8, 0, 1), (8, 1025, 1), (9, 0, 1),
        (9, 65537, 1), (10, 0, 1), (10, 65537, 1), (12, None, 1), (12, FAKE + 1, 1),
        ((4, 7, 8, 9), (None, (1 << 31) - 1025, 1, 65536), 4)])
    _rejects(dl, "do_expert_swiglu_fp8",
             [FAKE, FAKE, FAKE, FAKE, FAKE, 1, FAKE, FAKE, 10, 20, 4, 64, 64, FAKE, FAKE, FAKE, FAKE, None], [
                 (0, None, 1), (1, None, 1), (2, None, 1), (3, None, 1), (4, FAKE + 1, 1), (5, 3, 2), (6, None, 1),
                 (7, None, 1), (8, 0, 1), (9, 0, 1), (10, 0, 1), (11, 0, 1), (12, 65537, 1), (13, None, 1),
                 (14, None, 1), (15, None, 1), (16, None, 1)])
    good = [FAKE, FAKE, FAKE, FAKE, FAKE, 1, FAKE, FAKE, FAKE, FAKE, 10, 4, 2, 64, 64, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
            20 * 4, None]
    _rejects(dl, "do_expert_swiglu_grad_fp8", good, [
        (0, None, 1), (1, None, 1), (2, None, 1), (3, None, 1), (4, None, 1), (4, FAKE + 1, 1), (5, 3, 2), (6, None, 1),
        (7, None, 1), (8, None, 1), (9, None, 1), (10, 0, 1), (11, 0, 1), (12, 5, 1), (13, 0, 1), (14, 0, 1),
        (15, None, 1), (16, None, 1), (17, None, 1), (17, FAKE + 1, 1), (18, None, 1), (19, FAKE + 1, 1), (20, None, 1),
        (21, 79, 1)])


def test_layer(dl):
    L = dl.lib()
    need = L.do_expert_layer_workspace(1, 10, 8, 2, 64, 60)
    assert need == 16 + 8 * 16 + 16 + 4 * 16 * 10 * 16 * 4 + 20 * 64 * 2
    assert L.do_expert_layer_workspace(0, 1, 8, 2, 65, 61) == 16 + 2 * 16 + 32 + 5 * 16 * 16 * 4 + 2 * 64 * 4
    good = (1, 10, 8, 2, 64, 60)
    for i, v in ((0, 2), (1, 0), (1, 65), (2, 0), (2, 1025), (3, 0), (3, 9), (4, 0), (4, 65537), (5, 0), (5, 65537)):
        bad = list(good)
        bad[i] = v
        assert L.do_expert_layer_workspace(*bad) == 0
    _rejects(dl, "do_expert_layer",
             [FAKE, 1, FAKE, 0, FAKE, 0, FAKE, FAKE, FAKE, FAKE, 10, 8, 2, 64, 60, FAKE, FAKE, need, None], [
                 (0, None, 1), (0, FAKE + 1, 1), (1, 2, 2), (2, None, 1), (2, FAKE + 2, 1), (3, 2, 2), (4, FAKE + 2, 1),
                 (5, 2, 2), (6, None, 1), (7, None, 1), (8, None, 1), (9, None, 1), (10, 0, 1), (10, 65, 1), (11, 0, 1),
                 (11, 1025, 1), (12, 0, 1), (12, 9, 1), (13, 0, 1), (13, 65537, 1), (14, 0, 1), (14, 65537, 1),
                 (15, None, 1), (15, FAKE + 1, 1), (16, None, 1), (16, FAKE + 8, 1), (17, need - 1, 1),
                 ((6, 7, 9), (FAKE + 1, None, None), 1)])


def _fp8(dl, *shape, e=None, dtype=E4M3):
    return dl.Fp8(torch.zeros(shape, dtype=dtype), torch.zeros(e or (*shape[:-1], -(-shape[-1] // 128)), dtype=torch.uint8))


def _refused(f, *args, say=None, **kw):
    with pytest.raises(ValueError) as err:
        f(*args, **kw)
    assert say is None or say in str(err.value), err.value


def test_binding(dl):
    # shapes and types are looked at before the device, so that CPU tensors show them
    rows = dl.ExpertRows(torch.zeros(5, dtype=torch.int32), torch.zeros(20, dtype=torch.int32),
                         torch.zeros(10, 2, dtype=torch.int32), torch.zeros(10, 2, dtype=torch.int32))
    _refused(dl.do_fp8_pack, torch.zeros(0, 4), say="at least one")
    _refused(dl.do_fp8_pack, torch.zeros(4), weights=True, say="[..., O, I]")
    _refused(dl.do_fp8_pack, torch.zeros(4, dtype=torch.float16), say="dtype")
    _refused(dl.do_fp8_pack, torch.zeros(4, 6)[:, ::2], say="contiguous")
    _refused(dl.do_fp8_pack, torch.zeros(4, 6), say="device tensor")
    _refused(dl.do_fp8_unpack, (1, 2), torch.float32, say="Fp8")
    _refused(dl.do_fp8_unpack, _fp8(dl, 4, 200), torch.float16, say="dtype")
    _refused(dl.do_fp8_unpack, _fp8(dl, 4, 200, e=(4, 1)), torch.float32, say="device")  # q's device comes first
    _refused(dl.do_fp8_unpack, dl.Fp8(None, None), torch.float32, say="Fp8")
    _refused(dl.do_expert_matmul_fp8, _fp8(dl, 10, 64), _fp8(dl, 1, 32, 64, e=(1, 1, 1)), None, gather=True, say="gather")
    _refused(dl.do_expert_matmul_fp8, _fp8(dl, 10, 64), _fp8(dl, 2, 32, 64, e=(2, 1, 1)), None, say="[1, O, I]")
    _refused(dl.do_expert_matmul_fp8, torch.zeros(10, 64), _fp8(dl, 1, 32, 64, e=(1, 1, 1)), None)
    _refused(dl.do_expert_matmul_fp8, _fp8(dl, 20, 64), _fp8(dl, 4, 32, 64, e=(4, 1, 1)), "rows", say="ExpertRows")
    w1, w2 = torch.zeros(4, 16, 64), torch.zeros(4, 64, 8)
    _refused(dl.do_expert_layer, torch.zeros(65, 64), torch.zeros(65, 4), 2, w1, w2, say="1 to 64 tokens")
    _refused(dl.do_expert_layer, torch.zeros(0, 64), torch.zeros(0, 4), 2, w1, w2, say="1 to 64 tokens")
    _refused(dl.do_expert_layer, torch.zeros(2, 64), torch.zeros(2, 4), 2, w1, w2, say="device tensor")
    _refused(dl.do_expert_swiglu_fp8, _fp8(dl, 10, 64), torch.zeros(4, 32, 64), rows)
    _refused(dl.do_expert_swiglu_grad_fp8, _fp8(dl, 10, 64), torch.zeros(4, 64, 32), rows, None)


@pytest.mark.gpu
def test_layer_binding_on_the_device(dl):
    # what is looked at behind the tokens' and the scores' device
    x, s = torch.zeros(2, 64, device="cuda"), torch.zeros(2, 4, device="cuda")
    w1, w2 = torch.zeros(4, 16, 64, device="cuda"), torch.zeros(4, 64, 8, device="cuda")
    q1, q2 = dl.do_fp8_pack(w1, True), dl.do_fp8_pack(w2, True)
    f = dl.do_expert_layer
    _refused(f, x, s, 0, w1, w2, say="k = 0")
    _refused(f, x, s, 5, w1, w2, say="k = 5")
    _refused(f, x, s[:1], 2, w1, w2, say="scores")
    _refused(f, x, s.double(), 2, w1, w2, say="dtype")
    _refused(f, x, s, 2, w1, q2, say="both")
    _refused(f, x, s, 2, w1[:, :15].contiguous(), w2, say="w1")
    _refused(f, x, s, 2, w1, w2.bfloat16(), say="dtype")
    _refused(f, x, s, 2, w1, w2.transpose(1, 2), say="w2")
    _refused(f, x, s, 2, q1, dl.Fp8(q2.q, q2.e[:, :, :0].contiguous()), say="w2.e")
    _refused(f, x, s, 2, dl.Fp8(None, None), q2, say="w1")
    _refused(f, x, s, 2, dl.Fp8(q1.q.view(torch.uint8), q1.e), q2, say="w1.q")
    _refused(f, x, s, 2, w1, w2, torch.zeros(2, 5, device="cuda"), say="p has shape")
    _refused(f, x, s, 2, w1, w2, out=torch.zeros(2, 64, device="cuda", dtype=torch.bfloat16), say="out")
    _refused(dl.do_expert_matmul_fp8, dl.do_fp8_pack(x), q1, None, say="[1, O, I]")
    _refused(dl.do_expert_matmul_fp8, dl.do_fp8_pack(x), dl.Fp8(q1.q[:1], q1.e[:1]), None, transposed=True, say="x.q")
    _refused(dl.do_fp8_unpack, dl.Fp8(q1.q, q1.e[:, :, :0].contiguous()), torch.float32, say="e has shape")
    torch.cuda.synchronize()
