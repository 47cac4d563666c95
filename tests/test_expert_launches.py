"""What the experts' entry points ask of HIP, recorded on the host in place of a GPU."""
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

# Run in a process of its own: the stand-ins are found before the HIP library's functions.
RUN = r"""
import ctypes, json, sys

class Record(ctypes.Structure):
    _fields_ = [("func", ctypes.c_void_p), ("limit", ctypes.c_int64), ("shared", ctypes.c_int64),
                ("blocks", ctypes.c_int64), ("threads", ctypes.c_int64)]

hip = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
i64, i32, vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
FAKE = 0x10000
for name, types, args in json.loads(sys.argv[3]):
    f = getattr(lib, name)
    f.argtypes, f.restype = [{"l": i64, "i": i32, "p": vp}[t] for t in types], i32
    print(f(*[FAKE if a == "p" else a for a in args]), file=sys.stderr)
records = (Record * 4096).in_dll(hip, "records")
print(json.dumps([[r.func, r.limit, r.shared, r.blocks, r.threads]
                  for r in records[:ctypes.c_int.in_dll(hip, "n_records").value]]))
"""


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    import paper_2609_32398_amd as p

    if not os.path.exists(p.LIB_PATH):
        p.build()
    so = str(tmp_path_factory.mktemp("hip") / "libhip_recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", os.path.join(HERE, "hip_recorder.c"), "-o", so], check=True)

    def run(calls, expect=None):
        r = subprocess.run([sys.executable, "-c", RUN, so, p.LIB_PATH, json.dumps(calls)], capture_output=True,
                           text=True, timeout=100)
        assert r.returncode == 0, r.stderr[-2000:]
        statuses = [int(s) for s in r.stderr.split()]
        assert len(statuses) == len(calls), r.stderr[-2000:]
        assert statuses == ([0] * len(calls) if expect is None else expect)
        return json.loads(r.stdout)

    return run


def _rows(N, E, k):
    return ["do_expert_rows", "pliippppplp", ["p", N, E, k, "p", "p", "p", "p", "p", 1 << 40, None]]


def test_rows_of_many_and_of_few_experts_share_one_limit(record):
    # Another thread may launch between a call's limit and its launch: a call must not lower it.
    got = record([_rows(600, 1024, 8), _rows(600, 8, 2), _rows(100, 512, 2), _rows(5000, 1024, 1)])
    limits, launches = {}, 0
    for func, limit, shared, blocks, threads in got:
        if limit >= 0:
            assert limit >= limits.get(func, 0), "a call lowers the limit that another one's launch needs"
            limits[func] = limit
        else:
            assert shared <= limits[func]
            launches += 1
    assert launches == 2 + 2 + 1 + 2  # counts and rows; one unit: the rows alone


def test_rows_whose_sums_pass_int32_are_refused(record):
    # the kernels add up to a tile of rows and a list of tokens to a row's number in int32
    most, E = (1 << 31) - 1024, 8

    def calls(R):
        return [["do_expert_matmul", "ppipplliiiipp", ["p", "p", 1, "p", "p", 50, R, E, 1, 1, 0, "p", None]],
                ["do_expert_weight_grad", "ppippplliiiipp", ["p", "p", 1, "p", None, None, 50, R, E, 1, 1, 0, "p", None]],
                ["do_expert_swiglu", "ppipipplliiipppp", ["p", "p", 1, "p", 0, "p", "p", 50, R, E, 1, 1, "p", "p", "p", None]],
                ["do_expert_swiglu_grad", "ppipippppliiiipppppplp",
                 ["p", "p", 1, "p", 0, "p", "p", "p", "p", R // 2, E, 2, 1, 1, "p", "p", "p", "p", "p", "p", 1 << 40, None]]]

    record(calls(most))
    assert record(calls(most + 2), expect=[4, 4, 4, 4]) == []  # refused, and nothing launched


def test_an_act8_of_no_tensors_is_refused():
    import torch

    import paper_2609_32398_amd as dl

    for a in (dl.Act8(None, None), dl.Act8(3, 4), dl.Act8([1], [2])):
        with pytest.raises(ValueError):
            dl.do_act8_unpack(a, torch.float32)


def _matmul(N, R, E, O, I, dtype, transposed=0):
    return ["do_expert_matmul", "ppipplliiiipp", ["p", "p", dtype, "p", "p", N, R, E, O, I, transposed, "p", None]]


def _swiglu(N, R, E, H, F, dtype):
    return ["do_expert_swiglu", "ppipipplliiipppp", ["p", "p", dtype, "p", 0, "p", "p", N, R, E, H, F, "p", "p", "p", None]]


def _wgrad(N, R, E, O, I, dtype, dy_token=None, x_token=None):
    return ["do_expert_weight_grad", "ppippplliiiipp", ["p", "p", dtype, "p", dy_token, x_token, N, R, E, O, I, 0, "p", None]]


def _threads(record, call):
    launches = [r for r in record([call]) if r[1] < 0]
    assert len(launches) == 1
    return launches[0][4], launches[0][3], launches[0][2]


@pytest.mark.parametrize("dtype", [0, 1])
def test_the_gpu_tests_shapes_reach_their_tiles(record, dtype):
    import test_gpu_expert_tiles as t

    for N, E, k, O, I in t.FEW:
        assert _threads(record, _matmul(N, N * k, E, O, I, dtype))[0] == 128
        assert _threads(record, _matmul(N, N * k, E, I, O, dtype, 1))[0] == (128 if O * (4 >> dtype) % 16 == 0 and I * (4 >> dtype) % 16 == 0 else 256)
    for N, E, k, H, F in t.FEW_GATED:
        assert _threads(record, _swiglu(N, N * k, E, H, F, dtype))[0] == 128
    # the kernel of few rows: four waves and no dynamic shared memory
    for N, E, k, O, I in t.SKINNY:
        assert _threads(record, _matmul(N, N * k, E, O, I, dtype))[::2] == (256, 0)
    for N, E, k, H, F in t.SKINNY_GATED:
        assert _threads(record, _swiglu(N, N * k, E, H, F, dtype))[::2] == (256, 0)
    for E, O, I in t.LARGE:
        for dy, x in ((None, None), ("p", None), (None, "p"), ("p", "p")):
            assert _threads(record, _wgrad(2600, 5200, E, O, I, dtype, dy, x))[0] == 512
