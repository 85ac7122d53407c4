"""Argument checks of the exchange of answers: every refusal comes from the host, before anything is launched, so the
buffers here are host memory that no kernel sees."""
import ctypes as C

import numpy as np
import pytest

from paper_2207_04604_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2207_04604_amd import build
        build.build_library()
    return B.lib()


ROWS, V, K = 3, 10, 4
_raw = np.zeros(4096, dtype=np.uint8)
BASE = _raw.ctypes.data + (-_raw.ctypes.data) % 16                  # 16-byte aligned
ZERO = dict(logits=BASE, index=BASE + 512, sum=BASE + 768, weight=BASE + 1024, loss=BASE + 1280, lse=BASE + 1536,
            grad=BASE + 1792, logprob=BASE + 2304, scratch=BASE + 2560)


def call(name, status, **change):
    a = dict(ZERO, dtype=B.F32, rows=ROWS, classes=V, row_stride=V, k=K, members=2, temperature=1.0, grad_stride=V,
             scratch_bytes=None)
    a.update(change)
    z = B.make_logits(a["logits"], a["dtype"], a["rows"], a["classes"], a["row_stride"])
    t = B.make_teacher(a["index"], a["sum"], a["k"], a["members"], a["temperature"], a["weight"])
    n = a["scratch_bytes"]
    if n is None:
        n = B.logits_scratch_bytes(z, a["k"])
    calls = {
        "top": lambda: B.top_logprobs(z, a["k"], a["index"], a["logprob"], a["scratch"], n),
        "at": lambda: B.logprobs_at(z, a["index"], a["k"], a["logprob"], a["scratch"], n),
        "distill": lambda: B.distill(z, t, a["loss"], a["lse"], a["grad"], a["grad_stride"], a["scratch"], n),
        "backward": lambda: B.distill_backward(z, t, a["lse"], a["grad"], a["grad_stride"]),
    }
    if status == B.OK:
        calls[name]()
        return
    with pytest.raises(B.D2mheError) as e:
        calls[name]()
    assert e.value.status == status, (name, change, e.value)


ALL = ("top", "at", "distill", "backward")


@pytest.mark.parametrize("name", ALL)
def test_no_rows_is_no_work(lib, name):
    call(name, B.OK, rows=0)


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(classes=0), dict(classes=1 << 31, row_stride=1 << 31), dict(rows=1 << 31), dict(row_stride=V - 1),
    dict(row_stride=1 << 60), dict(rows=1 << 30, row_stride=1 << 31), dict(k=0), dict(k=B.MAX_TOP + 1),
])
def test_sizes_out_of_range(lib, name, change):
    call(name, B.ERR_RANGE, **change)


@pytest.mark.parametrize("name", ["distill", "backward"])
@pytest.mark.parametrize("change", [
    dict(members=0), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
    dict(temperature=float("inf")), dict(temperature=0.009), dict(temperature=101.0), dict(grad_stride=V - 1),
    dict(grad_stride=1 << 60), dict(grad=ZERO["logits"]), dict(grad=ZERO["logits"] + 4 * V * (ROWS - 1)),
    dict(logits=ZERO["grad"] + 16 * 7),
])
def test_teachers_and_gradients_out_of_range(lib, name, change):
    call(name, B.ERR_RANGE, **change)


USES = {"top": ("logits", "index", "logprob", "scratch"), "at": ("logits", "index", "logprob", "scratch"),
        "distill": ("logits", "index", "sum", "loss", "lse", "scratch"), "backward": ("logits", "index", "sum", "lse", "grad")}


@pytest.mark.parametrize("name,field", [(n, f) for n in ALL for f in USES[n]])
def test_missing_and_misaligned_buffers(lib, name, field):
    call(name, B.ERR_NULL, **{field: None})
    call(name, B.ERR_ALIGN, **{field: ZERO[field] + 8})


@pytest.mark.parametrize("name", ["distill", "backward"])
def test_optional_buffers_are_aligned_too(lib, name):
    call(name, B.ERR_ALIGN, weight=ZERO["weight"] + 4)
    call(name, B.ERR_ALIGN, grad=ZERO["grad"] + 4)
    call(name, B.OK, weight=None, rows=0)


@pytest.mark.parametrize("name", ["top", "at", "distill"])
def test_scratch_too_small(lib, name):
    z = B.make_logits(ZERO["logits"], B.F32, ROWS, V)
    n = B.logits_scratch_bytes(z, K)
    assert n > 0 and n % 256 == 0
    call(name, B.ERR_WORKSPACE, scratch_bytes=n - 1)
    call(name, B.ERR_WORKSPACE, scratch_bytes=0)


def test_missing_descriptors(lib):
    z, t = B.make_logits(BASE, B.F32, ROWS, V), B.make_teacher(BASE, BASE, K, 2)
    p = BASE + 2048
    assert lib.d2mhe_top_logprobs(None, K, p, p, p, 256, None) == B.ERR_NULL
    assert lib.d2mhe_logprobs_at(None, p, K, p, p, 256, None) == B.ERR_NULL
    assert lib.d2mhe_distill(None, C.byref(t), p, p, p, V, p, 256, None) == B.ERR_NULL
    assert lib.d2mhe_distill(C.byref(z), None, p, p, p, V, p, 256, None) == B.ERR_NULL
    assert lib.d2mhe_distill_backward(None, C.byref(t), p, p, V, None) == B.ERR_NULL
    assert lib.d2mhe_distill_backward(C.byref(z), None, p, p, V, None) == B.ERR_NULL


def test_scratch_of_invalid_descriptors_is_zero(lib):
    assert lib.d2mhe_logits_scratch_bytes(None, 4) == 0
    good = B.make_logits(None, B.BF16, 1 << 20, 131072)
    assert B.logits_scratch_bytes(good, 64) > 0
    assert B.logits_scratch_bytes(good, 0) == 0 and B.logits_scratch_bytes(good, B.MAX_TOP + 1) == 0
    for bad in (dict(dtype=7), dict(classes=0), dict(row_stride=5)):
        a = dict(dtype=B.F32, rows=1, classes=10, row_stride=10)
        a.update(bad)
        assert B.logits_scratch_bytes(B.make_logits(None, **a), 4) == 0
