"""The operators on device tensors refuse what they document as refused, before anything reaches a GPU (the pointers here are
made up: a call that went through would return a CUDA error at best)."""
import ctypes as C

import pytest

import paper_2108_09413_b200 as isc

torch = pytest.importorskip("torch")

OK, ARG, UNSUPPORTED = 0, -1, -3
AT = 0x10000                                  # an aligned address nobody owns


def changed(call, good, at, value):
    a = list(good)
    a[at] = value
    return call(*a)


NORM = dict(x=0, ldx=1, residual=2, ldr=3, weight=4, weight_type=5, type=6, rows=7, width=8, eps=9, sum=10, lds=11, q=12, ldq=13, scale=14)
NORM_GOOD = [AT, 64, AT, 64, AT, 0, 0, 4, 64, 1e-6, AT, 64, AT, 64, AT, None]


@pytest.mark.parametrize("what,value,expected", [
    ("x", None, ARG), ("weight", None, ARG), ("q", None, ARG), ("scale", None, ARG), ("x", AT + 1, ARG), ("scale", AT + 2, ARG), ("weight", AT + 1, ARG),
    ("residual", AT + 1, ARG), ("sum", AT + 1, ARG), ("ldx", 63, ARG), ("ldr", 63, ARG), ("lds", 63, ARG), ("ldq", 63, ARG), ("ldx", 0, ARG), ("ldx", -64, ARG),
    ("type", 3, ARG), ("type", -1, ARG), ("type", 4, ARG), ("weight_type", 1, ARG), ("weight_type", 3, ARG), ("rows", -1, ARG), ("width", 0, ARG), ("width", -5, ARG),
    ("eps", -1e-9, ARG), ("eps", float("nan"), ARG), ("eps", float("inf"), ARG), ("rows", 2**31, UNSUPPORTED), ("width", 2**31, UNSUPPORTED), ("rows", 0, OK)])
def test_norm(what, value, expected):
    assert changed(isc.lib().isc_rms_norm_quant, NORM_GOOD, NORM[what], value) == expected


LOGS = dict(logits=0, ld=1, type=2, rows=3, vocab=4, scale=5, targets=6, top=7, log_probs=8, entropy=9, top_ids=10, top_log_probs=11, votes=12)
LOGS_GOOD = [AT, 100, 0, 4, 100, 1.0, AT, 5, AT, AT, AT, AT, AT, None]


@pytest.mark.parametrize("what,value,expected", [
    ("logits", None, ARG), ("logits", AT + 1, ARG), ("ld", 99, ARG), ("ld", 0, ARG), ("type", 4, ARG), ("type", -1, ARG), ("rows", -1, ARG), ("vocab", 0, ARG),
    ("scale", 0.0, ARG), ("scale", -1.0, ARG), ("scale", float("nan"), ARG), ("scale", float("inf"), ARG), ("scale", 2e38, ARG), ("targets", None, ARG), ("log_probs", None, ARG),
    ("targets", AT + 4, ARG), ("entropy", AT + 2, ARG), ("votes", AT + 1, ARG), ("top_ids", None, ARG), ("top_log_probs", None, ARG), ("top", 33, ARG), ("top", -1, ARG),
    ("rows", 2**31, UNSUPPORTED), ("vocab", 2**31, UNSUPPORTED), ("rows", 0, OK)])
def test_log_probs(what, value, expected):
    good = list(LOGS_GOOD)
    if what == "vocab":
        good[LOGS["ld"]] = 2**40
    assert changed(isc.lib().isc_log_probs, good, LOGS[what], value) == expected


LINEAR = dict(x=0, ldx=1, x_scale=2, rows=3, w=4, ldw=5, w_scale=6, k=7, n=8, bias=9, adapters=10, y=11, ldy=12, y_type=13, work=14, work_bytes=15)
LINEAR_GOOD = [AT, 64, AT, 8, AT, 64, AT, 64, 100, AT, None, AT, 100, 0, AT, 1 << 20, None]


@pytest.mark.parametrize("what,value,expected", [
    ("x", None, ARG), ("x_scale", None, ARG), ("w", None, ARG), ("w_scale", None, ARG), ("y", None, ARG), ("ldx", 63, ARG), ("ldw", 63, ARG), ("ldy", 99, ARG), ("ldx", 0, ARG),
    ("x_scale", AT + 2, ARG), ("w_scale", AT + 1, ARG), ("bias", AT + 2, ARG), ("y", AT + 1, ARG), ("y_type", 3, ARG), ("y_type", -1, ARG), ("rows", -1, ARG), ("k", 0, ARG), ("n", 0, ARG),
    ("x", AT + 8, UNSUPPORTED), ("w", AT + 1, UNSUPPORTED), ("ldx", 72, UNSUPPORTED), ("ldw", 65, UNSUPPORTED), ("rows", 2**30, UNSUPPORTED), ("n", 2**30, UNSUPPORTED), ("k", 65537, UNSUPPORTED),
    ("rows", 0, OK)])
def test_linear(what, value, expected):
    good = list(LINEAR_GOOD)
    if what == "k" and value > 64:
        good[LINEAR["ldx"]] = good[LINEAR["ldw"]] = 1 << 20
    if what == "n" and value > 100:
        good[LINEAR["ldy"]] = 2**32
    assert changed(isc.lib().isc_quant_linear, good, LINEAR[what], value) == expected


@pytest.mark.parametrize("what,value,expected", [
    ("a", None, ARG), ("b", None, ARG), ("scale", None, ARG), ("ids", None, ARG), ("scale", AT + 1, ARG), ("ids", AT + 2, ARG), ("type", 2, ARG), ("type", 3, ARG), ("n_adapters", 0, ARG),
    ("n_adapters", -1, ARG), ("rank", 0, ARG), ("a", AT + 8, UNSUPPORTED), ("b", AT + 2, UNSUPPORTED), ("rank", 6, UNSUPPORTED), ("rank", 132, UNSUPPORTED)])
def test_linear_s_adapters(what, value, expected):
    from paper_2108_09413_b200.operators import _Adapters
    parts = _Adapters(AT, AT, AT, AT, 0, 4, 16)
    setattr(parts, what, value)
    good = list(LINEAR_GOOD)
    good[LINEAR["adapters"]] = C.addressof(parts)
    assert isc.lib().isc_quant_linear(*good) == expected


def test_linear_s_work_space():
    from paper_2108_09413_b200.operators import _Adapters
    size = C.c_int64()
    for rows, rank in ((1, 4), (8, 16), (100, 17), (3, 128)):
        assert isc.lib().isc_quant_linear_work_space(rows, rank, C.byref(size)) == OK and size.value == -(-rank // 16) * rows * 64
    for rows, rank in ((-1, 4), (4, -1), (4, 129)):
        assert isc.lib().isc_quant_linear_work_space(rows, rank, C.byref(size)) == ARG
    assert isc.lib().isc_quant_linear_work_space(1, 4, None) == ARG
    parts = _Adapters(AT, AT, AT, AT, 0, 4, 16)
    for at, value in ((LINEAR["work"], None), (LINEAR["work"], AT + 8), (LINEAR["work_bytes"], 8 * 64 - 1)):
        good = list(LINEAR_GOOD)
        good[LINEAR["adapters"]] = C.addressof(parts)
        good[at] = value
        assert isc.lib().isc_quant_linear(*good) == ARG


def test_tensors_of_the_host_are_refused():
    x, w = torch.zeros(2, 8), torch.ones(8)
    for call in (lambda: isc.rms_norm_quant(x, w), lambda: isc.log_probs(x), lambda: isc.log_probs([1.0, 2.0]),
                 lambda: isc.quant_linear(x.to(torch.int8), w, x.to(torch.int8), w)):
        with pytest.raises(isc.IscError) as e:
            call()
        assert e.value.code == ARG


def test_a_stream_of_another_device_is_refused():
    from types import SimpleNamespace
    from paper_2108_09413_b200 import operators
    operators._start()
    with pytest.raises(isc.IscError) as e:
        operators._enqueue("isc_log_probs", torch.device("cuda", 0), SimpleNamespace(device_index=1), lambda raw: pytest.fail("went through"))
    assert e.value.code == ARG


def test_more_rows_than_the_work_space_s_size_can_tell():
    from paper_2108_09413_b200.operators import _Adapters
    size = C.c_int64(7)
    for rows in (2**30, 2**56, 2**62):
        assert isc.lib().isc_quant_linear_work_space(rows, 128, C.byref(size)) == UNSUPPORTED and size.value == 7
        parts = _Adapters(AT, AT, AT, AT, 0, 4, 128)
        good = list(LINEAR_GOOD)
        good[LINEAR["adapters"]], good[LINEAR["rows"]] = C.addressof(parts), rows
        assert isc.lib().isc_quant_linear(*good) == UNSUPPORTED
