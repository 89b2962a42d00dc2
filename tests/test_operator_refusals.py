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
    ("scale", 0.0, ARG), ("scale", -1.0, ARG), ("scale", float("nan"), ARG), ("scale", float("inf"), ARG), ("targets", None, ARG), ("log_probs", None, ARG),
    ("targets", AT + 4, ARG), ("entropy", AT + 2, ARG), ("votes", AT + 1, ARG), ("top_ids", None, ARG), ("top_log_probs", None, ARG), ("top", 33, ARG), ("top", -1, ARG),
    ("rows", 2**31, UNSUPPORTED), ("vocab", 2**31, UNSUPPORTED), ("rows", 0, OK)])
def test_log_probs(what, value, expected):
    good = list(LOGS_GOOD)
    if what == "vocab":
        good[LOGS["ld"]] = 2**40
    assert changed(isc.lib().isc_log_probs, good, LOGS[what], value) == expected


def test_tensors_of_the_host_are_refused():
    x, w = torch.zeros(2, 8), torch.ones(8)
    for call in (lambda: isc.rms_norm_quant(x, w), lambda: isc.log_probs(x), lambda: isc.log_probs([1.0, 2.0])):
        with pytest.raises(isc.IscError) as e:
            call()
        assert e.value.code == ARG
