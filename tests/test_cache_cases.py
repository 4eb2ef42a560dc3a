"""The cases of perf/operators.py: its plain form, its request-by-request form and the kernels on the same inputs.  All outputs
are whole numbers, so the tolerance is equality."""
import importlib.util
import os
import random

import numpy as np
import pytest
import torch

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")


def _operators(device, own):
    spec = importlib.util.spec_from_file_location("operators_under_test", _PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.DEVICE, m.own = device, own
    return m


def _cases(m, count):
    """Drawn cases of one fleet each, cut to sizes that the request-by-request form takes a moment for: `count` of each operator."""
    rng, left, out = random.Random(7), dict.fromkeys(("tables", "slots", "pages"), count), []
    while any(left.values()):
        c = dict(m.draw(rng), N=1)
        tokens = c["G"] * c["B"] * m._mean_length(c)
        if left[c["op"]] and c["G"] * c["B"] * c["columns"] < 2e6 and c["G"] * c["pool"] < 5e5 and tokens < 2e6:
            left[c["op"]] -= 1
            out.append(c)
    return out


_CASES = _cases(_operators("cpu", False), 6)
_IDS = [f"{c['op']}_{c['G']}x{c['B']}_{c['block']}" for c in _CASES]


def _same(m, case, seed):
    want = m.exact(case, seed)
    have = m.run(m.prepare(case, seed))
    assert want is not None and list(want) == list(have)
    for name, h in have.items():
        assert np.array_equal(h.cpu().numpy(), want[name]), name
    return have


@pytest.mark.parametrize("case", _CASES, ids=_IDS)
def test_plain_form_is_the_definition(case):
    m = _operators("cpu", False)
    first, other = _same(m, case, 1), _same(m, case, 2)
    assert any(not torch.equal(first[n], other[n]) for n in first)               # other inputs


@pytest.mark.gpu
@pytest.mark.parametrize("case", _CASES, ids=_IDS)
def test_kernels_are_the_definition(case):
    _same(_operators("cuda:0", True), case, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["tables_c0_step", "tables_ragged_burst", "slots_c1_decode", "slots_ragged_chunks", "pages_h80_one",
                                  "pages_ragged"])
def test_kernels_are_the_plain_form_on_listed_cases(name):
    plain, own = _operators("cuda:0", False), _operators("cuda:0", True)
    case = next(c for c in plain.listed() if c["name"] == name)
    want, have = plain.run(plain.prepare(case, 5)), own.run(own.prepare(case, 5))
    for n, t in want.items():
        assert torch.equal(t, have[n]), n
