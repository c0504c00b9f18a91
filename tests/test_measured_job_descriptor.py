"""The descriptor that the example makes of a measured student: what is outside its layers counts once, not once a layer."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import measure_job
    return measure_job


def test_only_the_layers_are_scaled(example):
    """Two of the layers and a head measured: 4 of 10 seconds forward and 9 of 22 back, 600 of 1,000 bytes and 700 of 800 parameters are the layers'."""
    import workloads
    wl = workloads.tiny()
    col = {n: i for i, n in enumerate(workloads.COEF_FIELDS)}
    wl.coef[0, col["hidden"]], wl.ints[0, 0] = 5, 24
    constant = float(wl.coef[0, col["mem_const"]])
    m = dict(forward=10.0, forward_layers=4.0, backward=22.0, backward_layers=9.0, bytes_kept=1000, bytes_layers=600, params_layers=700, params_rest=100)
    coef, ints = example.descriptor(wl, 0, m, layers=2, seq=3, micro_batch=2)
    got = {n: float(coef[0, i]) for n, i in col.items()}
    forward, backward = 4.0 * 12 + 6.0, 9.0 * 12 + 13.0
    assert got["t_fwd_sample"] == forward / 2
    assert got["k_bwd"] == pytest.approx(backward / forward, rel=1e-6)
    assert got["mem_act"] == 600 / (3 * 2 * 5 * 2) and got["mem_const"] - constant == pytest.approx(400, abs=constant * 2.0 ** -24)
    assert got["P_bytes"] == 2 * (700 * 12 + 100)
    assert (ints == wl.ints).all() and (coef[1:] == wl.coef[1:]).all()


@pytest.mark.gpu
def test_a_larger_output_changes_nothing_of_the_layers(example):
    # (two steps: the first product of all takes room for the library that runs it; a rate of 0: the same choices in both)
    small, large = (example.measure(256, 64, 2, layers=2, experts=4, top_k=2, vocab=v, kept=16, steps=2, rate=0.0) for v in (512, 4096))
    assert small["bytes_layers"] == large["bytes_layers"] > 0 and small["params_layers"] == large["params_layers"]
    assert large["bytes_kept"] - small["bytes_kept"] == 2 * 128 * (4096 - 512)
    assert large["params_rest"] - small["params_rest"] == 256 * (4096 - 512)
    for m in (small, large):
        assert 0 < m["forward_layers"] < m["forward"] and 0 < m["backward_layers"] < m["backward"] and 0 < m["bytes_layers"] < m["bytes_kept"]
