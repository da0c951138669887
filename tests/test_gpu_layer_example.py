"""The example that runs planner, replica executor and layer operators together (needs a B200)."""
import importlib.util
import os

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_decode_equals_the_layer_without_replicas():
    m = _example()
    d = m.decode()
    pl = d["planner"]
    assert ((d["instances"] % pl.s_phys) >= pl.e_loc).any()      # replicas take part
    # the same experts by their ids: expert e is local expert e % e_loc of rank e // e_loc
    n = m.EXPERTS
    want, bound = ref.experts_forward(d["x"], d["ids"], d["weights"], d["main"].view(1, n, -1), None,
                                      n, 0, n, m.HIDDEN, m.FFN)
    assert ((d["y"].cpu().double() - want).abs() <= bound).all()


def test_train_clips_every_gradient_to_one_norm():
    m = _example()
    free = m.train(max_norm=1e9)
    done = m.train(max_norm=0.5)
    assert torch.equal(free["norm"], done["norm"]) and float(done["norm"]) > 0.5
    factor = 0.5 / (float(done["norm"]) + 1e-6)
    for name, unit in (("gate", 2.0 ** -22), ("experts", 2.0 ** -8)):
        want = free[name].double() * factor
        assert ((done[name].double() - want).abs() <= want.abs() * (unit + 2.0 ** -20) + 1e-30).all()
    total = sum(float((done[k].double() ** 2).sum()) for k in ("gate", "experts")) ** 0.5
    assert abs(total - 0.5) <= 0.5 * 2.0 ** -8
    assert done["replicas"] > 0
