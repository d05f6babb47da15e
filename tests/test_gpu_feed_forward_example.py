"""The feed-forward block's operators run together, compared as two systems."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "feed_forward_energy.py")
    spec = importlib.util.spec_from_file_location("feed_forward_energy", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype,tokens,hidden,inner",
                         [("f32", 130, 96, 260), ("bf16", 200, 136, 320), ("f16", 64, 65, 99)])
def test_two_systems_agree_and_are_ranked(dtype, tokens, hidden, inner):
    names, ranking, same, outputs = _example().compare(tokens, hidden, inner, dtype)
    assert sorted(names[int(k)] for k in ranking["key"]) == sorted(names) and len(names) == 10
    assert bool((ranking["energy_a"] > 0).all()) and bool((ranking["energy_b"] > 0).all())
    assert same and all(same.values()), same
    # a few roundings to the type apart, element by element
    for name in ("y", "dx", "dw1", "db1", "dw2", "db2", "dnorm_w", "dnorm_b", "tokens"):
        a, b = (o[name].double() for o in outputs)
        bound = (1e-5 if dtype == "f32" else 2 ** -5 if dtype == "bf16" else 2 ** -8) * float(b.abs().max())
        assert float((a - b).abs().max()) <= bound, name
