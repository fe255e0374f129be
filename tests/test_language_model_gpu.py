"""The example that runs the token operators together: the model learns its
corpus (embed, dropout and their gradients), and what it writes follows it and
the grammar (penalties, mask and draws)."""
import importlib.util
import math
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(ROOT, "examples", "language_model.py")
    spec = importlib.util.spec_from_file_location("language_model", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_learns_and_writes(example):
    r = example.main(steps=400)
    print(f"loss {r['first']:.3f} -> {r['last']:.3f}, follows {r['follows']:.3f}", flush=True)
    assert abs(r["first"] - math.log(example.VOCABULARY)) < 3  # nothing learned yet
    assert r["last"] < 2.5  # the floor is log 4 = 1.39; unlearned it is 6.9
    assert r["follows"] > 0.7  # by chance 0.004
    words = r["words"]
    assert int(words.min()) >= example.SPECIAL and int(words.max()) < example.VOCABULARY

