"""The example that trains and serves a map of dense documents."""

import importlib.util
import os

import pytest

from conftest import ROOT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_the_dense_map_learns_and_is_served():
    spec = importlib.util.spec_from_file_location("dense_map", os.path.join(ROOT, "examples", "dense_map.py"))
    dense_map = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(dense_map)
    lines = []
    losses, same = dense_map.main(steps=25, docs=300, states=200, side=9, features=75, say=lines.append)
    # the distance falls with the steps, to less than half of where it began
    assert losses[-1] < 0.5 * losses[0] and lines
    # 8 bits (3 of fraction) move few documents to another unit
    assert same > 0.5
