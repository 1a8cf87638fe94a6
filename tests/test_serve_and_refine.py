"""The example that learns factor pairs, serves requests with them and refines them."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_the_example_learns_serves_and_refines():
    spec = importlib.util.spec_from_file_location("serve_and_refine", os.path.join(ROOT, "examples", "serve_and_refine.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, off = example.run(m=256, n=200, tasks=4, requests=9, iters=40, steps=20, verbose=False)
    # tasks of ranks 2 and 4 cannot hold changes of rank 6: what is left out is there to be refined
    assert losses[-1] < losses[0]
    # two ways to one gradient, both in floats: sums over 256 + 200 terms and up to 360 rows, at most 2^-23 of their
    # magnitudes for each; the magnitudes exceed the sums by less than a hundred here (random signs)
    assert off < 816 * 2.0 ** -23 * 100
