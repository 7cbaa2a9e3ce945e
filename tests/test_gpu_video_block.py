"""The example runs the operators together; against the same block with their plain forms."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "video_block.py")


@pytest.mark.parametrize("grid,D,heads,C", [((2, 5, 7), 256, 2, 64), ((3, 9, 11), 512, 4, 96)])
def test_block_and_decoder(grid, D, heads, C):
    spec = importlib.util.spec_from_file_location("video_block", PATH)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    mine, plain = ex.run(grid, D, heads, C), ex.run(grid, D, heads, C, ex.PLAIN)
    # eight roundings to bf16 (2^-8 each) between the inputs and the tokens, two to the latents, where the two sides may differ by one place
    for got, ref, bound in zip(mine, plain, (8 * 2.0 ** -8, 2 * 2.0 ** -8)):
        assert bool(got.isfinite().all()) and got.shape == ref.shape
        assert float((got.float() - ref.float()).norm() / ref.float().norm()) < bound
