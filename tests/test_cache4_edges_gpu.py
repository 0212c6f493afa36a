"""Edges of the 4-bit cache's calls, against the plain form in 64 bits."""
import numpy as np
import pytest
import torch

from tests.test_cache4_gpu import run_attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads,group,lens,qlens,window", [(1, 1, [705], [1345], 258), (2, 1, [769, 30], [1921, 5], 256), (1, 4, [200], [500], 40)])
def test_many_more_queries_than_tokens_under_a_window(heads, group, lens, qlens, window, dtype):
    """Whole row tiles of queries stand in front of the first token: they see nothing and get 0 and -inf, the others what they see."""
    run_attend(np.random.default_rng(window), heads, group, 16, lens, qlens, window, dtype, garbage=False)
