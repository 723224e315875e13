"""Edges of the serving operators: against the 64-bit forms of test_gpu_serve.py,
with its tolerances where no other is derived here."""
import pytest

from test_gpu_serve import BF, Case, tree  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- chunk attention --------------------------------------------------------------
@pytest.mark.parametrize("eight", [False, True])
def test_a_workspace_of_a_larger_batch(tree, eight):  # noqa: F811
    """Made for many single tokens, used for a piece of a prompt of as many tokens and fewer, and for the batch again."""
    ws = tree.chunk_attention_workspace(256, 256, 32, 8, 128)
    for new, ctx in (([33], [700]), ([1] * 256, [40] * 256), ([256], [0]), ([200, 3], [9000, 4]), ([1], [3000])):
        Case(BF, 32, 8, 128, new, ctx, eight, seed=len(new)).check(tree, workspace=ws)
    assert int(ws[:1296].sum()) == 0
