"""Edges of the tree operators that a wrong share, cut or rounding would show at:
against the 64-bit forms of test_gpu_tree.py, with its tolerances where no other
is derived here."""
import numpy as np
import pytest
import torch

from test_gpu_tree import check_attention, check_sample, tree  # noqa: F401  (tree: the module's fixture)

pytestmark = pytest.mark.gpu


class Given:
    """Attention into outputs that start as NaN, with one workspace for all calls."""

    def __init__(self, tree, workspace):
        self.tree, self.workspace = tree, workspace

    def tree_attention(self, q, *args, **kw):
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        return self.tree.tree_attention(q, *args, out=out, workspace=self.workspace, **kw)


@pytest.mark.parametrize("batch,Hkv,active", [
    (65, 1, {3: (60, 3)}), (65, 1, {64: (12, 1)}), (128, 1, {0: (148, 2)}), (65, 2, {40: (72, 5)}), (65, 4, {7: (34, 1)}),
    (65, 8, {0: (13, 2)}), (65, 8, {64: (15, 2)}), (128, 2, {5: (12, 1), 127: (20, 4)}), (400, 1, {399: (60, 2)}), (65, 1, {}),
])
def test_attention_large_batch_mostly_idle(tree, batch, Hkv, active):  # noqa: F811
    """More sequences than a CTA keeps at hand and less work than CTAs: most CTAs' ranges are empty, also in
    the middle of a unit.  active: sequence -> (tiles of 128 keys, nodes).  An ordinary call follows on the same
    workspace, whose arrival counts must be as it wants them."""
    lens, nodes = [0] * batch, [0] * batch
    for b, (tiles, n) in active.items():
        lens[b], nodes[b] = tiles * 128 - n - 3 * (b % 5), n
    given = Given(tree, tree.tree_attention_workspace(batch, 5, 4 * Hkv, Hkv, 64))
    for seed in (1, 2):
        check_attention(given, torch.bfloat16, 4 * Hkv, Hkv, 64, lens, nodes, 5, seed=seed)
        check_attention(given, torch.bfloat16, 4 * Hkv, Hkv, 64, [3000, 40], [5, 4], 5, seed=seed)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k,m", [(0, 0.0), (3500, 0.0), (0, 1.0)])
def test_sample_empty_nucleus_among_ties(tree, dtype, k, m):  # noqa: F811
    """top_p = 0 (or below) where thousands of entries tie at the maximum and the lowest indices are not among
    them: the first of the tied is kept, alone."""
    V = 5003
    z = torch.zeros((5, V))
    z[0, 0] = float("-inf")
    z[1, :700] = -4.0
    z[2, :1500] = float("nan")
    z[3, :2000], z[3, 4000:] = -1e30, 3.0
    z[4, 1:3000] = 7.5
    R = len(z)
    for p in (0.0, -1.0, 1e-30):
        for T in (1.0, 1e-20):
            full = lambda v: np.full(R, v)  # noqa: E731
            assert check_sample(tree, z.to(dtype).cuda(), np.linspace(0, 0.99, R), full(T), full(k), full(p), full(m)) == R
