"""Attention over pages on both sides of the numbers of sequences, of blocks of rows and of K/V heads from which keys are not cut, with
one sequence that is far longer than the others."""
import pytest
import torch

from gpu_helpers import say
from test_gpu_paged_attn import _check, _state, ress  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

# Blocks of 32 rows: cut up to 1,024 blocks of all K/V heads; of 128 rows, below 1,000; up to 256 sequences.
CASES = [(64, 16, 16, 1, True), (65, 16, 16, 1, False), (96, 16, 16, 1, False), (198, 10, 5, 1, True), (199, 10, 5, 1, False),
         (256, 2, 2, 1, True), (257, 2, 2, 1, False), (42, 16, 16, 150, True), (43, 16, 16, 150, False), (224, 8, 2, 40, True),
         (225, 8, 2, 40, False), (256, 4, 1, 20, True), (257, 4, 1, 20, False)]


@pytest.mark.parametrize("B,H,H_kv,new,cut", CASES)
@pytest.mark.parametrize("at", [0, -1])
def test_one_long_sequence(ress, B, H, H_kv, new, cut, at):  # noqa: F811
    """The long one first or last, an empty one and one without new tokens among the others."""
    lens = [40 + i % 61 for i in range(B)]
    lens[at] = 5000
    new = [min(n, new) for n in lens]
    lens[3], new[3], new[5] = 0, 0, 0
    q, k, v, cu, tables = _state(B + H, H, H_kv, 16, lens, new, padding=2)
    n = ress.ress_paged_attn_workspace_size(B, H, H_kv, q.shape[1], page=16, max_pages=tables.shape[1], n_pages=k.shape[0], window=10 ** 9)
    say(f"[cut limits] B {B} H {H}/{H_kv} rows {q.shape[1]} workspace {n}")
    assert (n > 0) == cut  # (parts of cut keys are what it holds)
    _check(ress, q, k, v, cu, lens, tables)
    _check(ress, q, k, v, cu, lens, tables, 3, 400, 7)
