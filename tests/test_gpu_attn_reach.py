"""Biases that reach far and the kernels' plans that they choose: wide heads whose table leaves room for two tiles on the way
instead of four (a reach beyond about 690), and tables that leave room for one block per SM.  The formulas and tolerances are
those of the forward and backward tests."""
import pytest
import torch

import test_gpu_attn_bwd as bwd
import test_gpu_attn_fwd as fwd
from attn_ref import Case

pytestmark = pytest.mark.gpu


def check(c, dtype=torch.float32, seed=0):
    fwd.check(c, dtype, seed)
    bwd.check(c, dtype, seed)


@pytest.mark.parametrize("dim", [72, 128])
@pytest.mark.parametrize("buckets,max_distance", [(32, 1000), (64, 2048)])
@pytest.mark.parametrize("causal,two_sided", [(True, False), (False, True), (False, False), (True, True)])
def test_wide_heads(dim, buckets, max_distance, causal, two_sided):
    """Lengths beyond the reach, so that tiles with a table, with the last bucket alone and with holes in the end all occur."""
    c = Case(batch=2, len_q=300, len_kv=2500, heads_q=4, heads_kv=1, dim=dim, causal=causal, buckets=buckets, max_distance=max_distance,
             two_sided=two_sided, q_pos=1900, kv_len=(2500, 1777))
    check(c)


@pytest.mark.parametrize("heads", [(1, 1), (6, 3)])
@pytest.mark.parametrize("n", [1, 63, 65, 129, 700])
@pytest.mark.parametrize("causal", [False, True])
def test_wide_heads_with_two_tiles_on_the_way(n, causal, heads):
    check(Case(batch=2, len_q=n, heads_q=heads[0], heads_kv=heads[1], dim=128, causal=causal, buckets=64, max_distance=2048))


def test_wide_heads_with_more_items_than_blocks():
    lens = [(0, 300, 1, 129, 260)[i % 5] for i in range(50)]
    for kv_len in (lens, None):
        check(Case(batch=50, len_q=300, heads_q=4, heads_kv=4, dim=128, buckets=32, max_distance=1000, kv_len=kv_len))
    check(Case(batch=150, len_q=130, heads_q=2, heads_kv=1, dim=128, causal=False, buckets=64, max_distance=2048, two_sided=True,
               kv_len=[(37 * i) % 131 for i in range(150)]))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("max_distance", [180, 256, 400, 800])
@pytest.mark.parametrize("causal", [False, True])
def test_reaches_on_both_sides_of_one_block_per_sm(max_distance, causal, dim):
    check(Case(batch=2, len_q=1000, heads_q=2, dim=dim, causal=causal, buckets=32, max_distance=max_distance, two_sided=not causal),
          torch.bfloat16)


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 56, 72, 80, 96, 104, 120])
@pytest.mark.parametrize("n", [1, 200])
def test_head_sizes_two_sided(dim, n):
    check(Case(batch=2, len_q=n, len_kv=n + 50, heads_q=3, dim=dim, causal=False, buckets=32, two_sided=True, kv_len=(n + 50, n // 2 + 1)))
