"""Serving from the 4-bit cache at its limits: rows that leave a warp in part, arrays that lie on top of one another, more CTAs than 16 bits count,
numbers that are none, bindings that were not built."""
import pytest
import torch

from paper_2608_23843_b200 import pkv
from q4_select_reference import window_seen
from test_q4_cache import BF16, FP16, Filled, check
from test_q4_serve import seen_by


# ---- clusters whose joins leave a warp in part ---------------------------------------------------------------------------
# A segment's states are rows * d / 4 pieces for 96 threads, and rows * d / 4 / cluster for each CTA of a cluster: these end inside a warp.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype, d, g", [(BF16, 128, 32), (FP16, 64, 32), (BF16, 64, 64)])
@pytest.mark.parametrize("G", [1, 3, 5, 7])
@pytest.mark.parametrize("S, T, W, n_ctas, cluster", [(20, 300, 200, 20, 1), (8, 700, 300, 20, 2), (2, 1500, 1400, 8, 4), (2, 1500, 1400, 0, 8)])
def test_clusters_join_any_number_of_rows(dtype, d, g, G, S, T, W, n_ctas, cluster):
    f = Filled([T - 50 * s % T for s in range(S)], seed=G, dtype=dtype, d=d, g=g, H=2, G=G, n_ctas=n_ctas)
    assert pkv.pkv_q4_attention_route(f.cache.handle, S, 1, f.table.shape[1] * 64, W, 3)[::2] == (2, cluster)
    qs = f.queries([1] * S)
    q = torch.stack(qs).cuda()
    out = f.cache.attention(f.table, f.lengths, q, window=W, sinks=3).cpu()
    state = f.cache.attention_partial(f.table, f.lengths, q, window=W, sinks=3).to("cpu", torch.float64)
    for s in range(S):
        ref, _, tol = seen_by(f, qs[s], s, window_seen(f.lens[s], 1, W, 3))
        check(out[s], ref, tol)
        check(state[s][..., :d] / state[s][..., d + 1:], ref, tol)
    f.clean()
