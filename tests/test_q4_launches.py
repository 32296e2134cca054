"""The 4-bit cache's kernels in a process that has no page cache whose decodes overlap freely: there each lets the next one start
early.  Other test files make such a cache, so everything here runs in processes of its own."""
import os
import subprocess
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))


def child(*args):
    r = subprocess.run([sys.executable, *args], capture_output=True, text=True, timeout=900, cwd=HERE,
                       env={**os.environ, "PYTHONPATH": os.pathsep.join([os.path.dirname(HERE), HERE])})
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]


@pytest.mark.gpu
@pytest.mark.parametrize("name, leave_out", [("test_q4_cache.py", "decodes_of_the_page_cache or in_a_process or whole_file"), ("test_q4_precision.py", "nothing")])
def test_the_cache_s_own_tests(name, leave_out):
    child("-m", "pytest", "-q", "-x", "-m", "gpu", "-k", "not (%s)" % leave_out, "-p", "no:cacheprovider", name)


def between_decodes(overlap):
    """Rows that change, decodes of a page cache in between, attention and reading behind them: each sees the rows just written."""
    import math

    from paper_2608_23843_b200 import pkv
    from q4_reference import attention
    H, G, T, dtype = 2, 4, 30000, torch.bfloat16
    gen = torch.Generator().manual_seed(overlap)
    draw = lambda *s: torch.randn(*s, generator=gen).to(dtype).cuda()         # noqa: E731
    cache = pkv.Q4Cache(pkv.make_q4_config(n_kv_heads=H, n_q_heads=H * G, n_pages=600))
    table, lengths = torch.randperm(600, generator=gen).to(torch.int32).view(1, 600).cuda(), torch.tensor([T], dtype=torch.int32).cuda()
    sets = [(draw(1, T, H, 128), draw(1, T, H, 128)) for _ in range(3)]
    qs = [draw(1, n, H * G, 128) for n in (1, 4, 40)]
    c = pkv.Cache(pkv.make_config(n_layers=1, n_kv_heads=H, n_q_heads=H * G, rank=16, sink_tokens=64, recent_tokens=64, max_seqs=1,
                                  max_pages_per_seq=8, n_dense_slots=8, n_factor_slots=1, decode_overlap=overlap))
    k, v, q = draw(130, H, 128), draw(130, H, 128), draw(1, H * G, 128)
    c.append_kv(0, [0], [130], k, v)
    dense, _, tol = attention(q.cpu(), k.cpu().double(), v.cpu().double(), 129, 1 / math.sqrt(128), dtype)
    tol = tol + 2.0 ** -9 * v.abs().max().item()           # (bf16 weights in the page cache: half a step of the largest value)
    want = []
    for rows in sets:
        cache.append_kv(table, lengths, *rows)
        torch.cuda.synchronize()
        want.append([cache.attention(table, lengths, x) for x in qs] + [x.clone() for x in cache.read_kv(table, lengths, *(torch.empty_like(x) for x in rows))])
        torch.cuda.synchronize()
    assert not torch.equal(want[0][0], want[1][0]) and not torch.equal(want[1][3], want[2][3])
    kept = []
    for i in range(24):
        rows = sets[i % 3]
        cache.append_kv(table, lengths, *rows)
        a = torch.empty(1, H * G, 128, dtype=dtype, device="cuda")
        c.decode_attention(0, [0], q, out=a)
        b = cache.attention(table, lengths, qs[i % 2 + i // 12])
        c.decode_attention(0, [0], q, out=torch.empty_like(a))
        st = cache.attention_partial(table, lengths, qs[0])
        back = cache.read_kv(table, lengths, *(torch.empty_like(x) for x in rows))
        kept.append((a, b, back, st))
    torch.cuda.synchronize()
    for i, (a, b, back, st) in enumerate(kept):
        w = want[i % 3]
        assert torch.equal(b, w[i % 2 + i // 12]), i
        assert torch.equal(back[0], w[3]) and torch.equal(back[1], w[4]), i
        assert ((a.cpu().double() - dense).abs() <= tol).all(), i
        o = st[..., :128] / st[..., 129:]
        assert ((o - w[0].float()).abs() <= 2.0 ** -7 * w[0].float().abs() + 1e-6).all(), i      # (one was rounded to bf16)
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("overlap", [0, 1, 2])
def test_between_decodes_of_a_page_cache(overlap):
    child("-c", "import test_q4_launches as t; t.between_decodes(%d)" % overlap)


@pytest.mark.gpu
def test_the_bindings_of_the_c_calls():
    """append, read and attention through the module's functions, as a caller that keeps its own pool makes them."""
    from paper_2608_23843_b200 import pkv
    from q4_reference import quantised
    H, n = 2, 50
    cfg = pkv.make_q4_config(n_kv_heads=H, n_q_heads=H, n_pages=4, dtype=torch.float16)
    sizes = pkv.pkv_q4_query_sizes(cfg)
    pool, meta = (torch.empty(b, dtype=torch.uint8, device="cuda") for b in (sizes.pool_bytes, sizes.meta_bytes))
    handle = pkv.pkv_q4_init_cache(cfg, pool, meta)
    stream = torch.cuda.current_stream()
    table, lengths = torch.tensor([[3]], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    x = torch.randn(n, 3 * H, 128, generator=torch.Generator().manual_seed(1)).half()
    fused, strides = x.cuda(), (3 * H * 128, 128)
    k, v = fused[:, :H], fused[:, H:2 * H]
    pkv.pkv_q4_append_kv(handle, 1, table, 1, lengths, n, None, k, strides, v, strides, stream)
    back = torch.zeros(2, n, H, 128, dtype=torch.float16, device="cuda")
    pkv.pkv_q4_read_kv(handle, 1, table, 1, lengths, n, None, back[0], (H * 128, 128), back[1], (H * 128, 128), stream)
    assert torch.equal(back[0].cpu(), quantised(x[:, :H], 32).half()) and torch.equal(back[1].cpu(), quantised(x[:, H:2 * H], 32).half())
    out = torch.empty(1, H, 128, dtype=torch.float16, device="cuda")
    assert pkv.pkv_q4_attention_workspace(handle, 1, 1, 64) == 0
    pkv.pkv_q4_attention(handle, 1, table, 1, lengths, 1, None, 1, 64, fused[-1:, 2 * H:], strides, out, (H * 128, 128), None, None, 0, stream)
    assert torch.isfinite(out).all() and out.abs().max() > 0
    assert pkv.pkv_q4_get_stats(handle, stream) == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}
    with pytest.raises(pkv.PkvError):
        pkv.pkv_q4_append_kv(handle, 1, table, 1, lengths, n, None, k, (1, 128), v, strides, stream)
    pkv.pkv_q4_destroy_cache(handle)
