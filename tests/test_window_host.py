"""Refusals of the attention with a window, its gradient, the paged cache and its attention: all on the host, no GPU needed."""
import pytest
import torch

Q, K, V, O, LSE, DO, DQ, DK, DV, W = (0x1000000 * (i + 1) for i in range(10))
NULL, SHAPE, ALIAS, WORKSPACE = 1, 2, 4, 6


@pytest.fixture(scope="module")
def pkg():
    import os
    import paper_2511_09987_amd as p
    if not os.path.exists(p.lib_path()):
        from paper_2511_09987_amd import build
        build.build()
    return p


def window(pkg, q=Q, k=K, v=V, o=O, lse=LSE, batch=1, heads=4, kv=2, N=8, M=8, d=64, strides=None, w=0, sinks=0, work=0, size=0):
    return pkg.cyc_recurrence_attention_window(q, k, v, o, lse, batch, heads, kv, N, M, d, strides, w, sinks, work, size)


def dense(batch, heads, N, d):
    return [heads * N * d, N * d, d]


@pytest.mark.parametrize("status,changes", [
    (SHAPE, dict(N=-1)), (SHAPE, dict(M=-1)), (SHAPE, dict(batch=-1)), (SHAPE, dict(d=32)), (SHAPE, dict(d=96)), (SHAPE, dict(heads=3)),
    (SHAPE, dict(kv=0)), (SHAPE, dict(w=-1)), (SHAPE, dict(sinks=-1)), (SHAPE, dict(N=1 << 30)), (SHAPE, dict(N=1 << 29, heads=4, kv=2)),
    (SHAPE, dict(M=1 << 30)), (SHAPE, dict(batch=1 << 24)), (SHAPE, dict(q=Q + 8)), (SHAPE, dict(o=O + 2)), (SHAPE, dict(lse=LSE + 2)),
    (NULL, dict(q=0)), (NULL, dict(k=0)), (NULL, dict(v=0)), (NULL, dict(o=0)),
    (ALIAS, dict(o=Q)), (ALIAS, dict(o=K + 16)), (ALIAS, dict(o=V)), (ALIAS, dict(lse=O)), (ALIAS, dict(lse=Q + 64)),
    (SHAPE, dict(work=W + 8, size=64)), (ALIAS, dict(work=O, size=64)), (ALIAS, dict(work=K, size=64)), (ALIAS, dict(work=LSE, size=64)),
])
def test_window_refusals(pkg, status, changes):
    assert window(pkg, **changes) == status


def test_window_strides(pkg):
    good = dense(1, 4, 8, 64), dense(1, 2, 8, 64), dense(1, 2, 8, 64), dense(1, 4, 8, 64)
    flat = lambda x: [n for s in x for n in s]  # noqa: E731
    for which, stride in ((0, [512, -64, 64]), (1, [512, 512, 60]), (3, [2048, 512, 0]), (3, [2048, 64, 64]), (3, [2048, 512, 32]),
                          (0, [1 << 60, 0, 64])):
        bad = list(good)
        bad[which] = stride
        assert window(pkg, strides=flat(bad), batch=2) == SHAPE, (which, stride)


def test_window_nothing_to_do(pkg):
    for changes in (dict(N=0), dict(batch=0), dict(heads=0, kv=0), dict(heads=0)):
        assert window(pkg, q=0, k=0, v=0, o=0, lse=0, **changes) == 0
    assert pkg.cyc_attention_window_workspace(0, 4, 2, 8, 8, 64, 0, 0) == 0
    assert pkg.cyc_attention_window_workspace(1, 3, 2, 8, 8, 64, 0, 0) == 0
    assert pkg.cyc_attention_window_workspace(1, 4, 2, 8, 8, 65, 0, 0) == 0


def grad(pkg, q=Q, k=K, v=V, o=O, lse=LSE, do=DO, dq=DQ, dk=DK, dv=DV, batch=1, heads=4, kv=2, N=8, M=8, d=64, strides=None, w=0, sinks=0,
         work=W, size=1 << 20):
    return pkg.cyc_recurrence_attention_window_grad(q, k, v, o, lse, do, dq, dk, dv, batch, heads, kv, N, M, d, strides, w, sinks, work, size)


@pytest.mark.parametrize("status,changes", [
    (SHAPE, dict(N=-1)), (SHAPE, dict(d=32)), (SHAPE, dict(heads=3)), (SHAPE, dict(w=-2)), (SHAPE, dict(M=1 << 29)), (SHAPE, dict(dq=DQ + 4)),
    (NULL, dict(q=0)), (NULL, dict(lse=0)), (NULL, dict(do=0)), (NULL, dict(dk=0)), (NULL, dict(o=0)),
    (ALIAS, dict(dq=Q)), (ALIAS, dict(dk=K)), (ALIAS, dict(dv=DK)), (ALIAS, dict(dq=LSE)), (ALIAS, dict(dv=DO)), (ALIAS, dict(work=DQ)),
    (ALIAS, dict(work=LSE)), (SHAPE, dict(work=W + 4)), (WORKSPACE, dict(work=0, size=0)), (WORKSPACE, dict(size=16)), (WORKSPACE, dict(work=0)),
])
def test_grad_refusals(pkg, status, changes):
    assert grad(pkg, **changes) == status


def test_grad_nothing_to_do(pkg):
    for changes in (dict(batch=0), dict(N=0, M=0), dict(heads=0, kv=0)):
        assert grad(pkg, q=0, k=0, v=0, o=0, lse=0, do=0, dq=0, dk=0, dv=0, work=0, size=0, **changes) == 0


TABLE, LENGTHS, STARTS = 0x20000000, 0x21000000, 0x22000000


def cache(pkg, **changes):
    fields = dict(K=K, V=V, table=TABLE, lengths=LENGTHS, starts=STARTS, seqs=2, pages=8, max_pages=4, kv_heads=2, page=16, d=64, table_stride=4,
                  page_stride=2 * 16 * 64, head_stride=16 * 64, row_stride=64)
    fields.update(changes)
    return pkg.cyc_cache(**fields)


BAD_CACHES = [(SHAPE, dict(pages=0)), (SHAPE, dict(max_pages=0)), (SHAPE, dict(page=24)), (SHAPE, dict(page=0)), (SHAPE, dict(page=1 << 17)),
              (SHAPE, dict(d=80)), (SHAPE, dict(seqs=-1)), (SHAPE, dict(kv_heads=0)), (SHAPE, dict(table_stride=-1)),
              (SHAPE, dict(row_stride=32)), (SHAPE, dict(page_stride=1024)), (SHAPE, dict(head_stride=4)),
              (SHAPE, dict(max_pages=1 << 28)), (SHAPE, dict(pages=1 << 40)), (SHAPE, dict(K=K + 8)), (SHAPE, dict(table=TABLE + 2)),
              (NULL, dict(K=0)), (NULL, dict(V=0)), (NULL, dict(table=0)), (NULL, dict(lengths=0)), (NULL, dict(starts=0))]


@pytest.mark.parametrize("status,changes", BAD_CACHES)
def test_caches_that_are_refused(pkg, status, changes):
    c = cache(pkg, **changes)
    assert pkg.cyc_cache_append(Q, O, c, 3, None) == status
    assert pkg.cyc_recurrence_attention_paged(Q, c, O, 3, 4, None, 0, 0, 0) == status


def test_append_refusals(pkg):
    f, c = pkg.cyc_cache_append, cache(pkg)
    assert f(Q, O, None, 3, None) == NULL
    assert f(0, O, c, 3, None) == NULL and f(Q, 0, c, 3, None) == NULL
    assert f(Q, O, c, -1, None) == SHAPE and f(Q, O, c, 1 << 30, None) == SHAPE
    assert f(Q + 4, O, c, 3, None) == SHAPE
    assert f(Q, O, c, 3, [128, 60, 128, 64]) == SHAPE and f(Q, O, c, 3, [128, -64, 128, 64]) == SHAPE
    assert f(K + 64, O, c, 3, None) == ALIAS and f(Q, V, c, 3, None) == ALIAS
    assert f(Q, O, cache(pkg, table=K), 3, None) == ALIAS and f(Q, O, cache(pkg, V=K), 3, None) == ALIAS
    assert f(0, 0, c, 0, None) == 0 and f(0, 0, cache(pkg, seqs=0), 3, None) == 0


def test_paged_refusals(pkg):
    f, c = pkg.cyc_recurrence_attention_paged, cache(pkg)
    ok = dict(tokens=3, heads=4, strides=None, max_new=0, window=0, sinks=0)
    call = lambda q=Q, o=O, c=c, work=0, size=0, **changes: f(q, c, o, *{**ok, **changes}.values(), work, size)  # noqa: E731
    assert f(Q, None, O, 3, 4, None, 0, 0, 0) == NULL
    assert call(q=0) == NULL and call(o=0) == NULL
    for changes in (dict(tokens=-1), dict(tokens=1 << 30), dict(heads=3), dict(heads=-2), dict(max_new=-1), dict(window=-1), dict(sinks=-1),
                    dict(heads=1 << 20), dict(strides=[256, 64, 0, 64]), dict(strides=[256, 64, 256, 0]), dict(strides=[250, 64, 256, 64])):
        assert call(**changes) == SHAPE, changes
    assert call(q=Q + 2) == SHAPE and call(o=O + 8) == SHAPE and call(work=W + 8, size=64) == SHAPE
    for changes in (dict(o=Q), dict(o=K), dict(o=V + 256), dict(o=TABLE), dict(o=LENGTHS - 16), dict(work=O, size=64), dict(work=V, size=64),
                    dict(work=STARTS, size=64), dict(work=Q, size=64)):
        assert call(**changes) == ALIAS, changes
    assert call(q=0, o=0, tokens=0) == 0 and call(q=0, o=0, heads=0) == 0 and call(q=0, o=0, c=cache(pkg, seqs=0)) == 0
    assert pkg.cyc_attention_paged_workspace(c, 0, 4, 0, 0, 0) == 0 and pkg.cyc_attention_paged_workspace(c, 3, 3, 0, 0, 0) == 0


def test_tensors_that_are_refused(pkg):
    """The tensor-level calls look at tensors before anything else: those of the CPU are refused, as there is no CPU path."""
    x = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        pkg.recurrence_attention_window(x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        pkg.recurrence_attention_window_grad(x, x, x, x, x[..., 0].float(), x)
    with pytest.raises(ValueError, match="shape mismatch"):
        pkg.recurrence_attention_window(x[0], x, x)
    with pytest.raises(ValueError, match="divide among"):
        pkg.recurrence_attention_window(torch.zeros((1, 3, 4, 64), dtype=torch.bfloat16), x, x)
    with pytest.raises(ValueError, match="64 or 128"):
        pkg.recurrence_attention_window(x[..., :32], x[..., :32], x[..., :32])
    t, n, s = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        pkg.cache_append(x[0], x[0], x, x, t, n, s)
    with pytest.raises(ValueError, match="device tensor"):
        pkg.recurrence_attention_paged(x[0], x, x, t, n, s)
    with pytest.raises(ValueError, match="same strides"):
        pkg.recurrence_attention_paged(x[0], x, x.transpose(1, 2), t, n, s)


def test_caches_whose_keys_and_values_meet(pkg):
    """Appending to keys and values that have memory in common is refused.  (False: they lie between one another; the append that this
    allows is among the tests on the device.)"""
    row, page = 64 * 2, 2 * 16 * 64 * 2                                       # bytes of cache()'s rows and pages
    wide = dict(row_stride=128, head_stride=16 * 128, page_stride=2 * 16 * 128)   # keys and values side by side, row by row
    above = dict(page_stride=2 * 2 * 16 * 64)                                 # page by page
    for met, at, strides in ((True, row, {}), (True, -row, {}), (True, page, {}), (True, 7 * page, {}), (True, 16, {}), (False, 8 * page, {}),
                             (False, row, wide), (True, 2 * row, wide), (True, 16, wide), (False, 31 * 2 * row + row, wide), (False, page, above),
                             (True, 2 * page, above), (True, page - row, above), (True, 3 * page - 16, above), (True, -page + 16, above)):
        c = cache(pkg, V=K + at, **strides)
        taken, meet = set(), False
        for k in (0, 1):
            for n in range(8 * 2 * 16):
                first = at * k // 2 + n // 32 * c.page_stride + n // 16 % 2 * c.head_stride + n % 16 * c.row_stride
                row_of = set(range(first, first + 64, 8))
                meet |= bool(row_of & taken) if k else False
                taken |= set() if k else row_of
        assert meet == met, (at, strides)
        if met:
            assert pkg.cyc_cache_append(Q, O, c, 3, None) == ALIAS, (at, strides)


def test_gradient_of_keys_without_queries(pkg):
    assert pkg.cyc_attention_window_grad_workspace(1, 0, 2, 8, 8, 64, 0, 0) == pkg.cyc_attention_window_grad_workspace(1, 2, 2, 0, 8, 64, 0, 0) > 0
    assert pkg.cyc_attention_window_grad_workspace(1, 0, 0, 8, 8, 64, 0, 0) == 0
    assert grad(pkg, heads=0, dk=0) == NULL and grad(pkg, heads=0, dv=DK) == ALIAS and grad(pkg, heads=0, size=16) == WORKSPACE
    assert grad(pkg, heads=0, M=0, q=0, k=0, v=0, o=0, lse=0, do=0, dq=0, dk=0, dv=0) == 0
    assert grad(pkg, batch=0, kv=1 << 40, heads=1 << 40, M=1 << 29) == 0


@pytest.mark.parametrize("N,window,sinks", [(500, 16, 4), (1 << 20, 1, 1), (500, 0, 0), (500, 16, 0), (1, 16, 4)])
def test_gradient_of_queries_without_keys(pkg, N, window, sinks):
    """No keys: room for the statistics of the queries alone, 8 bytes for each row of whole tiles of 32, whatever the mask."""
    rows = -(-N // 32) * 32
    for d in (64, 128):
        assert pkg.cyc_attention_window_grad_workspace(1, 4, 2, N, 0, d, window, sinks) == -(-4 * rows * 8 // 256) * 256
    assert grad(pkg, N=500, M=0, w=window, sinks=sinks, size=16) == WORKSPACE     # (a million queries would meet the next operand)


@pytest.mark.parametrize("case", [(4, 16, 16, 8192, 8192, 128, 4096, 8191), (4, 16, 16, 8192, 8192, 128, 4096, 8000), (8, 256, 128, 4096, 3, 64, 2690, 511),
                                  (2, 64, 8, 8192, 8192, 64, 700, 5000), (1, 32, 8, 30000, 30000, 128, 1024, 29000)], ids=str)
def test_partial_sums_of_many_sinks_are_bounded(pkg, case):
    """8 bytes for each row, 64 MB at most for each of the partial sums of rows, of keys with sinks and of other keys, and 32 bytes for each
    workgroup, of which there are at most 256 for each tile of 128 keys."""
    batch, heads, kv, N, M, d, window, sinks = case
    rows, tiles = -(-N // 32) * 32, -(-M // 128)
    wanted = pkg.cyc_attention_window_grad_workspace(*case)
    assert 0 < wanted <= batch * heads * rows * 8 + 3 * (64 << 20) + batch * kv * tiles * 256 * 32
    assert wanted <= 2 * pkg.cyc_attention_window_grad_workspace(batch, heads, kv, N, M, d, window, 0) + (192 << 20)


def test_the_largest_append(pkg):
    """One launch has 2^32 - 1 threads in workgroups of 256, and a thread moves eight elements of K: 2^29 tokens of 64 are too many, 32 fewer are
    not (and meet the check of the pointers that follows)."""
    c, f = cache(pkg, kv_heads=1), pkg.cyc_cache_append
    assert f(0, 0, c, 1 << 29, None) == SHAPE
    assert f(0, 0, c, (1 << 29) - 32, None) == NULL
    assert f(0, 0, cache(pkg), 1 << 28, None) == SHAPE and f(0, 0, cache(pkg), (1 << 28) - 16, None) == NULL


def test_strides_that_nothing_takes(pkg):
    """An extent of one element may have any stride (the check of the pointers comes after that of the strides)."""
    odd = [7, 64, -3], [5, 1, 64], [-1, 9, 64], [3, 64, 3]                      # Q, O: four heads of one query; K, V: one head of eight keys
    assert window(pkg, q=0, kv=1, N=1, strides=[s for x in odd for s in x]) == NULL
    assert window(pkg, q=0, kv=1, N=2, strides=[s for x in odd for s in x]) == SHAPE
    c = cache(pkg, pages=1, kv_heads=1, page_stride=3, head_stride=-5)
    assert pkg.cyc_cache_append(0, O, c, 1, [3, 1, 1, 5]) == NULL and pkg.cyc_cache_append(0, O, c, 2, [3, 1, 1, 5]) == SHAPE
    assert pkg.cyc_recurrence_attention_paged(0, c, O, 1, 4, [3, 64, 5, 64], 0, 0, 0) == NULL
    assert pkg.cyc_recurrence_attention_paged(0, cache(pkg, pages=2, kv_heads=1, page_stride=3), O, 1, 4, None, 0, 0, 0) == SHAPE
