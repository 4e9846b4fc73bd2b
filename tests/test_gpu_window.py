"""GPU parity of attention with a window and sinks, and of its gradient, against the definition in 64 bits.

Every element is held to the bounds derived in attention_reference.py."""
import math

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    import paper_2511_09987_amd as pkg
    return pkg


def normal(shape, seed, sigma=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, sigma, generator=g)


def operands(batch, heads, kv, N, M, d, seed):
    return normal((batch, heads, N, d), seed), normal((batch, kv, M, d), seed + 1), normal((batch, kv, M, d), seed + 2)


# batch, heads, kv_heads, N, M, d, window, sinks
CASES = [
    (1, 1, 1, 1, 1, 64, None, 0), (1, 2, 1, 1, 1, 128, 1, 0), (2, 4, 2, 1, 77, 128, None, 0), (1, 3, 1, 5, 3, 64, None, 0),
    (1, 2, 2, 70, 70, 64, 1, 0), (1, 2, 1, 130, 130, 128, 64, 1), (1, 4, 4, 64, 64, 64, 32, 4), (2, 6, 2, 129, 257, 64, 100, 70),
    (1, 8, 1, 33, 1000, 128, 256, 300), (1, 5, 5, 300, 300, 128, None, 0), (1, 2, 1, 7, 0, 64, None, 0), (3, 12, 4, 200, 333, 64, 65, 17),
    (1, 16, 1, 1, 5000, 128, None, 0), (1, 2, 1, 513, 2100, 64, 2000, 4), (1, 2, 2, 100, 90, 128, 16, 3), (1, 7, 1, 45, 300, 128, 5000, 9),
    (1, 1, 1, 257, 257, 128, 128, 1000), (2, 40, 1, 3, 129, 64, 128, 0), (1, 4, 2, 400, 64, 64, 7, 2), (1, 2, 1, 1, 4097, 64, 1024, 5),
    (5, 3, 3, 17, 65, 128, 33, 31), (1, 1, 1, 128, 128, 64, 129, 0), (1, 9, 3, 31, 31, 128, 64, 64), (1, 64, 8, 2, 1500, 128, 600, 65),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(lib, case):
    batch, heads, kv, N, M, d, window, sinks = case
    Q, K, V = operands(batch, heads, kv, N, M, d, 11 * N + M)
    O, lse = lib.recurrence_attention_window(Q, K, V, window, sinks)
    want, wlse, bound, lbound = ref.forward(Q, K, V, window, sinks)
    ref.within(O, want, bound, "O")
    ref.within(lse, wlse, lbound, "lse")
    again, lagain = lib.recurrence_attention_window(Q, K, V, window, sinks)
    assert torch.equal(O.view(torch.int16), again.view(torch.int16)) and torch.equal(lse.view(torch.int32), lagain.view(torch.int32))


@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradient(lib, case):
    batch, heads, kv, N, M, d, window, sinks = case
    Q, K, V = operands(batch, heads, kv, N, M, d, 13 * N + M)
    dO = normal(Q.shape, 17 * N + M)
    O, lse, _, _ = ref.forward(Q, K, V, window, sinks)
    O, lse = O.to(torch.bfloat16), lse.float()
    got = lib.recurrence_attention_window_grad(Q, K, V, O, lse, dO, window, sinks)
    want, bounds = ref.gradient(Q, K, V, O, lse, dO, window, sinks)
    for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bounds):
        ref.within(g, w, b, name)
    again = lib.recurrence_attention_window_grad(Q, K, V, O, lse, dO, window, sinks)
    for g, a in zip(got, again):
        assert torch.equal(g.view(torch.int16), a.view(torch.int16))


def test_gradient_against_differences_of_the_forward(lib):
    """The whole step as a program makes it, O and lse from the call: <dQ, u> against central differences in 64 bits.  O is
    rounded, which moves D_i by up to 2^-8 sum_c |dO_c O_c| and dS_ij by P_ij times that."""
    case = (1, 4, 2, 40, 90, 64, 33, 5)
    batch, heads, kv, N, M, d, window, sinks = case
    Q, K, V = operands(batch, heads, kv, N, M, d, 5)
    dO = normal(Q.shape, 6)
    O, lse = lib.recurrence_attention_window(Q, K, V, window, sinks)
    got = lib.recurrence_attention_window_grad(Q, K, V, O, lse, dO, window, sinks)
    _, bounds = ref.gradient(Q, K, V, O, lse, dO, window, sinks)
    O64, lse64, obound, _ = ref.forward(Q, K, V, window, sinks)
    moved = (dO.double().abs() * obound).sum(-1, keepdim=True)                   # of D
    zero = torch.zeros_like(dO)
    # P times the shift of D, through K and Q: the reference gradient of |.| operands with dO = 0 and D = -moved
    P = torch.exp((torch.where(ref.visible(N, M, window, sinks, DEV), 0.0, -math.inf) +
                   Q.double() @ K.double().repeat_interleave(2, 1).transpose(-1, -2) / 8.0) - lse64[..., None])
    extra = ((P * moved) @ K.double().repeat_interleave(2, 1).abs() / 8.0,
             ((P * moved).transpose(-1, -2) @ Q.double().abs()).view(batch, kv, 2, M, d).sum(2) / 8.0, zero[:, :kv, :1].double() * 0)
    h = 1e-4
    for which, (g, b, e) in enumerate(zip(got, bounds, extra)):
        u = torch.randn(g.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(which)).to(DEV)
        ends = []
        for sign in (1, -1):
            x = [Q.double(), K.double(), V.double()]
            x[which] = x[which] + sign * h * u
            ends.append((ref.forward(*x, window, sinks)[0] * dO.double()).sum().item())
        diff = (ends[0] - ends[1]) / (2 * h)
        allowed = ((b + e) * u.abs()).sum().item() + 1e-5 * (1 + abs(diff))
        assert abs((g.double() * u).sum().item() - diff) <= allowed, which


@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("rising", (True, False))
def test_scores_that_rise_or_fall_along_the_keys(lib, d, rising):
    """Every key's score is 2 above (below) the last one's, exactly: the reference of the running sum has to move all the time."""
    M = 250
    c = torch.arange(M, device=DEV, dtype=torch.float32) * (0.25 if d == 64 else 0.125)
    c = c if rising else c.flip(0)
    K = c[:, None].expand(M, d).to(torch.bfloat16).view(1, 1, M, d)
    Q = torch.ones((1, 2, M, d), dtype=torch.bfloat16, device=DEV)
    V = normal((1, 1, M, d), 3)
    for window, sinks in ((None, 0), (40, 3)):
        O, lse = lib.recurrence_attention_window(Q, K, V, window, sinks)
        want, wlse, bound, lbound = ref.forward(Q, K, V, window, sinks)
        ref.within(O, want, bound, "O")
        ref.within(lse, wlse, lbound, "lse")


@pytest.mark.parametrize("bad", (float("nan"), float("inf"), -float("inf")))
@pytest.mark.parametrize("d", (64, 128))
def test_what_is_masked_never_reaches_a_query(lib, bad, d):
    """Keys and values that are no numbers: the queries that see them get NaN or infinities, all others what they get without."""
    N = M = 300
    window, sinks = 50, 3
    Q, K, V = operands(1, 2, 1, N, M, d, 21)
    want, wlse, bound, lbound = ref.forward(Q, K, V, window, sinks)
    seen = ref.visible(N, M, window, sinks, DEV)
    for at in (1, 17, 64, 130, 255, 299):
        Kb, Vb = K.clone(), V.clone()
        Vb[:, :, at] = bad
        Kb[:, :, at, ::3] = bad
        clean = ~seen[:, at]
        O, lse = lib.recurrence_attention_window(Q, Kb, Vb, window, sinks)
        ref.within(O[:, :, clean], want[:, :, clean], bound[:, :, clean], f"O beside key {at}")
        ref.within(lse[:, :, clean], wlse[:, :, clean], lbound[:, :, clean], f"lse beside key {at}")
        Vb[:, :, at] = bad
        O, _ = lib.recurrence_attention_window(Q, K, Vb, window, sinks)          # finite scores: every query that sees it
        ref.within(O[:, :, clean], want[:, :, clean], bound[:, :, clean], f"O beside value {at}")
        assert not torch.isfinite(O[:, :, ~clean]).any()


def test_nan_in_keys_that_no_query_sees(lib):
    """A window has passed the first keys: they may hold anything, and take no gradient."""
    N, M, window = 40, 400, 64
    Q, K, V = operands(2, 4, 2, N, M, 128, 31)
    want, wlse, bound, lbound = ref.forward(Q, K, V, window, 0)
    K[:, :, :M - N - window] = float("nan")
    V[:, :, :M - N - window] = float("inf")
    O, lse = lib.recurrence_attention_window(Q, K, V, window)
    ref.within(O, want, bound, "O")
    ref.within(lse, wlse, lbound, "lse")
    dO = normal(Q.shape, 32)
    dQ, dK, dV = lib.recurrence_attention_window_grad(Q, K, V, O, lse, dO, window)
    assert torch.isfinite(dQ).all() and torch.isfinite(dK).all() and torch.isfinite(dV).all()
    assert not dK[:, :, :M - N - window].any() and not dV[:, :, :M - N - window].any()


def test_gradients_beside_what_is_masked(lib):
    """One key, one query's dO, one query without numbers: every gradient that does not meet them in a visible pair stays what it is."""
    N = M = 200
    window, sinks = 40, 2
    Q, K, V = operands(1, 2, 1, N, M, 128, 41)
    dO = normal(Q.shape, 42)
    O, lse, _, _ = ref.forward(Q, K, V, window, sinks)
    O, lse = O.to(torch.bfloat16), lse.float()
    want, bounds = ref.gradient(Q, K, V, O, lse, dO, window, sinks)
    seen = ref.visible(N, M, window, sinks, DEV)
    for at in (70, 133, 199):
        for which in ("K", "V", "Q", "dO"):
            x = {"Q": Q, "K": K, "V": V, "dO": dO}
            x[which] = x[which].clone()
            x[which][:, :, at] = float("nan")
            dQ, dK, dV = lib.recurrence_attention_window_grad(x["Q"], x["K"], x["V"], O, lse, x["dO"], window, sinks)
            if which in ("K", "V"):        # queries that do not see the key; keys that share no query with it
                queries = ~seen[:, at]
                keys = ~(seen[seen[:, at]].any(0))
            else:
                queries = torch.ones(N, dtype=torch.bool, device=DEV)
                queries[at] = False
                keys = ~seen[at]
            ref.within(dQ[:, :, queries], want[0][:, :, queries], bounds[0][:, :, queries], f"dQ, {which} {at}")
            ref.within(dK[:, :, keys], want[1][:, :, keys], bounds[1][:, :, keys], f"dK, {which} {at}")
            ref.within(dV[:, :, keys], want[2][:, :, keys], bounds[2][:, :, keys], f"dV, {which} {at}")


@pytest.mark.parametrize("d", (64, 128))
def test_views(lib, d):
    """(batch, rows, heads, d) tensors, one buffer for queries, keys and values, keys that the whole batch shares; results into views."""
    batch, heads, kv, N, window, sinks = 2, 6, 2, 150, 60, 3
    fused = normal((batch, N, heads + 2 * kv, d), 51)
    Q, K, V = (t.transpose(1, 2) for t in fused.split((heads, kv, kv), 2))
    out = torch.zeros((batch, N, heads, d), dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    O, lse = lib.recurrence_attention_window(Q, K, V, window, sinks, out=out)
    assert O is out
    want, wlse, bound, lbound = ref.forward(Q, K, V, window, sinks)
    ref.within(O, want, bound, "O")
    ref.within(lse, wlse, lbound, "lse")
    dO = normal((batch, N, heads, d), 52).transpose(1, 2)
    grads = [torch.zeros((batch, N, h, d), dtype=torch.bfloat16, device=DEV).transpose(1, 2) for h in (heads, kv, kv)]
    lib.recurrence_attention_window_grad(Q, K, V, O, lse, dO, window, sinks, *grads)
    want, bounds = ref.gradient(Q, K, V, O, lse, dO, window, sinks)
    for name, g, w, b in zip(("dQ", "dK", "dV"), grads, want, bounds):
        ref.within(g, w, b, name)
    # keys of stride 0 along the batch, gradients of each batch element
    Ks, Vs = K[:1].expand(batch, -1, -1, -1), V[:1].expand(batch, -1, -1, -1)
    O, lse = lib.recurrence_attention_window(Q, Ks, Vs, window, sinks)
    want, wlse, bound, lbound = ref.forward(Q, Ks, Vs, window, sinks)
    ref.within(O, want, bound, "O, shared keys")
    got = lib.recurrence_attention_window_grad(Q, Ks, Vs, O, lse, dO, window, sinks)
    want, bounds = ref.gradient(Q, Ks, Vs, O, lse, dO, window, sinks)
    for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bounds):
        ref.within(g, w, b, name + ", shared keys")


def test_refusals_of_device_tensors(lib):
    Q, K, V = operands(1, 2, 1, 8, 8, 64, 61)
    call = lib.recurrence_attention_window
    with pytest.raises(ValueError, match="bfloat16"):
        call(Q.float(), K, V)
    with pytest.raises(ValueError, match="contiguous rows"):
        call(normal((1, 2, 8, 128), 1)[..., ::2], K, V)
    with pytest.raises(ValueError, match="contiguous rows"):
        call(normal((1, 2, 8, 68), 1)[..., :64], K, V)
    with pytest.raises(ValueError, match="shape mismatch"):
        call(Q, K, V[:, :, :7])
    with pytest.raises(ValueError, match="window"):
        call(Q, K, V, 0)
    with pytest.raises(ValueError, match="sinks"):
        call(Q, K, V, 4, -1)
    with pytest.raises(ValueError, match="lse"):
        call(Q, K, V, lse=torch.zeros((1, 2, 8), dtype=torch.float64, device=DEV))
    with pytest.raises(lib.CycError, match="ALIAS"):
        call(Q, K, V, out=Q)
    with pytest.raises(lib.CycError, match="SHAPE"):
        call(Q, K, V, out=normal((1, 1, 8, 64), 1).expand(1, 2, 8, 64))


def test_a_workspace_too_small_counts_as_none(lib):
    batch, heads, kv, N, M, d = 1, 2, 1, 1, 4000, 128
    Q, K, V = operands(batch, heads, kv, N, M, d, 71)
    want, wlse, bound, lbound = ref.forward(Q, K, V, None, 0)
    wanted = lib.cyc_attention_window_workspace(batch, heads, kv, N, M, d, 0, 0)
    assert wanted > 0
    work = torch.full((wanted + 64,), 255, dtype=torch.uint8, device=DEV)
    for size in (0, wanted - 1, wanted):
        O, lse = torch.empty_like(Q), torch.empty(Q.shape[:3], device=DEV)
        s = torch.cuda.current_stream().cuda_stream
        assert lib.cyc_recurrence_attention_window(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), lse.data_ptr(), batch, heads, kv, N, M,
                                                   d, None, 0, 0, work.data_ptr() if size else 0, size, s) == 0
        ref.within(O, want, bound, "O")
        ref.within(lse, wlse, lbound, "lse")
    assert bool((work[wanted:] == 255).all())


def test_another_stream_and_no_lse(lib):
    Q, K, V = operands(2, 4, 2, 300, 300, 64, 81)
    want, wlse, bound, lbound = ref.forward(Q, K, V, 77, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    O, lse = lib.recurrence_attention_window(Q, K, V, 77, 2, stream=side)
    dO = normal(Q.shape, 82)
    side.wait_stream(torch.cuda.current_stream())
    grads = lib.recurrence_attention_window_grad(Q, K, V, O, lse, dO, 77, 2, stream=side)
    side.synchronize()
    ref.within(O, want, bound, "O")
    gwant, gbounds = ref.gradient(Q, K, V, O, lse, dO, 77, 2)
    for g, w, b in zip(grads, gwant, gbounds):
        ref.within(g, w, b)
    out = torch.empty_like(Q)
    s = torch.cuda.current_stream().cuda_stream
    assert lib.cyc_recurrence_attention_window(Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), 0, 2, 4, 2, 300, 300, 64, None, 77, 2, 0, 0, s) == 0
    assert torch.equal(out.view(torch.int16), O.view(torch.int16))


def test_a_captured_step(lib):
    """Forward and gradient in one graph, replayed on new inputs with eager calls between the replays."""
    shape = (1, 4, 2, 2, 1500, 128)
    Q, K, V = operands(*shape, 91)
    dO = normal(Q.shape, 92)
    step = lambda: (lambda f: (*f, *lib.recurrence_attention_window_grad(Q, K, V, *f, dO, 700, 4)))(lib.recurrence_attention_window(Q, K, V, 700, 4))  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for n in range(4):
        for t, new in zip((Q, K, V, dO), (*operands(*shape, 100 + 4 * n), normal(Q.shape, 103 + 4 * n))):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        for g, e in zip(got, step()):
            assert torch.equal(g, e)


@pytest.mark.parametrize("heads,N", ((0, 5), (4, 0)))
def test_gradients_of_keys_that_no_query_reads(lib, heads, N):
    Q, K, V = operands(2, heads, 2, N, 70, 64, 3)
    O, lse = lib.recurrence_attention_window(Q, K, V)
    dK, dV = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    lib.recurrence_attention_window_grad(Q, K, V, O, lse, torch.ones_like(Q), dK=dK, dV=dV)
    assert not dK.any() and not dV.any()


@pytest.mark.parametrize("case", [(1, 4, 2, 300, 2100, 64, None, 0), (2, 3, 1, 65, 1500, 128, 700, 70), (1, 2, 2, 1300, 1300, 128, None, 0),
                                  (1, 1, 1, 1, 700, 64, 600, 3), (1, 6, 2, 900, 800, 64, 620, 1)], ids=str)
def test_gradients_of_few_rows_against_many_keys(lib, case):
    """The keys of a row are cut into runs, as its queries' are."""
    test_gradient(lib, case)
    batch, heads, kv, N, M, d, window, sinks = case
    whole, less = (lib.cyc_attention_window_grad_workspace(batch, heads, kv, n, M, d, window or 0, sinks) for n in (N, 0))
    assert whole - less > batch * heads * N * d * 4                                # of two runs and more


@pytest.mark.parametrize("d", (64, 128))
def test_queries_that_are_no_numbers_among_many_heads(lib, d):
    """One query of three of 64 heads, far apart: what does not meet them stays what it is, in their heads and in all others."""
    N, window, sinks, where = 700, 100, 3, ((0, 0, 650), (2, 7, 90), (3, 15, 699))
    Q, K, V = operands(4, 16, 16, N, N, d, 51)
    dO = normal(Q.shape, 52)
    O, lse = lib.recurrence_attention_window(Q, K, V, window, sinks)
    want, bounds = ref.gradient(Q, K, V, O, lse, dO, window, sinks)
    seen = ref.visible(N, N, window, sinks, DEV)
    for x in (Q, dO):
        kept = x.clone()
        for b, h, i in where:
            x[b, h, i] = float("inf")
        dQ, dK, dV = lib.recurrence_attention_window_grad(Q, K, V, O, lse, dO, window, sinks)
        x.copy_(kept)
        clean = [torch.ones(t.shape[:3], dtype=torch.bool, device=DEV) for t in (dQ, dK)]
        for b, h, i in where:
            clean[0][b, h, i] = False
            clean[1][b, h, seen[i]] = False
            assert not torch.isfinite(dK[b, h, i]).any()
        for g, w, e, c, name in zip((dQ, dK, dV), want, bounds, (clean[0], clean[1], clean[1]), ("dQ", "dK", "dV")):
            ref.within(g[c], w[c], e[c], name)


def test_rows_far_apart(lib):
    """Rows of keys, values and queries 36 MB apart, more than 2^32 bytes from the first to the last: offsets past 32 bits, and strides that the
    copies of whole tiles do not take."""
    N, M, d, step = 100, 130, 64, 18 << 20
    pool = torch.empty(step * M, dtype=torch.bfloat16, device=DEV)
    at = lambda offset, rows: pool.as_strided((1, 1, rows, d), (0, 0, step, 1), offset)  # noqa: E731
    Q, K, V, dO = (at(i * 4096, M if i in (1, 2) else N) for i in range(4))
    for i, t in enumerate((Q, K, V, dO)):
        t.copy_(normal(t.shape, 71 + i))
    own = [t.clone(memory_format=torch.contiguous_format) for t in (Q, K, V, dO)]
    want, lse = lib.recurrence_attention_window(*own[:3], 50, 3)
    grads = lib.recurrence_attention_window_grad(*own[:3], want, lse, own[3], 50, 3)
    got, glse = lib.recurrence_attention_window(Q, K, V, 50, 3)
    assert torch.equal(got, want) and torch.equal(glse, lse)
    for g, w in zip(lib.recurrence_attention_window_grad(Q, K, V, want, lse, dO, 50, 3), grads):
        assert torch.equal(g, w)
    ref.within(got, *(lambda f: (f[0], f[2]))(ref.forward(*own[:3], 50, 3)), "O")


# batch, heads, kv_heads, N, M, d, window, sinks: calls whose keys have their rows cut into runs, and tiles of queries that all see all keys of a tile
CUT_CASES = [(1, 2, 2, 1024, 1024, 64, None, 0), (1, 2, 1, 1024, 1024, 128, 300, 0), (1, 2, 2, 2000, 2000, 64, 300, 4), (1, 2, 1, 1500, 1500, 128, 400, 200)]


@pytest.mark.parametrize("case", CUT_CASES, ids=str)
def test_no_numbers_beside_runs_of_rows(lib, case):
    """One query, dO, key or value without numbers where the rows of a tile of keys are cut into runs: gradients that meet it in no visible pair
    stay what they are, those that do are no numbers.  A query is in a masked tile for the keys around it and in a whole one for those before."""
    batch, heads, kv, N, M, d, window, sinks = case
    Q, K, V = operands(batch, heads, kv, N, M, d, 61)
    dO = normal(Q.shape, 62)
    O, lse, _, _ = ref.forward(Q, K, V, window, sinks)
    O, lse = O.to(torch.bfloat16), lse.float()
    want, bounds = ref.gradient(Q, K, V, O, lse, dO, window, sinks)
    seen = ref.visible(N, M, window, sinks, DEV)
    none = torch.zeros(M, dtype=torch.bool, device=DEV)
    for at in (300, 655, 1000):
        for which in ("Q", "dO", "K", "V"):
            for bad in (math.nan, math.inf):
                x = {"Q": Q, "dO": dO, "K": K, "V": V}
                x[which] = x[which].clone()
                x[which][:, :, at] = bad
                got = lib.recurrence_attention_window_grad(x["Q"], x["K"], x["V"], O, lse, x["dO"], window, sinks)
                if which in ("Q", "dO"):
                    queries, keys = none[:N].clone(), seen[at]
                    queries[at] = True
                else:
                    queries, keys = seen[:, at], none.clone()
                    keys[at] = True
                spoilt = queries, keys, keys if which != "V" else none             # (dV does not depend on V)
                for name, g, w, b, off in zip(("dQ", "dK", "dV"), got, want, bounds, spoilt):
                    ref.within(g[:, :, ~off], w[:, :, ~off], b[:, :, ~off], f"{name}, {which} {at} {bad}")
                    assert not torch.isfinite(g[:, :, off]).any(), f"{name}, {which} {at} {bad}"


@pytest.mark.parametrize("d", (64, 128))
def test_many_queries_without_keys(lib, d):
    """Far more queries than the window is wide, and no keys: outputs and gradients of zeros."""
    Q, K, V = operands(1, 4, 2, 500, 0, d, 71)
    O, lse = lib.recurrence_attention_window(Q, K, V, 16, 4)
    assert not O.any() and lse.isneginf().all()
    dQ, dK, dV = lib.recurrence_attention_window_grad(Q, K, V, O, lse, normal(Q.shape, 72), 16, 4, dQ=torch.full_like(Q, 7.0))
    assert not dQ.any() and dK.shape == K.shape and dV.shape == V.shape


@pytest.mark.parametrize("case", [(1, 2, 1, 1500, 1500, 128, 400, 1400), (1, 2, 2, 2000, 2000, 64, 300, 2000), (2, 12, 2, 700, 600, 64, 128, 500)], ids=str)
def test_gradients_of_almost_all_keys_as_sinks(lib, case):
    test_gradient(lib, case)


def test_a_stream_of_another_library(lib):
    """Any object with a stream's handle: all calls take it, and have their memory from that stream's pool."""
    from types import SimpleNamespace
    side = torch.cuda.Stream()
    other = SimpleNamespace(cuda_stream=side.cuda_stream)
    Q, K, V = operands(1, 4, 2, 300, 2100, 64, 85)
    dO = normal(Q.shape, 86)
    O, lse = lib.recurrence_attention_window(Q, K, V, 700, 3)
    grads = lib.recurrence_attention_window_grad(Q, K, V, O, lse, dO, 700, 3)
    cache, table, count = K[0].view(2, -1, 4, 64).transpose(0, 1), torch.arange(525, dtype=torch.int32, device=DEV).view(1, -1), torch.tensor([2100], dtype=torch.int32, device=DEV)
    starts, values = torch.tensor([0, 300], dtype=torch.int32, device=DEV), V[0].view(2, -1, 4, 64).transpose(0, 1)
    rows = Q[0].transpose(0, 1)
    paged = lib.recurrence_attention_paged(rows, cache, values, table, count, starts, 700, 3)
    torch.cuda.synchronize()
    again = lib.recurrence_attention_window(Q, K, V, 700, 3, stream=other)
    gagain = lib.recurrence_attention_window_grad(Q, K, V, *again, dO, 700, 3, stream=other)
    pagain = lib.recurrence_attention_paged(rows, cache, values, table, count, starts, 700, 3, stream=other)
    keys, old = K[0].transpose(0, 1), (cache.clone(), values.clone())
    lib.cache_append(keys.contiguous(), V[0].transpose(0, 1).contiguous(), cache, values, table, count, torch.tensor([0, 2100], dtype=torch.int32, device=DEV), stream=other)
    side.synchronize()
    torch.cuda.synchronize()
    for g, w in zip((*again, *gagain, pagain, cache, values), (O, lse, *grads, paged, *old)):
        assert torch.equal(g, w)


def test_a_gradient_without_memory(lib):
    """Where the memory for partial sums is not to be had the error says so."""
    Q, K, V = operands(1, 2, 1, 1500, 1500, 128, 87)
    O, lse = lib.recurrence_attention_window(Q, K, V, 400, 200)
    dQ, dK, dV = (torch.empty_like(t) for t in (Q, K, V))
    assert lib.cyc_attention_window_grad_workspace(1, 2, 1, 1500, 1500, 128, 400, 200) > 4 << 20
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    torch.cuda.set_per_process_memory_fraction(0.0)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            lib.recurrence_attention_window_grad(Q, K, V, O, lse, O, 400, 200, dQ, dK, dV)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    lib.recurrence_attention_window_grad(Q, K, V, O, lse, O, 400, 200, dQ, dK, dV)


def test_strides_of_one_element(lib):
    """Dimensions of one element may have any stride: a single query out of (heads, d, 1), a key head out of a tensor of odd rows."""
    batch, heads, M, d = 1, 4, 90, 64
    Q, K, V = operands(batch, heads, 1, 1, M, d, 95)
    odd = Q.view(batch, heads, d, 1).transpose(2, 3)                               # strides 256, 64, 1, 1
    assert odd.stride(2) == 1
    shared = K[0, 0].as_strided((1, 1, M, d), (7, 3, d, 1))
    tall = torch.zeros((M, 2, d), dtype=torch.bfloat16, device=DEV)
    tall[:, 0] = V[0, 0]
    views = odd, shared, tall[:, :1].permute(1, 0, 2)[None]                         # (the last is not contiguous: strides are looked at)
    want, wlse, bound, lbound = ref.forward(Q, K, V, 33, 2)
    O, lse = lib.recurrence_attention_window(*views, 33, 2)
    ref.within(O, want, bound, "O")
    ref.within(lse, wlse, lbound, "lse")
    out = torch.zeros_like(Q).view(batch, heads, d, 1).transpose(2, 3)
    lib.recurrence_attention_window(*views, 33, 2, out=out)
    assert torch.equal(out, O)
    grads = lib.recurrence_attention_window_grad(*views, O, lse, odd, 33, 2, dQ=torch.zeros_like(Q).view(batch, heads, d, 1).transpose(2, 3))
    for g, w in zip(grads, lib.recurrence_attention_window_grad(Q, K, V, O, lse, Q, 33, 2)):
        assert torch.equal(g, w)
