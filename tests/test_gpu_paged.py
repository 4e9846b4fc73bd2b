"""GPU parity of the paged cache and its attention against the definition in 64 bits, at the bounds of attention_reference.py."""
import random

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    import paper_2511_09987_amd as pkg
    return pkg


def normal(shape, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)


def whole(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Batch:
    """Sequences of known keys and values, laid out in shuffled pages of a pool that holds NaN everywhere else.  Table entries that no key
    needs, and the keys before `evicted[b]`, are garbage."""

    def __init__(self, new, lengths, heads, kv, d, page, seed, token_major=False, evicted=None, before_new=False):
        rng = random.Random(seed)
        self.new, self.lengths, self.heads, self.kv, self.d, self.page = new, lengths, heads, kv, d, page
        need = [-(-n // page) for n in lengths]
        pages = sum(need) + 2
        order = list(range(pages))
        rng.shuffle(order)
        shape = (pages, page, kv, d) if token_major else (pages, kv, page, d)
        self.pool = [torch.full(shape, float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        self.caches = [p.transpose(1, 2) if token_major else p for p in self.pool]
        self.keys = [normal((2, kv, max(n, 1), d), seed * 1000 + b)[:, :, :n] for b, n in enumerate(lengths)]
        wide = max(max(need, default=0), 1) + 2
        table = [[-7, 10 ** 9, pages][i % 3] for i in range(wide)]
        table = [list(table) for _ in lengths]
        at = 0
        for b, n in enumerate(lengths):
            for i in range(need[b]):
                count = min(page, n - i * page)
                if before_new:                    # the new tokens are appended later
                    count = min(count, n - new[b] - i * page)
                gone = evicted and (i + 1) * page <= evicted[b][1] and i * page >= evicted[b][0]
                if gone:
                    continue
                table[b][i] = order[at]
                for c, k in zip(self.caches, self.keys[b]):
                    if count > 0:
                        c[order[at], :, :count] = k[:, i * page:i * page + count]
                at += 1
        self.table, self.lens = whole(table), whole(lengths)
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        self.starts, self.rows = whole(starts), starts
        self.Q = normal((starts[-1], heads, d), seed * 1000 + 999)

    def arguments(self):
        return (*self.caches, self.table, self.lens, self.starts)

    def check(self, O, window, sinks, only=None):
        for b, n in enumerate(self.new):
            if n == 0 or (only is not None and b not in only):
                continue
            rows = slice(self.rows[b], self.rows[b + 1])
            K, V = (k[None] for k in self.keys[b])
            want, _, bound, _ = ref.forward(self.Q[rows].transpose(0, 1)[None], K, V, window, sinks)
            ref.within(O[rows].transpose(0, 1)[None], want, bound, f"sequence {b}")


# new tokens, lengths, heads, kv_heads, d, page, window, sinks
CASES = [
    ([1], [1], 2, 1, 64, 16, None, 0), ([1], [130], 8, 2, 128, 16, None, 0), ([1, 1, 1], [5, 1000, 64], 8, 8, 64, 16, None, 0),
    ([1] * 20, [17 * i + 1 for i in range(20)], 12, 4, 128, 32, None, 0), ([5, 1, 0, 33], [5, 700, 40, 300], 4, 2, 128, 16, None, 0),
    ([300], [300], 4, 4, 64, 64, None, 0), ([129, 1, 64], [1029, 2000, 64], 8, 1, 128, 16, None, 0), ([7, 2], [3, 2], 4, 1, 64, 16, None, 0),
    ([1, 3], [0, 0], 2, 2, 128, 16, None, 0), ([1] * 8, [900 + 37 * i for i in range(8)], 16, 2, 128, 16, 256, 4),
    ([100, 1, 250], [400, 3000, 251], 6, 2, 64, 64, 128, 70), ([1, 2, 4, 8, 16], [4000, 50, 77, 1300, 16], 32, 2, 64, 1, 100, 1),
    ([1, 9], [2500, 2600], 40, 1, 128, 256, None, 0), ([2] * 6, [100, 2, 1025, 64, 65, 63], 5, 5, 128, 128, 64, 0),
    ([1], [20000], 8, 1, 128, 16, None, 0), ([512], [2600], 8, 4, 128, 32, 300, 5), ([1, 1], [3000, 8], 3, 3, 64, 2, 2000, 3),
    ([0, 0, 4], [9, 0, 4], 16, 16, 64, 8, None, 0), ([1, 1], [600, 601], 96, 2, 64, 16, None, 0),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("token_major", (False, True))
def test_against_the_definition(lib, case, token_major):
    new, lengths, heads, kv, d, page, window, sinks = case
    batch = Batch(new, lengths, heads, kv, d, page, 3 + len(new), token_major)
    for max_new in (None, max(new)):
        O = lib.recurrence_attention_paged(batch.Q, *batch.arguments(), window=window, sinks=sinks, max_new=max_new)
        batch.check(O, window, sinks)
        again = lib.recurrence_attention_paged(batch.Q, *batch.arguments(), window=window, sinks=sinks, max_new=max_new)
        assert torch.equal(O.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("window,sinks", [(100, 0), (100, 20), (333, 64)])
def test_pages_that_a_window_has_passed(lib, window, sinks):
    """Entries of pages that no query sees hold garbage, the pages themselves are in other hands."""
    new, lengths, page = [1, 40, 3], [1500, 900, 1111], 16
    evicted = [(-(-sinks // page) * page, n - m - window + 1) for m, n in zip(new, lengths)]
    batch = Batch(new, lengths, 8, 2, 128, page, 8, evicted=evicted)
    batch.check(lib.recurrence_attention_paged(batch.Q, *batch.arguments(), window=window, sinks=sinks), window, sinks)


@pytest.mark.parametrize("new,lengths", [([1, 1, 1], [700, 40, 1300]), ([1, 150, 3, 1], [2000, 1500, 64, 300]), ([260], [3000])])
@pytest.mark.parametrize("workspace", (True, False))
def test_a_table_far_wider_than_its_sequences(lib, new, lengths, workspace):
    """How the keys are split goes by the lengths on the device, not by what the table could hold; and without memory they are not."""
    batch = Batch(new, lengths, 8, 2, 128, 16, 13)
    table = torch.full((len(new), 8192), -1, dtype=torch.int32, device=DEV)
    table[:, :batch.table.shape[1]] = batch.table
    O = torch.empty_like(batch.Q)
    cache = lib.cyc_cache(batch.caches[0].data_ptr(), batch.caches[1].data_ptr(), table.data_ptr(), batch.lens.data_ptr(), batch.starts.data_ptr(),
                          len(new), batch.caches[0].shape[0], 8192, 2, 16, 128, 8192, *batch.caches[0].stride()[:3])
    wanted = lib.cyc_attention_paged_workspace(cache, batch.rows[-1], 8, 0, 0, 0)
    assert wanted > 0
    work = torch.full((wanted + 64,), 255, dtype=torch.uint8, device=DEV)
    for size in (wanted, wanted - 1) if workspace else (0,):
        assert lib.cyc_recurrence_attention_paged(batch.Q.data_ptr(), cache, O.data_ptr(), batch.rows[-1], 8, None, 0, 0, 0,
                                                  work.data_ptr() if size else 0, size, torch.cuda.current_stream().cuda_stream) == 0
        batch.check(O, None, 0)
    assert bool((work[wanted:] == 255).all())


def test_rows_that_belong_to_nobody(lib):
    batch = Batch([3, 0, 20], [70, 5, 300], 4, 2, 64, 16, 5)
    Q = torch.cat([batch.Q, normal((9, 4, 64), 1)])
    out = torch.full(Q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lib.recurrence_attention_paged(Q, *batch.arguments(), out=out)
    batch.check(out[:-9], None, 0)
    assert bool((out[-9:] == 7.0).all())


def test_wrong_numbers_give_nan_in_their_sequence_alone(lib):
    batch = Batch([1, 60, 1, 2, 1], [900, 500, 300, 64, 70], 8, 2, 128, 16, 6)
    table, lens = batch.table.clone(), batch.lens.clone()
    table[0, 20] = 10 ** 8
    table[1, 0] = -1
    lens[2] = -5
    lens[4] = table.shape[1] * 16 + 1
    O = lib.recurrence_attention_paged(batch.Q, *batch.caches, table, lens, batch.starts)
    batch.check(O, None, 0, only=(3,))
    for b in (0, 1, 2, 4):
        assert bool(O[batch.rows[b]:batch.rows[b + 1]].isnan().all()), b
    # more new tokens than were announced
    O = lib.recurrence_attention_paged(batch.Q, *batch.arguments(), max_new=2)
    batch.check(O, None, 0, only=(0, 2, 3, 4))
    assert bool(O[1:61].isnan().all())
    # starts outside the tokens there are
    starts = batch.starts.clone()
    starts[-1] += 1
    O = lib.recurrence_attention_paged(batch.Q, *batch.caches, batch.table, batch.lens, starts)
    batch.check(O, None, 0, only=(0, 1, 2, 3))
    assert bool(O[64:].isnan().all())


def test_nan_behind_the_last_key_and_in_masked_ones(lib):
    """The pool holds NaN wherever no key lies (Batch); here keys of the new tokens themselves are no numbers, which earlier rows of the
    chunk do not see."""
    batch = Batch([90], [400], 4, 1, 128, 16, 7)
    want = lib.recurrence_attention_paged(batch.Q, *batch.arguments())
    at, page = 350, batch.table[0, 350 // 16].item()
    for c in batch.caches:
        c[page, :, at % 16] = float("nan")
    O = lib.recurrence_attention_paged(batch.Q, *batch.arguments())
    first = at - 310
    # (another route through a masked tile may round its weights against another reference: both are held to the definition)
    K, V = (k[None] for k in batch.keys[0])
    ref64, _, bound, _ = ref.forward(batch.Q.transpose(0, 1)[None], K, V, None, 0)
    ref.within(want.transpose(0, 1)[None], ref64, bound, "without")
    ref.within(O[:first].transpose(0, 1)[None], ref64[:, :, :first], bound[:, :, :first], "beside")
    assert bool(O[first:].isnan().all())


def test_a_pool_beyond_32_bits(lib):
    """Pages whose byte offsets pass 2^32."""
    pages, kv, page, d = 150000, 8, 16, 128
    K_cache, V_cache = (torch.empty((pages, kv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    used = whole([[149999, 131072, 140001, 131071, 7, 149998, 131073]])
    n = 100
    K, V = normal((n, kv, d), 1), normal((n, kv, d), 2)
    lib.cache_append(K, V, K_cache, V_cache, used, whole([n]), whole([0, n]))
    for c, x in ((K_cache, K), (V_cache, V)):
        got = c[used[0].long()].transpose(1, 2).reshape(-1, kv, d)[:n]
        assert torch.equal(got.view(torch.int16), x.view(torch.int16))
    Q = normal((40, 16, d), 3)
    O = lib.recurrence_attention_paged(Q, K_cache, V_cache, used, whole([n]), whole([0, 40]))
    want, _, bound, _ = ref.forward(Q.transpose(0, 1)[None], K.transpose(0, 1)[None], V.transpose(0, 1)[None], None, 0)
    ref.within(O.transpose(0, 1)[None], want, bound)
    O = lib.recurrence_attention_paged(Q[-1:], K_cache, V_cache, used, whole([n]), whole([0, 1]), max_new=1)
    ref.within(O.transpose(0, 1)[None], want[:, :, -1:], bound[:, :, -1:])


@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("new,lengths,kv,page", [([1], [1], 1, 16), ([3, 0, 40, 1], [3, 9, 100, 64], 2, 16), ([5, 300], [5, 1000], 8, 1), ([7], [3], 4, 32)])
def test_append(lib, new, lengths, kv, page, d):
    """Every token at its place (tokens before key 0 have none), everything else untouched; from and into views."""
    batch = Batch(new, lengths, kv, kv, d, page, 4, token_major=True)
    total = batch.rows[-1]
    fused = normal((total, 2 * kv, d), 9)
    K, V = fused[:, :kv], fused[:, kv:]
    for c in batch.pool:
        c.fill_(2.0)
    want = [c.clone() for c in batch.pool]
    for b, n in enumerate(new):
        for t in range(n):
            j = lengths[b] - n + t
            if j >= 0:
                for w, x in zip(want, (K, V)):
                    w[batch.table[b, j // page], j % page] = x[batch.rows[b] + t]
    lib.cache_append(K, V, *batch.arguments())
    for c, w in zip(batch.pool, want):
        assert torch.equal(c.view(torch.int16), w.view(torch.int16))


def test_append_without_a_place(lib):
    """Wrong lengths, starts and pages: those tokens are not written, and nothing else is."""
    K_cache, V_cache = torch.zeros((4, 1, 16, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((4, 1, 16, 64), dtype=torch.bfloat16, device=DEV)
    K, V = normal((6, 1, 64), 1), normal((6, 1, 64), 2)
    lib.cache_append(K, V, K_cache, V_cache, whole([[-1, 9], [4, 2], [1, 3], [2, 0]]), whole([5, 16, 33, -3]), whole([0, 1, 3, 4, 5]))
    assert not K_cache.any() and not V_cache.any()
    lib.cache_append(K, V, K_cache, V_cache, whole([[1, 3]]), whole([20]), whole([0, 7]))
    assert not K_cache.any() and not V_cache.any()


def test_refusals_of_device_tensors(lib):
    batch = Batch([1], [20], 2, 1, 64, 16, 5)
    K_cache, V_cache, table, lens, starts = batch.arguments()
    call = lib.recurrence_attention_paged
    for bad, match in (((K_cache, V_cache, table.long(), lens, starts), "int32"), ((K_cache, V_cache, table, lens.repeat(2), starts), "lengths"),
                       ((K_cache, V_cache, table[0], lens, starts), "table"), ((K_cache.float(), V_cache, table, lens, starts), "bfloat16"),
                       ((K_cache[:, :, :12], V_cache[:, :, :12], table, lens, starts), "power of two")):
        with pytest.raises(ValueError, match=match):
            call(batch.Q, *bad)
        with pytest.raises(ValueError, match=match):
            lib.cache_append(batch.Q[:, :1], batch.Q[:, :1], *bad)
    with pytest.raises(ValueError, match="max_new"):
        call(batch.Q, *batch.arguments(), max_new=0)
    with pytest.raises(ValueError, match="divide among"):
        call(normal((1, 3, 64), 1), *Batch([1], [20], 2, 2, 64, 16, 5).arguments())
    with pytest.raises(lib.CycError, match="ALIAS"):
        call(batch.Q, *batch.arguments(), out=batch.Q)
    with pytest.raises(lib.CycError, match="ALIAS"):
        lib.cache_append(K_cache[0].transpose(0, 1), V_cache[0].transpose(0, 1), *batch.arguments())


@pytest.mark.parametrize("window,sinks", [(None, 0), (90, 6)])
def test_a_text_read_in_chunks_and_continued(lib, window, sinks):
    """Append and attend, chunk by chunk, then token by token, two sequences side by side: what one forward pass over the whole texts gives."""
    heads, kv, d, page = 8, 2, 128, 16
    totals, chunks = (333, 190), ((100, 64), (1, 0), (130, 100), (96, 20), (1, 1), (1, 1), (4, 4))
    X = [tuple(normal((1, h, n, d), 7 * b + c) for c, h in enumerate((heads, kv, kv))) for b, n in enumerate(totals)]
    pages = 60
    K_cache, V_cache = (torch.full((pages, kv, page, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(2))[:44].view(2, 22).to(torch.int32).to(DEV)
    done, out = [0, 0], [[], []]
    for sizes in chunks:
        rows = [tuple(x[0, :, done[b]:done[b] + n].transpose(0, 1) for x in X[b]) for b, n in enumerate(sizes)]
        Q, K, V = (torch.cat(part) for part in zip(*rows))
        done = [a + n for a, n in zip(done, sizes)]
        where = table, whole(done), whole([0, sizes[0], sizes[0] + sizes[1]])
        lib.cache_append(K, V, K_cache, V_cache, *where)
        O = lib.recurrence_attention_paged(Q, K_cache, V_cache, *where, window=window, sinks=sinks, max_new=max(sizes))
        for b, part in enumerate(O.split(sizes)):
            out[b].append(part)
    assert done == list(totals)
    for b in range(2):
        want, _, bound, _ = ref.forward(*X[b], window, sinks)
        ref.within(torch.cat(out[b]).transpose(0, 1)[None], want, bound, f"sequence {b}")
        O, _ = lib.recurrence_attention_window(*X[b], window, sinks)
        ref.within(O, want, bound, f"sequence {b} in one")


def test_a_captured_decoding_step(lib):
    """Append and attend in one graph; lengths, tables and inputs change between replays, eager calls in between."""
    new, lengths = [1] * 6, [40, 700, 1, 333, 64, 2000]
    batch = Batch(new, lengths, 8, 2, 128, 16, 9, before_new=True)
    K, V = (torch.empty((6, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def step():
        lib.cache_append(K, V, *batch.arguments())
        return lib.recurrence_attention_paged(batch.Q, *batch.arguments(), max_new=1, window=900, sinks=4)

    for b in range(6):
        K[b], V[b] = batch.keys[b][0][:, -1], batch.keys[b][1][:, -1]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O = step()
    for n in range(4):
        batch.Q.copy_(normal(batch.Q.shape, 50 + n))
        for b in range(6):
            batch.keys[b][:, :, -1] = normal((2, 2, 128), 60 + 7 * n + b)
            K[b], V[b] = batch.keys[b][0][:, -1], batch.keys[b][1][:, -1]
        graph.replay()
        torch.cuda.synchronize()
        batch.check(O, 900, 4)
        assert torch.equal(O, step())


def test_two_streams_at_once(lib):
    batches = [Batch([1] * 4, [500, 900, 64, 2000], 8, 2, 128, 16, 11 + i) for i in range(2)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(6):
        for i in range(2):
            outs[i].append(lib.recurrence_attention_paged(batches[i].Q, *batches[i].arguments(), max_new=1, stream=sides[i]))
    torch.cuda.synchronize()
    for b, out in zip(batches, outs):
        b.check(out[0], None, 0)
        for o in out[1:]:
            assert torch.equal(o.view(torch.int16), out[0].view(torch.int16))


@pytest.mark.parametrize("dim", (1, 3, 4))
def test_append_to_keys_and_values_in_one_pool(lib, dim):
    """Keys and values page by page, row by row, and halves of a row: they lie between one another and are written as if apart."""
    shape = [6, 2, 16, 64]
    pool = torch.zeros(shape[:dim] + [2] + shape[dim:], dtype=torch.bfloat16, device=DEV) if dim < 4 else \
        torch.zeros(shape[:3] + [128], dtype=torch.bfloat16, device=DEV)
    K_cache, V_cache = pool.unbind(dim) if dim < 4 else pool.split(64, -1)
    g = torch.Generator(device=DEV).manual_seed(dim)
    K, V = (torch.empty((9, 2, 64), dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    number = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    lib.cache_append(K, V, K_cache, V_cache, number(3, 1).view(1, 2), number(20), number(0, 9))
    for cache, rows in ((K_cache, K), (V_cache, V)):
        flat = torch.cat([cache[3], cache[1]], 1).transpose(0, 1)             # keys x heads x d
        assert torch.equal(flat[11:20], rows) and not flat[:11].any() and not flat[20:].any()
        assert not cache[[0, 2, 4, 5]].any()


def test_few_rows_with_runs_beside_many_without(lib):
    """Many tokens whose keys are not split, and sequences of a few whose are: also one that sees nothing with its first token, one with a
    wrong length and one that reaches past the last token."""
    new, lengths, heads, window, sinks = [1, 700, 3, 16, 17, 0, 4, 5, 2], [1500, 900, 1100, 1030, 800, 5, 3, 200, 1200], 64, 1000, 70
    batch = Batch(new, lengths, heads, heads, 64, 16, 21)
    out = torch.full(batch.Q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lib.recurrence_attention_paged(batch.Q, *batch.arguments(), window=window, sinks=sinks, out=out)
    batch.check(out, window, sinks)
    lens, starts = batch.lens.clone(), batch.starts.clone()
    lens[7] = -1
    starts[-1] += 3
    lib.recurrence_attention_paged(batch.Q, *batch.caches, batch.table, lens, starts, window=window, sinks=sinks, out=out)
    batch.check(out, window, sinks, only=range(7))
    assert bool(out[batch.rows[7]:].isnan().all())
    starts = batch.starts.clone()
    starts[0] = -3
    lib.recurrence_attention_paged(batch.Q, *batch.caches, batch.table, batch.lens, starts, window=window, sinks=sinks, out=out)
    batch.check(out, window, sinks, only=range(1, 9))
    assert bool(out[:1].isnan().all())


@pytest.mark.parametrize("case", [
    ([1] * 70 + [3], [50 + i for i in range(70)] + [900], 8, 8, 64, 16, None, 0),
    ([129] * 3 + [1] * 80 + [40], [129 + i for i in range(3)] + [1000 + i for i in range(80)] + [2222], 16, 2, 64, 32, None, 0),
    ([17] * 66, [700 + 3 * i for i in range(66)], 16, 1, 128, 16, None, 0), ([300, 2], [6000, 9000], 64, 8, 128, 16, None, 0),
    ([2, 40], [600, 50], 12, 3, 128, 65536, None, 0), ([1, 5, 300, 1], [3000, 5, 700, 1], 4, 2, 128, 4096, 100, 7),
], ids=lambda c: f"{len(c[0])} sequences, page {c[5]}")
def test_many_sequences_and_large_pages(lib, case):
    test_against_the_definition(lib, case, False)


def test_a_captured_step_whose_lengths_grow(lib):
    """How many runs there are is chosen anew in every replay."""
    batch = Batch([260, 1, 1], [5000, 4000, 700], 8, 2, 128, 16, 31)
    lens = batch.lens.clone()
    step = lambda: lib.recurrence_attention_paged(batch.Q, *batch.caches, batch.table, lens, batch.starts)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for lengths in ([300, 20, 4], [2000, 4000, 1], [5000, 1500, 700], [261, 1, 700], [5000, 4000, 700]):
        lens.copy_(whole(lengths))
        graph.replay()
        torch.cuda.synchronize()
        got = captured.clone()
        assert torch.equal(got, step())
    batch.check(got, None, 0)


def test_a_stream_of_another_device_is_refused(lib):
    from types import SimpleNamespace
    batch, other = Batch([1], [40], 2, 2, 64, 16, 9), SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0)
    K = batch.keys[0][0].transpose(0, 1)[-1:].contiguous()
    Q = batch.Q[None].transpose(1, 2)
    lse = torch.zeros(Q.shape[:3], device=DEV)
    for call in (lambda: lib.recurrence_attention_paged(batch.Q, *batch.arguments(), stream=other), lambda: lib.cache_append(K, K, *batch.arguments(), stream=other),
                 lambda: lib.recurrence_attention_window(Q, Q, Q, stream=other), lambda: lib.recurrence_attention_window_grad(Q, Q, Q, Q, lse, Q, stream=other)):
        with pytest.raises(ValueError, match="the stream is on cuda:1"):
            call()
    lib.cache_append(K, K, *batch.arguments(), stream=torch.cuda.Stream(DEV))
    torch.cuda.synchronize()


@pytest.mark.parametrize("new,lengths,heads,kv", [([1, 1, 1], [1500, 900, 2100], 8, 2), ([2, 5, 3], [1500, 900, 2100], 4, 4), ([40, 1, 60], [1500, 900, 2100], 8, 2)])
def test_starts_far_outside_the_tokens(lib, new, lengths, heads, kv):
    """Sequences whose runs are joined: the one with the wrong start has NaN in its rows, the others what they had."""
    batch = Batch(new, lengths, heads, kv, 64, 16, 41)
    for max_new in (None, max(new)):
        for at, value, wrong in ((0, -1, 0), (0, -3, 0), (0, -2 ** 31, 0), (3, batch.rows[-1] + 1, 2), (3, 2 ** 31 - 1, 2)):
            starts = batch.starts.clone()
            starts[at] = value
            out = torch.full(batch.Q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
            lib.recurrence_attention_paged(batch.Q, *batch.caches, batch.table, batch.lens, starts, max_new=max_new, out=out)
            batch.check(out, None, 0, only=[b for b in range(3) if b != wrong])
            assert bool(out[batch.rows[wrong]:batch.rows[wrong + 1]].isnan().all()), (max_new, at, value)


def test_more_sequences_than_a_launch_takes(lib):
    """2^22 sequences x 16 key heads x 64 threads are 2^32, one more than a launch has: refused, and nothing is written."""
    seqs, cache = 1 << 22, torch.zeros((1, 16, 16, 64), dtype=torch.bfloat16, device=DEV)
    starts = torch.zeros(seqs + 1, dtype=torch.int32, device=DEV)
    starts[-1] = 1
    out = torch.full((1, 16, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(lib.CycError, match="LAUNCH"):
        lib.recurrence_attention_paged(torch.zeros_like(out), cache, cache, starts[:-1].view(-1, 1), starts[:-1], starts, max_new=1, out=out)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


def test_strides_of_one_element(lib):
    """One key head, one page, one token: the strides of such dimensions may be any, and differ between keys and values."""
    page, d = 128, 64
    keys, values = normal((page, d), 1), normal((page, d), 2)
    K_cache, V_cache = torch.zeros_like(keys), torch.zeros_like(values)
    views = K_cache.as_strided((1, 1, page, d), (3, 5, d, 1)), V_cache.as_strided((1, 1, page, d), (8, d, d, 1))
    table, lengths = whole([[0]]), whole([100])
    lib.cache_append(keys[:100].view(100, 1, d), values[:100].as_strided((100, 1, d), (d, 1, 1)), *views, table, lengths, whole([0, 100]))
    assert torch.equal(K_cache[:100], keys[:100]) and torch.equal(V_cache[:100], values[:100]) and not K_cache[100:].any()
    Q = normal((1, 6, d), 3)
    O = lib.recurrence_attention_paged(Q.as_strided((1, 6, d), (1, d, 1)), *views, table, lengths, whole([0, 1]))
    want, _, bound, _ = ref.forward(Q[:, :, None], keys[None, None, :100], values[None, None, :100], None, 0)
    ref.within(O[:, :, None], want, bound)
