"""Page tables of the paged cache in states that a run of extensions does not make: missing pages, entries past the pool, requests
that do not fit."""
import numpy as np
import pytest
import torch

from oracle import pages4 as ref
import paper_2609_36835_gb300 as pk

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu(lib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same_tables(p, t):
    assert p.table.tolist() == t.table.tolist() and p.len.tolist() == t.len.tolist()
    n = int(p.n_free[0])
    assert p.free[:n].tolist() == [int(x) for x in t.free]


@pytest.mark.parametrize("S,M,longest,gone", [(1, 4, 256, 1), (3, 5, 300, 2), (40, 40, 2560, 9), (300, 9, 500, 60), (7, 300, 19000, 500)])
def test_missing_pages_are_not_given_back(S, M, longest, gone):
    """More than a round of 512 entries among them; then an extension that takes every page there is."""
    g = np.random.default_rng(S)
    lens = g.integers(1, longest + 1, S)
    P = int((-(-lens // 64)).sum()) + 5
    p, t = pk.pages_alloc(S, 1, P, M * 64), ref.Tables(S, M, P)
    pk.pages_extend(p, i32(lens.tolist()), int(lens.sum()))
    t.extend(lens, int(lens.sum()))
    for _ in range(gone):
        s = int(g.integers(S))
        j = int(g.integers(-(-lens[s] // 64)))
        t.table[s, j] = -1
        p.table[s, j] = -1
    to = np.where(g.random(S) < 0.5, 0, (lens * g.random(S)).astype(int))
    pk.pages_truncate(p, i32(to.tolist()))                   # (raises where something is recorded: nothing is)
    t.truncate(to)
    same_tables(p, t)
    free = p.free[:int(p.n_free[0])]
    assert int(free.min()) >= 0 and len(free.unique()) == len(free)
    pk.pages_truncate(p, i32([0] * S))
    t.truncate([0] * S)
    same_tables(p, t)
    counts = [min(64 * M, 64 * len(t.free))] + [0] * (S - 1)
    for got, want in zip(pk.pages_extend(p, i32(counts), counts[0]), t.extend(counts, counts[0])):
        assert got.tolist() == list(want)
    same_tables(p, t)


def test_entries_past_the_pool_are_recorded_and_not_given_back():
    p, t = pk.pages_alloc(2, 1, 9, 256), ref.Tables(2, 4, 9)
    pk.pages_extend(p, i32([200, 130]), 330)
    t.extend([200, 130], 330)
    for s, j, page in ((0, 1, 9), (1, 2, 10 ** 6), (0, 3, -1)):
        t.table[s, j] = page
        p.table[s, j] = page
    pk.pages_truncate(p, i32([64, 0]), check=False)
    t.truncate([64, 0])
    assert pk.arckv_query_status(p.state) == 1
    same_tables(p, t)


def test_a_length_whose_pages_are_nearly_all_missing():
    """As many entries as the pool has no room for, of which one is a page."""
    p, t = pk.pages_alloc(1, 1, 4, 640), ref.Tables(1, 10, 4)
    pk.pages_extend(p, i32([10]), 10)
    t.extend([10], 10)
    p.table[0, 7], p.table[0, 0] = p.table[0, 0].clone(), -1
    t.table[0, 7], t.table[0, 0] = t.table[0, 0], -1
    p.len.fill_(640)
    t.len[0] = 640
    pk.pages_truncate(p, i32([0]))
    t.truncate([0])
    same_tables(p, t)
    assert int(p.n_free[0]) == 4


def test_an_extension_that_does_not_fit_hands_its_rows_over():
    """The requests that fit are extended, and the error has what the call returned: on with them, or back to where they were."""
    p, t = pk.pages_alloc(3, 1, 6, 256), ref.Tables(3, 4, 6)
    pk.pages_extend(p, i32([60, 200, 10]), 270)
    t.extend([60, 200, 10], 270)
    before = p.len.clone()
    with pytest.raises(pk.ArckvError) as e:
        pk.pages_extend(p, i32([3, 100, 2]), 105)
    for got, want in zip(e.value.rows, t.extend([3, 100, 2], 105)):
        assert got.tolist() == list(want)
    same_tables(p, t)
    assert e.value.code == 2 and p.len.tolist() == [63, 200, 12]
    pk.pages_truncate(p, before)
    t.truncate(before.tolist())
    same_tables(p, t)


@pytest.mark.parametrize("n", [2, 12, 40])
def test_a_request_that_did_not_fit_leaves_the_others_right(n):
    """Its rows are attended over as well, to no purpose; those of the others are what they are without it."""
    H, G = 2, 4
    p = pk.pages_alloc(3, H, 9, 256)
    gen = torch.Generator().manual_seed(n)
    x = [torch.randn(300, H, 128, generator=gen).bfloat16().cuda() for _ in range(2)]
    _, slots, _ = pk.pages_extend(p, i32([70, 220, 10]), 300)
    pk.pages_append(p, *x, slots)
    starts, slots, positions = pk.pages_extend(p, i32([n, n, n]), 3 * n, check=False)
    fits = 220 + n <= 256
    assert pk.arckv_query_status(p.state) == (0 if fits else 2) and p.len.tolist() == [70 + n, 220 + n * fits, 10 + n]
    assert bool((slots[n:2 * n] >= 0).all() if fits else (slots[n:2 * n] == -1).all())
    new = [torch.randn(3 * n, H, 128, generator=gen).bfloat16().cuda() for _ in range(2)]
    pk.pages_append(p, *new, slots)
    Q = torch.randn(3 * n, H, G, 128, generator=gen).bfloat16().cuda()
    O = pk.pages_attend(p, Q, starts, max_count=n)
    two = pk.pages_alloc(2, H, 9, 256)
    _, slots, _ = pk.pages_extend(two, i32([70 + n, 10 + n]), 80 + 2 * n)
    pk.pages_append(two, *[torch.cat([a[:70], b[:n], a[290:], b[2 * n:]]) for a, b in zip(x, new)], slots)
    keep = torch.cat([torch.arange(n), torch.arange(2 * n, 3 * n)]).cuda()
    want = pk.pages_attend(two, Q[keep], i32([0, n, 2 * n]), max_count=n).float()
    # The same tokens, cut into items elsewhere.  Each is off by half a bf16 step and by 2^-10 (A + B) + 2 d A, where weights sum
    # A <= 1 of the values' magnitudes, B <= 4 of a token's largest, and keys' roundings move logits by d <= 2^-11 * 9.
    assert bool(((O[keep].float() - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -5).all())
