"""The paged 4-bit cache and rotary positions on the GPU against their plain form (``oracle.pages4``), through the public
calls.

Tables, slots and what the rows are held as are compared exactly.  An output of attention is a bf16: it is off by at most
2^-8 of itself, half a step.  What comes before that, with M the largest magnitude of the values:
 - Each weight p is rounded to f16: 2^-11 of it, and below f16's normal range 2^-25 of the weights' unit.  The values' unit is at
   most 4 M, and one where their codes count 15 at most: a weight costs 2^-22 M there.
 - It may multiply a value's code times scale alone, c s = v - m, where m is the row's least value and enters with the weight as it
   was: with |m| <= (1 + 2^-8) max |v| that is 2^-11 p (|v| + 1.01 max |v|).  Or it multiplies a value rounded to f16: 2^-10 p |v|.
 - Values and keys may be rounded to f16, in units that leave a page's largest below 2^-6: 2^-11 of each element, and twice 2^-25 of
   the unit below the normal range, m's rounding and the sum's, which is 2^-17 of the page's largest.  For keys that moves a logit
   by up to 2^-11 scale sum |q_e k_e| + 2^-17 scale sum |q_e| max |k|, its weight by as much, relatively, and the sum of weights
   likewise.
 - A query's sums over groups of its elements, which the keys' least values multiply, are two bf16: 2^-17 scale sum |q_e| max |k| too.
 - fp32 logits and sums add less than 2^-14 of a weight.
With A = sum p |v|, B = sum p max |v| and d the largest move of a logit,
    |O - ref| <= 2^-8 |ref| + (2^-10 + 2^-13 + 2 d) A + 2^-10 B + (2^-17 + T 2^-22) M
"""
import numpy as np
import pytest
import torch

from oracle import pages4 as ref
import paper_2609_36835_gb300 as pk

pytestmark = pytest.mark.gpu
SC = 1.0 / np.sqrt(128.0)
LOWEST = float(np.finfo(np.float32).min)


@pytest.fixture(scope="module", autouse=True)
def _gpu(lib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rows(seed, n, H, dtype=torch.bfloat16, outliers=True):
    x = torch.randn(n, H, 128, generator=gen(seed))
    if outliers:
        x[..., 5] *= 6.0
    return x.to(dtype).cuda()


def host(x):
    return x.detach().float().cpu().numpy()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def filled(seed, lens, H, bias=False, spare=3, M=None, dtype=torch.bfloat16, scale=1.0):
    """Pages whose requests hold lens[s] tokens, in pages of any order, and the rows that were written."""
    S, n = len(lens), sum(lens)
    M = M or max(1, -(-max(lens) // 64))
    need = sum(-(-x // 64) for x in lens) + spare
    p = pk.pages_alloc(S, H, need, M * 64, bias=bias)
    p.data.fill_(0xff)                                       # what no row has written is NaN
    if bias:
        p.bias.fill_(float("nan"))
    p.free.copy_(torch.randperm(need, generator=gen(seed)).to(torch.int32))
    starts, slots, _ = pk.pages_extend(p, i32(lens), n)
    k, v = rows(seed, n, H, dtype) * scale, rows(seed + 1, n, H, dtype, outliers=False) * scale
    b = (torch.rand(n, H, generator=gen(seed + 2)) * 3 - 2).cuda() if bias else None
    if n:
        pk.pages_append(p, k, v, slots, bias=b)
    return p, k, v, b


def queries(seed, N, H, G, size=1.5):
    return (torch.randn(N, H, G, 128, generator=gen(seed)) * size).to(torch.bfloat16).cuda()


def check_rows(O, q, k, v, bias, sees, scale=SC):
    """Rows O [n, 128] of one head against the plain form over what the pages hold of k, v [T, 128]."""
    k, v = ref.held_rows(host(k), host(v))
    want, size = ref.attend(host(q), k, v, scale, sees, None if bias is None else host(bias))
    _, large = ref.attend(host(q), k, np.abs(v).max(1, keepdims=True), scale, sees, None if bias is None else host(bias))
    got = host(O).astype(np.float64)
    T = max(max(sees, default=0), 1)
    q, most_k = np.abs(host(q)).astype(np.float64), np.abs(k[:T]).max(initial=0.0)
    moved = scale * (2.0 ** -11 * (q @ np.abs(k[:T]).T).max(1, initial=0.0) + 2.0 ** -16 * q.sum(1) * most_k)[:, None]
    most = np.abs(v[:T]).max(initial=0.0)
    bound = (2.0 ** -8 * np.abs(want) + (2.0 ** -10 + 2.0 ** -13 + 2 * moved) * size + 2.0 ** -10 * large
             + (2.0 ** -17 + T * 2.0 ** -22) * most)
    empty = ~size.any(-1)
    assert not got[empty].any()
    assert np.all(np.abs(got - want) <= bound), float(np.max(np.abs(got - want) / np.maximum(bound, 1e-300)))


def check_attend(p, k, v, b, lens, counts, Q, O, causal=True, heads=None, requests=None, first=0):
    """All (or the listed) requests and heads of a packed call; k, v, b: all tokens, request after request."""
    at, row, G = 0, first, Q.shape[2]
    for s, (T, c) in enumerate(zip(lens, counts)):
        for h in (range(Q.shape[1]) if heads is None else heads):
            if c and (requests is None or s in requests):
                sees = np.repeat([max(0, T - c + i + 1) if causal else T for i in range(c)], G)
                check_rows(O[row:row + c, h].reshape(-1, 128), Q[row:row + c, h].reshape(-1, 128), k[at:at + T, h], v[at:at + T, h],
                           None if b is None else b[at:at + T, h], sees)
        at += T
        row += c


def starts_of(counts, first=0):
    return i32(list(first + np.concatenate([[0], np.cumsum(counts)])))


# -------------------------------------------------------------------- tables

def same_tables(p, t):
    assert p.table.tolist() == t.table.tolist() and p.len.tolist() == t.len.tolist()
    n = int(p.n_free[0])
    assert p.free[:n].tolist() == [int(x) for x in t.free]


@pytest.mark.parametrize("S,M,P", [(1, 1, 1), (3, 5, 9), (40, 7, 150), (600, 3, 900), (4096, 2, 5000)])
def test_a_run_of_extensions_and_truncations(S, M, P):
    g = np.random.default_rng(S)
    p, t = pk.pages_alloc(S, 2, P, M * 64), ref.Tables(S, M, P)
    for step in range(6):
        counts = g.integers(0, 90, S) * (g.random(S) < 0.7)
        n = int(counts.sum()) + int(g.integers(0, 9))
        st = pk.pages_extend(p, i32(counts.tolist()), n, check=False)
        for got, want in zip(st, t.extend(counts, n)):
            assert got.tolist() == list(want)
        same_tables(p, t)
        to = (t.len * g.random(S)).astype(int)
        to[g.random(S) < 0.5] = 0 if step % 2 else 10 ** 6
        to = np.minimum(to, t.len)
        pk.pages_truncate(p, i32(to.tolist()), check=False)
        t.truncate(to)
        same_tables(p, t)
    pk.arckv_query_status(p.state)


def test_many_rows_take_several_blocks():
    counts = [5000, 0, 1, 130, 0, 9000]
    p, t = pk.pages_alloc(6, 1, 400, 150 * 64), ref.Tables(6, 150, 400)
    for n in (sum(counts) + 77, sum(counts)):
        for got, want in zip(pk.pages_extend(p, i32(counts), n, check=False), t.extend(counts, n)):
            assert got.tolist() == list(want)
        same_tables(p, t)
        p.len.zero_(), p.table.fill_(-1)
        p.free.copy_(torch.arange(399, -1, -1)), p.n_free.fill_(400)
        t = ref.Tables(6, 150, 400)


@pytest.mark.parametrize("counts,n,M,P,code", [([64, 65, 3], 132, 1, 9, 2), ([64, 64, 0, 10], 138, 4, 2, 2), ([10, 20, 5], 20, 4, 9, 2),
                                               ([3, -5, 4], 7, 4, 9, 1)])
def test_what_does_not_fit_is_left_out_and_recorded(counts, n, M, P, code):
    S = len(counts)
    p, t = pk.pages_alloc(S, 1, P, M * 64), ref.Tables(S, M, P)
    got = pk.pages_extend(p, i32(counts), n, check=False)
    for x, want in zip(got, t.extend(counts, n)):
        assert x.tolist() == list(want)
    same_tables(p, t)
    assert pk.arckv_query_status(p.state) == code and pk.arckv_query_status(p.state) == 0
    with pytest.raises(pk.ArckvError):
        pk.pages_extend(p, i32(counts), n)


def test_truncation_refuses_lengths_that_are_not_held():
    p, t = pk.pages_alloc(3, 1, 9, 256), ref.Tables(3, 4, 9)
    pk.pages_extend(p, i32([100, 70, 10]), 180)
    t.extend([100, 70, 10], 180)
    with pytest.raises(pk.ArckvError):
        pk.pages_truncate(p, i32([101, 64, -1]))
    t.truncate([101, 64, -1])
    same_tables(p, t)


# ------------------------------------------------------------ write and read

@pytest.mark.parametrize("n", [1, 2, 7, 63, 64, 65, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [1, 3])
def test_rows_are_held_as_defined(n, dtype, H):
    P = -(-n // 64) + 1
    p = pk.pages_alloc(1, H, P, P * 64)
    p.data.fill_(0xff)
    slots = torch.randperm(P * 64, generator=gen(n))[:n].to(torch.int32).cuda()
    k, v = rows(n, n, H, dtype), rows(n + 1, n, H, dtype)
    pk.pages_append(p, k, v, slots)
    K, V = pk.pages_read(p, slots, dtype=torch.float32)
    wk, wv = ref.held_rows(host(k), host(v))
    assert np.array_equal(host(K), wk.astype(np.float32)) and np.array_equal(host(V), wv.astype(np.float32))
    K, V = pk.pages_read(p, slots)
    assert torch.equal(K, torch.from_numpy(wk.astype(np.float32)).cuda().to(torch.bfloat16))
    assert torch.equal(V, torch.from_numpy(wv.astype(np.float32)).cuda().to(torch.bfloat16))


def test_rows_of_every_magnitude():
    x = torch.randn(40, 2, 128, generator=gen(3))
    scale = torch.tensor([0.0, 1e-38, 2.0 ** -101, 1e-20, 1.0, 3e4, 1e12, 2.0 ** 66]).repeat(5).view(40, 1, 1)
    x = x * scale
    x[8] = 7.0                                               # constant rows, negative ones, one that an element dominates
    x[9], x[10, :, 3] = -x[9].abs() - 1, 1e9
    x = x.cuda()
    p, slots = pk.pages_alloc(1, 2, 1, 64), torch.arange(40, dtype=torch.int32, device="cuda")
    pk.pages_append(p, x, x, slots)
    K, V = pk.pages_read(p, slots, dtype=torch.float32)
    wk, wv = ref.held_rows(host(x), host(x))
    assert np.array_equal(host(K), wk.astype(np.float32)) and np.array_equal(host(V), wv.astype(np.float32))


def test_elements_that_are_not_finite_are_zero_and_huge_ones_cut():
    x = rows(1, 3, 2, torch.float32)
    x[1, 0, 7], x[1, 1, 9], x[2, 0, 3] = float("nan"), float("inf"), -3e38
    p, slots = pk.pages_alloc(1, 2, 1, 64), i32([4, 9, 63])
    pk.pages_append(p, x, x, slots, check=False)
    assert pk.arckv_query_status(p.state) == 5
    K, V = pk.pages_read(p, slots, dtype=torch.float32)
    wk, wv = ref.held_rows(host(x), host(x))
    assert np.array_equal(host(K), wk.astype(np.float32)) and np.array_equal(host(V), wv.astype(np.float32))


def test_rows_are_passed_over_and_rows_read_as_zero():
    p = pk.pages_alloc(2, 2, 2, 128, bias=True)
    p.data.zero_(), p.bias.zero_()
    before = p.data.clone()
    x = rows(5, 3, 2)
    pk.pages_append(p, x, x, i32([-1, 128, -7]), bias=torch.ones(3, 2, device="cuda"), check=False)
    assert pk.arckv_query_status(p.state) == 1
    assert torch.equal(p.data, before) and not p.bias.any()
    K, V = pk.pages_read(p, i32([-1, 5000, -2]), check=False)
    assert not K.any() and not V.any() and pk.arckv_query_status(p.state) == 1


def test_a_written_row_leaves_the_others_as_they_were():
    p = pk.pages_alloc(1, 2, 2, 128, bias=True)
    slots = torch.arange(128, dtype=torch.int32, device="cuda")
    x, b = rows(6, 128, 2), torch.randn(128, 2, generator=gen(1)).cuda()
    pk.pages_append(p, x, x, slots, bias=b)
    K, V = pk.pages_read(p, slots)
    y = rows(7, 1, 2)
    pk.pages_append(p, y, y, i32([77]))                      # no bias given: zero
    K2, V2 = pk.pages_read(p, slots)
    other = torch.arange(128, device="cuda") != 77
    assert torch.equal(K[other], K2[other]) and torch.equal(V[other], V2[other]) and not torch.equal(K[77], K2[77])
    held = p.bias.permute(0, 2, 1).reshape(128, 2)
    assert torch.equal(held[other], b[other]) and not held[77].any()


def test_rows_of_a_fused_projection():
    qkv = torch.randn(50, 10, 128, generator=gen(8)).to(torch.bfloat16).cuda()
    p, slots = pk.pages_alloc(1, 2, 1, 64), torch.arange(50, dtype=torch.int32, device="cuda")
    pk.pages_append(p, qkv[:, 6:8], qkv[:, 8:], slots)
    K, V = pk.pages_read(p, slots)
    pk.pages_append(p, qkv[:, 6:8].contiguous(), qkv[:, 8:].contiguous(), slots)
    K2, V2 = pk.pages_read(p, slots)
    assert torch.equal(K, K2) and torch.equal(V, V2)


# ----------------------------------------------------------------- attention

@pytest.mark.parametrize("T", [1, 2, 31, 63, 64, 65, 127, 128, 300, 1000])
@pytest.mark.parametrize("G", [1, 4, 7, 8, 16])
def test_single_tokens(T, G):
    p, k, v, b = filled(T, [T], 2)
    Q = queries(T + 1, 1, 2, G)
    O = pk.pages_attend(p, Q, starts_of([1]))
    check_attend(p, k, v, b, [T], [1], Q, O)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("G", [1, 2, 4, 8, 9])
def test_ragged_single_tokens(bias, G):
    lens = [0, 1, 64, 100, 129, 700, 63, 1500]
    p, k, v, b = filled(G, lens, 3, bias=bias)
    Q = queries(G, len(lens), 3, G)
    O = pk.pages_attend(p, Q, starts_of([1] * len(lens)), max_count=1)
    check_attend(p, k, v, b, lens, [1] * len(lens), Q, O)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,G", [(2, 4), (3, 4), (4, 4), (3, 1), (5, 3), (2, 8), (16, 1), (17, 1), (5, 4), (30, 4), (33, 8), (70, 4), (257, 1)])
def test_drafts_and_chunks(n, G, causal, bias):
    lens, counts = [n, 64 + n, 1200, 333], [n, n, n, max(1, n - 2)]
    p, k, v, b = filled(n, lens, 2, bias=bias)
    Q = queries(n, sum(counts), 2, G)
    O = pk.pages_attend(p, Q, starts_of(counts), max_count=n, causal=causal)
    check_attend(p, k, v, b, lens, counts, Q, O, causal, heads=[1], requests=[0, 1, 3] if n > 60 else None)


@pytest.mark.parametrize("bias", [False, True])
def test_a_mixed_batch_with_rows_of_no_request(bias):
    lens, counts = [500, 0, 129, 2000, 64, 77, 1], [1, 0, 100, 1, 64, 0, 1]
    p, k, v, b = filled(20, lens, 2, bias=bias)
    N = sum(counts) + 9
    Q = queries(21, N, 2, 4)
    Q[:2], Q[-7:] = float("nan"), float("nan")               # rows of no request: before the first one and behind the last
    out = torch.full((N, 2, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    st = starts_of(counts, first=2)
    got = pk.pages_attend(p, Q, st, max_count=100, out=out)
    assert got is out and bool((out[:2] == 7).all()) and bool((out[-7:] == 7).all())
    check_attend(p, k, v, b, lens, counts, Q, out, first=2)


def test_a_request_of_more_rows_than_announced_is_left_out():
    lens, counts = [100, 200, 50], [1, 30, 1]
    p, k, v, b = filled(30, lens, 2)
    Q, out = queries(31, 32, 2, 4), torch.full((32, 2, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    for most in (1, 2, 29):
        out.fill_(7.0)
        ws = pk.pages_workspace(p, most, 4)
        pk.pages_attend(p, Q, starts_of(counts), max_count=most, out=out, ws=ws, check=False)
        assert pk.arckv_query_status(ws) == 2 and bool((out[1:31] == 7).all())
        check_attend(p, k, v, b, lens, counts, Q, out, requests=[0, 2])


@pytest.mark.parametrize("n", [1, 40])
def test_masks_of_infinity_and_of_the_lowest_value(n):
    lens = [150, 150, 150]
    p, k, v, b = filled(40, lens, 2, bias=True)
    b = b.clone()
    b[:150] = -float("inf")                                  # nothing left
    b[150:300] = LOWEST                                      # everything equally far away
    b[300:400] = -float("inf")
    b[430:450] = LOWEST
    slots = torch.cat([p.table[s, torch.arange(150, device="cuda") // 64] * 64 + torch.arange(150, device="cuda") % 64 for s in range(3)])
    pk.pages_append(p, k, v, slots.to(torch.int32), bias=b)
    Q = queries(41, 3 * n, 2, 4)
    O = pk.pages_attend(p, Q, starts_of([n] * 3), max_count=n)
    assert not O[:n].any()
    check_attend(p, k, v, b, lens, [n] * 3, Q, O, requests=[0, 2])
    # with a bias that swallows every logit the weights are equal, over the tokens that a row sees
    for i in range(n):
        want = ref.held_rows(host(k), host(v))[1][150:300 - n + 1 + i, 0].mean(0)
        assert np.abs(host(O[n + i, 0, 0]) - want).max() <= 2.0 ** -7 * np.abs(want).max() + 2.0 ** -10


@pytest.mark.parametrize("n", [1, 50])
def test_missing_pages_and_pages_past_the_pool(n):
    p, k, v, b = filled(50, [300], 2)
    p.table[0, 1], p.table[0, 3] = -1, 10 ** 6
    Q = queries(51, n, 2, 4)
    ws = pk.pages_workspace(p, n, 4)
    O = pk.pages_attend(p, Q, starts_of([n]), max_count=n, ws=ws, check=False)
    assert pk.arckv_query_status(ws) == 1
    keep = [j for j in range(300) if j // 64 not in (1, 3)]
    for h in range(2):
        sees = np.repeat([sum(j < 300 - n + i + 1 for j in keep) for i in range(n)], 4)
        check_rows(O[:, h].reshape(-1, 128), Q[:, h].reshape(-1, 128), k[keep, h], v[keep, h], None, sees)


@pytest.mark.parametrize("n", [1, 4, 60])
def test_values_and_keys_of_every_size(n):
    """Pages that are large, ordinary, tiny and zero side by side; queries of every size with them."""
    T = 400
    p = pk.pages_alloc(1, 2, 8, T)
    _, slots, _ = pk.pages_extend(p, i32([T]), T)
    size = torch.tensor([1.0, 2.0 ** -40, 2.0 ** 30, 0.0, 1.0, 1e-30, 1.0]).cuda().repeat_interleave(64)[:T, None, None]
    k, v = rows(60, T, 2, torch.float32, outliers=False), rows(61, T, 2, torch.float32) * size
    pk.pages_append(p, k, v, slots)
    for q_size in (1.5, 1e-20, 3.0):
        Q = queries(62, n, 2, 4, q_size)
        O = pk.pages_attend(p, Q, starts_of([n]), max_count=n)
        check_attend(p, k, v, None, [T], [n], Q, O)
    pk.pages_append(p, k * 2.0 ** 20, v, slots)
    Q = queries(63, n, 2, 4, 2.0 ** -20)
    check_attend(p, k * 2.0 ** 20, v, None, [T], [n], Q, pk.pages_attend(p, Q, starts_of([n]), max_count=n))
    pk.pages_append(p, k * 2.0 ** -30, v, slots)
    Q = queries(64, n, 2, 4, 2.0 ** 30)
    check_attend(p, k * 2.0 ** -30, v, None, [T], [n], Q, pk.pages_attend(p, Q, starts_of([n]), max_count=n))


@pytest.mark.parametrize("n", [1, 40])
def test_a_row_that_one_token_takes(n):
    """Logits far apart: the weights of all but one token vanish."""
    T = 300
    p, k, v, b = filled(70, [T], 1)
    Q = (k[[10, 130, 299], None].repeat(n, 1, 1, 1)[:n] * 8).to(torch.bfloat16)
    O = pk.pages_attend(p, Q, starts_of([n]), max_count=n, causal=False)
    check_attend(p, k, v, b, [T], [n], Q, O, causal=False)


@pytest.mark.parametrize("n", [1, 40])
def test_strided_queries_and_outputs(n):
    lens, counts = [200, 77], [n, n]
    p, k, v, b = filled(80, lens, 3)
    wide = torch.randn(2 * n, 3 * 4 + 6, 128, generator=gen(81)).to(torch.bfloat16).cuda()
    Q = wide[:, :12].view(2 * n, 3, 4, 128)
    room = torch.zeros(2 * n, 4, 6, 128, dtype=torch.bfloat16, device="cuda")
    out = room[:, 1:, 1:5]
    pk.pages_attend(p, Q, starts_of(counts), max_count=n, out=out)
    check_attend(p, k, v, b, lens, counts, Q, out)
    assert not room[:, 0].any() and not room[:, :, 0].any() and not room[:, :, 5].any()


@pytest.mark.parametrize("n", [1, 30])
def test_calls_repeat_bit_for_bit(n):
    p, k, v, b = filled(90, [3000, 100, 5000], 4)
    Q, ws = queries(91, 3 * n, 4, 4), pk.pages_workspace(p, n, 4)
    first = pk.pages_attend(p, Q, starts_of([n] * 3), max_count=n, ws=ws)
    for _ in range(3):
        assert torch.equal(first, pk.pages_attend(p, Q, starts_of([n] * 3), max_count=n, ws=ws))


@pytest.mark.parametrize("n", [1, 20])
def test_many_requests(n):
    S = 700
    lens = torch.randint(1, 200, (S,), generator=gen(100)).tolist()
    counts = [min(n, x) for x in lens]
    p, k, v, b = filled(101, lens, 1)
    Q = queries(102, sum(counts), 1, 2)
    O = pk.pages_attend(p, Q, starts_of(counts), max_count=n)
    check_attend(p, k, v, b, lens, counts, Q, O, requests=[0, 1, 57, 300, 698, 699])


def test_more_requests_than_a_block_keeps_in_shared_memory():
    S = 1300
    lens = torch.randint(1, 150, (S,), generator=gen(105)).tolist()
    counts = [20 if s % 400 == 399 and lens[s] >= 20 else 1 for s in range(S)]
    p, k, v, b = filled(106, lens, 1)
    Q = queries(107, sum(counts), 1, 4)
    listed = [0, 399, 799, 1023, 1024, 1025, 1199, 1299]
    check_attend(p, k, v, b, lens, counts, Q, pk.pages_attend(p, Q, starts_of(counts), max_count=20), requests=listed)
    Q = queries(108, S, 1, 4)
    check_attend(p, k, v, b, lens, [1] * S, Q, pk.pages_attend(p, Q, starts_of([1] * S), max_count=1), requests=listed)


@pytest.mark.parametrize("n", [1, 3, 64])
def test_a_long_request(n):
    T = 20000
    p, k, v, b = filled(110, [T, 5], 2)
    Q = queries(111, n + 1, 2, 4)
    O = pk.pages_attend(p, Q, starts_of([n, 1]), max_count=n)
    check_attend(p, k, v, b, [T, 5], [n, 1], Q, O, heads=[1])


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("G", [2, 3, 5, 10])
def test_a_long_request_among_many_short_ones(G, bias):
    """Shares of all pages: a request's end, the next ones' whole and another's beginning; rows of both tiles or of one."""
    S, H = 60, 4
    lens = torch.randint(0, 200, (S,), generator=gen(112)).tolist()
    lens[0], lens[20], lens[21], lens[59] = 65, 30000, 6000, 4097
    counts = [min(T, 1 + s % 3) if s % 7 else 1 for s, T in enumerate(lens)]
    p, k, v, b = filled(113, lens, H, bias)
    Q = queries(114, sum(counts), H, G)
    ws = pk.pages_workspace(p, 3, G)
    for causal in (True, False):
        O = pk.pages_attend(p, Q, starts_of(counts), max_count=3, causal=causal, ws=ws)
        check_attend(p, k, v, b, lens, counts, Q, O, causal, heads=[0, 3])
    again = [pk.pages_attend(p, Q, starts_of(counts), max_count=3, ws=ws) for _ in range(8)]
    assert all(torch.equal(x, again[0]) for x in again)


def test_missing_pages_of_many_requests():
    S, H, T = 50, 4, 700
    p, k, v, b = filled(115, [T] * S, H)
    Q = queries(116, S, H, 4)
    gone = torch.arange(S, device="cuda") % 2 == 0
    p.table[gone, 2:5] = -1
    p.table[1, 3] = p.data.shape[0]
    starts, ws = starts_of([1] * S), pk.pages_workspace(p, 1, 4)
    O = pk.pages_attend(p, Q, starts, max_count=1, ws=ws, check=False)
    assert pk.arckv_query_status(ws) == 1
    for s in (0, 1, 2, 49):
        out = range(2, 5) if s % 2 == 0 else [3] if s == 1 else []
        held = [j for j in range(T) if j // 64 not in out]
        kk, vv = k[s * T:(s + 1) * T, 3][held], v[s * T:(s + 1) * T, 3][held]
        check_rows(O[s, 3], Q[s, 3], kk, vv, None, [len(held)] * 4)


def test_another_scale():
    p, k, v, b = filled(120, [90], 1)
    Q = queries(121, 1, 1, 4)
    O = pk.pages_attend(p, Q, starts_of([1]), 0.25)
    check_rows(O[0, 0], Q[0, 0], k[:, 0], v[:, 0], None, [90] * 4, scale=0.25)


# -------------------------------------------------------------------- rotation

def check_rotation(y, x, pos, r, **kw):
    """sincospi is good to 2 ulp and its argument to 2^-25 half turns: 2^-22 in all; three roundings more; bf16 outputs half a step."""
    turns = [int(t) % 2 ** 64 for t in r.turns]
    x, want = host(x), ref.rotate(host(x), pos.tolist(), turns, r.factor, r.interleaved, **kw)
    pair = np.abs(x).max(-1, keepdims=True) * max(1.0, r.factor)
    step = 2.0 ** -8 if y.dtype == torch.bfloat16 else 0.0
    assert np.all(np.abs(host(y) - want) <= pair * 2.0 ** -20 + np.abs(want) * step)


@pytest.mark.parametrize("N,Hq,H,d,width", [(1, 1, 0, 64, 64), (1, 32, 8, 128, 128), (5, 3, 2, 128, 32), (33, 4, 1, 256, 64), (700, 2, 2, 80, 48),
                                            (2500, 3, 1, 128, 128), (3, 1, 1, 512, 512), (6000, 1, 1, 16, 16)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotation(N, Hq, H, d, width, layout, dtype):
    r = pk.rotary(width, 10000.0, layout=layout)
    pos = torch.randint(-1, 140000, (N,), generator=gen(N)).to(torch.int32).cuda()
    q, k = torch.randn(N, Hq, d, generator=gen(1)).to(dtype).cuda(), torch.randn(N, H, d, generator=gen(2)).to(dtype).cuda()
    yq, yk = pk.rotate(r, pos, q, k)
    check_rotation(yq, q, pos, r)
    check_rotation(yk, k, pos, r)
    if width < d:
        assert torch.equal(yq[..., width:], q[..., width:])
    alone = pk.rotate(r, pos, q)
    assert torch.equal(alone, yq)
    back = pk.rotate(r, pos, q, transpose=True)
    check_rotation(back, q, pos, r, transpose=True)
    a, b = q.clone(), k.clone()
    same = pk.rotate(r, pos, a, b, out=(a, b))
    assert same[0] is a and torch.equal(a, yq) and torch.equal(b, yk)


def test_rotation_at_the_farthest_positions():
    r = pk.rotary(128, 500000.0, scaling={"kind": "ramp", "factor": 32, "fast": 32, "slow": 1, "context": 4096})
    pos = i32([0, 1, 2 ** 24 + 1, 2 ** 31 - 1, 2 ** 31 - 2, 123456789])
    x = torch.randn(6, 2, 128, generator=gen(4)).cuda()
    y = pk.rotate(r, pos, x)
    check_rotation(y, x, pos, r)
    assert r.factor > 1 and torch.allclose(y[0], x[0] * r.factor)


def test_rotation_gradient():
    """<g, R x> has the gradient R^T g: against the formula's, and against differences along random directions."""
    r = pk.rotary(64, layout="interleaved", scaling={"kind": "ramp", "factor": 4, "fast": 32, "slow": 1, "context": 4096})
    pos = torch.arange(7, dtype=torch.int32, device="cuda") * 1000
    x, g, e = (torch.randn(7, 3, 128, generator=gen(i)).cuda() for i in range(3))
    grad = pk.rotate(r, pos, g, transpose=True).double()
    f = lambda z: float((g.double() * pk.rotate(r, pos, z).double()).sum())
    size = float(g.norm() * e.norm()) * r.factor
    # the map is linear: a difference over a step of one is exact but for fp32 roundings, 2^-21 of each term's size
    assert abs(f(x + e) - f(x) - float((grad * e.double()).sum())) <= 2.0 ** -19 * (size + float(g.norm() * x.norm()) * r.factor)


def test_rotation_of_a_fused_projections_rows():
    r = pk.rotary(128)
    qkv = torch.randn(40, 12, 128, generator=gen(5)).to(torch.bfloat16).cuda()
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    q, k = pk.rotate(r, pos, qkv[:, :8].contiguous(), qkv[:, 8:10].contiguous())
    v = qkv[:, 10:].clone()
    pk.rotate(r, pos, qkv[:, :8], qkv[:, 8:10], out=(qkv[:, :8], qkv[:, 8:10]))
    assert torch.equal(qkv[:, :8], q) and torch.equal(qkv[:, 8:10], k) and torch.equal(qkv[:, 10:], v)


# ---------------------------------------------------- streams, graphs, together

def test_on_another_stream():
    p, k, v, b = filled(130, [400, 90], 2)
    Q, stream = queries(131, 2, 2, 4), torch.cuda.Stream()
    want = pk.pages_attend(p, Q, starts_of([1, 1]), max_count=1)
    r, pos = pk.rotary(128), i32([5, 9])
    turned = pk.rotate(r, pos, k[:2])
    stream.wait_stream(torch.cuda.current_stream())
    got = pk.pages_attend(p, Q, starts_of([1, 1]), max_count=1, stream=stream)
    also = pk.rotate(r, pos, k[:2], stream=stream)
    starts, slots, positions = pk.pages_extend(p, i32([1, 1]), 2, stream=stream)
    pk.pages_append(p, k[:2], v[:2], slots, stream=stream)
    back, _ = pk.pages_read(p, slots, stream=stream)
    pk.pages_truncate(p, i32([400, 90]), stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(want, got) and torch.equal(turned, also) and positions.tolist() == [400, 90]
    assert np.array_equal(host(back), host(torch.from_numpy(ref.held(host(k[:2]), 32).astype(np.float32)).to(torch.bfloat16)))


@pytest.mark.parametrize("n", [1, 24])
def test_a_serving_loop_in_a_replayed_graph(n):
    """Steps of rotation, tables, writes and attention, captured once and replayed while the requests grow."""
    S, H, G, steps = 5, 2, 4, 6
    lens = [0, 60, 64, 130, 500]
    r = pk.rotary(128, 500000.0)
    p, k, v, _ = filled(140, lens, H, spare=3 * S + steps * n * S // 64, M=20)
    held = {s: (k[sum(lens[:s]):sum(lens[:s + 1])], v[sum(lens[:s]):sum(lens[:s + 1])]) for s in range(S)}
    counts = i32([n, 1, 0, n, 1])
    c = counts.tolist()
    N = sum(c) + 3                                           # padded rows behind
    q_in, k_in, v_in = (torch.zeros(N, h, 128, dtype=torch.bfloat16, device="cuda") for h in (H * G, H, H))
    ws, out = pk.pages_workspace(p, n, G), torch.zeros(N, H, G, 128, dtype=torch.bfloat16, device="cuda")

    def step():
        starts, slots, positions = pk.pages_extend(p, counts, N, check=False)
        q, kk = pk.rotate(r, positions, q_in, k_in)
        pk.pages_append(p, kk, v_in, slots, check=False)
        pk.pages_attend(p, q.view(N, H, G, 128), starts, max_count=n, out=out, ws=ws, check=False)
        return q, kk

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                               # what a first call sets up
        pk.pages_truncate(p, i32(lens))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, kk = step()
    for i in range(steps):
        for x, seed in ((q_in, 1), (k_in, 2), (v_in, 3)):
            x.copy_(torch.randn(x.shape, generator=gen(10 * i + seed)))
        graph.replay()
        torch.cuda.synchronize()
        row = 0
        for s in range(S):
            held[s] = tuple(torch.cat([old, new[row:row + c[s]]]) for old, new in zip(held[s], (kk, v_in)))
            row += c[s]
    assert pk.arckv_query_status(p.state) == 0 and pk.arckv_query_status(ws) == 0
    now = [len(held[s][0]) for s in range(S)]
    assert p.len.tolist() == now and now == [a + steps * b for a, b in zip(lens, c)]
    pos = torch.cat([torch.arange(a - b, a) for a, b in zip(now, c)] + [torch.full((3,), -1)])
    check_rotation(kk, k_in, pos, r)
    K, V = (torch.cat([held[s][i] for s in range(S)]) for i in range(2))
    check_attend(p, K, V, None, now, c, q.view(N, H, G, 128), out)


def test_two_graphs_with_a_workspace_each_run_side_by_side():
    p, k, v, b = filled(150, [2000, 900], 2)
    st, graphs = starts_of([1, 1]), []
    for seed in (1, 2):
        Q, ws = queries(seed, 2, 2, 4), pk.pages_workspace(p, 1, 4)
        want = pk.pages_attend(p, Q, st, max_count=1)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = pk.pages_attend(p, Q, st, max_count=1, ws=ws, check=False)
        graphs.append((graph, want, got, ws, Q, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, *_, stream in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, want, got, ws, _, _ in graphs:
        assert torch.equal(want, got) and pk.arckv_query_status(ws) == 0


def test_single_tokens_without_an_announced_maximum():
    """N rows that could be one request's: the heavier path is there and finds nothing."""
    lens = [70, 3, 300, 1000, 64, 9]
    p, k, v, b = filled(160, lens, 2)
    Q = queries(161, 6, 2, 4)
    check_attend(p, k, v, b, lens, [1] * 6, Q, pk.pages_attend(p, Q, starts_of([1] * 6)))


def test_a_workspace_that_is_too_small_is_refused():
    p, k, v, b = filled(170, [70], 2)
    ws = pk.pages_workspace(p, 1, 4)
    with pytest.raises(pk.ArckvError):
        pk.pages_attend(p, queries(1, 64, 2, 4), starts_of([64]), max_count=64, ws=ws)


def test_pages_past_four_gigabytes():
    """Offsets of pages and of queries' and outputs' rows past 32 bits."""
    P, H, T = 60000, 8, 200
    p = pk.pages_alloc(2, H, P, 256)                                 # 4.5 GB
    p.free[:8] = torch.arange(P - 1, P - 9, -1, dtype=torch.int32, device="cuda")
    p.n_free.fill_(8)
    starts, slots, _ = pk.pages_extend(p, i32([T, T]), 2 * T)
    assert int(p.table.max()) == P - 1 and int(slots.min()) > (P - 9) * 64
    k, v = rows(180, 2 * T, H), rows(181, 2 * T, H, outliers=False)
    pk.pages_append(p, k, v, slots)
    K, V = pk.pages_read(p, slots, dtype=torch.float32)
    wk, wv = ref.held_rows(host(k), host(v))
    assert np.array_equal(host(K), wk.astype(np.float32)) and np.array_equal(host(V), wv.astype(np.float32))
    del K, V
    for n in (1, 30):
        step = (1 << 31) // (2 * n)                                  # elements between rows: the last is past 2^31 bytes, and 2^32
        base = torch.zeros(step * (2 * n - 1) + H * 4 * 128, dtype=torch.bfloat16, device="cuda")
        Q = base.as_strided((2 * n, H, 4, 128), (step // 8 * 8, 512, 128, 1))
        Q.copy_(queries(182, 2 * n, H, 4))
        room = torch.zeros_like(base)
        out = room.as_strided((2 * n, H, 4, 128), (step // 8 * 8, 512, 128, 1))
        pk.pages_attend(p, Q, starts_of([n, n]), max_count=n, out=out)
        check_attend(p, k, v, None, [T, T], [n, n], Q.contiguous(), out.contiguous(), heads=[0, 7])
        del base, room, Q, out


def test_the_serving_example():
    import sys
    from pathlib import Path
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
    import serve_4bit
    f = serve_4bit.main(["--requests", "5", "--longest", "700", "--chunk", "128", "--steps", "24"])
    assert f["pages_free_after"] == f["pages"] and 0 < f["pages_used"] <= f["pages"] and f["tokens"] > f["length"] > 0
    # values of a standard deviation of one in steps of their range / 15, about 5.4 / 15, are off by 5.4 / 15 / sqrt(12) = 0.10;
    # keys, in groups of 32, by 4.1 / 15 / sqrt(12) = 0.08, which moves logits of that size by 0.08 and weights alike: with
    # independent errors 0.13 of the outputs' size; twice that is never reached
    assert f["error"] < 0.26
