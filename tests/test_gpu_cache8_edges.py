"""Edges of the 8-bit cache's calls on the GPU, against its plain form (``oracle.cache8``) as in test_gpu_cache8:
codes, scales, bounds and chosen blocks exactly, attention to a relative 2e-5."""
import numpy as np
import pytest
import torch

from oracle import cache8 as ref
import paper_2609_36835_gb300 as pk

pytestmark = pytest.mark.gpu
TOL = 2e-5
SC = 1.0 / np.sqrt(128.0)


@pytest.fixture(scope="module", autouse=True)
def _gpu(lib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def rows(seed, S, H, n, dtype=torch.bfloat16, grow=0.02):
    """Rows with one strong channel, whose magnitudes grow: blocks are quantised again."""
    x = torch.randn(S, H, n, 128, generator=torch.Generator().manual_seed(seed))
    x[..., 5] *= 6.0
    x *= 1.0 + grow * torch.arange(n).view(1, 1, n, 1)
    return x.to(dtype).cuda()


def biases(seed, *shape):
    return (torch.rand(*shape, generator=torch.Generator().manual_seed(seed)) * 3 - 2).cuda()


def queries(seed, S, H, n_pos, G):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(S, H, n_pos, G, 128, generator=g) * 1.5).to(torch.bfloat16).cuda()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def host(x):
    return x.detach().float().cpu().numpy()


def held(c, s, h):
    """Codes, scales and bounds of the tokens that one head holds."""
    T = int(c.len[s])
    nb = -(-T // 64)
    code = lambda x: (x[s, h, :T].cpu().numpy().astype(np.int16) - 128).astype(np.int8)
    return (code(c.K), host(c.k_scale[s, h, :nb]), c.bounds[s, h, :nb].cpu().numpy(), code(c.V),
            host(c.v_scale[s, h, :nb]))


def assert_holds(c, s, h, k, v):
    """The head holds exactly the rows k, v [T, 128]."""
    K, ks, bounds, V, vs = held(c, s, h)
    for got, want in zip((K, ks, bounds), ref.quantise(host(k))):
        assert np.array_equal(got, want)
    for got, want in zip((V, vs), ref.quantise(host(v))[:2]):
        assert np.array_equal(got, want)


def check_attend(c, Q, O, causal=False, blocks=None):
    got, q = host(O).astype(np.float64), host(Q)
    for s in range(Q.shape[0]):
        for h in range(Q.shape[1]):
            K, ks, _, V, vs = held(c, s, h)
            bias = None if c.bias is None else host(c.bias[s, h, :len(K)])
            bl = None if blocks is None else blocks[s, h].cpu().numpy()
            want = ref.attend(q[s, h], ref.values(K, ks), ref.values(V, vs), SC, bias, causal, bl)
            assert not got[s, h][~want.any(-1)].any()
            err = np.linalg.norm(got[s, h] - want) / max(np.linalg.norm(want), 1e-300)
            assert err <= TOL, (s, h, err)


# ----------------------------------------------------------------- writing

LENS = [0, 1, 55, 57, 60, 62, 63, 64, 127]


@pytest.mark.parametrize("n", [2, 5, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("grow", [0.02, 0.0])
def test_few_rows_over_a_block_end(n, dtype, grow):
    """Calls of 2 to 8 rows that end in the block where they began, with its end, or in the next, with biases."""
    S, H, most = len(LENS), 2, max(LENS)
    k, v = rows(1, S, H, most + 3 * n, dtype, grow), rows(2, S, H, most + 3 * n, dtype, 0.0)
    b = biases(3, S, H, most + 3 * n)
    c = pk.cache_alloc(S, H, most + 3 * n, bias=True)
    pk.cache_append(c, k[:, :, :most], v[:, :, :most], bias=b[:, :, :most].contiguous(), counts=i32(LENS))
    part = lambda x, i: torch.stack([x[s, :, t + i * n:t + (i + 1) * n] for s, t in enumerate(LENS)])
    for i in range(3):
        pk.cache_append(c, part(k, i), part(v, i), bias=part(b, i))
    for s, t in enumerate(LENS):
        T = t + 3 * n
        assert int(c.len[s]) == T
        assert torch.equal(c.bias[s, :, :T], b[s, :, :T])
        for h in range(H):
            assert_holds(c, s, h, k[s, h, :T], v[s, h, :T])


def test_few_rows_without_biases_clear_them():
    c = pk.cache_alloc(1, 2, 192, bias=True)
    k, b = rows(4, 1, 2, 68), biases(5, 1, 2, 60)
    c.bias.fill_(float("nan"))
    pk.cache_append(c, k[:, :, :60], k[:, :, :60], bias=b)
    pk.cache_append(c, k[:, :, 60:], k[:, :, 60:])
    assert torch.equal(c.bias[:, :, :60], b) and not c.bias[:, :, 60:68].any()
    assert torch.isnan(c.bias[:, :, 68:]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_rows_that_are_not_finite(dtype):
    """They are written as zeros on both sides of a block's end, staged as zeros, and reported."""
    k, v = rows(6, 1, 2, 68, dtype), rows(7, 1, 2, 68, dtype)
    c = pk.cache_alloc(1, 2, 128)
    pk.cache_append(c, k[:, :, :61], v[:, :, :61])
    bad, worse = k[:, :, 61:].clone(), v[:, :, 61:].clone()
    bad[0, 0, 1, 5], bad[0, 1, 5, 0], worse[0, 1, 2, 127] = float("nan"), float("inf"), -float("inf")
    pk.cache_append(c, bad, worse, check=False)
    assert pk.arckv_query_status(c.state) == 5
    clean = lambda x: torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    more = rows(8, 1, 2, 3, dtype) * 20                       # the newest block's staged rows are quantised again
    pk.cache_append(c, more, more)
    for h in range(2):
        assert_holds(c, 0, h, torch.cat([k[0, h, :61], clean(bad[0, h]), more[0, h]]),
                     torch.cat([v[0, h, :61], clean(worse[0, h]), more[0, h]]))


@pytest.mark.parametrize("n", [3, 8, 9, 70, 200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_written_over_earlier_ones(n, dtype):
    """at within the newest block, at its first row and at an earlier block's, for few rows and for many; the rows that
    go were the largest of their blocks."""
    T = 150
    ats = [140, 129, 128, 64, 0, 150, 149]
    S, H = len(ats), 2
    k, v = rows(9, S, H, T, dtype, grow=0.2), rows(10, S, H, T, dtype, grow=0.2)
    k2, v2 = rows(11, S, H, n, dtype, grow=0.0), rows(12, S, H, n, dtype, grow=0.0)
    b, b2 = biases(13, S, H, T), biases(14, S, H, n)
    c = pk.cache_alloc(S, H, T + n, bias=True)
    pk.cache_append(c, k, v, bias=b)
    pk.cache_append(c, k2, v2, bias=b2, at=i32(ats))
    more = rows(15, S, H, 2, dtype, grow=0.0)
    pk.cache_append(c, more, more)                            # what is staged is the newest block
    for s, at in enumerate(ats):
        assert int(c.len[s]) == at + n + 2
        assert torch.equal(c.bias[s, :, :at + n], torch.cat([b[s, :, :at], b2[s]], 1))
        for h in range(H):
            assert_holds(c, s, h, torch.cat([k[s, h, :at], k2[s, h], more[s, h]]),
                         torch.cat([v[s, h, :at], v2[s, h], more[s, h]]))


# --------------------------------------------------------------- attention

@pytest.mark.parametrize("G", [17, 20, 24, 33, 40])
@pytest.mark.parametrize("behind", [float("nan"), float("inf")])
def test_rows_that_do_not_exist_report_nothing(G, behind):
    """Listed blocks, and query heads that leave a tile of 8 rows empty: what lies behind the end is nobody's."""
    c = pk.cache_alloc(1, 2, 192, bias=True)
    pk.cache_append(c, rows(21, 1, 2, 70), rows(22, 1, 2, 70, grow=0.0), bias=biases(23, 1, 2, 70))
    c.bias[:, :, 70:] = behind
    Q = queries(24, 1, 2, 1, G)
    blocks = i32([0, 1, -1]).expand(1, 2, 1, 3).contiguous()
    check_attend(c, Q, pk.cache_attend(c, Q, blocks=blocks), False, blocks)


def large(seed, n, exponent, most=4.0):
    """Positive values up to 2^(exponent + 2): sums of them do not cancel."""
    x = torch.randn(1, 1, n, 128, generator=torch.Generator().manual_seed(seed)).abs().clamp(0.25, most)
    return (x * 2.0 ** exponent).cuda()


@pytest.mark.parametrize("n_pos", [16, 70])
@pytest.mark.parametrize("exponent", [100, 110, 118, 125])
@pytest.mark.parametrize("bias", [False, True])
def test_large_values_in_many_rows(n_pos, exponent, bias):
    n = 320
    c = pk.cache_alloc(1, 1, n, bias=bias)
    pk.cache_append(c, rows(25, 1, 1, n, grow=0.0).float(), large(26, n, exponent), bias=biases(27, 1, 1, n) if bias else None)
    Q = queries(28, 1, 1, n_pos, 4)
    check_attend(c, Q, pk.cache_attend(c, Q, causal=True), True)


@pytest.mark.parametrize("n_pos", [16, 70])
@pytest.mark.parametrize("n", [320, 6400])
@pytest.mark.parametrize("order", [[0, 1, 2, 3, 4], [4, 3, 2, 1, 0], [2, 0, 4, 1, 3]])
@pytest.mark.parametrize("bias", [False, True])
def test_magnitudes_from_end_to_end_in_many_rows(n_pos, n, order, bias):
    """Zeros, ordinary values and the largest ones in one sequence, equal logits but for biases: each takes its share."""
    v = large(29, n, 0)
    for b in range(n // 64):
        v[:, :, 64 * b:64 * (b + 1)] *= [0.0, 2.0 ** -60, 1.0, 2.0 ** 60, 2.0 ** 123][order[b * 5 * 64 // n]]
    c = pk.cache_alloc(1, 1, n, bias=bias)
    pk.cache_append(c, torch.zeros_like(v), v, bias=biases(36, 1, 1, n) * 4 / 3 if bias else None)
    Q = queries(30, 1, 1, n_pos, 4)
    check_attend(c, Q, pk.cache_attend(c, Q, causal=False))


@pytest.mark.parametrize("n_pos", [16, 33])
@pytest.mark.parametrize("order", [[0, 4, 1, 3, 2], [4, 2, 0, 3, 1]])
@pytest.mark.parametrize("bias", [False, True])
def test_magnitudes_side_by_side_in_many_rows(n_pos, order, bias):
    """As above with several blocks of one sequence for each SM, so that one follows the other in the same sums."""
    n = 64 * 5 * torch.cuda.get_device_properties(0).multi_processor_count
    v = large(37, n, 0).view(1, 1, n // 64, 64, 128)
    for i, k in enumerate(order):
        v[:, :, i::5] *= [0.0, 2.0 ** -60, 1.0, 2.0 ** 60, 2.0 ** 123][k]
    v = v.view(1, 1, n, 128)
    c = pk.cache_alloc(1, 1, n, bias=bias)
    pk.cache_append(c, torch.zeros_like(v), v, bias=biases(38, 1, 1, n) * 4 / 3 if bias else None)
    Q = queries(39, 1, 1, n_pos, 4)
    check_attend(c, Q, pk.cache_attend(c, Q, causal=False))


@pytest.mark.parametrize("G,n_pos", [(4, 1), (8, 1), (4, 4)])
@pytest.mark.parametrize("n,exponent", [(320, 118), (6400, 112), (131072, 105)])
@pytest.mark.parametrize("bias", [False, True])
def test_large_values_in_few_rows(G, n_pos, n, exponent, bias):
    """Equal logits: every token weighs the same, and their sum is below 2^126."""
    v = large(31, n, exponent, most=3.0)
    c = pk.cache_alloc(1, 1, n, bias=bias)
    pk.cache_append(c, torch.zeros_like(v), v)
    Q = queries(32, 1, 1, n_pos, G)
    check_attend(c, Q, pk.cache_attend(c, Q))


@pytest.mark.parametrize("G,n_pos", [(4, 1), (8, 1), (4, 4)])
def test_large_values_in_listed_blocks(G, n_pos):
    v = large(33, 640, 116)
    c = pk.cache_alloc(1, 1, 640)
    pk.cache_append(c, rows(34, 1, 1, 640, grow=0.0).float(), v)
    Q = queries(35, 1, 1, n_pos, G)
    blocks = i32([0, 3, 4, 9]).expand(1, 1, n_pos, 4).contiguous()
    check_attend(c, Q, pk.cache_attend(c, Q, blocks=blocks), False, blocks)


# --------------------------------------------------------------- selection

@pytest.mark.parametrize("T", [0, 1, 64, 700])
def test_one_block_is_the_newest(T):
    """m = 1 leaves no room for the first block beside the newest one."""
    c = pk.cache_alloc(1, 2, 704)
    if T:
        pk.cache_append(c, rows(44, 1, 2, T), rows(45, 1, 2, T))
    Q = queries(46, 1, 2, 3, 4)
    for causal in (False, True):
        got = pk.cache_select(c, Q, 1, causal=causal).cpu().numpy()
        for h in range(2):
            _, ks, bounds, _, _ = held(c, 0, h)
            assert np.array_equal(got[0, h], ref.select(host(Q[0, h]), bounds, ks, T, 1, 0, 1, causal))
