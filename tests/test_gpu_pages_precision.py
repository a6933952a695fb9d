"""How far outputs of the paged cache's attention are off, row by row, where single elements say little: attention spread over
thousands of tokens, whose outputs are far smaller than the values, values and queries of very different sizes side by side.

The error of a row is the norm of its difference from the plain form in 64 bits (over what the pages hold), relative to the
row's norm.  An output is a bf16: half a step is 2^-8 of an element, so 2^-8 of the norm at most.  Every rounding before it
(weights 2^-11; values 2^-11, in units of their page twice 2^-25, 2^-10 of an ordinary value beside one 2^6 to 2^7 larger; parts
of an item 2^-11; keys, which move a logit x by 2^-11 of sum |q k|) is independent of the others over thousands of
tokens, so that their norms add up in squares: below 2^-9 in all."""
import numpy as np
import pytest
import torch

from oracle import pages4 as ref
import paper_2609_36835_gb300 as pk

pytestmark = pytest.mark.gpu
SC = 1.0 / np.sqrt(128.0)
BOUND = 2.0 ** -8 + 2.0 ** -9


@pytest.fixture(scope="module", autouse=True)
def _gpu(lib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(seed, *shape):
    return torch.randn(*shape, generator=gen(seed))


def host(x):
    return x.detach().float().cpu().numpy()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def pages_of(k, v, bias=None):
    """Pages of one request that hold k, v [T, H, 128] and biases [T, H]."""
    T, H, _ = k.shape
    p = pk.pages_alloc(1, H, -(-T // 64), T, bias=bias is not None)
    _, slots, _ = pk.pages_extend(p, i32([T]), T)
    pk.pages_append(p, k.cuda(), v.cuda(), slots, bias=None if bias is None else bias.cuda())
    return p


def errors(O, Q, k, v, bias=None, rows=None, dims=slice(None), causal=True):
    """Relative errors of the (listed) rows of O [n, H, G, 128] over the given dims."""
    n, H, G, _ = O.shape
    T, out = len(k), []
    for h in range(H):
        K, V = ref.held_rows(host(k[:, h]), host(v[:, h]))
        for i in range(n) if rows is None else rows:
            sees = [T - n + 1 + i if causal else T] * G
            want = ref.attend(host(Q[i, h]), K, V, SC, sees, None if bias is None else host(bias[:, h]))[0][:, dims]
            diff = host(O[i, h]).astype(np.float64)[:, dims] - want
            out.append(np.linalg.norm(diff, axis=1) / np.linalg.norm(want, axis=1))
    return np.concatenate(out)


def attend(p, Q, n, **kw):
    return pk.pages_attend(p, Q, i32([0, n]), max_count=n, **kw)


ORDINARY = [i for i in range(128) if i != 7]


@pytest.mark.parametrize("outlier", [1, 16, 64])
@pytest.mark.parametrize("n,T", [(40, 8192), (40, 32768), (300, 8192), (300, 32768)])
def test_spread_attention_of_many_rows(n, T, outlier):
    """Items that many CTAs share; one channel of the values larger than the others, which are the ones that count."""
    k, v = randn(T, T, 2, 128), randn(T + 1, T, 2, 128)
    v[..., 7] *= outlier
    Q = (randn(n, n, 2, 1, 128) * 0.05).bfloat16().cuda()
    O = attend(pages_of(k, v), Q, n)
    assert errors(O, Q, k, v, rows=range(0, n, max(1, n // 20)), dims=ORDINARY).max() <= BOUND


@pytest.mark.parametrize("outlier", [1, 16, 64])
@pytest.mark.parametrize("n,T", [(1, 8192), (1, 131072), (7, 32768), (12, 8192), (16, 32768), (30, 8192)])
def test_spread_attention_of_few_rows(n, T, outlier):
    """The same, where a value's code, least value and scale enter apart."""
    k, v = randn(T, T, 1, 128), randn(T + 1, T, 1, 128)
    v[..., 7] *= outlier
    Q = (randn(n, n, 1, 1, 128) * 0.05).bfloat16().cuda()
    O = attend(pages_of(k, v), Q, n)
    assert errors(O, Q, k, v, rows=range(0, n, max(1, n // 6)), dims=ORDINARY).max() <= BOUND


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 2.0 ** 60, 2.0 ** -60])
@pytest.mark.parametrize("n", [2, 12, 40, 300])
def test_a_row_is_nothing_to_the_others(n, bad):
    """A row that holds an infinity, a NaN or an element far from the others' size: the other rows are what they are without it."""
    T = 1000
    k, v = randn(1, T, 2, 128), randn(2, T, 2, 128)
    p, Q = pages_of(k, v), randn(3, n, 2, 4, 128).bfloat16()
    ws, plain = pk.pages_workspace(p, n, 4), attend(p, Q.cuda(), n)
    Q[1, 0, 2], Q[n // 2, 1, 3, 9] = bad, bad
    O = attend(p, Q.cuda(), n, ws=ws, check=False)
    assert pk.arckv_query_status(ws) == (0 if bad < 1 else 5)
    keep = torch.ones(n, 2, 4, dtype=torch.bool)
    keep[1, 0, 2] = keep[n // 2, 1, 3] = False
    assert torch.equal(O[keep], plain[keep])
    if bad < 1:                                              # (a row of next to nothing sees all tokens alike)
        assert errors(O, Q, k, v, rows=[1, n // 2]).max() <= BOUND


def requests(S, k, v, n, bias=None):
    """Pages of S requests that hold k, v [T, H, 128] and biases [T, H] each, and starts of n rows for each: with as many items as SMs
    none is cut into many parts, which would each see little of what the others do."""
    T, H, _ = k.shape
    p = pk.pages_alloc(S, H, S * -(-T // 64), T, bias=bias is not None)
    _, slots, _ = pk.pages_extend(p, i32([T] * S), S * T)
    pk.pages_append(p, k.cuda().repeat(S, 1, 1), v.cuda().repeat(S, 1, 1), slots, bias=None if bias is None else bias.cuda().repeat(S, 1))
    return p, i32([n * s for s in range(S + 1)])


def check_requests(S, k, v, Q, bound, bias=None):
    """Q [n, H, G, 128], the same for every request."""
    n = len(Q)
    p, starts = requests(S, k, v, n, bias)
    O = pk.pages_attend(p, Q.cuda().repeat(S, 1, 1, 1), starts, max_count=n)
    for s in (0, S // 3, S - 1):
        e = errors(O[s * n:(s + 1) * n], Q, k, v, bias, rows=range(0, n, max(1, n // 5)))
        assert e.max() <= bound, (s, e.max())


@pytest.mark.parametrize("nats", [8, 12, 16])
@pytest.mark.parametrize("n,H", [(1, 8), (12, 8), (40, 8), (300, 4)])
def test_what_lies_far_below_a_token_of_no_value(n, H, nats):
    """An attention sink: its weight is e^nats of another token's, its value zero, so that the others are the output.  Keys as f16
    (many rows) move its logit, sum q k > 0, by 2^-11 of it twice, for their least values and for themselves, and so the sum."""
    T = 4096
    k, v = randn(1, T, H, 128) * 0.3, randn(2, T, H, 128) + 1.0
    d = torch.sign(randn(3, H, 128)) / 128 ** 0.5
    k -= (k * d).sum(-1, keepdim=True) * d
    k[0], v[0] = d * 8, 0.0
    q = randn(4, n, H, 1, 128) * 0.05
    q += (nats / 8 / SC - (q * d[:, None]).sum(-1, keepdim=True)) * d[:, None]
    check_requests(40, k, v, q.bfloat16(), BOUND + 2 * nats * 2.0 ** -11)


@pytest.mark.parametrize("size", [2.0 ** 8, 2.0 ** 20, 2.0 ** 40, 2.0 ** -20])
@pytest.mark.parametrize("n,H", [(1, 8), (12, 8), (40, 8), (300, 4)])
def test_values_behind_a_page_of_another_size(n, H, size):
    """The first page's values are larger (or smaller) and have next to no weight.  Behind it the peak is a token whose value is zero;
    the others of its page, 2^-6 of its weight each, are the output, and then pages 2^-12 of it."""
    T = 640
    k, v, b = randn(1, T, H, 128), randn(2, T, H, 128), torch.zeros(T, H)
    v[:64] *= size
    v[64] = 0.0
    b[:64], b[64], b[128:] = -100.0, 6 * np.log(2.0), -6 * np.log(2.0)
    check_requests(40, k, v, (randn(3, n, H, 1, 128) * 0.05).bfloat16(), BOUND, b)
    # the same without biases: by one dimension of the keys, whose rounding to f16, twice, moves logits of up to 4.2 by 2^-10 of them
    k[..., 0] = SC ** -1 / 16 * b
    k[:64, :, 1:] = 0.0
    q = randn(4, n, H, 1, 128) * 0.05
    q[..., 0] = 16.0
    check_requests(40, k, v, q.bfloat16(), BOUND + 2.0 ** -10 * 5)


@pytest.mark.parametrize("n", [1, 4, 12, 40])
def test_logits_past_the_range_are_recorded(n):
    """Logits of a standard deviation of 2^19 stay below 2^22, those of 2^26 pass it."""
    k, v = randn(1, 300, 2, 128), randn(2, 300, 2, 128)
    p, Q, ws = pages_of(k, v), randn(3, n, 2, 2, 128), None
    for size, status in ((2.0 ** 19, 0), (2.0 ** 26, 5), (2.0 ** 60, 5)):
        ws = pk.pages_workspace(p, n, 2)
        O = attend(p, (Q * size).bfloat16().cuda(), n, ws=ws, check=False)
        assert pk.arckv_query_status(ws) == status
        if status == 0:   # (one token of all but those that come near it)
            assert bool(torch.isfinite(O).all()) and bool((O.float().abs().amax(-1) > 0.5).all())
