"""The 8-bit cache on the GPU against its plain form (``oracle.cache8``), through the public calls.

Codes, scales, bounds and selected blocks are compared exactly: they are defined down to their roundings.  Attention
reads exact codes and exact bf16 queries, sums in 32 bits and keeps the softmax weights to 2^-22 or better.  A logit
of |q||k|/sqrt(d) up to 60 then carries at most 60 * 2^-23 = 7e-6, a weight the same relative error, and an output row
twice that: outputs are held to a relative 2-norm of 2e-5.
"""
import numpy as np
import pytest
import torch

from oracle import cache8 as ref
import paper_2609_36835_gb300 as pk

pytestmark = pytest.mark.gpu
TOL = 2e-5
SC = 1.0 / np.sqrt(128.0)
LOWEST = float(np.finfo(np.float32).min)


@pytest.fixture(scope="module", autouse=True)
def _gpu(lib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def rows(seed, S, H, n, dtype=torch.bfloat16, outliers=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(S, H, n, 128, generator=g)
    if outliers:
        x[..., 5] *= 6.0
        x *= 1.0 + 0.02 * torch.arange(n).view(1, 1, n, 1)   # magnitudes grow: blocks are quantised again
    return x.to(dtype).cuda()


def host(x):
    return x.detach().float().cpu().numpy()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


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


def filled(seed, lens, H, cap=None, bias=False, dtype=torch.bfloat16):
    """A cache whose sequences hold lens[s] tokens, written in one ragged call."""
    S, n = len(lens), max(max(lens), 1)
    c = pk.cache_alloc(S, H, cap or n, bias=bias)
    k, v = rows(seed, S, H, n, dtype), rows(seed + 1, S, H, n, dtype, outliers=False)
    b = None
    if bias:
        b = (torch.rand(S, H, n, generator=torch.Generator().manual_seed(seed + 2)) * 3 - 2).cuda()
    pk.cache_append(c, k, v, bias=b, counts=i32(lens))
    assert c.len.tolist() == list(lens)
    return c, k, v


def queries(seed, c, n_pos, G):
    g = torch.Generator().manual_seed(seed)
    S, H = c.K.shape[:2]
    return (torch.randn(S, H, n_pos, G, 128, generator=g) * 1.5).to(torch.bfloat16).cuda()


def rel(a, b):
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    return np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-300)


def check_attend(c, Q, O, causal=False, blocks=None, heads=None):
    S, H = Q.shape[:2]
    got, q = host(O), host(Q)
    for s, h in heads or [(s, h) for s in range(S) for h in range(H)]:
        K, ks, _, V, vs = held(c, s, h)
        T = len(K)
        bias = None if c.bias is None else host(c.bias[s, h, :T])
        bl = None if blocks is None else blocks[s, h].cpu().numpy()
        want = ref.attend(q[s, h], ref.values(K, ks), ref.values(V, vs), SC, bias, causal, bl)
        empty = ~want.any(-1)
        assert not got[s, h][empty].any()
        assert rel(got[s, h], want) <= TOL, (s, h, rel(got[s, h], want))


# ------------------------------------------------------------ write and read

@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 127, 128, 200, 643])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_write_matches_the_definition(T, dtype):
    k, v = rows(T, 2, 3, T, dtype), rows(T + 1, 2, 3, T, dtype)
    c = pk.cache_alloc(2, 3, T)
    pk.cache_append(c, k, v)
    assert c.len.tolist() == [T, T]
    for s in range(2):
        for h in range(3):
            assert_holds(c, s, h, k[s, h], v[s, h])


@pytest.mark.parametrize("cuts", [[1] * 70, [63, 1, 1, 63, 2], [10, 200, 1, 7], [64, 64, 3], [127, 66, 65]])
def test_content_does_not_depend_on_the_cuts(cuts):
    T = sum(cuts)
    k, v = rows(3, 2, 2, T), rows(4, 2, 2, T)
    c = pk.cache_alloc(2, 2, T)
    at = 0
    for n in cuts:
        pk.cache_append(c, k[:, :, at:at + n], v[:, :, at:at + n])   # strided views
        at += n
    for s in range(2):
        for h in range(2):
            assert_holds(c, s, h, k[s, h], v[s, h])


def test_ragged_counts_and_bias():
    lens = [0, 1, 64, 100, 129]
    c, k, v = filled(7, lens, 2, cap=192, bias=True)
    kept = c.bias.clone()
    more = [5, 64, 0, 29, 63]
    k2, v2 = rows(8, 5, 2, 64), rows(9, 5, 2, 64)
    pk.cache_append(c, k2, v2, counts=i32(more))                     # no biases given: zeros
    for s in range(5):
        assert int(c.len[s]) == lens[s] + more[s]
        for h in range(2):
            assert_holds(c, s, h, torch.cat([k[s, h, :lens[s]], k2[s, h, :more[s]]]),
                         torch.cat([v[s, h, :lens[s]], v2[s, h, :more[s]]]))
        assert torch.equal(c.bias[s, :, :lens[s]], kept[s, :, :lens[s]])
        assert not c.bias[s, :, lens[s]:lens[s] + more[s]].any()


def test_token_major_sources():
    """Keys and values as a fused projection leaves them: [S, n, 2, H, 128]."""
    S, n, H = 2, 70, 3
    kv = torch.randn(S, n, 2, H, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    k, v = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    c = pk.cache_alloc(S, H, n)
    pk.cache_append(c, k, v)
    for s in range(S):
        for h in range(H):
            assert_holds(c, s, h, k[s, h], v[s, h])


def test_rejected_tokens_are_written_over():
    """A draft of 5 tokens, of which 2 stay, then 3 others: the scale falls back with the rejected rows."""
    k, v = rows(11, 1, 2, 75, outliers=False), rows(12, 1, 2, 75)
    k[:, :, 72:75] *= 30.0
    c = pk.cache_alloc(1, 2, 128)
    pk.cache_append(c, k, v)
    k2, v2 = rows(13, 1, 2, 3, outliers=False), rows(14, 1, 2, 3)
    pk.cache_append(c, k2, v2, at=i32([72]))
    assert c.len.tolist() == [75]
    for h in range(2):
        assert_holds(c, 0, h, torch.cat([k[0, h, :72], k2[0, h]]), torch.cat([v[0, h, :72], v2[0, h]]))
    pk.cache_append(c, k2, v2, at=i32([64]))                          # back to a block's start
    assert c.len.tolist() == [67]
    for h in range(2):
        assert_holds(c, 0, h, torch.cat([k[0, h, :64], k2[0, h]]), torch.cat([v[0, h, :64], v2[0, h]]))


@pytest.mark.parametrize("bad", [dict(at=[70]), dict(at=[131]), dict(at=[-1]), dict(counts=[9]), dict(counts=[-1])])
def test_positions_that_cannot_be_written_are_reported(bad):
    """at inside an older block, past the end or negative; counts out of [0, n]: the sequence stays as it was."""
    c, k, v = filled(15, [130], 1, cap=192)
    with pytest.raises(pk.ArckvError) as e:
        pk.cache_append(c, rows(1, 1, 1, 8), rows(2, 1, 1, 8), **{n: i32(x) for n, x in bad.items()})
    assert e.value.code == 2 and c.len.tolist() == [130]
    assert_holds(c, 0, 0, k[0, 0], v[0, 0])
    pk.cache_append(c, rows(1, 1, 1, 8), rows(2, 1, 1, 8))            # the status was cleared
    assert c.len.tolist() == [138]


def test_a_full_cache_refuses_more():
    c, _, _ = filled(16, [60, 10], 1, cap=64)
    with pytest.raises(pk.ArckvError):
        pk.cache_append(c, rows(1, 2, 1, 5), rows(2, 2, 1, 5))
    assert c.len.tolist() == [60, 15]


def test_nonfinite_rows_and_tiny_blocks():
    k = torch.zeros(1, 1, 130, 128, device="cuda")
    k[0, 0, 64:] = 1e-38                                              # below the least magnitude
    k[0, 0, 128, 3] = float("nan")
    k[0, 0, 129, 4] = float("inf")
    k[0, 0, 129, 5] = 2.0
    c = pk.cache_alloc(1, 1, 130)
    pk.cache_append(c, k, k, check=False)
    assert pk.arckv_query_status(c.state) == 5 and pk.arckv_query_status(c.state) == 0
    clean = torch.where(torch.isfinite(k), k, torch.zeros_like(k))
    assert_holds(c, 0, 0, clean[0, 0], clean[0, 0])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("start,count", [(0, 200), (-64, 64), (-1, 1), (60, 9), (-300, 301), (190, 30)])
def test_read_back(start, count, dtype):
    lens = [0, 1, 64, 200]
    c, _, _ = filled(21, lens, 2)
    K, V = pk.cache_read(c, start, count, dtype=dtype)
    for s, T in enumerate(lens):
        for h in range(2):
            kc, ks, _, vc, vs = held(c, s, h)
            for got, codes, scale in ((K, kc, ks), (V, vc, vs)):
                val = codes.astype(np.float32) * np.repeat(scale, 64)[:T, None]
                want = np.zeros((count, 128), np.float32)
                for i in range(count):
                    j = (T if start < 0 else 0) + start + i
                    if 0 <= j < T:
                        want[i] = val[j]
                want = torch.from_numpy(want).to(dtype)
                assert torch.equal(got[s, h].cpu(), want)


# ------------------------------------------------------------------- attention

@pytest.mark.parametrize("G,n_pos,causal", [(1, 1, False), (4, 1, False), (3, 2, True), (8, 1, True), (4, 5, False),
                                            (5, 3, True), (16, 1, False), (4, 33, True), (8, 40, False)])
def test_attention_over_ragged_lengths(G, n_pos, causal):
    lens = [0, 1, 2, 63, 64, 65, 200, 331]
    c, _, _ = filled(31, lens, 2)
    Q = queries(32, c, n_pos, G)
    check_attend(c, Q, pk.cache_attend(c, Q, causal=causal), causal)


@pytest.mark.parametrize("n_pos,G", [(1, 4), (3, 4), (40, 4)])
def test_attention_with_biases_and_masks(n_pos, G):
    lens = [70, 70, 130, 192]
    c, _, _ = filled(41, lens, 2, bias=True)
    c.bias[0, 0, :] = -float("inf")                # a row that nothing is left of
    c.bias[0, 1, :64] = -float("inf")              # a whole block
    c.bias[1, 0, :70] = LOWEST                     # every entry the type's lowest value: uniform weights
    c.bias[1, 1, 3:69] = LOWEST
    c.bias[2, 0, 1::2] = -float("inf")
    Q = queries(42, c, n_pos, G)
    for causal in (False, True):
        check_attend(c, Q, pk.cache_attend(c, Q, causal=causal), causal)


def test_nan_bias_behind_the_end_is_not_read():
    c, _, _ = filled(43, [70], 1, bias=True)
    c.bias[:, :, 70:] = float("nan")
    c.k_scale[:, :, 2:] = float("nan")
    Q = queries(44, c, 1, 4)
    check_attend(c, Q, pk.cache_attend(c, Q))
    c.bias[0, 0, 5] = float("nan")                 # a visible one shows
    with pytest.raises(pk.ArckvError) as e:
        pk.cache_attend(c, Q)
    assert e.value.code == 5


@pytest.mark.parametrize("n_pos", [1, 2, 48])
def test_strided_queries_and_outputs(n_pos):
    """Queries as a projection leaves them [S, n_pos, H, G, 128], outputs written the same way."""
    c, _, _ = filled(51, [100, 64], 3)
    q = torch.randn(2, n_pos, 3, 4, 128, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    Q = q.transpose(1, 2)
    out = torch.full((2, n_pos, 3, 4, 128), float("nan"), device="cuda")
    O = pk.cache_attend(c, Q, out=out.transpose(1, 2))
    check_attend(c, Q, O)
    assert torch.equal(O, pk.cache_attend(c, Q.contiguous()))
    assert not torch.isnan(out).any()


def test_sharp_and_large_logits():
    """Logits of several hundred and one-hot rows; the largest key sits in the last block."""
    c, k, _ = filled(61, [300], 2)
    Q = (k[:, :, 299:300] * 4).view(1, 2, 1, 1, 128).expand(1, 2, 1, 4, 128).contiguous()
    O = host(pk.cache_attend(c, Q))
    for h in range(2):
        K, ks, _, V, vs = held(c, 0, h)
        want = ref.attend(host(Q[0, h]), ref.values(K, ks), ref.values(V, vs), SC)
        # logits near 2000: 2000 * 2^-23 relative error of a weight, twice for the row
        assert rel(O[0, h], want) <= 5e-4


def test_values_far_apart_in_magnitude():
    """Blocks of values 2^60 apart, zero blocks between: no weight or partial sum overflows."""
    n = 320
    k, v = rows(62, 1, 1, n, torch.float32), rows(63, 1, 1, n, torch.float32, outliers=False)
    v[0, 0, :64] *= 2.0 ** 60
    v[0, 0, 64:128] = 0.0
    v[0, 0, 128:192] *= 2.0 ** -60
    c = pk.cache_alloc(1, 1, n)
    pk.cache_append(c, k, v)
    Q = queries(64, c, 1, 4)
    check_attend(c, Q, pk.cache_attend(c, Q))


@pytest.mark.parametrize("n_pos", [1, 4, 32, 70])
@pytest.mark.parametrize("bias", [False, True])
def test_zero_queries_over_zero_keys(n_pos, bias):
    """All logits are zero, down to products of two factors of 2^-100: rows are means of the visible values."""
    n = 200
    k, v = torch.zeros(1, 2, n, 128, device="cuda"), rows(65, 1, 2, n, torch.float32)
    c = pk.cache_alloc(1, 2, n, bias=bias)
    pk.cache_append(c, k, v)
    Q = torch.zeros(1, 2, n_pos, 4, 128, device="cuda", dtype=torch.bfloat16)
    check_attend(c, Q, pk.cache_attend(c, Q, causal=True), True)


@pytest.mark.parametrize("n_pos", [4, 32, 70])
def test_values_far_apart_for_many_rows(n_pos):
    """As above in causal rows, of which the first see only small values."""
    n = 320
    k, v = rows(66, 1, 1, n, torch.float32), rows(67, 1, 1, n, torch.float32, outliers=False)
    v[0, 0, :64] = 0.0
    v[0, 0, 64:128] *= 2.0 ** -60
    v[0, 0, 256:] *= 2.0 ** 60
    c = pk.cache_alloc(1, 1, n)
    pk.cache_append(c, k, v)
    Q = queries(68, c, n_pos, 4)
    O = pk.cache_attend(c, Q, causal=True)
    check_attend(c, Q, O, True)
    K, ks, _, V, vs = held(c, 0, 0)
    want = ref.attend(host(Q[0, 0]), ref.values(K, ks), ref.values(V, vs), SC, None, True)
    assert rel(host(O[0, 0, 0]), want[0]) <= TOL      # each row by its own magnitude


@pytest.mark.parametrize("n_pos", [1, 4, 32, 70])
@pytest.mark.parametrize("bias", [False, True])
def test_zeros_weigh_beside_large_values(n_pos, bias):
    """Equal logits: a block of zeros takes its share of the weight, whatever the other block's magnitude."""
    k, v = torch.zeros(1, 1, 128, 128, device="cuda"), rows(69, 1, 1, 128, torch.float32, outliers=False)
    v[0, 0, :64] = 0.0
    v[0, 0, 64:] *= 2.0 ** 60
    c = pk.cache_alloc(1, 1, 128, bias=bias)
    pk.cache_append(c, k, v)
    Q = queries(70, c, n_pos, 4)
    check_attend(c, Q, pk.cache_attend(c, Q, causal=False))


@pytest.mark.parametrize("n_pos", [1, 4, 32, 70])
@pytest.mark.parametrize("n", [320, 6400])
def test_zeros_weigh_behind_large_values(n_pos, n):
    """As above with the zeros last, in one piece and in parts of several CTAs."""
    k, v = torch.zeros(1, 1, n, 128, device="cuda"), rows(71, 1, 1, n, torch.float32, outliers=False)
    v[0, 0, :64] *= 2.0 ** 60
    v[0, 0, 128:] = 0.0
    c = pk.cache_alloc(1, 1, n)
    pk.cache_append(c, k, v)
    Q = queries(72, c, n_pos, 4)
    check_attend(c, Q, pk.cache_attend(c, Q, causal=True), True)


@pytest.mark.parametrize("G,n_pos,bias", [(4, 1, False), (8, 1, False), (16, 1, True), (4, 8, False), (4, 40, True)])
def test_as_many_sequences_as_are_taken(G, n_pos, bias):
    S = 4096
    lens = [(37 * s) % 65 for s in range(S)]
    c, _, _ = filled(73, lens, 1, cap=64, bias=bias)
    Q = queries(74, c, n_pos, G)
    O = pk.cache_attend(c, Q)
    assert not host(O)[[s for s in range(S) if lens[s] == 0]].any()
    check_attend(c, Q, O, heads=[(s, 0) for s in (0, 1, 2, 63, 1000, 2047, 2048, 4094, 4095)])


@pytest.mark.parametrize("G,n_pos", [(4, 1), (4, 16), (8, 64)])
def test_long_sequences_split_over_the_device(G, n_pos):
    lens = [20001, 64 * 150, 17]
    c, _, _ = filled(71, lens, 2)
    Q = queries(72, c, n_pos, G)
    check_attend(c, Q, pk.cache_attend(c, Q, causal=True), True)
    assert torch.equal(pk.cache_attend(c, Q, causal=True), pk.cache_attend(c, Q, causal=True))


@pytest.mark.parametrize("G,n_pos,bias", [(4, 1, False), (8, 1, False), (4, 3, True), (16, 1, False), (3, 2, True)])
def test_rings_go_round(G, n_pos, bias):
    """Many blocks for each SM, for every number of rows of the decode kernel: the shared-memory ring is refilled."""
    lens = [24000, 19937, 23041]
    c, _, _ = filled(75, lens, 4, bias=bias)
    Q = queries(76, c, n_pos, G)
    O = pk.cache_attend(c, Q, causal=True)
    check_attend(c, Q, O, True, heads=[(0, 0), (1, 2), (2, 3)])
    assert torch.equal(O, pk.cache_attend(c, Q, causal=True))


def test_offsets_past_32_bits():
    """More than 2^32 bytes of codes: the last head of the last sequence, whose rows lie behind them."""
    S, H, cap = 5, 9, 1 << 20
    c = pk.cache_alloc(S, H, cap)
    assert c.K.numel() > 1 << 32
    lens = [0, 0, 64, 0, 130]
    k, v = rows(81, S, H, 130), rows(82, S, H, 130)
    pk.cache_append(c, k, v, counts=i32(lens))
    assert_holds(c, 4, 8, k[4, 8], v[4, 8])
    c.len[4] = cap                                                    # the tail of the longest sequence
    c.K[4], c.V[4] = 128, 128
    c.k_scale[4], c.v_scale[4] = 1e-3, 1e-3
    c.bounds[4] = 0
    c.K[4, 8, cap - 1], c.V[4, 8, cap - 1] = 255, 200
    c.bounds[4, 8, cap // 64 - 1, 1] = 127
    c.k_scale[4, 8, cap // 64 - 1] = 1.0
    Q = torch.ones(S, H, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    O = pk.cache_attend(c, Q)
    want = 72 * 1e-3                                                  # the one large logit takes all the weight
    assert torch.allclose(O[4, 8], torch.full_like(O[4, 8], want), rtol=1e-6)
    assert not O[4, 7].any() and not O[3].any()
    b = pk.cache_select(c, Q, 3, keep_first=0, keep_last=0)
    assert b[4, 8, 0].tolist() == [0, 1, cap // 64 - 1]
    K, _ = pk.cache_read(c, -1, 1, dtype=torch.float32)
    assert torch.equal(K[4, 8, 0], torch.full((128,), 127.0, device="cuda"))


# --------------------------------------------------------- selection, sparse

@pytest.mark.parametrize("m,first,last", [(1, 0, 0), (2, 1, 1), (7, 1, 2), (16, 0, 3), (40, 1, 1)])
@pytest.mark.parametrize("G,n_pos,causal", [(4, 1, False), (1, 3, True), (8, 70, True)])
def test_selected_blocks_are_exact(m, first, last, G, n_pos, causal):
    lens = [0, 1, 64, 700, 2050]
    c, _, _ = filled(91, lens, 2)
    Q = queries(92, c, n_pos, G)
    got = pk.cache_select(c, Q, m, keep_first=first, keep_last=last, causal=causal).cpu().numpy()
    q = host(Q)
    for s, T in enumerate(lens):
        for h in range(2):
            _, ks, bounds, _, _ = held(c, s, h)
            assert np.array_equal(got[s, h], ref.select(q[s, h], bounds, ks, T, m, first, last, causal)), (s, h)


@pytest.mark.parametrize("n,m", [(20000, 9), (20000, 300), (140000, 100)])
def test_ties_go_to_the_lower_block(n, m):
    """Blocks of three kinds, many equal: the order among equals is the index."""
    kind = torch.randint(0, 3, (1, 2, -(-n // 64)), generator=torch.Generator().manual_seed(1))
    base = rows(93, 1, 1, 3 * 64, outliers=False).view(1, 1, 3, 64, 128)
    k = torch.stack([base[0, 0, kind[0, h].cuda()].view(-1, 128)[:n] for h in range(2)])[None]
    c = pk.cache_alloc(1, 2, n)
    pk.cache_append(c, k, k)
    Q = queries(94, c, 2, 4)
    got = pk.cache_select(c, Q, m).cpu().numpy()
    for h in range(2):
        _, ks, bounds, _, _ = held(c, 0, h)
        assert np.array_equal(got[0, h], ref.select(host(Q[0, h]), bounds, ks, n, m, 1, 1, False))


def test_zero_queries_select_the_lowest_blocks():
    c, _, _ = filled(95, [1000], 1)
    Q = torch.zeros(1, 1, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    assert pk.cache_select(c, Q, 4, keep_first=0, keep_last=1).flatten().tolist() == [0, 1, 2, 15]
    Q[0, 0, 0, 0, 0] = -0.0
    assert pk.cache_select(c, Q, 4, keep_first=0, keep_last=0).flatten().tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("G,n_pos,m", [(4, 1, 5), (4, 17, 3), (1, 2, 40), (12, 3, 8), (20, 1, 4)])
def test_sparse_attention_over_the_selected_blocks(G, n_pos, m):
    lens = [0, 5, 64, 700, 2050]
    c, _, _ = filled(101, lens, 2)
    Q = queries(102, c, n_pos, G)
    causal = n_pos > 1
    blocks = pk.cache_select(c, Q, m, causal=causal) if m > 1 else None
    check_attend(c, Q, pk.cache_attend(c, Q, blocks=blocks, causal=causal), causal, blocks)


def test_sparse_attention_over_any_list():
    """Unordered lists with gaps, blocks behind the end, lists of nothing; an index past the cache is reported."""
    c, _, _ = filled(103, [700, 30], 2, bias=True)
    Q = queries(104, c, 2, 4)
    blocks = torch.full((2, 2, 2, 6), -1, dtype=torch.int32, device="cuda")
    blocks[0, 0, 0] = i32([10, -1, 3, 0, -1, 7])
    blocks[0, 0, 1] = i32([-1, -1, -1, -1, -1, 2])
    blocks[1, 1, 0] = i32([5, 0, -1, -1, 3, -1])
    check_attend(c, Q, pk.cache_attend(c, Q, blocks=blocks), False, blocks)
    blocks[0, 1, 0, 2] = 11                                           # capacity 704: blocks 0 .. 10
    ws = pk.cache_workspace(c, 2, 4)
    O = pk.cache_attend(c, Q, blocks=blocks, ws=ws, check=False)
    assert pk.arckv_query_status(ws) == 1
    check_attend(c, Q, O, False, blocks)


def test_every_block_listed_equals_dense():
    c, _, _ = filled(105, [515], 2)
    Q = queries(106, c, 1, 4)
    blocks = torch.arange(9, dtype=torch.int32, device="cuda").expand(1, 2, 1, 9).contiguous()
    assert rel(host(pk.cache_attend(c, Q, blocks=blocks)), host(pk.cache_attend(c, Q))) <= TOL


# ------------------------------------------------------------ use in programs

def test_another_stream():
    c, k, v = filled(111, [100], 2, cap=192)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    Q, k2, v2 = queries(112, c, 1, 4), rows(113, 1, 2, 3), rows(114, 1, 2, 3)
    side.wait_stream(torch.cuda.current_stream())
    pk.cache_append(c, k2, v2, stream=side, check=False)
    b = pk.cache_select(c, Q, 2, stream=side, check=False)
    O = pk.cache_attend(c, Q, blocks=b, stream=side.cuda_stream, check=False)
    side.synchronize()
    assert c.len.tolist() == [103]
    check_attend(c, Q, O, False, b)


def test_decode_loop_in_a_graph():
    """One captured step (write a token, select, attend) replayed while the cache grows past block ends."""
    c, k, v = filled(121, [62, 3], 2, cap=256)
    n = 70
    ks, vs = rows(122, 2, 2, n), rows(123, 2, 2, n)
    Q, ws = queries(124, c, 1, 4), pk.cache_workspace(c, 1, 4)
    kin, vin = ks[:, :, :1].clone(), vs[:, :, :1].clone()
    dense, sparse = torch.empty(2, 2, 1, 4, 128, device="cuda"), torch.empty(2, 2, 1, 4, 128, device="cuda")

    def step():
        pk.cache_append(c, kin, vin, check=False)
        b = pk.cache_select(c, Q, 2, ws=ws, check=False)
        pk.cache_attend(c, Q, ws=ws, out=dense, check=False)
        pk.cache_attend(c, Q, blocks=b, ws=ws, out=sparse, check=False)
        return b

    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        step()
    torch.cuda.current_stream().wait_stream(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b = step()
    for i in range(1, n):
        kin.copy_(ks[:, :, i:i + 1])
        vin.copy_(vs[:, :, i:i + 1])
        graph.replay()
    torch.cuda.synchronize()
    assert c.len.tolist() == [62 + n, 3 + n]
    for s, T in enumerate((62, 3)):
        assert_holds(c, s, 1, torch.cat([k[s, 1, :T], ks[s, 1]]), torch.cat([v[s, 1, :T], vs[s, 1]]))
    check_attend(c, Q, dense)
    check_attend(c, Q, sparse, False, b)
    assert pk.arckv_query_status(ws) == 0 and pk.arckv_query_status(c.state) == 0


def test_compact_cache_in_8_bits():
    """What arckv_compact leaves (fp32 rows, beta) held in 8 bits stays close to the compact operator itself."""
    g = torch.Generator().manual_seed(131)
    H, t = 2, 409
    C_k, C_v = torch.randn(H, t, 128, generator=g).cuda(), torch.randn(H, t, 128, generator=g).cuda()
    beta = (torch.rand(H, t, generator=g) * 3 - 2).cuda()
    c = pk.cache_alloc(1, H, t, bias=True)
    pk.cache_append(c, C_k[None], C_v[None], bias=beta[None])
    Q = queries(132, c, 1, 4)
    O = pk.cache_attend(c, Q)
    check_attend(c, Q, O)
    full = pk.attend(Q.view(H, 4, 128), C_k, beta, C_v)
    # a code is off by at most half a step of a / 127 with a near 4.4: about 0.5 % of a value's magnitude
    assert rel(host(O).reshape(H, 4, 128), host(full)) <= 0.03


def test_example_runs_them_together():
    """The decode example: compaction, 8-bit caches, selection and attention in a replayed graph."""
    import importlib.util
    from pathlib import Path
    path = Path(__file__).resolve().parent.parent / "examples" / "decode_8bit.py"
    spec = importlib.util.spec_from_file_location("decode_8bit", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    f = mod.main(["--context", "1500", "--steps", "70", "--blocks", "24"])
    assert f["tokens"] == 1570 and f["compact_tokens"] == 220
    # a code is off by at most half a step: 0.5 / 127 of a block's magnitude, which outlier channels of 8 times the rest
    # (keys) and single values of 4 deviations (values) set; logits of |q||k|/sqrt(d) up to 60 move by a few tenths
    assert max(f["full_error"], f["compact_error"], f["sparse_error"]) <= 0.2
