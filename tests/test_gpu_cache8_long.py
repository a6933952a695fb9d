"""Many-row attention over the 8-bit cache where one CTA holds many blocks of an item: its outputs then go to sums in
memory every 32 blocks and start again.  Compared with the same attention in 64 bits on the device, to the bound of
test_gpu_cache8 (2e-5 for logits up to 60).

An item is (sequence, head, 128 or 256 rows); equal shares of all blocks go to as many CTAs as the GPU has SMs, so the
sizes below give a CTA over 96 blocks of an item in pieces that begin anywhere, or exactly 32, 33 or 65.
"""
import math

import pytest
import torch

import paper_2609_36835_gb300 as pk

pytestmark = pytest.mark.gpu
TOL = 2e-5
GROW = 50.0      # a logit's growth: 72 in powers of two, past the 60 up to which earlier sums keep their reference


@pytest.fixture(scope="module", autouse=True)
def _gpu(lib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def cache_of(seed, S, H, n, bias=False, grown=None):
    """S x H heads of n tokens; from token grown[h] on, keys of head h have a large dimension 3."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c = pk.cache_alloc(S, H, n, bias=bias)
    k, v = normal(g, S, H, n, 128), normal(g, S, H, n, 128)
    k[..., 3] = 0.0
    for h, t in enumerate(grown or []):
        k[:, h, t:, 3] = GROW * math.sqrt(128.0) / 4.0
    b = torch.rand(S, H, n, generator=g, device="cuda") * 3 - 2 if bias else None
    pk.cache_append(c, k.to(torch.bfloat16), v.to(torch.bfloat16), bias=b)
    return c, g


def queries(g, S, H, n_pos, G):
    """Rows of odd query heads (with one query head: of odd positions) see the large dimension, the others do not."""
    q = normal(g, S, H, n_pos, G, 128)
    q[..., 3] = 0.0
    odd = q[:, :, :, 1::2] if G > 1 else q[:, :, 1::2]
    odd[..., 3] = 4.0
    return q.to(torch.bfloat16)


def exact(c, Q, s, h, causal):
    """O [n_pos, G, 128] of one head in 64 bits."""
    T, (n_pos, G) = int(c.len[s]), Q.shape[2:4]
    step = torch.arange(T, device="cuda") // 64
    k = (c.K[s, h, :T].double() - 128) * c.k_scale[s, h].double()[step, None]
    v = (c.V[s, h, :T].double() - 128) * c.v_scale[s, h].double()[step, None]
    a = Q[s, h].double().view(-1, 128) @ k.T / math.sqrt(128.0)
    if c.bias is not None:
        a += c.bias[s, h, :T].double()
    if causal:
        sees = (T - n_pos + 1 + torch.arange(n_pos, device="cuda")).repeat_interleave(G)
        a.masked_fill_(torch.arange(T, device="cuda") >= sees[:, None], -math.inf)
    top = a.amax(1, keepdim=True)
    e = torch.exp(a - torch.where(torch.isinf(top), 0.0, top))
    z = e.sum(1, keepdim=True)
    return (e @ v / torch.where(z == 0, 1.0, z)).view(n_pos, G, 128)


def check(c, Q, causal, heads):
    O = pk.cache_attend(c, Q, causal=causal)
    for s, h in heads:
        want = exact(c, Q, s, h, causal)
        got = O[s, h].double()
        err = ((got - want).norm(dim=-1) / want.norm(dim=-1).clamp_min(1e-300)).amax()
        assert float(err) <= TOL, (s, h, float(err))         # each row by its own magnitude
        assert not got[want.norm(dim=-1) == 0].any()
    assert torch.equal(O, pk.cache_attend(c, Q, causal=causal))


ONE_TILE, TWO_TILES = (8, 8, 8, 4), (1, 8, 256, 8)          # sequences, heads, positions, query heads
HEADS = {ONE_TILE: [(0, 0), (0, 1), (3, 2), (5, 5), (7, 7)], TWO_TILES: [(0, 0), (0, 1), (0, 2), (0, 5), (0, 7)]}


@pytest.mark.parametrize("shape", [ONE_TILE, (8, 8, 32, 4), TWO_TILES])
@pytest.mark.parametrize("bias", [False, True])
def test_sums_over_many_blocks(shape, bias):
    S, H, n_pos, G = shape
    c, g = cache_of(1, S, H, 16384 - 5, bias)
    check(c, queries(g, S, H, n_pos, G), True, HEADS[TWO_TILES if S == 1 else ONE_TILE])


@pytest.mark.parametrize("shape", [ONE_TILE, TWO_TILES])
@pytest.mark.parametrize("bias", [False, True])
def test_references_that_outgrow_the_sums(shape, bias):
    """Half of the rows meet logits 50 larger behind the first or second time that their sums went to memory."""
    S, H, n_pos, G = shape
    c, g = cache_of(2, S, H, 16384, bias, grown=[64 * b for b in (70, 40, 33, 65, 100, 20, 128, 250)])
    check(c, queries(g, S, H, n_pos, G), False, HEADS[shape])


@pytest.mark.parametrize("shape", [ONE_TILE, TWO_TILES])
def test_masks_and_biases_that_grow(shape):
    """Heads whose first blocks are all masked, whose biases grow or fall, and one with nothing but masks."""
    S, H, n_pos, G = shape
    c, g = cache_of(3, S, H, 16384, True)
    low = torch.finfo(torch.float32).min
    c.bias[:, 0, :64 * 40] = -math.inf
    c.bias[:, 1, :64 * 70] = -math.inf
    c.bias[:, 2, 64 * 50:] += GROW
    c.bias[:, 3] = -math.inf
    c.bias[:, 4, :64 * 36] = low
    c.bias[:, 5, 64 * 45:] -= GROW
    c.bias[:, 6, 64 * 35:64 * 100] = -math.inf
    heads = [(0, h) for h in range(8)] + ([(4, h) for h in range(8)] if S > 4 else [])
    check(c, queries(g, S, H, n_pos, G), True, heads)


@pytest.mark.parametrize("blocks", [32, 33, 64, 65])
@pytest.mark.parametrize("n_pos", [10, 32, 64])
@pytest.mark.parametrize("bias", [False, True])
def test_shares_that_end_with_the_sums(blocks, n_pos, bias):
    """One item a CTA, of exactly so many blocks."""
    S = torch.cuda.get_device_properties(0).multi_processor_count
    c, g = cache_of(4, S, 1, 64 * blocks, bias, grown=[64 * 20])
    check(c, queries(g, S, 1, n_pos, 4), False, [(0, 0), (1, 0), (S // 2, 0), (S - 1, 0)])
