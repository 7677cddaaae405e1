"""The 8-bit paged cache at the ends of its types' ranges: values as large as BF16 holds, queries
and keys whose factors are beyond binary32."""
import pytest
import torch

import paper_2609_35800_gb300 as hg
from test_gpu_pages8 import BF16, D, Pool, _begins, _check_decode, _gen, _ints, _randn, _random_pool, _run_decode, _tables
from test_gpu_pages8 import _workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [4, 12])
@pytest.mark.parametrize("tokens", [1, 40, 1000, 20011])
@pytest.mark.parametrize("scale,codes", [(2.0 ** 103, (0, 0x7f)), (2.0 ** 112, (0, 0x7f)), (2.0 ** 119, (0, 0x7f)), (2.0 ** 126, (0x30, 0x3e))])
def test_decode_largest_values(scale, codes, tokens, group):
    """Averages of values up to BF16's end are in its range, whatever the number of tokens and the sums on the way."""
    g = _gen(tokens)
    tab, pages = _tables(g, [tokens], 64)
    pool = _random_pool(g, pages, 2, 64)
    c = torch.randint(*codes, pool.codes[1].shape, generator=g, device="cuda", dtype=torch.uint8)
    c[:, 1] |= torch.randint(0, 2, c[:, 1].shape, generator=g, device="cuda", dtype=torch.uint8) << 7  # both signs in one head
    pool.codes[1].copy_(c)
    pool.scales[1].copy_(torch.where(torch.rand(pool.scales[1].shape, generator=g, device="cuda") < 0.3, scale * 2.0 ** -9, scale))
    q = _randn(g, 1, 2 * group, D, scale=0.2)
    out, lse = _run_decode(pool, q, tab, [tokens])
    assert bool(out.isfinite().all())
    _check_decode(q, pool, tab, [tokens], out, lse)


@pytest.mark.parametrize("value", [2.0 ** 111, 2.0 ** 121, 1.75 * 2.0 ** 127, -1.75 * 2.0 ** 127])
def test_values_that_e4m3_holds_come_back(value):
    """One value for all tokens, which a code and a power of two hold: the average of any number of them."""
    g = _gen(3)
    lens = [1, 17, 700]
    tab, pages = _tables(g, lens, 16)
    pool = Pool(g, pages, 1, 16)
    k = _randn(g, sum(lens), 1, D)
    v = torch.full_like(k, value)
    hg.hg_pages8_append(pool.hg, None, k, v, None, None, _begins(lens), tab, _ints(lens))
    q = torch.zeros((3, 4, D), dtype=BF16, device="cuda")  # even probabilities
    out, lse = _run_decode(pool, q, tab, lens)
    assert torch.equal(out, torch.full_like(out, value))
    # a step's new token: a query far along its key, so that it is the sum
    lens = [n + 1 for n in lens]
    k1 = torch.full((3, 1, D), 16.0, dtype=BF16, device="cuda")
    out = torch.empty_like(out)
    tab2, pages2 = _tables(g, lens, 16)
    pool = Pool(g, pages2, 1, 16)
    pool.fill(g, tab2, [n - 1 for n in lens])
    hg.hg_pages8_decode_step(pool.hg, torch.ones_like(q), k1, torch.full_like(k1, value), None, None, tab2, _ints(lens), out, None,
                             0.0, _workspace(pool, 3, 4))
    assert torch.equal(out, torch.full_like(out, value))


@pytest.mark.parametrize("group", [4, 12])
@pytest.mark.parametrize("q_at,k_at", [(2.0 ** 100, 2.0 ** 60), (2.0 ** 70, 2.0 ** 90), (2.0 ** 120, 2.0 ** 119)])
def test_decode_far_factors_of_zeros(q_at, k_at, group):
    """Queries and keys that share no channel: every score is 0, however large both are."""
    g = _gen(5)
    lens = [1, 33, 500]
    tab, pages = _tables(g, lens, 16)
    pool = Pool(g, pages, 2, 16)
    k, v = (_randn(g, sum(lens), 2, D) for _ in "kv")
    k = k.clamp(-4, 4) * k_at
    k[..., ::3] = 0.0
    hg.hg_pages8_append(pool.hg, None, k, v, None, None, _begins(lens), tab, _ints(lens))
    q = torch.zeros((3, 2 * group, D), dtype=BF16, device="cuda")
    q[..., ::3] = q_at
    out, lse = _run_decode(pool, q, tab, lens)
    _check_decode(q, pool, tab, lens, out, lse)
