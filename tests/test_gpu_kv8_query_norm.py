"""The norm of queries beside the 8-bit cache, over the whole range of their type: the mean of the
squares is no float long before the elements are none."""
import pytest
import torch

from . import kv8_ref as R
from .test_gpu_kv8 import BF, DEV, F32, bd, cu_of, gen_of, ints, make_cache, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,batch,rows", [((4, 2, 64), 3, [1, 1, 1]), ((16, 8, 128), 2, [1, 1]), ((4, 2, 64), 2, [5, 20]),
                                              ((5, 1, 128), 1, [40]), ((8, 2, 64), 2, [17000, 3]), ((8, 1, 128), 1, [20000])])
@pytest.mark.parametrize("size,eps", [(1e20, 1e-6), (3e38, 1e-6), (1e-22, 1e-40), (1e-30, 1e-6), (1.0, 1e-6)])
def test_queries_of_any_size_are_normalised(heads, batch, rows, size, eps, dtype):
    nq, nkv, hd = heads
    n = sum(rows)
    gen = gen_of(n)
    cache = make_cache(batch, max(rows) // 16 + 1, nkv, hd, 3)
    k, v = (torch.randn((n, nkv, hd), generator=gen, device=DEV).to(dtype) for _ in range(2))
    # (uniform: `size` is the largest)
    q = ((torch.rand((n, nq, hd), generator=gen, device=DEV) * 2 - 1) * size).to(dtype)
    q[0, 0] = 0.0
    q[0, 1, 1:] = 0.0                                     # one element alone
    gain = (1 + 0.2 * torch.randn(hd, generator=gen, device=DEV)).to(dtype)
    cos, sin = tables(max(rows), hd)
    out = torch.empty_like(q)
    err = ints([0])
    one = all(r == 1 for r in rows)
    bd().kv8_append(cache, k, v, ints([0] * batch), q=q, q_out=out, cu_rows=None if one else ints(cu_of(rows)), q_norm=gain, eps=eps,
                    rope_cos=cos.to(DEV), rope_sin=sin.to(DEV), errors=err)
    torch.cuda.synchronize()
    assert int(err) == 0
    at = torch.cat([torch.arange(r) for r in rows])
    eps32 = float(torch.tensor(eps, dtype=torch.float32))
    want = R.norm_rope(q.cpu().double(), gain.cpu(), eps32, cos[at], sin[at])
    half = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    # a sum of hd squares, a root, a quotient, two gains, two products: fp32; and half of the output's smallest step
    big = torch.maximum(want.abs(), want.roll(hd // 2, -1).abs())
    tol = half * want.abs() + (hd + 16) * 2.0 ** -24 * big * 2 ** 0.5 * 2 + (2.0 ** -134 if dtype == BF else 2.0 ** -150)
    assert bool(((out.cpu().double() - want).abs() <= tol).all())


def test_a_query_that_is_not_finite_stays_a_matter_of_its_head():
    hd, nq, rows = 64, 4, 6
    for dtype in (BF, F32):
        cache = make_cache(1, 1, 1, hd, 3)
        gen = gen_of(3)
        k = torch.randn((rows, 1, hd), generator=gen, device=DEV).to(dtype)
        q = torch.randn((rows, nq, hd), generator=gen, device=DEV).to(dtype)
        q[1, 2, 5], q[3, 0, 63] = float("nan"), float("inf")
        q[4, 1] = 1e25
        gain = torch.ones(hd, device=DEV, dtype=dtype)
        out = torch.empty_like(q)
        bd().kv8_append(cache, k, k, ints([0]), q=q, q_out=out, cu_rows=ints([0, rows]), q_norm=gain)
        bad = ~torch.isfinite(out).all(-1).cpu()
        want = torch.zeros((rows, nq), dtype=torch.bool)
        want[1, 2] = want[3, 0] = True
        assert torch.equal(bad, want)
        assert bool(((out[4, 1].float() - 1.0).abs() <= 2.0 ** -8).all())
