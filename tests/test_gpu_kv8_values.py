"""Attention over the 8-bit cache where value blocks differ by more than f16 spans: a row's output
comes from what the row sees, whatever lies in the other positions of its pass."""
import pytest
import torch

from . import kv8_seen as S
from .test_gpu_kv8 import BF, DEV, F32, bd, cu_of, gen_of, ints, make_cache, ref_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def attend(cache, cached, rows, q, masks=None, max_context=None):
    nq, n = q.shape[1], sum(rows)
    ctx = max_context or max(c + r for c, r in zip(cached, rows))
    out = torch.full_like(q, 7.0)
    ws = torch.empty(bd().kv8_attention_workspace(cache, n, nq, max(rows), ctx), dtype=torch.uint8, device=DEV)
    err = ints([0])
    tree = None if masks is None else torch.tensor([[m, 0] for s in masks for m in s], dtype=torch.int64, device=DEV)
    bd().kv8_attention(cache, q, out, ints(cached), ws, max_rows=max(rows), max_context=ctx, cu_rows=ints(cu_of(rows)), tree_mask=tree,
                       errors=err)
    torch.cuda.synchronize()
    assert int(err) == 0
    return out


def check(cache, cached, rows, q, masks=None, max_context=None):
    out = attend(cache, cached, rows, q, masks, max_context)
    ref, r0 = ref_of(cache), 0
    for b, (c, r) in enumerate(zip(cached, rows)):
        sees = S.causal(c, r)
        if masks is not None:
            sees = torch.ones((r, c + r), dtype=torch.bool)
            sees[:, c:] = torch.tensor([[bool(m >> i & 1) for i in range(r)] for m in masks[b]])
        want, tol = S.attention(ref, b, q[r0:r0 + r], sees, q.shape[2] ** -0.5, q.dtype)
        off = (out[r0:r0 + r].cpu().double() - want).abs()
        bad = (off > tol).any(-1).any(-1)
        assert not bool(bad.any()), f"sequence {b}, rows {bad.nonzero().flatten().tolist()[:8]}: off by {float((off - tol).max()):.3g}"
        r0 += r


# heads, cached positions, rows: 1 to 16 vectors a kv head and sequence, 17 to 32 (either form, by the
# context the call is planned for), more
FORMS = [
    ((4, 4, 64), [15], [2], None),
    ((16, 8, 128), [15, 40], [2, 8], None),
    ((8, 2, 64), [60, 3], [4, 4], 4000),
    ((8, 2, 64), [1500, 31], [8, 5], 1),
    ((8, 2, 128), [1500, 31], [8, 5], 1 << 20),
    ((8, 2, 128), [200], [40], None),
    ((8, 2, 64), [9, 0], [300, 50], None),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,cached,rows,max_context", FORMS)
@pytest.mark.parametrize("old,new", [(1.0, 1e12), (1.0, 1e6), (1.0, 3e37), (1e-26, 1e30)])
def test_a_later_rows_values_leave_earlier_rows_alone(heads, cached, rows, max_context, old, new, dtype):
    """The last row's own value is larger than every other by `new / old`."""
    nq, nkv, hd = heads
    gen = gen_of(11)
    cache = make_cache(len(rows), max(c + r for c, r in zip(cached, rows)) // 16 + 1, nkv, hd, 3)
    n = sum(c + r for c, r in zip(cached, rows))
    k, v = (torch.randn((n, nkv, hd), generator=gen, device=DEV) for _ in range(2))
    total = cu_of([c + r for c, r in zip(cached, rows)])
    last = torch.zeros(n, dtype=torch.bool, device=DEV)
    last[[t - 1 for t in total[1:]]] = True
    v *= torch.where(last, new, old)[:, None, None]
    bd().kv8_append(cache, k, v, ints([0] * len(rows)), cu_rows=ints(total))
    q = torch.randn((sum(rows), nq, hd), generator=gen, device=DEV).to(dtype)
    check(cache, cached, rows, q, max_context=max_context)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("group,rows", [(1, 9), (2, 16), (2, 40)])
def test_a_masked_branchs_values_leave_the_others_alone(group, rows, dtype):
    """Two branches of a tree, the second's values 2^70 times the first's; each sees its own."""
    nkv, hd, cached = 2, 64, 32 - rows // 2     # (the second branch begins a page)
    gen = gen_of(12)
    cache = make_cache(1, 6, nkv, hd, 3)
    k, v = (torch.randn((cached + rows, nkv, hd), generator=gen, device=DEV) for _ in range(2))
    half = rows // 2
    v[cached + half:] *= 2.0 ** 70
    masks = [[sum(1 << j for j in range(i + 1) if (j >= half) == (i >= half)) for i in range(rows)]]
    bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, cached + rows]))
    q = torch.randn((rows, nkv * group, hd), generator=gen, device=DEV).to(dtype)
    check(cache, [cached], [rows], q, masks=masks)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("step", [2.3, -2.3, 0.0])
def test_values_that_grow_or_fall_from_page_to_page(step, hd, dtype):
    """A prompt whose scales go over 2^200 in one direction, or jump between two sizes; several
    chunks of 64 pages for a block to walk, and single rows over the same positions."""
    n, nkv, nq = 1400, 1, 1
    gen = gen_of(13)
    cache = make_cache(1, n // 16 + 1, nkv, hd, 3)
    k, v = (torch.randn((n, nkv, hd), generator=gen, device=DEV) for _ in range(2))
    page = torch.arange(n, device=DEV) // 16
    e = page * step + (-85 if step > 0 else 115) if step else (page % 7 == 3) * 90 - 60
    v *= (2.0 ** e.double().round()).float()[:, None, None]
    v[640:672] = 0.0                                            # blocks of the smallest scale
    bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, n]))
    q = torch.randn((n, nq, hd), generator=gen, device=DEV).to(dtype)
    check(cache, [0], [n], q)
    for last in (1, 8):
        check(cache, [n - last], [last], q[-last:].contiguous())
        check(cache, [n - last], [last], q[-last:].contiguous(), max_context=1)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 40])
def test_small_values_before_large_ones_in_a_later_chunk(rows, dtype):
    """4096 small positions (a whole chunk of pages of each wavefront), then large ones whose keys
    nobody attends to: exponents 2^-60 and less, which P holds as nothing."""
    nkv, hd, n = 1, 64, 9000
    gen = gen_of(14)
    cache = make_cache(1, n // 16 + 1, nkv, hd, 3)
    k = torch.zeros((n, nkv, hd), device=DEV)
    k[:, :, 1:] = torch.randn((n, nkv, hd - 1), generator=gen, device=DEV)
    k[8000:8960, :, 0] = -2000.0
    v = torch.randn((n, nkv, hd), generator=gen, device=DEV)
    v[8000:8960] *= 2.0 ** 80
    bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, n]))
    q = torch.randn((rows, 2, hd), generator=gen, device=DEV)
    q[:, :, 0] = 8.0
    q = q.to(dtype)
    out = attend(cache, [n - rows], [rows], q, max_context=1)
    # as if the large ones were masked: their weights are below 2^-2000
    sees = S.causal(n - rows, rows)
    sees[:, 8000:8960] = False
    want, tol = S.attention(ref_of(cache), 0, q, sees, hd ** -0.5, dtype)
    assert bool(((out.cpu().double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("spread", [False, True])
@pytest.mark.parametrize("rows", [1, 8, 40])
def test_many_of_the_largest_values_in_one_sum(rows, spread, dtype):
    """6000 values of 3e38 whose probabilities lie 2^7 above what the first pages' maximum makes 2^6: sums of
    2^25 times the largest float, in one split, over blocks of one scale and beside a page of zeros."""
    nkv, hd, n = 1, 64, 6000
    cache = make_cache(1, n // 16 + 1, nkv, hd, 3)
    k = torch.zeros((n, nkv, hd), device=DEV)
    k[128:, :, 0] = 1.0
    v = 3.0e38 * (1 - 0.2 * torch.rand((n, nkv, hd), generator=gen_of(15), device=DEV))
    if spread:
        v[3200:3216] = 0.0
    bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, n]))
    q = torch.zeros((rows, 4, hd), device=DEV)
    q[:, :, 0] = 5.1875 * hd ** 0.5
    check(cache, [n - rows], [rows], q.to(dtype), max_context=1)
    check(cache, [n - rows], [rows], q.to(dtype), max_context=n)
