"""Attention over the 8-bit cache with scores of any size that fp32 holds: keys are kept up to the
largest floats, so a row's scores may all lie far below zero, or far above."""
import itertools

import pytest
import torch

from . import kv8_seen as S
from .test_gpu_kv8 import BF, DEV, F32, bd, cu_of, gen_of, ints, make_cache, ref_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def attend(cache, cached, rows, q, max_context, scale=None):
    out = torch.full_like(q, 7.0)
    n, nq = q.shape[:2]
    ws = torch.empty(bd().kv8_attention_workspace(cache, n, nq, rows, max_context), dtype=torch.uint8, device=DEV)
    err = ints([0])
    bd().kv8_attention(cache, q, out, ints([cached] * (n // rows)), ws, max_rows=rows, max_context=max_context,
                       cu_rows=ints(cu_of([rows] * (n // rows))), errors=err, scale=scale)
    torch.cuda.synchronize()
    assert int(err) == 0
    return out.cpu().double()


def definition(ref, q, sees, scale, dtype):
    """The softmax in 64 bits of scores that are one product each.  Their fp32 error, 4 roundings, counts where it
    can change a weight: past 2^28 two scores that differ at all do so by a sixteenth of themselves or more
    (codes of 4 significant bits), 2^24 against 2^6, so the largest share the weight."""
    half, p_step = (2.0 ** -8, 2.0 ** -11) if dtype is BF else (2.0 ** -24, 2.0 ** -22)
    n, nq, hd = q.shape
    k, v = ref.context(0, sees.shape[1])
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for h in range(nq):
        z = (q[:, h].cpu().double() @ k[h * ref.nkv // nq].T) * scale
        z = z.masked_fill(~sees, -torch.inf)
        w = torch.softmax(z, -1)
        big = torch.where(sees, z.abs(), 0.0).max(-1, keepdim=True).values
        assert bool(((big < 2.0 ** 8) | (big > 2.0 ** 28)).all())
        dz = torch.where(big > 2.0 ** 28, 0.0, 4 * 2.0 ** -24 * big)
        vh = v[h * ref.nkv // nq]
        out[:, h] = w @ vh
        tol[:, h] = half * out[:, h].abs() + (p_step + 2 * dz + 2.0 ** -18) * (w @ vh.abs()) \
            + sees.sum(-1, keepdim=True) * 2.0 ** -30 * vh.abs().max()
    return out, tol


PATTERNS = {
    "one": lambda n, a: [a] * n,                                  # all alike: the mean
    "last_larger": lambda n, a: [a] * (n - 1) + [a * 1.25],
    "first_larger": lambda n, a: [a * 1.25] + [a] * (n - 1),
    "two_of_many": lambda n, a: [a * (1.5 if i in (n // 3, n - 1) else 1.0) for i in range(n)],
    "among_zeros": lambda n, a: [0.0 if i % 5 == 2 else a for i in range(n)],
    "both_signs": lambda n, a: [a if i % 3 else -a for i in range(n)],
    "growing": lambda n, a: [a * 2.0 ** (2 * i // n - 2) for i in range(n)],
}
# rows, query heads a kv head, positions, planned for: the kernels for 1 to 16, 17 to 32 (two), more vectors
FORMS = [(1, 2, 1, 1), (1, 2, 16, 16), (1, 4, 700, 1), (1, 4, 5000, 5000), (8, 4, 100, 100), (8, 4, 2000, 1 << 20),
         (40, 1, 41, 41), (40, 2, 1500, 1500), (200, 1, 200, 1)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pattern", list(PATTERNS))
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("size", [2.0 ** 34, 2.0 ** 60, 2.0 ** 115])
def test_scores_far_from_zero(size, sign, pattern, dtype):
    """One key dim carries the score: size / 8 is its largest, in powers of two and codes that hold exactly."""
    hd, nkv = 64, 1
    for rows, group, n, planned in FORMS:
        cache = make_cache(1, n // 16 + 1, nkv, hd, 3)
        k = torch.zeros((n, nkv, hd), device=DEV)
        k[:, 0, 5] = torch.tensor(PATTERNS[pattern](n, size), device=DEV)
        v = torch.randn((n, nkv, hd), generator=gen_of(5), device=DEV)
        bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, n]))
        q = torch.zeros((rows, group, hd), device=DEV)
        q[:, :, 5] = sign
        q[:, :, 6] = 3.0
        q = q.to(dtype)
        out = attend(cache, n - rows, rows, q, planned)
        want, tol = definition(ref_of(cache), q, S.causal(n - rows, rows), hd ** -0.5, dtype)
        off = (out - want).abs()
        assert bool((off <= tol).all()), (rows, group, n, planned, float((off - tol).max()))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hd", [64, 128])
def test_rows_of_far_scores_beside_ordinary_ones(hd, dtype):
    """Every row of a pass has a size of its own, from 2^-3 to 2^60; the ordinary ones are as they would be alone."""
    nkv, n = 2, 900
    gen = gen_of(6)
    cache = make_cache(1, n // 16 + 1, nkv, hd, 3)
    k = torch.zeros((n, nkv, hd), device=DEV)
    k[:, :, 1] = (1 + torch.randint(0, 8, (n, nkv), generator=gen, device=DEV) / 8) * torch.where(
        torch.rand((n, nkv), generator=gen, device=DEV) < 0.5, -1.0, 1.0)
    v = torch.randn((n, nkv, hd), generator=gen, device=DEV)
    bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, n]))
    sizes = [2.0 ** -3, 2.0 ** 40, 1.0, -2.0 ** 60, 8.0, 2.0 ** 36, -4.0]
    for rows, group in ((1, 4), (4, 4), (8, 4), (70, 2)):
        q = torch.zeros((rows, nkv * group, hd), device=DEV)
        for (r, h), s in zip(itertools.product(range(rows), range(nkv * group)), itertools.cycle(sizes)):
            q[r, h, 1] = s
        q = q.to(dtype)
        want, tol = definition(ref_of(cache), q, S.causal(n - rows, rows), 1.0, dtype)
        for planned in (1, n):
            out = attend(cache, n - rows, rows, q, planned, scale=1.0)
            off = (out - want).abs()
            assert bool((off <= tol).all()), (rows, group, planned, float((off - tol).max()))


def test_one_position_returns_its_value_at_any_score():
    """out = v exactly as stored where one position is seen: its weight is 1 whatever the score."""
    hd = 64
    for dtype in (BF, F32):
        for key, q0, scale in ((1e32, -1.0, 0.125), (1e32, 1.0, 0.125), (3e37, -1.0, 1.0), (1e9, 3.0, 1.0), (-1e9, 7.0, 1.0),
                               (1.0, -2.0 ** 100, 0.125), (448.0, 2.0 ** 27, 1.0), (440.0, 1.7e8, 0.7)):
            cache = make_cache(1, 1, 1, hd, 3)
            k = torch.zeros((1, 1, hd), device=DEV)
            k[0, 0, 9] = key
            v = torch.randn((1, 1, hd), generator=gen_of(7), device=DEV)
            bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, 1]))
            q = torch.zeros((1, 4, hd), device=DEV)
            q[:, :, 9] = q0
            out = attend(cache, 0, 1, q.to(dtype), 1, scale=scale)
            stored = ref_of(cache).read(0, 0)[1][0]
            assert torch.equal(out, stored.expand(1, 4, hd)), (dtype, key, q0, scale)


def test_rows_that_see_nothing_are_zeros_beside_rows_of_far_scores():
    """A tree mask that leaves a row nothing, in tiles whose other rows score far below zero."""
    hd, rows = 64, 20
    for group in (1, 2):
        cache = make_cache(1, 3, 1, hd, 3)
        k = torch.zeros((rows, 1, hd), device=DEV)
        k[:, 0, 0] = 2.0 ** 110
        v = torch.randn((rows, 1, hd), generator=gen_of(8), device=DEV)
        bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, rows]))
        for dtype in (BF, F32):
            q = torch.zeros((rows, group, hd), device=DEV, dtype=dtype)
            q[:, :, 0] = -1.0
            masks = [0 if i % 3 == 0 else 1 << i for i in range(rows)]
            out = torch.full_like(q, 7.0)
            ws = torch.empty(bd().kv8_attention_workspace(cache, rows, group, rows, 300), dtype=torch.uint8, device=DEV)
            bd().kv8_attention(cache, q, out, ints([0]), ws, max_rows=rows, max_context=300, cu_rows=ints([0, rows]),
                               tree_mask=torch.tensor([[m, 0] for m in masks], dtype=torch.int64, device=DEV))
            ref = ref_of(cache)
            for i in range(rows):
                want = ref.read(0, i)[1][0] if masks[i] else torch.zeros(hd, dtype=torch.float64)
                assert torch.equal(out[i].cpu().double(), want.expand(group, hd)), (group, dtype, i)


@pytest.mark.parametrize("rows", [1, 40])
def test_large_queries_over_the_smallest_scales_keep_their_small_scores(rows):
    """Products of 2^125 with codes, a block's scale of 2^-100 and a small softmax scale: the factor of the
    scores lies below fp32's normal numbers (7 bits of it are left at 2^-142, all that a score of 2^-17 needs)."""
    hd, n = 64, 64
    cache = make_cache(1, n // 16, 1, hd, 3)
    k = torch.zeros((n, 1, hd), device=DEV)
    k[:, 0, 3] = torch.where(torch.arange(n, device=DEV) % 2 == 0, 256.0, -256.0) * 2.0 ** -100
    v = torch.where(torch.arange(n, device=DEV) % 2 == 0, 1.0, -1.0)[:, None, None].expand(n, 1, hd).contiguous()
    bd().kv8_append(cache, k, v, ints([0]), cu_rows=ints([0, n]))
    q = torch.zeros((rows, 2, hd), device=DEV, dtype=BF)
    q[:, :, 3] = 2.0 ** 117
    for scale, z in ((2.0 ** -24, 2.0), (2.0 ** -28, 2.0 ** -3), (2.0 ** -42, 2.0 ** -17)):
        out = attend(cache, n - rows, rows, q, 1, scale=scale)
        even = torch.arange(n - rows, n) // 2 + 1.0
        odd = (torch.arange(n - rows, n) + 1) // 2
        up, down = even * torch.exp(torch.tensor(z, dtype=torch.float64)), odd * torch.exp(torch.tensor(-z, dtype=torch.float64))
        want = ((up - down) / (up + down))[:, None, None]
        # the factor's rounding of 2^-8 of the score, P's 2^-11, the sums' 2^-18, the output's 2^-8
        assert bool(((out - want).abs() <= 2.0 ** -8 * want.abs() + 2 * z * 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18).all()), (scale, z)
