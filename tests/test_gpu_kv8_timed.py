"""Drafters over the 8-bit cache with attention timing on: a timed attention runs several times and
leaves what an untimed one leaves."""
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("kv8", [True, False])
@pytest.mark.parametrize("body,change", [
    # 32 query heads, or over 20 splits: the splits of a single row are merged by a kernel of their own
    ("p_single64", dict(n_q_heads=32, n_kv_heads=4, ctx_lo=40, ctx_hi=40)),
    ("p_single128", dict(n_q_heads=32, n_kv_heads=8, ctx_lo=700, ctx_hi=700)),
    ("p_single64", dict(ctx_lo=12000, ctx_hi=12000)),
    ("p_single64", {}),
    ("p_qwen_small", {}),
])
def test_a_timed_attention_leaves_what_an_untimed_one_does(body, change, kv8):
    """Two handles, one timed in its first iterations; the last ones run over the cache that these left."""
    from paper_2609_09338_amd import workload as WL
    n_it = 4
    w = synth.get(body).with_(**change)
    weights = synth.make_weights(w)
    runs = []
    for timed in (False, True):
        s = WL.make_drafter(w, n_it, weights=weights, kv8=kv8)
        WL.reset_sequences(s)
        out = WL.alloc_outputs(s)
        got = []
        for it in range(n_it):
            s.drafter.kernel_timing((1,) if timed and it < 2 else ())
            inp = WL.iter_inputs(s, it)
            WL.draft(s, it, inp, out)
            tl = WL.synthetic_target(s, it, out.logits)
            WL.verify(s, inp, tl, out)
            torch.cuda.synchronize()
            if timed and it < 2:
                assert s.drafter.kernel_time(1)[1] > 0
            got += [torch.nan_to_num(out.logits), out.drafts.clone(), out.accept_len.clone(), out.tokens.clone()]
        assert s.drafter.device_errors() == 0
        runs.append(got)
    for i, (a, b) in enumerate(zip(*runs)):
        assert torch.equal(a, b), i
