"""Most probable tokens of many rows in parts of 256 lanes each, and rows beyond those of one launch."""
import numpy as np
import pytest
import torch

from tests import more_operators_plain as M
from tests.operators_plain import assert_within
from tests.test_gpu_operators_logprob import BF16, DEV, F32, INF, backward, check_forward, forward, make

pytestmark = pytest.mark.gpu


# more rows than workgroups of 1024 lanes take in two turns: parts of 8192 tokens, the last one short
@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,top", [(600, 9001, 20), (520, 8193, 64), (520, 16384, 1), (520, 32768, 64), (180, 70001, 5), (40, 400001, 64), (33, 524288, 64)])
def test_rows_in_parts(rows, vocab, top, kind):
    print(f"case parts {rows} {vocab} {top} {kind}", flush=True)
    logits, ids = make(rows, vocab, kind)
    check_forward(logits, ids, top)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,top", [(600, 9001, 20), (520, 32768, 64)])
def test_masked_rows_and_rows_of_few_values_in_parts(rows, vocab, top, kind):
    """Parts in which more tokens reach the bound than the list holds: nothing left in a part, fewer than are wanted, equal logits, some far behind the others."""
    print(f"case masked parts {rows} {vocab} {top} {kind}", flush=True)
    gen = torch.Generator().manual_seed(2)
    logits = torch.randint(0, 3, (rows, vocab), generator=gen).float()
    logits[0::5] = -INF
    for i in range(0, rows, 5):
        at = torch.randperm(vocab, generator=gen)[:1 + i % 90]
        logits[i, at] = torch.randn(len(at), generator=gen)
    logits[1::5] = torch.finfo(kind).min
    logits[1::5, vocab - 7] = 1.5
    logits[2::5, :8192] = -INF
    logits[3::5] = torch.sort(torch.randn(len(logits[3::5]), vocab, generator=gen)).values
    logits, ids = logits.to(kind).to(DEV), torch.randint(0, vocab, (rows,), generator=gen).to(DEV)
    check_forward(logits, ids, top)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_rows_of_two_launches(index, kind):
    print(f"case launches {index} {kind}", flush=True)
    rows, vocab = (1 << 21) + 3, 5
    gen = torch.Generator().manual_seed(4)
    logits = (torch.randn(rows, vocab, generator=gen) * 2).to(kind).to(DEV)
    ids = torch.randint(-1, vocab, (rows,), generator=gen).to(index).to(DEV)
    r = forward(logits, ids, 2, index)
    none = forward(logits, ids, 0, index)
    lse, lp, entropy, lse_off, lp_off, ent_off = M.logprob(logits)
    where = ids.cpu().numpy().astype(np.int64)
    pick = np.maximum(where, 0)[:, None]
    for got in (r, none):
        assert_within(got["lse"], lse, lse_off, "lse")
        assert_within(got["entropy"], entropy, ent_off, "entropy")
        assert_within(got["logprob"], np.where(where >= 0, np.take_along_axis(lp, pick, 1)[:, 0], 0), np.take_along_axis(lp_off, pick, 1)[:, 0], "logprob")
    best = torch.sort(logits.cpu().float(), dim=1, descending=True, stable=True).indices[:, :2].numpy()
    assert np.array_equal(r["top_ids"].cpu().numpy(), best)
    assert_within(r["top_logprobs"], np.take_along_axis(lp, best, 1), np.take_along_axis(lp_off, best, 1), "top_logprobs")
    g, ge = torch.randn(rows, generator=gen).to(DEV), torch.randn(rows, generator=gen).to(DEV)
    for kw in (dict(), dict(entropy=r["entropy"], grad_entropy=ge)):
        ref, off = M.logprob_gradient(logits, ids, r["lse"], g, kw.get("entropy"), kw.get("grad_entropy"))
        assert_within(backward(logits, ids, r["lse"], g, **kw), ref, off, "gradient")
