"""Scores of tokens count every column of a row once: rows whose sum of exponentials is a
whole number, which float32 holds exactly.

Where every logit that is left is the same, x - m is 0 and z the number of columns, without
rounding; only ln z is rounded (two units in the last place), so that one column lost or
counted twice of V shows as 1 / V.  A row with a single logit has ln p = 0 for it if it was
counted once, ln 2 less if twice, and no probabilities if it was lost.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16, I32 = torch.float32, torch.bfloat16, torch.float16, torch.int32
DEV = "cuda"
INF = float("inf")

# one wave a row; 4 waves a row; 16 waves a row; parts of a row; many rows whole
PLANS = [(3, 40), (2, 1000), (4, 2048), (3, 2050), (2, 4097), (2, 16384), (300, 8200), (240, 126464),
         (1, 126464), (1, 152064), (120, 126464), (2, 300007), (400, 5000)]


def _scores(x, ids, mask_id, k=3):
    from paper_2608_23167_amd import api
    rows, vocab = x.shape
    lp, ent = torch.full(ids.shape, 7.0, device=DEV), torch.full((rows,), 7.0, device=DEV)
    top, tlp = torch.full((rows, k), -7, dtype=I32, device=DEV), torch.full((rows, k), 7.0, device=DEV)
    ws = torch.full((api.ssm_token_logprobs_workspace_size(rows, vocab, k),), 0xff, dtype=torch.uint8, device=DEV)
    api.ssm_token_logprobs(x, ids, mask_id, k, lp, ent, top, tlp, ws)
    return lp, ent, top, tlp


def _at(rows, vocab, dtype, shift, value):
    """Rows of `value` at an address `shift` elements past an aligned one."""
    flat = torch.full((rows * vocab + shift,), value, dtype=dtype, device=DEV)
    return flat[shift:].view(rows, vocab)


def _ln_tol(z):
    """Two units in the last place of ln z, and a rounding of the difference from 0."""
    return 2.5 * 2.0 ** (math.floor(math.log2(max(math.log(z), 2.0 ** -20))) - 23)


@pytest.mark.parametrize("rows,vocab", PLANS)
@pytest.mark.parametrize("dtype,shift", [(F32, 0), (F32, 1), (F32, 2), (F32, 3), (BF16, 0), (BF16, 1), (BF16, 3),
                                         (BF16, 7), (F16, 5)])
def test_equal_logits(gpu, rows, vocab, dtype, shift):
    """All columns, then random halves of them (a column lost does not make up for one counted
    twice in every half), with and without a mask."""
    g = torch.Generator(device=DEV)
    g.manual_seed(vocab + shift)
    x = _at(rows, vocab, dtype, shift, 1.25)
    ids = torch.zeros(rows, 1, dtype=I32, device=DEV)
    for half in range(4):
        keep = torch.ones(vocab, dtype=torch.bool, device=DEV)
        if half:
            keep = torch.rand(vocab, generator=g, device=DEV) < 0.5
            keep[0] = keep[vocab - 1] = True
            x.copy_(torch.where(keep, 1.25, -INF).to(dtype).expand(rows, vocab))
        for mask in (-1, vocab - 2):
            z = int(keep.sum()) - int(mask >= 0 and keep[mask])
            lp, ent, top, tlp = _scores(x, ids, mask)
            tol = _ln_tol(z)
            assert z < 3 or tol < math.log(z) - math.log(z - 1)      # one column is seen
            for got in (lp + math.log(z), ent - math.log(z)):
                assert float(got.abs().max()) <= tol + 2.0 ** -24 * math.log(z), (mask, z)
            first = torch.nonzero(keep & (torch.arange(vocab, device=DEV) != mask)).view(-1)[:3].to(I32)
            assert torch.equal(top, first.expand(rows, 3))


def _edges(vocab):
    """Columns around the ends of loads, tiles and parts, whatever their size."""
    at = {0, vocab - 1, vocab // 2}
    for step in (4, 8, 1024, 2048, 4096):
        ends = list(range(step, vocab, step))
        if len(ends) > 40:
            ends = ends[:12] + ends[-12:] + ends[12:-12:max(1, len(ends) // 16)]
        at.update(c + d for c in ends for d in (-1, 0, 1))
    # with the row's start off alignment, every end moves by up to 7 columns
    at = {c - d for c in at for d in range(8)} | at
    return sorted(c for c in at if 0 <= c < vocab)


@pytest.mark.parametrize("rows,vocab", [(3, 40), (64, 2050), (200, 16384), (1, 126464), (33, 152064), (120, 126464),
                                        (400, 8200)])
@pytest.mark.parametrize("dtype,shift", [(F32, 0), (F32, 3), (BF16, 0), (BF16, 1), (BF16, 6)])
def test_a_single_logit_at_every_edge(gpu, rows, vocab, dtype, shift):
    """Each row has one logit above -inf, at a column where a load, a tile or a part ends or begins."""
    cols = _edges(vocab)
    if rows == 1:
        cols = cols[::7] + cols[-3:]
    x = _at(rows, vocab, dtype, shift, -INF)
    r = torch.arange(rows, device=DEV)
    worst = torch.zeros((), device=DEV)
    for lo in range(0, len(cols), rows):
        c = torch.tensor((cols[lo:lo + rows] + cols[:1] * rows)[:rows], device=DEV)
        x[r, c] = -3.5
        lp, ent, top, tlp = _scores(x, c[:, None].to(I32), -1)
        want = torch.full_like(top, -1)
        want[:, 0] = c
        # ln p and entropy are 0 exactly: NaN compares as different
        worst += (lp[:, 0] != 0).sum() + (ent != 0).sum() + (top != want).sum() + (tlp[:, 0] != 0).sum()
        x[r, c] = -INF
    assert float(worst) == 0
