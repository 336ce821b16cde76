"""Log probabilities of given tokens, entropy and top alternatives against a
plain 64-bit form."""
import math

import pytest
import torch

import _i8_ref as R

pytestmark = pytest.mark.gpu

F32, BF16, F16, I32 = torch.float32, torch.bfloat16, torch.float16, torch.int32
DEV = "cuda"
NAN, INF = float("nan"), float("inf")


def _logits(seed, rows, vocab, dtype=F32, std=3.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g, device=DEV) * std).to(dtype)


def _run(x, ids, mask_id, k, stream=None):
    from paper_2608_23167_amd import api
    rows, vocab = x.shape
    t = 0 if ids is None else ids.shape[1]
    # guard rows behind the last must be left as they were
    lp, ent = torch.full((rows + 1, max(t, 1)), 7.0, device=DEV), torch.full((rows + 1,), 7.0, device=DEV)
    top = torch.full((rows + 1, max(k, 1)), -7, dtype=I32, device=DEV)
    tlp = torch.full((rows + 1, max(k, 1)), 7.0, device=DEV)
    need = api.ssm_token_logprobs_workspace_size(rows, vocab, k)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV) if need else None
    if stream is not None:                         # after the fills above, before the checks below
        stream.wait_stream(torch.cuda.current_stream())
    api.ssm_token_logprobs(x, ids, mask_id, k, lp[:rows] if t else None, ent[:rows],
                           top[:rows] if k else None, tlp[:rows] if k else None, ws, stream=stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    assert bool((lp[rows:] == 7).all()) and bool((ent[rows:] == 7).all())
    assert bool((top[rows:] == -7).all()) and bool((tlp[rows:] == 7).all())
    return lp[:rows], ent[:rows], top[:rows], tlp[:rows]


def _near(got, ref, tol):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    assert torch.equal(torch.isinf(got), torch.isinf(ref))
    fine = torch.isfinite(ref)
    if bool(fine.any()):
        off = (got - ref)[fine].abs() - R.SCORES_REL * ref[fine].abs()
        assert float(off.max()) <= tol, (float(off.max()), tol)


def _check(x, ids, mask_id, k):
    vocab = x.shape[1]
    lp, ent, top, tlp = _run(x, ids, mask_id, k)
    ref, logp, h = R.scores(x, mask_id)
    tol = R.scores_tol(vocab)
    if ids is not None:
        inside = (ids >= 0) & (ids < vocab)
        want = torch.where(inside, logp.gather(1, ids.long().clamp(0, vocab - 1)), NAN)
        _near(lp, want, tol)
    _near(ent, h, tol)
    if k:
        want = R.top(ref, k)
        assert torch.equal(top, want)
        _near(tlp, torch.where(want >= 0, logp.gather(1, want.long().clamp(0)), -INF), tol)


def _ids(seed, rows, t, vocab):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(0, vocab, (rows, t), generator=g, device=DEV, dtype=I32)


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 2), (3, 7), (2, 63), (5, 64), (4, 257), (33, 512), (1, 4097),
                                        (7, 8191), (130, 1000), (1, 126464), (3, 152064), (40, 30001),
                                        (600, 2050), (2, 300007), (150, 60001), (2, 16384), (300, 8200)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_scores(gpu, rows, vocab, dtype):
    x = _logits(rows + vocab, rows, vocab, dtype)
    _check(x, _ids(1, rows, 2, vocab), vocab - 1 if vocab > 1 else -1, 5)


@pytest.mark.parametrize("k", range(9))
@pytest.mark.parametrize("t", [0, 1, 3])
def test_every_k_and_number_of_targets(gpu, k, t):
    for rows, vocab in ((5, 3001), (2, 6), (300, 515)):
        x = _logits(k, rows, vocab)
        _check(x, _ids(2, rows, t, vocab) if t else None, 4, k)


@pytest.mark.parametrize("shift", [1, 2, 3, 5])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [4096, 126464])
def test_unaligned(gpu, shift, dtype, vocab):
    flat = torch.zeros(3 * vocab + shift, dtype=dtype, device=DEV)
    x = flat[shift:].view(3, vocab)
    x.copy_(_logits(3, 3, vocab, dtype))
    _check(x, _ids(3, 3, 1, vocab), 0, 8)


@pytest.mark.parametrize("vocab", [40, 5000, 126464])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ties(gpu, vocab, dtype):
    """Equal logits rank by id, within a thread's share, across shares and over the whole row."""
    x = torch.zeros(7, vocab, dtype=dtype, device=DEV)
    x[1] = torch.arange(vocab, device=DEV) % 3
    x[2, ::7] = 2.0
    x[3] = torch.arange(vocab, device=DEV).flip(0) // 5
    x[4, vocab - 6:] = 1.0
    x[5] = -0.0
    x[5, 3::5] = 0.0
    x[6] = _logits(1, 1, vocab)[0].round()
    _check(x, _ids(1, 7, 1, vocab), 1, 8)
    _check(x, _ids(1, 7, 1, vocab), -1, 8)


@pytest.mark.parametrize("vocab", [3000, 126464])
def test_orders(gpu, vocab):
    """Rising rows bring a better token at every step, falling ones never; peaks at the ends."""
    up = torch.linspace(-20, 20, vocab, device=DEV)
    x = torch.stack([up, up.flip(0), torch.zeros_like(up), torch.zeros_like(up), up.sin() * 9])
    x[2, 0], x[3, vocab - 1] = 30.0, 30.0
    for dtype in (F32, BF16):
        _check(x.to(dtype), _ids(4, 5, 2, vocab), vocab // 2, 8)


@pytest.mark.parametrize("vocab", [9, 2000, 126464])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_masked_logits(gpu, vocab, dtype):
    lowest = torch.finfo(dtype).min
    x = _logits(2, 9, vocab, dtype)
    x[0] = -INF                       # nothing left
    x[1, 3:] = -INF                   # three left, one of them the mask
    x[2] = -INF
    x[2, vocab - 1] = 4.0             # one left: entropy 0
    x[3] = lowest                     # every logit the type's lowest: uniform
    x[4, : vocab // 2] = lowest
    x[5, 1::2] = -INF
    x[6] = -INF
    x[6, 0] = 1.0                     # only the mask is left: nothing
    x[7, : vocab - 2] = -INF
    _check(x, _ids(5, 9, 3, vocab), 0, 6)


@pytest.mark.parametrize("vocab", [300, 126464])
def test_rows_with_nan_or_infinity(gpu, vocab):
    """A NaN or +inf spoils its own row alone."""
    x = _logits(6, 6, vocab)
    x[1, vocab // 3] = NAN
    x[3, vocab - 1] = INF
    x[4, 0] = NAN
    ids = _ids(6, 6, 2, vocab)
    lp, ent, top, tlp = _run(x, ids, 5, 4)
    bad = torch.tensor([1, 3, 4], device=DEV)
    assert bool(torch.isnan(lp[bad]).all()) and bool(torch.isnan(ent[bad]).all())
    assert bool(torch.isnan(tlp[bad]).all())
    y = x.clone()
    y[:, 5] = -INF
    assert torch.equal(top, R.top(y, 4))
    good = torch.tensor([0, 2, 5], device=DEV)
    a, b, c, d = _run(x[good].contiguous(), ids[good].contiguous(), 5, 4)
    assert torch.equal(lp[good], a) and torch.equal(ent[good], b) and torch.equal(tlp[good], d)


def test_targets_outside_and_masked(gpu):
    x = _logits(7, 4, 1000)
    ids = torch.tensor([[-1, 999, 3, 3], [1000, 0, 2 ** 31 - 1, -2 ** 31], [3, 3, 5, 6], [0, 1, 2, 3]],
                       dtype=I32, device=DEV)
    _check(x, ids, 3, 2)
    lp = _run(x, ids, 3, 2)[0]
    assert bool(torch.isneginf(lp[2, :2]).all()) and bool(torch.isnan(lp[1, [0, 2, 3]]).all())


def test_many_targets(gpu):
    x = _logits(8, 3, 2000)
    _check(x, _ids(8, 3, 1500, 2000), -1, 1)


def test_far_offsets(gpu):
    """Logits past 2^31 elements."""
    rows, vocab = 17100, 126464
    x = torch.zeros(rows, vocab, dtype=BF16, device=DEV)
    tail = _logits(9, 50, vocab, BF16)
    x[-50:] = tail
    ids = _ids(9, rows, 1, vocab)
    lp, ent, top, tlp = _run(x, ids, vocab - 1, 3)
    a, b, c, d = _run(tail, ids[-50:].contiguous(), vocab - 1, 3)
    # few rows may be cut into parts: the same sums in another order
    tol = R.scores_tol(vocab)
    assert float((lp[-50:] - a).abs().max()) <= 2 * tol and float((ent[-50:] - b).abs().max()) <= 2 * tol
    assert torch.equal(top[-50:], c)
    assert abs(float(ent[0]) - math.log(vocab - 1)) <= tol


def test_agrees_with_the_steps_statistics(gpu):
    """The confidence of the row statistics is the probability of the first alternative."""
    from paper_2608_23167_amd.decoder import Decoder
    from paper_2608_23167_amd.model import DeviceModel
    from synthetic import WORKLOADS, initial_tokens, make_weights
    wl = WORKLOADS["tiny"]
    dec = Decoder(wl, DeviceModel(wl.model, make_weights(wl.model, seed=0, norm_jitter=0.1).to("cuda:0")), device="cuda:0")
    dec.reset(initial_tokens(wl).to("cuda:0"))
    logits = torch.empty(dec.max_rows * wl.model.vocab, device=DEV)
    info = dec.step(0, True, logits=logits)
    x = logits[: info.n_out * wl.model.vocab].view(info.n_out, -1)
    argmax, conf = dec.argmax[: info.n_out], dec.conf[: info.n_out]
    lp, ent, top, tlp = _run(x, argmax[:, None].contiguous(), wl.model.mask_id, wl.topk)
    assert torch.equal(top.reshape(-1), dec.topk_ids[: info.n_out * wl.topk])
    tol = R.scores_tol(wl.model.vocab)
    # both sides are within tol of the exact value
    assert float((lp[:, 0].exp() / conf - 1).abs().max()) <= 2 * tol
    assert torch.equal(lp[:, 0], tlp[:, 0])


@pytest.mark.parametrize("rows,vocab", [(2, 126464), (50, 30000)])
def test_captured_and_on_another_stream(gpu, rows, vocab):
    from paper_2608_23167_amd import api
    x, ids = _logits(1, rows, vocab), _ids(1, rows, 1, vocab)
    lp, ent = torch.zeros(rows, 1, device=DEV), torch.zeros(rows, device=DEV)
    top, tlp = torch.zeros(rows, 4, dtype=I32, device=DEV), torch.zeros(rows, 4, device=DEV)
    ws = torch.zeros(max(16, api.ssm_token_logprobs_workspace_size(rows, vocab, 4)), dtype=torch.uint8, device=DEV)
    call = lambda: api.ssm_token_logprobs(x, ids, 0, 4, lp, ent, top, tlp, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        call()
    for seed in range(4):
        x.copy_(_logits(seed, rows, vocab))
        call()
        want = [t.clone() for t in (lp, ent, top, tlp)]
        for t in (lp, ent, tlp):
            t.fill_(5.0)
        ws.fill_(0xff)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip((lp, ent, top, tlp), want):
            assert torch.equal(t, w)
    other = _run(x, ids, 0, 4, stream=torch.cuda.Stream())
    for t, w in zip(other, (lp, ent, top, tlp)):
        assert torch.equal(t, w)
