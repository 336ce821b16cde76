"""Row operators at more rows than one launch can hold: a launch takes fewer than 2^32
threads along an axis, and a row takes up to 1024 of them."""
import pytest
import torch

import _i8_ref as R

pytestmark = pytest.mark.gpu

F32, BF16, I8, I32 = torch.float32, torch.bfloat16, torch.int8, torch.int32
DEV = "cuda"


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _rand(seed, *size):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*size, generator=g, device=DEV)


def _some(rows, at):
    """The first and last rows, and those around the end of a first launch of `at` rows."""
    return torch.tensor([0, 1, at - 2, at - 1, at, at + 1, rows - 2, rows - 1], device=DEV)


def _check_rows(q, s, some, y, rel):
    """Rows `some` have codes of y, all others are zero: written, and with nothing in them."""
    R.check_codes(q[some], s[some], y, rel)
    s[some] = 0.0
    q[some] = 0
    assert not bool(s.any())
    for part in q.split(1 << 20):
        assert not bool(part.any())


def test_quant_of_wide_rows(gpu):
    rows, d = (1 << 22) + 5, 4104                    # 1024 threads a row
    x = torch.zeros(rows, d, dtype=BF16, device=DEV)
    some = _some(rows, (1 << 22) - 1)
    x[some] = _rand(1, len(some), d).to(BF16)
    q, s = torch.full((rows, d), 99, dtype=I8, device=DEV), torch.full((rows,), -1.0, device=DEV)
    from paper_2608_23167_amd import api
    api.ssm_quant_i8(x, q, s)
    _check_rows(q, s, some, x[some].double(), 0.0)


def test_norm_of_the_most_rows(gpu):
    rows, d = 1 << 24, 1028                          # 256 threads a row
    x = torch.zeros(rows, d, device=DEV)
    some = _some(rows, (1 << 24) - 1 - 8)
    x[some] = _rand(2, len(some), d)
    q, s = torch.full((rows, d), 99, dtype=I8, device=DEV), torch.full((rows,), -1.0, device=DEV)
    gain = _rand(3, d).abs() + 0.5
    from paper_2608_23167_amd import api
    api.ssm_norm_i8(x, gain, 1e-5, q, s, resid=x)
    _check_rows(q, s, some, R.norm(x[some], gain, 1e-5), R.norm_rel(d))


def test_scores_of_the_most_rows(gpu):
    rows, vocab = 1 << 24, 2052                      # 4 waves a row
    x = torch.zeros(rows, vocab, dtype=BF16, device=DEV)
    some = _some(rows, (1 << 24) - 1 - 8)
    x[some] = _rand(4, len(some), vocab).to(BF16)
    ids = torch.zeros(rows, 1, dtype=I32, device=DEV)
    ids[some] = 2051
    lp, ent = torch.full((rows, 1), 7.0, device=DEV), torch.full((rows,), 7.0, device=DEV)
    top, tlp = torch.full((rows, 2), -7, dtype=I32, device=DEV), torch.full((rows, 2), 7.0, device=DEV)
    from paper_2608_23167_amd import api
    api.ssm_token_logprobs(x, ids, 1, 2, lp, ent, top, tlp, None)
    ref, logp, h = R.scores(x[some], 1)
    tol = R.scores_tol(vocab)
    assert float((lp[some, 0].double() - logp[:, 2051]).abs().max()) <= tol
    assert float((ent[some].double() - h).abs().max()) <= tol
    assert torch.equal(top[some], R.top(ref, 2))
    # the others: uniform over vocab - 1 tokens, all alike
    rest = torch.ones(rows, dtype=torch.bool, device=DEV)
    rest[some] = False
    for t in (lp, ent, top, tlp):
        t = t[rest]
        assert bool((t == t[0]).all())
    assert abs(float(ent[5]) - float(torch.log(torch.tensor(vocab - 1.0)))) <= tol
    assert top[5].tolist() == [0, 2]
