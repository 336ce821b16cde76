"""What the 8-bit projections and the scores of tokens refuse, on the host
before any GPU work (no GPU needed: no call here launches)."""
import ctypes as C

import pytest

from paper_2608_23167_amd import _lib as L

P1 = C.c_void_p(4096)          # never dereferenced: each call is refused, or has no rows
NULL = C.c_void_p(None)


def _refused(rc, code, word):
    assert rc == code, (rc, L.lib().ssm_last_error())
    assert word in L.lib().ssm_last_error().decode()


def _norm(rows=2, d=8, x=P1, delta=P1, ddt=0, gain=P1, gdt=1, eps=1e-5, resid=P1, q=P1, s=P1):
    return L.lib().ssm_norm_i8(rows, d, x, delta, ddt, gain, gdt, eps, resid, q, s, None)


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "sizes"), (dict(d=0), "sizes"), (dict(d=-4), "sizes"), (dict(rows=(1 << 24) + 1), "sizes"),
    (dict(d=(1 << 30) + 1), "sizes"),
    (dict(ddt=3), "delta_dtype"), (dict(gdt=2), "gain_dtype"), (dict(gdt=-1), "gain_dtype"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(x=NULL), "null"), (dict(gain=NULL), "null"), (dict(q=NULL), "null"), (dict(s=NULL), "null")])
def test_norm(kw, word):
    _refused(_norm(**kw), L.SSM_E_INVAL, word)


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "sizes"), (dict(d=0), "sizes"), (dict(d=(1 << 30) + 1), "sizes"), (dict(sw=2), "swiglu"),
    (dict(dt=3), "dtype"), (dict(x=NULL), "null"), (dict(q=NULL), "null"), (dict(s=NULL), "null")])
def test_quant(kw, word):
    a = dict(rows=2, d=8, sw=0, dt=0, x=P1, q=P1, s=P1) | kw
    _refused(L.lib().ssm_quant_i8(a["rows"], a["d"], a["sw"], a["dt"], a["x"], a["q"], a["s"], None),
             L.SSM_E_INVAL, word)


@pytest.mark.parametrize("kw,code,word", [
    (dict(m=-1), L.SSM_E_INVAL, "sizes"), (dict(n=0), L.SSM_E_INVAL, "sizes"), (dict(k=0), L.SSM_E_INVAL, "sizes"),
    (dict(k=131072), L.SSM_E_UNSUPPORTED, "overflow"), (dict(m=64 * 65535 + 1), L.SSM_E_UNSUPPORTED, "rows"),
    (dict(dt=3), L.SSM_E_INVAL, "out_dtype"), (dict(a=NULL), L.SSM_E_INVAL, "null"),
    (dict(sa=NULL), L.SSM_E_INVAL, "null"), (dict(w=NULL), L.SSM_E_INVAL, "null"),
    (dict(sw=NULL), L.SSM_E_INVAL, "null"), (dict(out=NULL), L.SSM_E_INVAL, "null")])
def test_gemm(kw, code, word):
    a = dict(m=2, n=8, k=32, a=P1, sa=P1, w=P1, sw=P1, dt=0, out=P1, ws=P1, wb=1 << 40) | kw
    _refused(L.lib().ssm_gemm_i8(a["m"], a["n"], a["k"], a["a"], a["sa"], a["w"], a["sw"], a["dt"], a["out"],
                                 a["ws"], a["wb"], None), code, word)


def _sizes():
    return [(1, 4096, 4096), (120, 4096, 4096), (240, 4096, 12288), (600, 1024, 8192), (1127, 3584, 18944)]


def test_gemm_workspace():
    b = C.c_size_t()
    for m, n, k in _sizes():
        assert L.lib().ssm_gemm_i8_workspace_size(m, n, k, C.byref(b)) == 0
        if b.value:
            _refused(L.lib().ssm_gemm_i8(m, n, k, P1, P1, P1, P1, 0, P1, P1, b.value - 1, None),
                     L.SSM_E_CAPACITY, "workspace")
            _refused(L.lib().ssm_gemm_i8(m, n, k, P1, P1, P1, P1, 0, P1, NULL, b.value, None),
                     L.SSM_E_INVAL, "workspace")
            _refused(L.lib().ssm_gemm_i8(m, n, k, P1, P1, P1, P1, 0, P1, C.c_void_p(4100), b.value, None),
                     L.SSM_E_INVAL, "aligned")
    for bad in ((1, 0, 1), (-1, 1, 1), (1, 1, 0)):
        _refused(L.lib().ssm_gemm_i8_workspace_size(*bad, C.byref(b)), L.SSM_E_INVAL, "sizes")
    _refused(L.lib().ssm_gemm_i8_workspace_size(1, 1, 1, None), L.SSM_E_INVAL, "null")


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "sizes"), (dict(vocab=0), "sizes"), (dict(k=9), "k 9"), (dict(k=-1), "k -1"),
    (dict(dt=3), "dtype"), (dict(mask=-2), "mask_id"), (dict(mask=100), "mask_id"), (dict(t=-1), "n_targets"),
    (dict(x=NULL), "null"), (dict(ids=NULL), "null"), (dict(lp=NULL), "null"), (dict(top=NULL), "null"),
    (dict(tlp=NULL), "null")])
def test_logprobs(kw, word):
    a = dict(rows=2, vocab=100, dt=0, x=P1, mask=99, t=1, ids=P1, k=3, lp=P1, ent=P1, top=P1, tlp=P1) | kw
    _refused(L.lib().ssm_token_logprobs(a["rows"], a["vocab"], a["dt"], a["x"], a["mask"], a["t"], a["ids"], a["k"],
                                        a["lp"], a["ent"], a["top"], a["tlp"], P1, 1 << 40, None),
             L.SSM_E_INVAL, word)


def test_logprobs_workspace():
    b = C.c_size_t()
    for rows, vocab in ((1, 152064), (120, 126464), (4000, 126464)):
        assert L.lib().ssm_token_logprobs_workspace_size(rows, vocab, 5, C.byref(b)) == 0
        if b.value:
            args = (rows, vocab, 0, P1, -1, 1, P1, 5, P1, P1, P1, P1)
            _refused(L.lib().ssm_token_logprobs(*args, P1, b.value - 1, None), L.SSM_E_CAPACITY, "workspace")
            _refused(L.lib().ssm_token_logprobs(*args, NULL, b.value, None), L.SSM_E_INVAL, "workspace")
    _refused(L.lib().ssm_token_logprobs_workspace_size(1, 1, 9, C.byref(b)), L.SSM_E_INVAL, "k 9")
    _refused(L.lib().ssm_token_logprobs_workspace_size(1, 1, 1, None), L.SSM_E_INVAL, "null")


def test_no_rows_need_no_pointers():
    assert _norm(rows=0, x=NULL, delta=NULL, gain=NULL, resid=NULL, q=NULL, s=NULL) == 0
    assert L.lib().ssm_quant_i8(0, 8, 0, 0, NULL, NULL, NULL, None) == 0
    assert L.lib().ssm_gemm_i8(0, 8, 32, NULL, NULL, NULL, NULL, 0, NULL, NULL, 0, None) == 0
    assert L.lib().ssm_token_logprobs(0, 8, 0, NULL, -1, 0, NULL, 0, NULL, NULL, NULL, NULL, NULL, 0, None) == 0


def test_binding_checks_shapes_and_places():
    import torch
    from paper_2608_23167_amd import api
    f, i8 = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.int8)
    s = torch.zeros(4)
    with pytest.raises(ValueError, match="gain"):
        api.ssm_norm_i8(f, torch.ones(7), 1e-5, i8, s)
    with pytest.raises(ValueError, match="delta"):
        api.ssm_norm_i8(f, torch.ones(8), 1e-5, i8, s, delta=torch.zeros(4, 7))
    with pytest.raises(ValueError, match="device"):
        api.ssm_norm_i8(f, torch.ones(8), 1e-5, i8, s)
    with pytest.raises(ValueError, match="x must be"):
        api.ssm_quant_i8(f, i8, s, swiglu=True)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        api.ssm_quant_i8(f.double(), i8, s)
    with pytest.raises(ValueError, match="w must be"):
        api.ssm_gemm_i8(i8, s, torch.zeros(3, 9, dtype=torch.int8), torch.zeros(3), torch.zeros(4, 3), None)
    with pytest.raises(ValueError, match="out must be"):
        api.ssm_gemm_i8(i8, s, i8, s, torch.zeros(4, 5), None)
    with pytest.raises(ValueError, match="go together"):
        api.ssm_token_logprobs(f, torch.zeros(4, 1, dtype=torch.int32), -1, 0, None, None, None, None, None)
    with pytest.raises(ValueError, match="needs top_ids"):
        api.ssm_token_logprobs(f, None, -1, 2, None, None, None, None, None)
