"""The 8-bit projections against plain 64-bit forms of the same operators."""
import pytest
import torch

import _i8_ref as R

pytestmark = pytest.mark.gpu

F32, BF16, F16, I8 = torch.float32, torch.bfloat16, torch.float16, torch.int8
DEV = "cuda"


def _rand(seed, *size, std=1.0, dtype=F32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(*size, generator=g, device=DEV) * std).to(dtype)


def _codes(seed, *size, lo=-128):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(lo, 128, size, generator=g, device=DEV, dtype=torch.int32).to(I8)


def _offset(t, elements):
    """The same values at an address `elements` elements past an aligned one."""
    flat = torch.empty(t.numel() + elements, dtype=t.dtype, device=t.device)
    v = flat[elements:].view(t.shape)
    v.copy_(t)
    return v


def _guarded(rows, d):
    """q [rows, d] and scale [rows], with a row behind the last that must be left as it was."""
    return torch.full((rows + 1, d), 99, dtype=I8, device=DEV), torch.full((rows + 1,), -1.0, device=DEV)


def _unguarded(q, s):
    assert bool((q[-1] == 99).all()) and float(s[-1]) == -1
    return q[:-1], s[:-1]


def _norm(x, gain, eps, delta=None, resid=None):
    from paper_2608_23167_amd import api
    q, s = _guarded(*x.shape)
    api.ssm_norm_i8(x, gain, eps, q[:-1], s[:-1], delta=delta, resid=resid)
    return _unguarded(q, s)


def _quant(x, swiglu=False):
    from paper_2608_23167_amd import api
    d = x.shape[1] // 2 if swiglu else x.shape[1]
    q, s = _guarded(x.shape[0], d)
    api.ssm_quant_i8(x, q[:-1], s[:-1], swiglu=swiglu)
    return _unguarded(q, s)


def _gemm(a, sa, w, sw, dtype, ws_extra=0):
    from paper_2608_23167_amd import api
    m, n, k = a.shape[0], w.shape[0], a.shape[1]
    need = api.ssm_gemm_i8_workspace_size(m, n, k)
    ws = torch.full((need + ws_extra,), 0x5a, dtype=torch.uint8, device=DEV) if need else None
    # a guard row behind the last one must be left as it was
    out = torch.full((m + 1, n), 7.0, dtype=dtype, device=DEV)
    api.ssm_gemm_i8(a, sa, w, sw, out[:m], ws)
    assert bool((out[m:] == 7.0).all())
    return out[:m]


# ---- norm ---------------------------------------------------------------------
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 4096), (3, 127), (5, 128), (17, 1000), (33, 512),
                                    (129, 3584), (7, 4096), (2, 8192), (3, 8196), (2, 20000),
                                    (300, 4095), (2, 8191), (2, 20001), (3, 33001), (2, 40000)])
@pytest.mark.parametrize("delta", [None, F32, BF16, F16])
def test_norm(gpu, rows, d, delta):
    gain = _rand(3, d, std=0.2, dtype=BF16 if rows % 2 else F32) + 1
    x = _rand(1, rows, d) * torch.exp(_rand(2, rows, 1))
    dl = None if delta is None else _rand(4, rows, d, std=0.5, dtype=delta)
    resid = torch.full_like(x, -7.0)
    q, s = _norm(x, gain, 1e-5, dl, resid)
    r = x if dl is None else x + dl.float()
    assert torch.equal(resid, r)
    R.check_codes(q, s, R.norm(r, gain, 1e-5), R.norm_rel(d))


@pytest.mark.parametrize("d", [512, 513, 4096])
def test_norm_in_place_and_without_residual_output(gpu, d):
    x, dl = _rand(1, 9, d), _rand(2, 9, d)
    gain = torch.ones(d, device=DEV)
    q0, s0 = _norm(x.clone(), gain, 1e-5, dl)
    for mine, other in ((0, 1), (1, 0)):
        both = [x.clone(), dl.clone()]
        q, s = _norm(both[0], gain, 1e-5, both[1], resid=both[mine])
        assert torch.equal(q, q0) and torch.equal(s, s0)
        assert torch.equal(both[mine], x + dl)
        assert torch.equal(both[other], [x, dl][other])


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("d", [256, 1000])
def test_norm_unaligned(gpu, d, shift):
    """Every operand at an address that only its element type allows."""
    x, dl, gain = _rand(1, 6, d), _rand(2, 6, d, dtype=BF16), _rand(3, d, dtype=BF16)
    q = _offset(torch.zeros(6, d, dtype=I8, device=DEV), shift)
    s, resid = torch.empty(6, device=DEV), _offset(x, shift)
    from paper_2608_23167_amd import api
    api.ssm_norm_i8(_offset(x, shift), _offset(gain, shift), 1e-6, q, s, delta=_offset(dl, shift), resid=resid)
    r = x + dl.float()
    assert torch.equal(resid, r)
    R.check_codes(q, s, R.norm(r, gain, 1e-6), R.norm_rel(d))


@pytest.mark.parametrize("d", [640, 4096, 4099, 33000])
def test_norm_special_rows(gpu, d):
    x = _rand(1, 6, d)
    x[0] = 0
    x[1, d // 2] = float("nan")
    x[2, d - 1] = float("inf")
    x[3] = 1e-30            # mean of squares below eps: y is tiny but above 2^-100
    x[4] = 0
    x[4, 3] = -5.0
    q, s = _norm(x, torch.ones(d, device=DEV), 1e-5)
    assert float(s[0]) == 0 and not bool(q[0].any())
    assert bool(torch.isnan(s[1:3]).all()) and not bool(q[1:3].any())
    ok = torch.tensor([0, 3, 4, 5], device=DEV)
    R.check_codes(q[ok], s[ok], R.norm(x[ok], torch.ones(d, device=DEV), 1e-5), R.norm_rel(d))


def test_norm_without_eps(gpu):
    """Without eps a row of zeros has no norm: NaN scale, codes 0; other rows are not touched by it."""
    x = _rand(1, 3, 200)
    x[1] = 0
    q, s = _norm(x, torch.ones(200, device=DEV), 0.0)
    assert bool(torch.isnan(s[1])) and not bool(q[1].any())
    ok = torch.tensor([0, 2], device=DEV)
    R.check_codes(q[ok], s[ok], R.norm(x[ok], torch.ones(200, device=DEV), 0.0), R.norm_rel(200))


# ---- rows to codes --------------------------------------------------------------
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 12288), (3, 127), (5, 128), (17, 1000), (240, 512),
                                    (7, 3584), (3, 6000), (2, 18944), (3, 20001), (2, 40000), (1, 40003)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("swiglu", [False, True])
def test_quant(gpu, rows, d, dtype, swiglu):
    x = _rand(5, rows, 2 * d if swiglu else d, std=2.0, dtype=dtype)
    q, s = _quant(x, swiglu)
    R.check_codes(q, s, R.swiglu(x, d) if swiglu else x.double(), R.SWIGLU_REL if swiglu else 0.0)


@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,shift", [(64, 1), (64, 2), (65, 0), (1027, 3), (4096, 1)])
def test_quant_unaligned(gpu, d, shift, dtype, swiglu):
    from paper_2608_23167_amd import api
    x = _rand(6, 5, 2 * d if swiglu else d, dtype=dtype)
    q = _offset(torch.zeros(5, d, dtype=I8, device=DEV), shift)
    s = torch.empty(5, device=DEV)
    api.ssm_quant_i8(_offset(x, shift), q, s, swiglu=swiglu)
    R.check_codes(q, s, R.swiglu(x, d) if swiglu else x.double(), R.SWIGLU_REL if swiglu else 0.0)


@pytest.mark.parametrize("d", [96, 3584, 20000, 33000])
def test_quant_special_rows(gpu, d):
    x = torch.zeros(8, d, device=DEV)
    x[1] = 1e-39                                   # denormals: zero, scale 0
    x[2] = 2.0 ** -99
    x[3] = 3e38
    x[3, 0] = -3.4e38
    x[4, d - 1] = float("nan")
    x[5, 0] = float("-inf")
    x[6] = torch.arange(d, device=DEV) % 255 - 127.0   # every code, exactly
    x[7, 5] = 1.0
    q, s = _quant(x)
    assert not bool(q[[0, 1, 4, 5]].any()) and not bool(s[:2].any()) and bool(torch.isnan(s[4:6]).all())
    ok = torch.tensor([0, 1, 2, 3, 6, 7], device=DEV)
    R.check_codes(q[ok], s[ok], x[ok].double(), 0.0)


def test_swiglu_of_large_gates(gpu):
    """exp(-gate) overflows for a gate far below zero: the product is zero, not NaN."""
    x = torch.tensor([[-200.0, 100.0, -88.8, 5.0, 2.0, 3.0, 4.0, -1.0]], device=DEV)
    q, s = _quant(x, swiglu=True)
    assert float(s[0]) > 0 and int(q[0, 0]) == 0 and int(q[0, 1]) == 127
    R.check_codes(q, s, R.swiglu(x, 4), R.SWIGLU_REL)


# ---- products -----------------------------------------------------------------
SIZES = [(1, 1, 1), (1, 16, 16), (1, 4096, 4096), (2, 33, 48), (5, 100, 100), (16, 64, 128), (17, 65, 144),
         (31, 257, 1040), (32, 512, 512), (33, 130, 2064), (48, 4096, 1024), (64, 96, 4096), (65, 640, 1008),
         (120, 1000, 4096), (127, 77, 511), (128, 128, 128), (129, 4100, 272), (240, 512, 12288),
         (250, 255, 1024), (256, 256, 256), (257, 513, 640), (376, 1536, 512), (513, 3584, 1152),
         (700, 300, 1001), (1127, 896, 2368), (2049, 1030, 400)]

# every tile, and every number of K splits, with rows, columns and K that end inside a tile
TILE_SIZES = [(30, 1008, 352), (1101, 157, 3904), (1084, 129, 3088), (68, 186, 2608), (191, 198, 3248),
              (25, 126, 5696), (1382, 603, 320), (950, 2114, 320), (1033, 9943, 1360), (27, 18307, 416),
              (949, 1156, 336), (517, 3333, 576), (1064, 2780, 528), (2498, 1597, 784), (262, 14266, 1168),
              (2105, 2519, 816), (301, 21310, 944), (2379, 277, 5648), (641, 663, 6624), (885, 587, 4768),
              (82, 1514, 4784), (79, 5656, 6160), (68, 8503, 6288), (2894, 323, 4112), (2915, 1493, 912),
              (412, 10959, 912), (262, 20255, 1392), (575, 16431, 1104), (2588, 1201, 672),
              (1351, 155, 5696), (133, 2058, 6176)]


@pytest.mark.parametrize("m,n,k", SIZES + TILE_SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gemm(gpu, m, n, k, dtype):
    a, w = _codes(m + k, m, k), _codes(n + 7, n, k)
    sa, sw = torch.exp(_rand(1, m)) / k, torch.exp(_rand(2, n)) / 100
    R.check_gemm(_gemm(a, sa, w, sw, dtype), a, sa, w, sw)


@pytest.mark.parametrize("m,n,k", [(3, 200, 256), (40, 96, 1024), (140, 260, 512), (300, 512, 384)])
@pytest.mark.parametrize("shift", [1, 4, 8])
def test_gemm_unaligned(gpu, m, n, k, shift):
    a, w = _codes(1, m, k), _codes(2, n, k)
    sa, sw = _rand(1, m).abs() + 0.1, _rand(2, n).abs() + 0.1
    for x, y in ((_offset(a, shift), w), (a, _offset(w, shift))):
        R.check_gemm(_gemm(x, sa, y, sw, F32), a, sa, w, sw)
    # outputs at an odd element
    from paper_2608_23167_amd import api
    need = api.ssm_gemm_i8_workspace_size(m, n, k)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    out = _offset(torch.zeros(m, n, dtype=BF16, device=DEV), shift)
    api.ssm_gemm_i8(a, _offset(sa, shift), w, _offset(sw, shift), out, ws)
    R.check_gemm(out, a, sa, w, sw)


@pytest.mark.parametrize("m,k", [(1, 131056), (20, 131056), (100, 131056), (300, 131071), (9, 131071)])
def test_gemm_largest_sums(gpu, m, k):
    """Every code -128 at the longest rows: the sums come to 2^31 - 2^14 k's
    remainder, the largest an int32 holds."""
    a, w = torch.full((m, k), -128, dtype=I8, device=DEV), torch.full((70, k), -128, dtype=I8, device=DEV)
    w[1] = 127
    sa, sw = torch.ones(m, device=DEV), torch.ones(70, device=DEV)
    R.check_gemm(_gemm(a, sa, w, sw, F32), a, sa, w, sw)


@pytest.mark.parametrize("m", [1, 50, 200])
def test_gemm_scales(gpu, m):
    """A NaN scale spoils its row alone, a zero scale clears it, float16 overflows to infinity."""
    a, w = _codes(1, m + 3, 512), _codes(2, 320, 512)
    sa, sw = torch.ones(m + 3, device=DEV), torch.ones(320, device=DEV)
    sa[0], sa[1], sa[2] = float("nan"), 0.0, 1e30
    out = _gemm(a, sa, w, sw, F16)
    ref = R.gemm(a, sa, w, sw)
    assert bool(torch.isnan(out[0]).all()) and not bool(out[1].any())
    assert torch.equal(out[2], torch.where(ref[2] == 0, 0.0, ref[2].sign() * float("inf")).to(F16))
    out = _gemm(a, sa, w, sw, F32)
    R.check_gemm(out[1:], a[1:], sa[1:], w, sw)


def test_gemm_far_offsets(gpu):
    """Outputs and weights past 2^31 elements."""
    m, n, k = 17000, 126464, 16
    a, w = _codes(1, m, k), _codes(2, n, k)
    sa, sw = _rand(1, m).abs() + 0.1, _rand(2, n).abs() + 0.1
    out = _gemm(a, sa, w, sw, BF16)
    R.check_gemm(out[-130:], a[-130:], sa[-130:], w, sw)
    del out
    k = 131056
    w = _codes(3, 16500, k)                      # 2.16e9 codes
    a = _codes(4, 24, k)
    sw = torch.ones(16500, device=DEV)
    out = _gemm(a, sa[:24].contiguous(), w, sw, F32)
    R.check_gemm(out[:, -130:], a, sa[:24], w[-130:], sw[-130:])


def test_gemm_same_result_every_time(gpu):
    for m, n, k in ((3, 4096, 4096), (120, 4096, 4096), (600, 1024, 8192)):
        a, w = _codes(1, m, k), _codes(2, n, k)
        sa, sw = _rand(1, m).abs(), _rand(2, n).abs()
        first = _gemm(a, sa, w, sw, F32)
        for _ in range(5):
            assert torch.equal(_gemm(a, sa, w, sw, F32, ws_extra=64), first)


def test_no_rows(gpu):
    from paper_2608_23167_amd import api
    z = torch.empty(0, 64, dtype=I8, device=DEV)
    s = torch.empty(0, device=DEV)
    api.ssm_gemm_i8(z, s, _codes(1, 32, 64), torch.ones(32, device=DEV), torch.empty(0, 32, device=DEV), None)
    api.ssm_quant_i8(torch.empty(0, 64, device=DEV), z, s)
    api.ssm_norm_i8(torch.empty(0, 64, device=DEV), torch.ones(64, device=DEV), 1e-5, z, s)
    torch.cuda.synchronize()


# ---- together -------------------------------------------------------------------
class Block:
    """A feed-forward block and a head in 8 bits, and the scores of its tokens,
    with every buffer kept."""

    def __init__(self, rows, d, ffn, vocab, seed=0):
        from paper_2608_23167_amd import api
        self.api, self.rows, self.d, self.ffn, self.vocab = api, rows, d, ffn, vocab
        e = lambda *s, t=F32: torch.zeros(*s, dtype=t, device=DEV)  # noqa: E731
        self.x, self.resid = _rand(seed, rows, d), e(rows, d)
        self.g1, self.g2 = _rand(11, d, std=0.1, dtype=BF16) + 1, _rand(12, d, std=0.1, dtype=BF16) + 1
        self.w, self.sw = [], []
        for i, (o, k) in enumerate(((2 * ffn, d), (d, ffn), (vocab, d))):
            w, q, s = _rand(20 + i, o, k, std=k ** -0.5, dtype=BF16), e(o, k, t=I8), e(o)
            api.ssm_quant_i8(w, q, s)
            self.w.append(q)
            self.sw.append(s)
        self.q, self.s = e(rows, d, t=I8), e(rows)
        self.gu, self.fq, self.fs = e(rows, 2 * ffn, t=BF16), e(rows, ffn, t=I8), e(rows)
        self.down, self.hq, self.hs = e(rows, d, t=BF16), e(rows, d, t=I8), e(rows)
        self.logits = e(rows, vocab, t=F32)
        self.ids = torch.randint(0, vocab, (rows, 2), device=DEV, dtype=torch.int32)
        self.lp, self.ent = e(rows, 2), e(rows)
        self.top, self.toplp = e(rows, 5, t=torch.int32), e(rows, 5)
        need = max(max(api.ssm_gemm_i8_workspace_size(rows, w.shape[0], w.shape[1]) for w in self.w),
                   api.ssm_token_logprobs_workspace_size(rows, vocab, 5), 16)
        self.ws = torch.zeros(need, dtype=torch.uint8, device=DEV)

    def run(self):
        api, w, sw, ws = self.api, self.w, self.sw, self.ws
        api.ssm_norm_i8(self.x, self.g1, 1e-5, self.q, self.s)
        api.ssm_gemm_i8(self.q, self.s, w[0], sw[0], self.gu, ws)
        api.ssm_quant_i8(self.gu, self.fq, self.fs, swiglu=True)
        api.ssm_gemm_i8(self.fq, self.fs, w[1], sw[1], self.down, ws)
        api.ssm_norm_i8(self.x, self.g2, 1e-5, self.hq, self.hs, delta=self.down, resid=self.resid)
        api.ssm_gemm_i8(self.hq, self.hs, w[2], sw[2], self.logits, ws)
        api.ssm_token_logprobs(self.logits, self.ids, self.vocab - 1, 5, self.lp, self.ent, self.top,
                               self.toplp, ws)

    def outputs(self):
        return [t.clone() for t in (self.resid, self.logits, self.lp, self.ent, self.top, self.toplp)]

    def check(self):
        """Each call against its 64-bit form on what it was given."""
        R.check_codes(self.q, self.s, R.norm(self.x, self.g1, 1e-5), R.norm_rel(self.d))
        R.check_gemm(self.gu, self.q, self.s, self.w[0], self.sw[0])
        R.check_codes(self.fq, self.fs, R.swiglu(self.gu, self.ffn), R.SWIGLU_REL)
        R.check_gemm(self.down, self.fq, self.fs, self.w[1], self.sw[1])
        assert torch.equal(self.resid, self.x + self.down.float())
        R.check_codes(self.hq, self.hs, R.norm(self.resid, self.g2, 1e-5), R.norm_rel(self.d))
        R.check_gemm(self.logits, self.hq, self.hs, self.w[2], self.sw[2])
        x, logp, ent = R.scores(self.logits, self.vocab - 1)
        tol = R.scores_tol(self.vocab)
        ref = logp.gather(1, self.ids.long())
        fine = ref > float("-inf")
        assert torch.equal(torch.isneginf(self.lp), ~fine)
        assert float((self.lp.double() - ref)[fine].abs().max()) <= tol
        assert float((self.ent.double() - ent).abs().max()) <= tol
        assert torch.equal(self.top, R.top(x, 5))
        assert float((self.toplp.double() - logp.gather(1, self.top.long())).abs().max()) <= tol


@pytest.mark.parametrize("rows,d,ffn,vocab", [(1, 128, 512, 512), (33, 256, 768, 1024), (120, 512, 1536, 4000),
                                              (300, 384, 1024, 2001)])
def test_feed_forward_and_head_in_8_bits(gpu, rows, d, ffn, vocab):
    b = Block(rows, d, ffn, vocab)
    b.run()
    b.check()


def test_captured_and_replayed(gpu):
    """A captured run replays with new inputs, with the same buffers used eagerly between."""
    for rows in (2, 40, 130):
        b = Block(rows, 512, 1536, 4000)
        b.run()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            b.run()
        for seed in range(4):
            b.x.copy_(_rand(50 + seed, rows, 512))
            b.run()
            want = b.outputs()
            for t in (b.resid, b.logits, b.lp, b.ent, b.toplp):
                t.fill_(-3.0)
            b.ws.fill_(0xff)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(b.outputs(), want):
                assert torch.equal(x, y)
            b.check()


def test_two_streams_at_once(gpu):
    """Two blocks on two streams, each with its own workspace, do not touch each other's."""
    bs = [Block(120, 512, 1536, 4000, seed=s) for s in (1, 2)]
    for b in bs:
        b.run()
    torch.cuda.synchronize()
    want = [b.outputs() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    for _ in range(10):
        for b, st in zip(bs, streams):
            with torch.cuda.stream(st):
                b.run()
    torch.cuda.synchronize()
    for b, w in zip(bs, want):
        for x, y in zip(b.outputs(), w):
            assert torch.equal(x, y)
