"""Child process of tests/test_gpu_debug_i8.py: runs the 8-bit projections and the token
scores through the library named on the command line and saves every output.  Not a
test module (pytest does not collect it)."""
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))


def run_cases():
    """(name -> array) of the outputs of the cases, through whatever library
    paper_2608_23167_amd._lib has loaded."""
    import torch
    from paper_2608_23167_amd import api
    from test_gpu_i8 import SIZES, TILE_SIZES
    out = {}
    dev, i8, i32 = "cuda:0", torch.int8, torch.int32
    g = torch.Generator(device=dev)

    def rand(*size):
        return torch.randn(*size, generator=g, device=dev)

    def codes(*size):
        return torch.randint(-127, 128, size, generator=g, device=dev, dtype=i32).to(i8)

    g.manual_seed(1)
    for d in (1, 130, 1000, 3584, 4099, 8192, 12288, 18944, 32768, 40000):
        x = rand(5, 2 * d)
        x[3] = 0
        q, s = torch.empty(5, d, dtype=i8, device=dev), torch.empty(5, device=dev)
        for name, call in (("norm", lambda: api.ssm_norm_i8(x[:, :d].contiguous(), rand(d), 1e-5, q, s)),
                           ("swiglu", lambda: api.ssm_quant_i8(x, q, s, swiglu=True)),
                           ("rows", lambda: api.ssm_quant_i8(x[:, :d].bfloat16(), q, s))):
            call()
            out[f"{name}_{d}_q"], out[f"{name}_{d}_s"] = q.cpu().numpy(), s.cpu().numpy()
    for m, n, k in SIZES + TILE_SIZES[::3]:
        a, w, sa, sw = codes(m, k), codes(n, k), rand(m), rand(n)
        ws = torch.empty(api.ssm_gemm_i8_workspace_size(m, n, k), dtype=torch.uint8, device=dev)
        y = torch.empty(m, n, device=dev)
        api.ssm_gemm_i8(a, sa, w, sw, y, ws)
        out[f"gemm_{m}_{n}_{k}"] = y.cpu().numpy()
    for rows, vocab, k in ((1, 1, 1), (3, 500, 8), (2, 4097, 0), (2, 16384, 5), (1, 152064, 5), (120, 60001, 8),
                           (400, 5000, 3)):
        x = rand(rows, vocab)
        ids = torch.randint(0, vocab, (rows, 2), generator=g, device=dev, dtype=i32)
        lp, ent = torch.empty(rows, 2, device=dev), torch.empty(rows, device=dev)
        top, tlp = torch.empty(rows, k, dtype=i32, device=dev), torch.empty(rows, k, device=dev)
        ws = torch.empty(api.ssm_token_logprobs_workspace_size(rows, vocab, k), dtype=torch.uint8, device=dev)
        api.ssm_token_logprobs(x, ids, vocab - 1 if vocab > 1 else -1, k, lp, ent, top, tlp, ws)
        for name, t in (("lp", lp), ("ent", ent), ("top", top), ("tlp", tlp)):
            out[f"{name}_{rows}_{vocab}"] = t.cpu().numpy()
    return out


if __name__ == "__main__":
    from paper_2608_23167_amd import _lib
    _lib.use_library(sys.argv[1])
    np.savez(sys.argv[2], **run_cases())
