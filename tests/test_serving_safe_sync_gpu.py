"""Packed prompts and 4-bit decoding in the library built with -DNAUT_SAFE_SYNC=1 (conservative synchronisation, see
tests/test_safe_sync_gpu.py): bit for bit what the shipped library gives."""
import math
import os

import numpy as np
import pytest
import torch

from paper_2604_14825_amd import binding as nb

pytestmark = pytest.mark.gpu

_libs = None


@pytest.fixture
def both(monkeypatch):
    """call(f) runs f with either library and returns what it gives, as bits."""
    global _libs
    if _libs is None:
        assert os.path.exists(nb.LIB_SAFE_PATH), "libnaut_attn_safe.so is missing: python -m paper_2604_14825_amd.build"
        _libs = (nb.lib(), nb.load(nb.LIB_SAFE_PATH))

    def call(f):
        out = []
        for L in _libs:
            monkeypatch.setattr(nb, "_lib", L)
            out.append([t.view(torch.int16 if t.element_size() == 2 else torch.int32).cpu().numpy() for t in f()])
        for a, b in zip(*out):
            assert np.array_equal(a, b), "the fast and the conservative build differ"
    return call


@pytest.mark.parametrize("D,variant", [(64, "w4q32"), (64, "w4q32g2"), (64, "w8q32"), (64, "bm128g4"), (80, "w4q32"), (96, "w4q32g2"), (128, "w4q32"),
                                       (128, "w4q32g2"), (128, "w8q32"), (128, "bm128g4"), (192, "w4q32"), (256, "w4q32"), (256, "w8q32")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_packed(D, variant, dtype, both, monkeypatch):
    monkeypatch.setenv("NAUT_ATTN_VARIANT", variant)
    gen = torch.Generator(device="cuda").manual_seed(D)
    q_lens, k_lens = [1, 63, 128, 500, 0, 257, 90], [40, 63, 700, 500, 3, 1300, 20]
    rows = lambda T, H, f: (torch.randn((T, H, D), device="cuda", generator=gen) * f).to(dtype)
    cu = lambda x: torch.tensor(np.concatenate([[0], np.cumsum(x)]).astype(np.int32), device="cuda")
    for causal in (True, False):
        for factor in (1.0, 6.0):  # moving maxima
            q, k, v = rows(sum(q_lens), 8, factor), rows(sum(k_lens), 2, 1.0), rows(sum(k_lens), 2, 1.0)

            def f():
                o, lse = torch.zeros_like(q), torch.zeros((8, q.shape[0]), device="cuda")
                nb.naut_attn_fwd_packed(q, k, v, o, lse, cu(q_lens), cu(k_lens), causal, 1 / math.sqrt(D))
                torch.cuda.synchronize()
                return o, lse
            print("packed", D, variant, dtype, causal, factor, flush=True)
            both(f)


@pytest.mark.parametrize("D", [32, 64, 128, 160, 256])
@pytest.mark.parametrize("Hq,Sq", [(4, 1), (40, 1), (8, 3)])
def test_decode(D, Hq, Sq, both):
    gen = torch.Generator(device="cuda").manual_seed(D)
    lens = [3000, 1, 700, 0, 33]
    cache = nb.KV4Cache.empty(5, 2, 3000, D)
    every = torch.arange(5 * 3000, dtype=torch.int32, device="cuda")
    nb.naut_kv4_store(*(torch.randn((5 * 3000, 2, D), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2)), cache, every)
    q = (3 * torch.randn((5, Hq, Sq, D), device="cuda", generator=gen)).to(torch.bfloat16)

    def f():
        o, lse = torch.zeros_like(q), torch.zeros((5, Hq, Sq), device="cuda")
        ws = torch.full((nb.decode_kv4_workspace_bytes(5, Hq, 2, Sq, 3000, D),), 0xFF, dtype=torch.uint8, device="cuda")
        nb.naut_attn_decode_kv4(q, o, lse, cache, torch.tensor(lens, dtype=torch.int32, device="cuda"), True, 1 / math.sqrt(D), ws)
        torch.cuda.synchronize()
        return o, lse
    print("decode", D, Hq, Sq, flush=True)
    both(f)
