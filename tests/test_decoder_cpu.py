"""The decoder's entry points refuse bad arguments on the host, before any HIP
call, and the float64 definitions of their tests agree with differences."""
import ctypes as C
import os

import pytest
import torch

import decoder_ref as R

FAKE = 0x1000  # never dereferenced: every call below fails validation first
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2608_27735_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2608_27735_amd import build
        build.build()
    return _lib.load()


def refuse(base, call, cases):
    for i, v in cases:
        a = list(base)
        a[i] = v
        assert call(*a) == 1, (i, v)


def test_layer_norm_refuses(lib):
    base = [F16, 4, 8, FAKE, 8, F16, FAKE, FAKE, 1e-5, FAKE, 8, FAKE, FAKE, None]
    refuse(base, lib.abcd_layer_norm,
           [(0, 3), (0, -1), (1, -1), (1, (1 << 30) + 1), (2, 0), (2, 65537), (3, None), (3, FAKE + 1), (4, 7),
            (5, BF16), (6, FAKE + 1), (8, -1.0), (8, float("nan")), (8, float("inf")), (9, None), (9, FAKE + 1),
            (10, 7), (11, FAKE + 2), (12, FAKE + 2)])
    assert b"rows" in lib.abcd_last_error() or lib.abcd_last_error()


def test_layer_norm_bwd_refuses(lib):
    need = C.c_size_t(0)
    assert lib.abcd_layer_norm_bwd_workspace_size(F16, 4, 8, C.byref(need)) == 0 and need.value >= 64
    assert lib.abcd_layer_norm_bwd_workspace_size(F16, 4, 0, C.byref(need)) == 1
    assert lib.abcd_layer_norm_bwd_workspace_size(F16, 4, 8, None) == 1
    base = [F16, 4, 8, FAKE, 8, FAKE, 8, FAKE, FAKE, F16, FAKE, FAKE, 8, FAKE, 8, FAKE, FAKE, FAKE, need.value, None]
    refuse(base, lib.abcd_layer_norm_bwd,
           [(0, 9), (1, -1), (2, 0), (3, None), (4, 7), (5, None), (6, 7), (7, None), (8, None), (8, FAKE + 2),
            (9, BF16), (10, FAKE + 1), (12, 7), (14, 7), (15, FAKE + 1), (17, None), (17, FAKE + 8),
            (18, need.value - 1)])


def test_dropout_refuses(lib):
    base = [BF16, 4, 8, FAKE, 8, FAKE, 8, FAKE, 8, 0.5, 1, 2, None]
    refuse(base, lib.abcd_dropout,
           [(0, 5), (1, -1), (2, 0), (3, None), (4, 7), (5, FAKE + 1), (6, 7), (7, None), (8, 7), (9, -0.1), (9, 1.1),
            (9, float("nan"))])


def test_reference_layer_norm_gradient_is_its_forwards():
    g = torch.Generator().manual_seed(0)
    x, dy = (torch.randn(4, 9, generator=g, dtype=R.F64).requires_grad_() for _ in range(2))
    w, b = (torch.randn(9, generator=g, dtype=R.F64).requires_grad_() for _ in range(2))
    y, mean, rstd, _ = R.layer_norm(x, w, b, 1e-5)
    want = torch.autograd.grad((y * dy.detach()).sum(), (x, w, b))
    got = R.layer_norm_bwd(dy.detach(), x.detach(), mean.detach(), rstd.detach(), w.detach(), None)
    for k, v in zip(("x", "weight", "bias"), want):
        assert torch.allclose(got[k][0], v, rtol=1e-10, atol=1e-12), k


def test_reference_generator_known_block():
    """The generator's rounds by hand for counter 0 and key 0: one round gives
    zeros under a zero key, and each later round the key's Weyl words mixed in."""
    M = 0xFFFFFFFF
    c, k0, k1 = [0, 0, 0, 0], 0, 0
    for _ in range(7):
        h0, l0 = divmod(0xD2511F53 * c[0], 1 << 32)
        h1, l1 = divmod(0xCD9E8D57 * c[2], 1 << 32)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & M, (k1 + 0xBB67AE85) & M
    for j, word in enumerate(c):
        for p in (word / 2.0 ** 32, (word + 1) / 2.0 ** 32):
            assert bool(R.keep_mask(1, 4, p, 0, 0)[0, j]) == (word >= int(p * 2 ** 32))
