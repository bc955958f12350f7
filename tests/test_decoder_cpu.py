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


def _ffn(**kw):
    from paper_2608_27735_amd import _lib
    f = _lib.abcd_ffn()
    f.dtype, f.act, f.d, f.h, f.o, f.p = F16, 0, 8, 16, 8, 0.1
    f.w_gate = f.w_up = f.w_down = FAKE
    for k, v in kw.items():
        setattr(f, k, v)
    return f


BAD_FFN = [dict(dtype=3), dict(act=3), dict(act=-1), dict(d=0), dict(h=0), dict(o=0), dict(d=65537), dict(h=65537),
           dict(p=-0.5), dict(p=1.5), dict(p=float("nan")), dict(w_gate=None), dict(w_up=None), dict(w_down=None),
           dict(w_up=FAKE + 1), dict(b_gate=FAKE + 1), dict(b_up=FAKE + 1), dict(b_down=FAKE + 1)]


def test_gated_ffn_refuses(lib):
    need = C.c_size_t(0)
    assert lib.abcd_gated_ffn_workspace_size(C.byref(_ffn()), 4, 0, C.byref(need)) == 0
    base = [C.byref(_ffn()), 4, FAKE, 8, FAKE, 8, FAKE, 8, FAKE, FAKE, FAKE, FAKE, need.value, None]
    refuse(base, lib.abcd_gated_ffn,
           [(0, None), (1, -1), (2, None), (3, 7), (4, FAKE + 1), (5, 7), (6, None), (7, 7), (8, None), (9, None),
            (10, None), (10, FAKE + 8), (11, None), (11, FAKE + 64), (12, 0)])
    refuse(base, lib.abcd_gated_ffn, [(0, C.byref(_ffn(**kw))) for kw in BAD_FFN])
    assert lib.abcd_gated_ffn_workspace_size(None, 4, 0, C.byref(need)) == 1
    assert lib.abcd_gated_ffn_workspace_size(C.byref(_ffn()), 4, 0, None) == 1


def test_gated_ffn_bwd_refuses(lib):
    need = C.c_size_t(0)
    assert lib.abcd_gated_ffn_bwd_workspace_size(C.byref(_ffn()), 4, 1, C.byref(need)) == 0
    base = [C.byref(_ffn()), 4, FAKE, 8, FAKE, 8, FAKE, FAKE, FAKE, FAKE, 8] + [FAKE] * 7 + [need.value, None]
    refuse(base, lib.abcd_gated_ffn_bwd,
           [(0, None), (1, -1), (2, None), (3, 7), (4, None), (5, 7), (6, None), (7, FAKE + 8), (8, None), (10, 7)] +
           [(i, FAKE + 1) for i in range(11, 17)] + [(17, None), (17, FAKE + 8), (18, need.value - 1)])
    refuse(base, lib.abcd_gated_ffn_bwd, [(0, C.byref(_ffn(**kw))) for kw in BAD_FFN])
    assert lib.abcd_gated_ffn_bwd_workspace_size(C.byref(_ffn()), -1, 1, C.byref(need)) == 1


@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
def test_reference_ffn_gradients_are_its_forwards(name):
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=R.F64)
    n, d, h, o = 5, 7, 9, 6
    x, dy, keep = r(n, d), r(n, o), r(n, o) > -0.3
    w = dict(w_gate=r(h, d), w_up=r(h, d), w_down=r(o, h), b_gate=r(h), b_up=r(h), b_down=r(o))
    leaves = {k: v.clone().requires_grad_() for k, v in {**w, "x": x}.items()}
    y = R.ffn(leaves["x"], {k: leaves[k] for k in w}, name, 0.0, None, keep, 0.25)["y"][0]
    want = dict(zip(leaves, torch.autograd.grad((y * dy).sum(), list(leaves.values()))))
    got = R.ffn(x, w, name, 0.0, None, keep, 0.25, dy)
    for k in want:
        assert torch.allclose(got[k][0], want[k], rtol=1e-10, atol=1e-12), k


def test_reference_generator_published_words():
    """Known answers published with the generator (4x32, 7 rounds): the words for
    counter 0 under key 0, and, as rows and offsets are counters too, for the digits of
    pi in both."""
    def words(quad, row, seed, offset):
        kept = []
        for j in range(4):  # the threshold at which a word is just kept, bit by bit
            at = 0
            for bit in range(31, -1, -1):
                p = (at + (1 << bit)) / 2.0 ** 32
                if _mask_row(quad, row, p, seed, offset)[j]:
                    at += 1 << bit
            kept.append(at)
        return kept

    assert words(0, 0, 0, 0) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    small = words(0, 3, (5 << 32) + 7, (9 << 32) + 11)
    assert small == _philox7([0, 3, 11, 9], [7, 5])
    assert _philox7([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == \
        [0x4DFCCABA, 0x190A87F0, 0xC47362BA, 0xB6B5242A]


def _mask_row(quad, row, p, seed, offset):
    return R.keep_mask(row + 1, 4 * quad + 4, p, seed, offset)[row, 4 * quad:]


def _philox7(c, k):
    """The generator in plain integers; the last case above pins it to the published
    words of a counter and key that no mask's row reaches."""
    for _ in range(7):
        h0, l0 = divmod(0xD2511F53 * c[0], 1 << 32)
        h1, l1 = divmod(0xCD9E8D57 * c[2], 1 << 32)
        c = [h1 ^ c[1] ^ k[0], l1, h0 ^ c[3] ^ k[1], l0]
        k = [(k[0] + 0x9E3779B9) % (1 << 32), (k[1] + 0xBB67AE85) % (1 << 32)]
    return c
