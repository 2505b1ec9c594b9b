"""CPU checks of the row operators (layer norm, rotary positions, gated feed-forward): host-side validation rejects
bad arguments before any HIP call, and the workspace sizes cover what the calls write."""
import ctypes
import math
import os

import pytest
import torch

from paper_1904_08755_amd import gsc

FAKE = ctypes.c_void_p(0x1000)   # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(gsc.LIB_PATH):
        pytest.skip("libgsc.so not built")
    return gsc.lib()


def _err(L):
    return L.gsc_last_error().decode()


def test_layer_norm_validation(L):
    fwd = lambda dt=0, n=10, c=8, X=FAKE, Y=FAKE, eps=1e-5: L.gsc_layer_norm_fwd(dt, X, n, c, None, None, eps, Y, None,
                                                                                None, None)
    assert fwd(dt=2) == gsc.GSC_EINVAL and "dtype" in _err(L)
    assert fwd(n=-1) == gsc.GSC_EINVAL
    assert fwd(c=0) == gsc.GSC_EINVAL and "c=0" in _err(L)
    assert fwd(c=(1 << 30) + 1) == gsc.GSC_EINVAL
    assert fwd(X=None) == gsc.GSC_EINVAL
    assert fwd(Y=None) == gsc.GSC_EINVAL
    for eps in (-1e-5, math.nan, math.inf):
        assert fwd(eps=eps) == gsc.GSC_EINVAL and "eps" in _err(L)
    assert fwd(n=0, X=None, Y=None) == gsc.GSC_OK   # no rows: nothing is read or launched
    need = L.gsc_layer_norm_bwd_ws_bytes(1000, 32)
    assert need >= 250 * 2 * 32 * 4 and L.gsc_layer_norm_bwd_ws_bytes(0, 32) == 2 * 32 * 4
    assert L.gsc_layer_norm_bwd_ws_bytes(-1, 32) == 0 and L.gsc_layer_norm_bwd_ws_bytes(5, 0) == 0
    assert L.gsc_layer_norm_bwd_ws_bytes(10**9, 32) == 1024 * 2 * 32 * 4
    bwd = lambda dt=0, n=1000, c=32, mean=FAKE, dX=FAKE, dg=FAKE, ws=FAKE, wsb=need: L.gsc_layer_norm_bwd(
        dt, FAKE, FAKE, n, c, None, mean, FAKE, dX, dg, None, ws, wsb, None)
    assert bwd(dt=-1) == gsc.GSC_EINVAL
    assert bwd(c=0) == gsc.GSC_EINVAL
    assert bwd(mean=None) == gsc.GSC_EINVAL
    assert bwd(ws=None) == gsc.GSC_ESHORT and str(need) in _err(L)
    assert bwd(wsb=need - 1) == gsc.GSC_ESHORT
    assert bwd(ws=ctypes.c_void_p(0x1002)) == gsc.GSC_EINVAL and "aligned" in _err(L)
    assert bwd(dX=None, dg=None, ws=None, wsb=0) == gsc.GSC_OK     # nothing asked for
    assert bwd(n=0, dg=None, ws=None, wsb=0) == gsc.GSC_OK


def test_rotary_validation(L):
    def rot(dt=0, X=FAKE, n=10, heads=2, d=8, ldx=16, coords=FAKE, D=3, pairs=(1, 1, 1), scale=None, base=1e4, pairing=0,
            Y=FAKE, ldy=16):
        pa = None if pairs is None else (ctypes.c_int32 * 8)(*pairs)
        sc = None if scale is None else (ctypes.c_double * 8)(*scale)
        return L.gsc_rotary(dt, X, n, heads, d, ldx, coords, D, pa, sc, base, pairing, 0, Y, ldy, None)

    for bad in (dict(dt=5), dict(n=-1), dict(heads=0), dict(d=7), dict(d=0), dict(d=4098, ldx=1 << 20, ldy=1 << 20),
                dict(ldx=15), dict(ldy=15), dict(D=0), dict(D=8, pairs=[0] * 8), dict(pairs=None), dict(pairs=(2, 2, 1)),
                dict(pairs=(1, -1, 1)), dict(pairs=(2**30, 2**30, 2**31 - 1)), dict(scale=(1, math.nan, 1)),
                dict(scale=(1, 1, 2e6)), dict(base=0.5), dict(base=math.inf), dict(base=math.nan), dict(pairing=2),
                dict(X=None), dict(Y=None), dict(coords=None), dict(ldy=17),
                dict(heads=1 << 20, d=1 << 10, ldx=1 << 40, ldy=1 << 40)):
        assert rot(**bad) == gsc.GSC_EINVAL, bad
        assert "rotary" in _err(L), bad
    assert rot(n=0, X=None, Y=None, coords=None) == gsc.GSC_OK


def test_gated_ffn_validation(L):
    need = L.gsc_gated_ffn_fwd_ws_bytes(gsc.GSC_BF16, 100, 64, 267, 64)
    assert need >= 100 * 272 * 2   # hidden rows padded to whole 16-byte pieces
    assert L.gsc_gated_ffn_fwd_ws_bytes(gsc.GSC_F32, 100, 64, 256, 64) >= 100 * 256 * 4
    for bad in ((7, 100, 64, 64, 64), (0, -1, 64, 64, 64), (0, 1, 0, 64, 64), (0, 1, 64, 0, 64), (0, 1, 64, 64, 0),
                (0, 1, (1 << 20) + 1, 64, 64)):
        assert L.gsc_gated_ffn_fwd_ws_bytes(*bad) == 0 and L.gsc_gated_ffn_bwd_ws_bytes(*bad) == 0
    fwd = lambda dt=1, X=FAKE, n=100, ci=64, f=267, co=64, act=0, Y=FAKE, ws=FAKE, wsb=need: L.gsc_gated_ffn_fwd(
        dt, X, n, ci, FAKE, FAKE, f, FAKE, co, act, Y, ws, wsb, None)
    for bad in (dict(dt=3), dict(X=None), dict(n=-1), dict(ci=0), dict(f=0), dict(co=0), dict(act=5), dict(act=-1),
                dict(Y=None), dict(f=1 << 21), dict(n=1 << 34, f=1 << 20), dict(n=1 << 40)):
        assert fwd(**bad) == gsc.GSC_EINVAL, bad
        assert "gated_ffn_fwd" in _err(L)
    assert fwd(ws=None) == gsc.GSC_ESHORT and fwd(wsb=need - 1) == gsc.GSC_ESHORT and str(need) in _err(L)
    assert fwd(ws=ctypes.c_void_p(0x1008)) == gsc.GSC_EINVAL and "aligned" in _err(L)
    assert fwd(n=0, X=None, ws=None, wsb=0) == gsc.GSC_OK
    nb = L.gsc_gated_ffn_bwd_ws_bytes(gsc.GSC_BF16, 100, 64, 267, 64)
    assert nb >= 3 * 100 * 272 * 2 + (64 * 2 * 272 + 267 * 64) * 4
    assert L.gsc_gated_ffn_bwd_ws_bytes(gsc.GSC_F32, 0, 64, 256, 64) > 0
    bwd = lambda dt=1, X=FAKE, n=100, f=267, act=0, dX=FAKE, dW=FAKE, ws=FAKE, wsb=nb: L.gsc_gated_ffn_bwd(
        dt, X, n, 64, FAKE, FAKE, f, FAKE, 64, FAKE, act, dX, dW, dW, dW, ws, wsb, None)
    for bad in (dict(dt=3), dict(X=None), dict(n=-1), dict(f=0), dict(act=5), dict(n=1 << 34, f=1 << 20)):
        assert bwd(**bad) == gsc.GSC_EINVAL, bad
        assert "gated_ffn_bwd" in _err(L)
    assert bwd(ws=None) == gsc.GSC_ESHORT and bwd(wsb=nb - 1) == gsc.GSC_ESHORT and str(nb) in _err(L)
    assert bwd(ws=ctypes.c_void_p(0x1008)) == gsc.GSC_EINVAL
    assert bwd(dX=None, dW=None, ws=None, wsb=0) == gsc.GSC_OK
    assert bwd(n=0, dW=None, ws=None, wsb=0) == gsc.GSC_OK


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="CUDA"):
        gsc.gsc_layer_norm_fwd(x)
    with pytest.raises(ValueError, match="CUDA"):
        gsc.gsc_layer_norm_bwd(x, x, x[:, 0], x[:, 0])
    with pytest.raises(ValueError, match="CUDA"):
        gsc.gsc_rotary(x.view(4, 1, 8), torch.zeros(4, 4, dtype=torch.int32), [1, 1, 1])
    with pytest.raises(ValueError, match="CUDA"):
        gsc.gsc_gated_ffn_fwd(x, torch.zeros(8, 4), torch.zeros(8, 4), torch.zeros(4, 8))
    with pytest.raises(ValueError, match="dtype"):
        gsc.gsc_layer_norm_fwd(x.half())


def test_layer_norm_wide_workspace(L):
    """Rows of over 2,048 columns: the chunks' column sums and three floats of each row."""
    assert L.gsc_layer_norm_bwd_ws_bytes(7, 2048) == 2 * 2 * 2048 * 4
    assert L.gsc_layer_norm_bwd_ws_bytes(7, 2049) == 2 * 2 * 2049 * 4 + 3 * 7 * 4
    assert L.gsc_layer_norm_bwd_ws_bytes(10**7, 4096) == 1024 * 2 * 4096 * 4 + 3 * 10**7 * 4


def test_gated_ffn_launch_sizes(L):
    """A launch takes fewer than 2^32 threads: sizes that would ask for more are refused before anything is launched, the
    ones just below are not (they come as far as the check of the workspace)."""
    def call(dt, n, ci, f, co, bwd):
        a = (dt, FAKE, n, ci, FAKE, FAKE, f, FAKE, co)
        if not bwd:
            return L.gsc_gated_ffn_fwd(*a, 0, FAKE, FAKE, 16, None)
        return L.gsc_gated_ffn_bwd(*a, FAKE, 0, FAKE, FAKE, FAKE, FAKE, FAKE, 16, None)

    top = 1 << 30
    for dt, n, ci, f, co, bwd in ((gsc.GSC_BF16, top, 8, 8, 8, 0),            # rows in registers, 512 threads a tile
                                  (gsc.GSC_F32, 2 * top, 8, 8, 8, 0),         # ... 256
                                  (gsc.GSC_BF16, 2 * top, 8, 8, 8, 1),        # tiles by 64 columns
                                  (gsc.GSC_F32, top, 200, 65, 65, 0), (gsc.GSC_BF16, top // 2, 64, 200, 8, 1)):
        assert call(dt, n, ci, f, co, bwd) == gsc.GSC_EINVAL and "launch" in _err(L), (dt, n, bwd)
        assert call(dt, n - 128, ci, f, co, bwd) == gsc.GSC_ESHORT, (dt, n, bwd)


def test_gated_ffn_workspace_is_what_the_kernels_use(L):
    """Upper bounds (256 bytes of padding a part): no hidden rows where they stay in registers, no copies where nothing is
    copied, one float32 hidden row each for a few rows.  (Without a device the library takes it to have 256 compute units.)"""
    fwd, bwd, B, F = L.gsc_gated_ffn_fwd_ws_bytes, L.gsc_gated_ffn_bwd_ws_bytes, gsc.GSC_BF16, gsc.GSC_F32
    assert fwd(B, 300_000, 256, 1024, 256) <= 3 * 256 * 1024 * 2 + 256         # the packed weights (771 MB with all parts)
    assert fwd(F, 120_011, 64, 256, 64) <= 256
    assert fwd(B, 13_000, 100, 267, 100) <= 3 * 128 * 320 * 2 + 256
    for n in (1, 4):
        assert fwd(B, n, 256, 1024, 256) <= n * 1024 * 4 + 256
        assert fwd(F, n, 256, 1024, 256) <= n * 1024 * 4 + 256
    # tiles: X, the weights and the hidden rows
    assert fwd(B, 1000, 300, 90, 129) <= 1000 * 304 * 2 + 2 * 300 * 96 * 2 + 90 * 136 * 2 + 1024 * 128 * 2 + 5 * 256
    assert fwd(F, 1000, 300, 90, 129) <= 1024 * 128 * 4 + 256
    # backward: X, dY and the projections' copies, hidden rows three times, at most 512 chunks' sums
    part = (256 * 2048 + 1024 * 256) * 4
    hid = 300_032 * 1024 * 2
    assert bwd(B, 300_000, 256, 1024, 256) <= 2 * 300_000 * 512 + 2 * 2**19 + 3 * 2**19 + 3 * hid + 64 * part + 8 * 256
    assert bwd(F, 1000, 64, 256, 64) <= 3 * 1024 * 256 * 4 + 8 * (64 * 512 + 256 * 64) * 4 + 3 * 256


def test_gated_ffn_rows_in_registers_from(L):
    """The forward pass of at most 64 channels writes no hidden rows from 40 tiles of 128 rows on, of at most 128 from 100."""
    size = L.gsc_gated_ffn_fwd_ws_bytes
    for c, tiles in ((8, 40), (64, 40), (65, 100), (128, 100)):
        n = 128 * (tiles - 1)
        pack = 3 * (64 if c <= 64 else 128) * 256 * 2
        assert size(gsc.GSC_BF16, n, c, 256, 8) > n * 256 * 2 and size(gsc.GSC_BF16, n + 1, c, 256, 8) == pack, c
        assert size(gsc.GSC_BF16, n, 8, 256, c) > n * 256 * 2 and size(gsc.GSC_BF16, n + 1, 8, 256, c) == pack, c


def test_stream_of_another_device_is_refused():
    class Stream:
        cuda_stream, device_index = 0x40, 1

    assert gsc._raw_stream(Stream(), 1) == 0x40
    with pytest.raises(ValueError, match="cuda:1"):
        gsc._raw_stream(Stream(), 0)


def test_gated_ffn_float32_rows_in_registers_from(L):
    """The float32 forward pass of at most 32 channels writes no hidden rows up to 128 hidden columns, and from 150 tiles of
    128 rows on; one of 64 channels where the tiles fill three quarters of a round of 256 compute units."""
    size = lambda n, c, f: L.gsc_gated_ffn_fwd_ws_bytes(gsc.GSC_F32, n, c, f, 8)
    assert size(5, 32, 128) == 256 and size(5, 32, 129) > 256 and size(5, 33, 128) > 256
    assert size(128 * 149, 32, 512) > 128 * 149 * 512 * 4 - 1 and size(128 * 149 + 1, 32, 512) == 256
    assert size(128 * 191, 64, 512) > 256 and size(128 * 192, 64, 512) == 256 and size(128 * 257, 64, 512) > 256
