"""CPU-side checks of the sequence layers: the oracle's gradients against differences, the symbols the header declares, and
the refusals that are decided before a device is touched."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import seq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "scan2d_seq.h")


@pytest.fixture(scope="module")
def lib():
    from paper_2412_00678_amd import scan2d
    return scan2d


def _differences(f, base, key, step=1e-6):
    v = base[key]
    out = np.zeros_like(v)
    for at in np.ndindex(*v.shape):
        hi, lo = v.copy(), v.copy()
        hi[at] += step
        lo[at] -= step
        out[at] = (f(**{**base, key: hi}) - f(**{**base, key: lo})) / (2 * step)
    return out


def test_recurrence_oracle_gradients_against_differences():
    rng = np.random.default_rng(0)
    T, C, spans = 30, 3, [(0, 9), (9, 9), (9, 10), (10, 28)]
    base = dict(x=rng.normal(size=(T, C)), r=rng.normal(size=(T, C)), i=rng.normal(size=(T, C)), lam=rng.normal(size=C) - 4,
                h0=rng.normal(size=(4, C)))
    dh, dhT = rng.normal(size=(T, C)), rng.normal(size=(4, C))

    def loss(**v):
        o = seq.recur(spans=spans, **v)
        return (o["h"][0] * dh).sum() + (o["hT"][0] * dhT).sum()

    got = seq.recur(spans=spans, dh=dh, dhT=dhT, **base)
    for key in base:
        assert np.abs(_differences(loss, base, key) - got["d" + key][0]).max() < 1e-7, key


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("masked", [False, True])
def test_group_norm_oracle_gradients_against_differences(act, masked):
    rng = np.random.default_rng(1)
    N, P, C, G = 3, 4, 6, 2
    mask = None
    if masked:
        mask = rng.integers(0, 2, (N, P))
        mask[1] = 1
    base = dict(x=rng.normal(size=(N, P, C)), gamma=rng.normal(size=C), beta=rng.normal(size=C))
    dy = rng.normal(size=(N, P, C))
    loss = lambda **v: (seq.group_norm(groups=G, eps=1e-5, act=act, mask=mask, **v)["y"][0] * dy).sum()
    got = seq.group_norm(groups=G, eps=1e-5, act=act, mask=mask, dy=dy, **base)
    for key in base:
        assert np.abs(_differences(loss, base, key) - got["d" + key][0]).max() < 1e-7, key


def test_library_exports_every_declared_symbol(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(scan2d_[a-z_0-9]+)\s*\(", text)))
    assert declared == sorted(lib.SEQ_EXPORTS)
    raw = ctypes.CDLL(lib.LIB_PATH)
    for name in declared:
        assert hasattr(raw, name), name


OK, ODD = 4096, 4098                    # fake addresses: never dereferenced


def _recur(lib, T=8, C=4, S=1, dtype=0, scale=8.0, **strides):
    d = lib.RecurDesc(T, C, S, dtype, scale)
    for k, v in strides.items():
        setattr(d, "stride_" + k, v)
    return d


def test_recurrence_forward_refusals(lib):
    def call(d, x=OK, r=2 * OK, i=3 * OK, lam=OK, off=None, lens=None, h0=None, h=4 * OK, hT=None, saved=None, sb=0, ws=5 * OK, wb=1 << 40):
        return lib.lib.scan2d_seq_recur_fwd(None if d is None else ctypes.byref(d), x, r, i, lam, off, lens, h0, h, hT, saved, sb, ws, wb, None)

    assert call(None) == -1
    for bad in (dict(T=-1), dict(T=1 << 31), dict(C=0), dict(S=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(x=3), dict(h=-8), dict(r=1 << 62), dict(T=9, S=2)):
        assert call(_recur(lib, **bad)) == -2, bad
    assert call(_recur(lib, dtype=2)) == -3
    d = _recur(lib)
    assert call(d, off=OK, lens=OK) == -4
    for bad in ("x", "r", "i", "lam", "h"):
        assert call(d, **{bad: None}) == -1, bad
        assert call(d, **{bad: ODD}) == -6, bad
    for bad in ("off", "lens", "h0", "hT"):
        assert call(d, **{bad: ODD}) == -6, bad
    assert call(d, saved=ODD, sb=1 << 40) == -6 and call(d, saved=6 * OK, sb=0) == -5
    assert call(d, h=OK) == -2 and call(d, h=2 * OK) == -2 and call(d, h=3 * OK) == -2          # in place
    assert call(d, h0=7 * OK, hT=7 * OK) == -2
    b = _recur(lib, dtype=1)
    assert call(b, x=ODD, saved=6 * OK, sb=0) == -5 and call(b, x=OK + 1) == -6      # rows: aligned to their element type
    long = _recur(lib, T=100000, C=64)
    assert lib.lib.scan2d_seq_recur_saved_bytes(ctypes.byref(long)) > 0
    need = lib.lib.scan2d_seq_recur_workspace_bytes(ctypes.byref(long), lib.PASS_FWD)
    if need:
        assert call(long, wb=need - 1) == -5 and call(long, ws=None) == -5
    assert lib.lib.scan2d_seq_recur_saved_bytes(ctypes.byref(_recur(lib, C=0))) == 0
    assert lib.lib.scan2d_seq_recur_workspace_bytes(ctypes.byref(long), 9) == 0


def test_recurrence_backward_refusals(lib):
    names = ["x", "r", "i", "lam", "off", "lens", "h0", "dh", "dhT", "saved"]

    def call(d, sb=1 << 40, ws=64 * OK, wb=1 << 40, **given):
        v = {n: (k + 1) * OK for k, n in enumerate(names + ["dx", "dr", "di", "dlam", "dh0"])}
        v["off"] = v["lens"] = None
        v.update(given)
        return lib.lib.scan2d_seq_recur_bwd(ctypes.byref(d), *(v[n] for n in names), sb, v["dx"], v["dr"], v["di"], v["dlam"], v["dh0"], ws, wb, None)

    d = _recur(lib)
    for bad in ("x", "r", "i", "lam", "dh", "saved", "dx", "dr", "di", "dlam"):
        assert call(d, **{bad: None}) == -1, bad
        assert call(d, **{bad: ODD}) == -6, bad
    for bad in ("h0", "dhT", "dh0"):
        assert call(d, **{bad: ODD}) == -6, bad
    assert call(d, off=OK, lens=OK) == -4
    assert call(d, dx=OK) == -2 and call(d, dr=8 * OK) == -2 and call(d, dr=13 * OK) == -2 and call(d, dh0=9 * OK) == -2
    assert call(d, sb=0) == -5
    need = lib.lib.scan2d_seq_recur_workspace_bytes(ctypes.byref(d), lib.PASS_BWD)
    if need:
        assert call(d, wb=need - 1) == -5 and call(d, ws=None) == -5
    assert call(_recur(lib, dx=3)) == -2


def test_recurrence_step_refusals(lib):
    def call(d, x=OK, r=2 * OK, i=3 * OK, lam=OK, state=5 * OK, slots=None, n=8, h=4 * OK):
        return lib.lib.scan2d_seq_recur_step(ctypes.byref(d), x, r, i, lam, state, slots, n, h, None)

    assert call(_recur(lib, T=0)) == -2 and call(_recur(lib, T=65536), n=65536) == -2
    assert call(_recur(lib), n=7) == -2 and call(_recur(lib), n=0, slots=OK) == -2 and call(_recur(lib), n=1 << 31) == -2
    assert call(_recur(lib, S=0), x=None) == -1                       # the sequences of the descriptor are not used
    for bad in ("x", "r", "i", "lam", "state", "h"):
        assert call(_recur(lib), **{bad: None}) == -1
        assert call(_recur(lib), **{bad: ODD}) == -6
    assert call(_recur(lib), slots=ODD) == -6
    assert call(_recur(lib), h=OK) == -2


def test_group_norm_refusals(lib):
    def desc(N=2, C=8, G=4, P=5, dtype=0, act=0, eps=1e-5, **strides):
        d = lib.GroupNormDesc(N, C, G, P, dtype, act, eps)
        for k, v in strides.items():
            setattr(d, "stride_" + k, v)
        return d

    def fwd(d, x=OK, g=OK, b=OK, m=None, y=2 * OK, st=3 * OK, ws=4 * OK, wb=1 << 40):
        return lib.lib.scan2d_group_norm_fwd(None if d is None else ctypes.byref(d), x, g, b, m, y, st, ws, wb, None)

    def bwd(d, x=OK, g=OK, b=OK, m=None, st=3 * OK, dy=5 * OK, dx=6 * OK, dg=7 * OK, db=8 * OK, ws=4 * OK, wb=1 << 40):
        return lib.lib.scan2d_group_norm_bwd(None if d is None else ctypes.byref(d), x, g, b, m, st, dy, dx, dg, db, ws, wb, None)

    assert fwd(None) == -1 and bwd(None) == -1
    for bad in (dict(N=0), dict(C=0), dict(G=0), dict(G=3), dict(P=0), dict(P=1 << 31), dict(N=1 << 16, P=1 << 15), dict(eps=-1.0), dict(eps=float("nan")),
                dict(x=7), dict(dy=-1)):
        assert fwd(desc(**bad)) == -2, bad
        assert bwd(desc(**bad)) == -2, bad
    assert fwd(desc(dtype=5)) == -3 and fwd(desc(act=3)) == -4 and bwd(desc(act=-1)) == -4
    d = desc()
    for bad in ("x", "y", "st"):
        assert fwd(d, **{bad: None}) == -1 and fwd(d, **{bad: ODD}) == -6
    for bad in ("x", "st", "dy", "dx"):
        assert bwd(d, **{bad: None}) == -1 and bwd(d, **{bad: ODD}) == -6
    assert fwd(d, g=ODD) == -6 and bwd(d, db=ODD) == -6
    assert fwd(desc(y=16), y=OK) == -2 and bwd(d, dx=OK) == -2 and bwd(desc(dx=16), dx=5 * OK) == -2
    big = desc(N=1, P=1 << 20, C=512, G=32)
    for p, call in ((lib.PASS_FWD, fwd), (lib.PASS_BWD, bwd)):
        need = lib.lib.scan2d_group_norm_workspace_bytes(ctypes.byref(big), p)
        if need:
            assert call(big, wb=need - 1) == -5 and call(big, ws=None) == -5
    assert lib.lib.scan2d_group_norm_workspace_bytes(ctypes.byref(desc(G=3)), lib.PASS_FWD) == 0


def test_binding_refuses_host_tensors(lib):
    x, lam = torch.zeros(4, 8), torch.zeros(8)
    with pytest.raises(ValueError, match="device"):
        lib.seq_recur_fwd(x, x, x, lam)
    with pytest.raises(ValueError, match="device"):
        lib.group_norm_fwd(torch.zeros(2, 4, 8), None, None, 2)
    with pytest.raises(TypeError):
        lib.seq_recur_step(None, x, x, lam, torch.zeros(4, 8))


def broadcasts(C=8):
    """Views that have one row for all of a dimension, at each place where such a dimension can stand."""
    return {"all rows": torch.zeros(1, C).expand(6, C), "inner": torch.zeros(4, 1, C).expand(4, 50, C), "outer": torch.zeros(1, 50, C).expand(4, 50, C),
            "both": torch.zeros(1, 1, C).expand(4, 50, C), "middle of three": torch.zeros(2, 1, 5, C).expand(2, 3, 5, C),
            "innermost of three": torch.zeros(2, 3, 1, C).expand(2, 3, 5, C), "two of three": torch.zeros(2, 1, 1, C).expand(2, 3, 5, C),
            "beside a one": torch.zeros(4, 1, 1, C).expand(4, 50, 1, C)}


@pytest.mark.parametrize("which", sorted(broadcasts()))
def test_binding_refuses_rows_that_are_broadcast(lib, which):
    """A broadcast dimension has fewer rows in memory than its size says.  Layouts are looked at before devices, so that this
    shows without one."""
    x, lam = broadcasts()[which], torch.zeros(8)
    if x.dim() <= 3:
        with pytest.raises(ValueError, match="rows at one stride"):
            lib.seq_recur_fwd(x, x, x, lam)
        with pytest.raises(ValueError, match="rows at one stride"):
            lib.seq_recur_bwd(x, x, x, lam, x, None)
    if x.dim() >= 3:
        with pytest.raises(ValueError, match="rows at one stride"):
            lib.group_norm_fwd(x, None, None, 2)
        with pytest.raises(ValueError, match="rows at one stride"):
            lib.group_norm_bwd(x, None, None, 2, None, x)


def test_binding_takes_the_layouts_of_rows(lib):
    """Views whose rows lie at one stride get as far as the device."""
    wide = torch.zeros(4, 50, 24)
    for x in (wide[..., 8:16], wide[:1, :, :8], wide[:, :1, :8], wide[:1, :1, 16:], torch.zeros(0, 5, 8), torch.zeros(4, 50, 8)[:, ::2].contiguous(),
              torch.zeros(50, 24)[::2, :8], torch.zeros(1, 1, 8).expand(1, 1, 8), torch.zeros(2, 6, 7, 8).permute(0, 1, 2, 3)):
        if x.dim() <= 3:
            with pytest.raises(ValueError, match="device tensor"):
                lib.seq_recur_fwd(x, x, x, torch.zeros(8))
        if x.dim() >= 3:
            with pytest.raises(ValueError, match="device tensor"):
                lib.group_norm_fwd(x, None, None, 2)


@pytest.mark.parametrize("T,C,fits", [(65535, 130560, True), (65535, 131072, True), (65535, 131073, False), (512, (1 << 24) - 1, False), (511, (1 << 24) - 1, True),
                                      (1, (1 << 24) - 1, True), (65535, 1, True)])
def test_step_is_refused_where_its_launch_would_hold_too_many_threads(lib, T, C, fits):
    """T ceil(C / 512) below 2^24, looked at before the pointers."""
    code = lib.lib.scan2d_seq_recur_step(ctypes.byref(_recur(lib, T=T, C=C)), None, None, None, OK, OK, OK, 8, OK, None)
    assert code == (-1 if fits else -2)
