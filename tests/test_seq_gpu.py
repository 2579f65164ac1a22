"""GPU parity of the sequence layers (scan2d_seq_recur_*, scan2d_group_norm_*) with oracle/seq.py, through the binding.

Tolerances: the oracle's own element-wise bound for fp32 arithmetic, plus the one rounding to the storage type (at most
half a step: 2^-8 of the value for bf16, 2^-24 for fp32)."""
import numpy as np
import pytest

from oracle import seq

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


@pytest.fixture(scope="module")
def s2d(torch):
    from paper_2412_00678_amd import scan2d          # raises if the library is not built
    return scan2d


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def close(name, got, ref, dtype):
    """|got - value| <= bound + half a step of the storage type."""
    value, bound = ref
    got = host(got).reshape(value.shape)
    assert np.isfinite(got).all() == np.isfinite(value).all(), name
    tol = bound + HALF_STEP[dtype] * (np.abs(value) + bound)
    off = np.abs(got - value)
    worst = np.unravel_index(np.argmax(off - tol), off.shape) if off.size else ()
    assert (off <= tol).all(), f"{name} at {worst}: {got[worst]!r} for {value[worst]!r}, off {off[worst]:.3e} > {tol[worst]:.3e}"


def rows(torch, rng, shape, dtype, scale=1.0, pad=None):
    """Rows in the storage type; pad = (channels before, channels behind): a view into wider rows."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    lo, hi = pad or (0, 0)
    wide = torch.from_numpy((rng.normal(size=(*shape[:-1], lo + shape[-1] + hi)) * scale).astype(np.float32)).to(dt).cuda()
    return wide[..., lo:lo + shape[-1]]


def decays(rng, C):
    """lam with softplus(lam) between 1e-4 and 1: decays from slow to fast."""
    sp = np.exp(rng.uniform(np.log(1e-4), 0, C))
    return np.log(np.expm1(sp)).astype(np.float32)


def spans_of(layout, lens, L=0):
    if layout == "packed":
        ends = np.cumsum(lens)
        return [(int(e - n), int(e)) for e, n in zip(ends, lens)]
    return [(s * L, s * L + n) for s, n in enumerate(lens)]


def recur_case(torch, s2d, layout, lens, L, C, dtype, seed, states=True, pad=None, behind=0, scale=8.0, gate=2.0):
    """Forward, backward and both again: compared with the oracle, rows of no sequence untouched, the same bits twice."""
    rng = np.random.default_rng(seed)
    S = len(lens)
    T = (sum(lens) if layout == "packed" else S * L) + behind
    spans = spans_of(layout, lens, L)
    shape = (T, C) if layout == "packed" else (S, L, C)
    x, r, i, dh = (rows(torch, rng, shape, dtype, s, pad) for s in (1.0, gate, gate, 1.0))
    lam = torch.from_numpy(decays(rng, C)).cuda()
    h0, dhT = (torch.from_numpy(rng.normal(size=(S, C)).astype(np.float32)).cuda() if states else None for _ in range(2))
    kw = dict(h0=h0, scale=scale)
    if layout == "packed":
        kw["offsets"] = torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device="cuda")
    elif layout == "padded":
        kw["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    flat = lambda t: host(t).reshape(T, C)
    ref = seq.recur(flat(x), flat(r), flat(i), host(lam), spans, None if h0 is None else host(h0), scale, flat(dh), None if dhT is None else host(dhT))
    print(f"recurrence {layout} S={S} T={T} C={C} {dtype} pad={pad} behind={behind}", flush=True)

    def once():
        out = [torch.full((*shape[:-1], C + sum(pad or (0, 0))), 7.0, dtype=x.dtype, device="cuda") for _ in range(4)]
        cut = [o[..., (pad or (0, 0))[0]:][..., :C] for o in out]
        h, hT, saved = s2d.seq_recur_fwd(x, r, i, lam, want_final=True, want_saved=True, h=cut[0], **kw)
        dx, dr, di, dlam, dh0 = s2d.seq_recur_bwd(x, r, i, lam, dh, saved, dhT=dhT, want_dh0=True, out=cut[1:], **kw)
        torch.cuda.synchronize()
        return dict(h=h, hT=hT, dx=dx, dr=dr, di=di, dlam=dlam, dh0=dh0), out

    got, wide = once()
    inside = np.zeros(T, bool)
    for lo, hi in spans:
        inside[lo:hi] = True
    for name in ("h", "dx", "dr", "di"):
        value, bound = ref[name]
        t = got[name].reshape(T, C)
        close(name, t[torch.from_numpy(inside).cuda()], (value[inside], bound[inside]), dtype)
        assert (host(t)[~inside] == 7.0).all(), name                          # rows of no sequence
    for o in wide:                                                            # and nothing beside the channels
        if pad is not None:
            flat_o = host(o).reshape(T, -1)
            assert (flat_o[:, :pad[0]] == 7.0).all() and (flat_o[:, pad[0] + C:] == 7.0).all()
    for name in ("hT", "dlam", "dh0"):
        close(name, got[name], ref[name], "fp32")
    again, _ = once()
    for name in got:
        assert torch.equal(got[name], again[name]), name
    return got


RECUR_CASES = [
    # layout, lengths, rows per sequence, channels, dtype, options
    ("packed", [1], 0, 1, "fp32", {}),
    ("packed", [1], 0, 64, "bf16", {"states": False}),
    ("packed", [2, 1], 0, 2, "bf16", {}),
    ("packed", [0], 0, 5, "fp32", {}),
    ("packed", [0, 5, 0, 0, 1, 131, 0], 0, 3, "fp32", {}),
    ("packed", [0, 0, 37, 0], 0, 65, "bf16", {"behind": 90}),
    ("packed", [64], 0, 64, "fp32", {}),
    ("packed", [65, 63, 1, 127, 128, 129], 0, 127, "bf16", {}),
    ("packed", [257], 0, 128, "bf16", {}),
    ("packed", [300, 0, 17], 0, 129, "fp32", {"behind": 3}),
    ("packed", [700], 0, 130, "bf16", {"pad": (1, 2)}),
    ("packed", [100, 411], 0, 33, "fp32", {"pad": (3, 0)}),
    ("packed", [1] * 300, 0, 40, "bf16", {}),
    ("packed", [3, 1, 2, 0, 4] * 60, 0, 31, "fp32", {}),
    ("packed", [2500], 0, 31, "bf16", {}),
    ("packed", [1700, 900], 0, 257, "fp32", {"states": False}),
    ("packed", [4000], 0, 8, "fp32", {"scale": 0.5}),
    ("padded", [0, 7, 50, 1], 50, 66, "bf16", {}),
    ("padded", [200, 0, 0, 129], 200, 24, "fp32", {"pad": (0, 24)}),
    ("padded", [0, 0], 3, 4, "bf16", {}),
    ("equal", [100] * 3, 100, 70, "bf16", {}),
    ("equal", [1] * 5, 1, 256, "fp32", {}),
    ("equal", [1000] * 2, 1000, 96, "fp32", {"gate": 8.0}),
    # several groups of chunks, 16 rows of a wavefront, one and two channels of a lane
    ("packed", [4150, 60], 0, 1030, "bf16", {}),
    ("packed", [9000], 0, 70, "bf16", {"states": False}),
    ("packed", [20011, 13000], 0, 40, "fp32", {}),
    # more sequences than a wavefront has lanes, some of them long, and empty ones in a row
    ("packed", [7, 0, 30, 1, 0, 0, 95, 2] * 25, 0, 90, "bf16", {"behind": 11}),
    ("packed", [0] * 150 + [40] + [0] * 90 + [3], 0, 20, "fp32", {}),
    ("padded", [0, 12, 3, 12, 7] * 30, 12, 68, "fp32", {}),
]


@pytest.mark.parametrize("case", RECUR_CASES, ids=lambda c: f"{c[0]}-{len(c[1])}x{sum(c[1])}-C{c[3]}-{c[4]}" + "".join(f"-{k}" for k in c[5]))
def test_recurrence_matches_the_oracle(torch, s2d, case):
    layout, lens, L, C, dtype, options = case
    recur_case(torch, s2d, layout, lens, L, C, dtype, seed=sum(lens) + C, **options)


def test_recurrence_random_shapes_match_the_oracle(torch, s2d):
    rng = np.random.default_rng(99)
    for k in range(12):
        layout = ("packed", "padded", "equal")[k % 3]
        S, L = int(rng.integers(1, 9)), int(np.exp(rng.uniform(0, np.log(500))))
        lens = [L] * S if layout == "equal" else [int(n) for n in rng.integers(0, L + 1, S)]
        recur_case(torch, s2d, layout, lens, L, int(np.exp(rng.uniform(0, np.log(400)))), ("fp32", "bf16")[int(rng.integers(2))], seed=k,
                   behind=int(rng.integers(0, 40)) if layout == "packed" else 0)


def test_recurrence_of_no_rows(torch, s2d):
    x = torch.empty((0, 6), device="cuda")
    lam = torch.zeros(6, device="cuda")
    h0, dhT = torch.randn(2, 6, device="cuda"), torch.randn(2, 6, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    h, hT, saved = s2d.seq_recur_fwd(x, x, x, lam, offsets=off, h0=h0, want_final=True, want_saved=True)
    dx, dr, di, dlam, dh0 = s2d.seq_recur_bwd(x, x, x, lam, x, saved, offsets=off, h0=h0, dhT=dhT)
    torch.cuda.synchronize()
    assert h.shape == (0, 6) and torch.equal(hT, h0) and torch.equal(dh0, dhT) and bool((dlam == 0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_recurrence_at_the_ends_of_the_gates(torch, s2d, dtype):
    """Gates that are shut or open to the last bit, decays of exactly 1 and 0, and the gradients through them."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    vals = [-1e30, -200.0, -88.0, -30.0, 0.0, 30.0, 88.0, 200.0, 1e30]
    r = torch.tensor(vals * 8, device="cuda").to(dt)[:, None].expand(72, 7).contiguous()
    i = torch.tensor([v for v in vals for _ in range(8)], device="cuda").to(dt)[:, None].expand(72, 7).contiguous()
    rng = np.random.default_rng(3)
    x, dh = rows(torch, rng, (72, 7), dtype), rows(torch, rng, (72, 7), dtype)
    lam = torch.tensor([-100.0, -40.0, -16.0, -5.0, 0.0, 19.0, 60.0], device="cuda")
    h0 = torch.ones(1, 7, device="cuda")
    h, hT, saved = s2d.seq_recur_fwd(x, r, i, lam, h0=h0, want_final=True, want_saved=True)
    dx, dr, di, dlam, dh0 = s2d.seq_recur_bwd(x, r, i, lam, dh, saved, h0=h0)
    torch.cuda.synchronize()
    ref = seq.recur(host(x), host(r), host(i), host(lam), [(0, 72)], host(h0), 8.0, host(dh))
    for name, t in dict(h=h, dx=dx, dr=dr, di=di).items():
        close(name, t, ref[name], dtype)
    for name, t in dict(hT=hT, dlam=dlam, dh0=dh0).items():
        close(name, t, ref[name], "fp32")


def test_recurrence_nan_stays_in_its_sequence_and_channel(torch, s2d):
    rng = np.random.default_rng(5)
    x, r, i = (rows(torch, rng, (600, 70), "fp32") for _ in range(3))
    off = torch.tensor([0, 200, 420, 600], dtype=torch.int32, device="cuda")
    lam = torch.from_numpy(decays(rng, 70)).cuda()
    clean, cT, _ = s2d.seq_recur_fwd(x, r, i, lam, offsets=off, want_final=True)
    x[250, 9], i[300, 30] = float("nan"), float("inf")                        # an open gate is no NaN
    h, hT, saved = s2d.seq_recur_fwd(x, r, i, lam, offsets=off, want_final=True, want_saved=True)
    torch.cuda.synchronize()
    bad = torch.isnan(h)
    want = torch.zeros_like(bad)
    want[250:420, 9] = True
    assert torch.equal(bad, want) and torch.equal(torch.isnan(hT), want[[199, 419, 599]])
    keep = ~want
    keep[300:420, 30] = False
    assert torch.equal(h[keep], clean[keep])


def test_recurrence_in_pieces_is_the_whole(torch, s2d):
    """A prompt in pieces, each from the state that the one before left, then token by token."""
    rng = np.random.default_rng(11)
    T, C = 700, 96
    x, r, i = (rows(torch, rng, (T, C), "bf16") for _ in range(3))
    lam = torch.from_numpy(decays(rng, C)).cuda()
    ref = seq.recur(host(x), host(r), host(i), host(lam), [(0, T)])
    state = torch.zeros(1, C, device="cuda")
    parts = []
    for lo, hi in ((0, 1), (1, 300), (300, 430), (430, 690)):
        h, state, _ = s2d.seq_recur_fwd(x[lo:hi], r[lo:hi], i[lo:hi], lam, h0=state, want_final=True)
        parts.append(h)
    for t in range(690, T):
        parts.append(s2d.seq_recur_step(x[t:t + 1], r[t:t + 1], i[t:t + 1], lam, state))
    torch.cuda.synchronize()
    close("h", torch.cat(parts), ref["h"], "bf16")
    close("hT", state, ref["hT"], "fp32")


@pytest.mark.parametrize("T,C,dtype,pad", [(1, 1, "fp32", None), (3, 2, "bf16", None), (4, 257, "bf16", (1, 0)), (65, 130, "fp32", (0, 130)),
                                           (300, 64, "bf16", None), (2, 1000, "bf16", None), (1025, 7, "fp32", None)])
def test_step_matches_the_oracle(torch, s2d, T, C, dtype, pad):
    rng = np.random.default_rng(T + C)
    x, r, i = (rows(torch, rng, (T, C), dtype, s, pad) for s in (1.0, 2.0, 2.0))
    lam = torch.from_numpy(decays(rng, C)).cuda()
    pool = torch.from_numpy(rng.normal(size=(2 * T + 1, C)).astype(np.float32)).cuda()
    slots = rng.permutation(2 * T + 1)[:T].astype(np.int32)
    if T > 3:
        slots[1], slots[T // 2], slots[T - 1] = -1, 2 * T + 1, -2 ** 31              # padding
    live = [(t, int(s)) for t, s in enumerate(slots) if 0 <= s <= 2 * T]
    for dev in (torch.from_numpy(slots).cuda(), None):
        state = pool.clone()
        order = live if dev is not None else [(t, t) for t in range(T)]
        h = torch.full((T, C), 7.0, dtype=x.dtype, device="cuda")
        s2d.seq_recur_step(x, r, i, lam, state, slots=dev, h=h)
        torch.cuda.synchronize()
        at, to = [t for t, _ in order], [s for _, s in order]
        ref = seq.recur(host(x)[at], host(r)[at], host(i)[at], host(lam), [(k, k + 1) for k in range(len(at))], host(pool)[to])
        close("h", h[at], ref["h"], dtype)
        close("state", state[to], ref["hT"], "fp32")
        rest = [s for s in range(2 * T + 1) if s not in set(to)]
        assert torch.equal(state[rest], pool[rest])
        skipped = [t for t in range(T) if t not in set(at)]
        assert bool((h[skipped] == 7.0).all())


def test_step_takes_a_repeated_slot_in_the_order_of_its_rows(torch, s2d):
    rng = np.random.default_rng(21)
    T, C = 400, 129
    x, r, i = (rows(torch, rng, (T, C), "fp32") for _ in range(3))
    lam = torch.from_numpy(decays(rng, C)).cuda()
    slots = torch.from_numpy(rng.integers(-1, 6, T).astype(np.int32)).cuda()
    pool = torch.from_numpy(rng.normal(size=(6, C)).astype(np.float32)).cuda()
    state, h = pool.clone(), torch.full((T, C), 7.0, device="cuda")
    s2d.seq_recur_step(x, r, i, lam, state, slots=slots, h=h)
    one, each = pool.clone(), torch.full((T, C), 7.0, device="cuda")
    for t in range(T):
        s2d.seq_recur_step(x[t:t + 1], r[t:t + 1], i[t:t + 1], lam, one, slots=slots[t:t + 1], h=each[t:t + 1])
    torch.cuda.synchronize()
    assert torch.equal(state, one) and torch.equal(h, each)


def test_recurrence_bad_offsets_stay_inside(torch, s2d):
    """Offsets and lengths outside the documented rules: any result, but nothing beside the tensors is touched."""
    rng = np.random.default_rng(31)
    T, C = 300, 66
    buf = torch.full((3 * T, C), 7.0, device="cuda")
    x, r, i, dh = (rows(torch, rng, (T, C), "fp32") for _ in range(4))
    lam = torch.from_numpy(decays(rng, C)).cuda()
    for off in ([0, 1000, 300], [-5, 100, 300], [0, 200, 100], [2 ** 31 - 1, -2 ** 31, 7], [300, 0, 0]):
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        h0 = torch.zeros(2, C, device="cuda")
        _, _, saved = s2d.seq_recur_fwd(x, r, i, lam, offsets=o, h0=h0, want_final=True, want_saved=True, h=buf[T:2 * T])
        s2d.seq_recur_bwd(x, r, i, lam, dh, saved, offsets=o, h0=h0, out=(buf[T:2 * T], None, None))
        torch.cuda.synchronize()
        assert bool((buf[:T] == 7.0).all()) and bool((buf[2 * T:] == 7.0).all())
    x3, lens = x.reshape(3, 100, C), torch.tensor([-4, 1000, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    h, hT, saved = s2d.seq_recur_fwd(x3, r.reshape(3, 100, C), i.reshape(3, 100, C), lam, lengths=lens, want_final=True, want_saved=True,
                                     h=buf[T:2 * T].reshape(3, 100, C))
    torch.cuda.synchronize()
    assert bool((buf[:T] == 7.0).all()) and bool((buf[2 * T:] == 7.0).all()) and bool(torch.isfinite(hT).all())


def test_recurrence_past_32_bit_offsets(torch, s2d):
    """Rows whose offsets pass 2^31 elements: the last rows against the same rows by themselves."""
    T, C = 2 ** 21 + 77, 1024
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((T, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    lam = torch.zeros(C, device="cuda")                                        # scale 8: a state is forgotten within some tokens
    h, hT, saved = s2d.seq_recur_fwd(x, x, x, lam, want_final=True, want_saved=True)
    n = 2000
    h2, hT2, saved2 = s2d.seq_recur_fwd(x[-n:], x[-n:], x[-n:], lam, want_final=True, want_saved=True)
    torch.cuda.synchronize()
    assert torch.equal(h[-n + 1000:], h2[1000:])
    assert float((hT - hT2).abs().max()) <= 1e-5
    dx, dr, di, dlam, _ = s2d.seq_recur_bwd(x, x, x, lam, x, saved)
    dx2, dr2, di2, _, _ = s2d.seq_recur_bwd(x[-n:], x[-n:], x[-n:], lam, x[-n:], saved2)
    torch.cuda.synchronize()
    for a, b in ((dx, dx2), (dr, dr2), (di, di2)):
        assert float((a[-n + 1000:].float() - b[1000:].float()).abs().max()) <= 2.0 ** -7 * float(b.float().abs().max())
    assert bool(torch.isfinite(dlam).all())


NORM_CASES = [
    # N, P, C, G, dtype, act, mask, affine, options
    (1, 1, 1, 1, "fp32", "none", False, True, {}),
    (2, 1, 8, 2, "bf16", "silu", False, True, {}),
    (5, 1, 64, 4, "fp32", "gelu", False, True, {}),
    (37, 1, 257, 1, "bf16", "silu", False, True, {}),
    (300, 1, 96, 96, "fp32", "none", False, True, {}),
    (7, 1, 2048, 16, "bf16", "silu", False, False, {}),
    (3, 1, 6000, 3, "fp32", "silu", False, True, {}),
    (64, 1, 640, 5, "bf16", "gelu", True, True, {}),
    (2, 3, 10, 5, "fp32", "gelu", False, True, {}),
    (3, 49, 32, 32, "bf16", "silu", True, True, {}),
    (2, 196, 96, 32, "fp32", "silu", False, True, {}),
    (8, 196, 64, 8, "bf16", "none", False, True, {"pad": (1, 3)}),
    (1, 1000, 36, 4, "bf16", "gelu", True, True, {}),
    (2, 777, 33, 11, "fp32", "silu", True, False, {"pad": (0, 5)}),
    (1, 5000, 130, 2, "bf16", "silu", True, True, {}),
    (4, 300, 513, 27, "fp32", "none", True, True, {}),
    (2, 4100, 24, 1, "bf16", "silu", False, True, {}),
    (70, 20, 48, 6, "fp32", "gelu", True, True, {}),
    (1, 9000, 7, 7, "fp32", "silu", True, True, {}),
    (1, 20000, 64, 32, "fp32", "silu", True, True, {}),
    # single rows: groups of many channels, odd ones, more rows than there are teams, channels below a load's width
    (9, 1, 1306, 2, "bf16", "gelu", False, True, {}),
    (33, 1, 1330, 1, "fp32", "silu", True, True, {"pad": (1, 0)}),
    (40, 1, 2048, 1, "bf16", "silu", True, True, {}),
    (21, 1, 2048, 1, "fp32", "none", False, True, {}),
    (12, 1, 1536, 3, "fp32", "gelu", False, False, {}),
    (5, 1, 2050, 1, "fp32", "silu", False, True, {}),
    (3, 1, 4200, 2, "bf16", "silu", True, True, {}),
    (5000, 1, 512, 8, "bf16", "silu", True, True, {}),
    (9001, 1, 33, 3, "fp32", "none", False, True, {}),
    (6, 1, 3, 1, "fp32", "silu", False, True, {}),
    (6, 1, 5, 1, "bf16", "none", False, True, {}),
    # a few positions, narrow and wide groups, slabs of a part of the row and of a part of a group
    (2, 9, 2, 1, "bf16", "silu", True, True, {}),
    (130, 2, 40, 4, "fp32", "silu", False, True, {}),
    (2, 700, 1602, 2, "bf16", "silu", True, True, {}),
    (1, 3000, 596, 1, "fp32", "gelu", True, True, {}),
    (3, 3, 4200, 2, "fp32", "none", False, True, {}),
    (1, 1500, 2600, 1, "bf16", "silu", True, True, {}),
]


def norm_case(torch, s2d, N, P, C, G, dtype, act, masked, affine, seed, pad=None, eps=1e-5):
    rng = np.random.default_rng(seed)
    x, dy = rows(torch, rng, (N, P, C), dtype, 1.5, pad), rows(torch, rng, (N, P, C), dtype, 1.0, pad)
    gamma, beta = (torch.from_numpy(v.astype(np.float32)).cuda() if affine else None
                   for v in (rng.normal(size=C) * 0.3 + 1, rng.normal(size=C) * 0.3))
    mask = None
    if masked:
        mask = (rng.random((N, P)) < 0.4).astype(np.uint8) * 3
        mask[N // 2] = 1                                                       # an item of no positions
        if N > 1:
            mask[0, :] = 1
            mask[0, P // 2] = 0                                                # and one of a single one
        x[torch.from_numpy(mask).cuda() != 0] = float("nan")
        dy[torch.from_numpy(mask).cuda() != 0] = float("inf")
        mask = torch.from_numpy(mask).cuda()
    code = {"none": s2d.ACT_NONE, "silu": s2d.ACT_SILU, "gelu": s2d.ACT_GELU}[act]
    param = lambda t: None if t is None else host(t)
    print(f"group norm N={N} P={P} C={C} G={G} {dtype} {act} masked={masked} affine={affine} pad={pad}", flush=True)
    ref = seq.group_norm(host(x), param(gamma), param(beta), G, eps, act, None if mask is None else mask.cpu().numpy(), host(dy))

    def once():
        out = [torch.full((N, P, C + sum(pad or (0, 0))), 7.0, dtype=x.dtype, device="cuda") for _ in range(2)]
        cut = [o[..., (pad or (0, 0))[0]:][..., :C] for o in out]
        y, stats = s2d.group_norm_fwd(x, gamma, beta, G, eps=eps, act=code, mask=mask, y=cut[0])
        dx, dgamma, dbeta = s2d.group_norm_bwd(x, gamma, beta, G, stats, dy, act=code, mask=mask, dx=cut[1])
        torch.cuda.synchronize()
        return dict(y=y, stats=stats, dx=dx, dgamma=dgamma, dbeta=dbeta), out

    got, wide = once()
    for name in ("y", "dx"):
        close(name, got[name], ref[name], dtype)
    close("stats", got["stats"], ref["stats"], "fp32")
    for name in ("dgamma", "dbeta"):
        if affine:
            close(name, got[name], ref[name], "fp32")
        else:
            assert got[name] is None
    if pad is not None:
        for o in wide:
            assert bool((o[..., :pad[0]] == 7.0).all()) and bool((o[..., pad[0] + C:] == 7.0).all())
    if masked:
        out = mask != 0
        assert bool((got["y"][out] == 0).all()) and bool((got["dx"][out] == 0).all())
    again, _ = once()
    for name in got:
        assert got[name] is None or torch.equal(got[name], again[name]), name
    return got


@pytest.mark.parametrize("case", NORM_CASES, ids=lambda c: "x".join(map(str, c[:4])) + f"-{c[4]}-{c[5]}" + ("-mask" if c[6] else "") + ("" if c[7] else "-plain"))
def test_group_norm_matches_the_oracle(torch, s2d, case):
    N, P, C, G, dtype, act, masked, affine, options = case
    norm_case(torch, s2d, N, P, C, G, dtype, act, masked, affine, seed=N + P + C, **options)


def test_group_norm_random_shapes_match_the_oracle(torch, s2d):
    rng = np.random.default_rng(7)
    for k in range(16):
        G = int(rng.choice([1, 2, 3, 4, 8, 16, 32]))
        C = G * int(np.exp(rng.uniform(0, np.log(600 // G))))
        N, P = int(np.exp(rng.uniform(0, np.log(40)))), int(np.exp(rng.uniform(0, np.log(3000))))
        P = max(1, min(P, 600000 // (N * C)))
        norm_case(torch, s2d, N, P, C, G, ("fp32", "bf16")[k % 2], ("none", "silu", "gelu")[k % 3], bool(rng.integers(2)), bool(rng.integers(4)), seed=k)


@pytest.mark.parametrize("P", [5, 4000])
def test_group_norm_of_a_large_mean_keeps_its_variance(torch, s2d, P):
    """Values around 1000 with a spread of 1: the squares are those of the deviations."""
    rng = np.random.default_rng(13)
    x = torch.from_numpy((1000 + rng.normal(size=(2, P, 64))).astype(np.float32)).cuda()
    y, stats = s2d.group_norm_fwd(x, None, None, 4)
    torch.cuda.synchronize()
    ref = seq.group_norm(host(x), None, None, 4, 1e-5)
    close("y", y, ref["y"], "fp32")
    assert float(np.abs(host(y) - ref["y"][0]).max()) < 2e-3                    # 2^-24 of 1000 on the mean, 6e-5, and some sums


def test_group_norm_in_place(torch, s2d):
    rng = np.random.default_rng(17)
    for shape in ((3, 50, 40), (1, 9000, 40), (50, 1, 320), (5000, 1, 36), (7, 1, 1100), (3, 5, 4100)):
        x, dy = rows(torch, rng, shape, "bf16"), rows(torch, rng, shape, "bf16")
        y, stats = s2d.group_norm_fwd(x, None, None, 4, act=s2d.ACT_SILU)
        dx, _, _ = s2d.group_norm_bwd(x, None, None, 4, stats, dy, act=s2d.ACT_SILU)
        x2, dy2 = x.clone(), dy.clone()
        y2, _ = s2d.group_norm_fwd(x2, None, None, 4, act=s2d.ACT_SILU, y=x2)
        dx2, _, _ = s2d.group_norm_bwd(x, None, None, 4, stats, dy2, act=s2d.ACT_SILU, dx=dy2)
        torch.cuda.synchronize()
        assert y2 is x2 and dx2 is dy2 and torch.equal(y, x2) and torch.equal(dx, dy2)


def test_group_norm_of_maps_and_of_views(torch, s2d):
    """[N][H][W][C] with a mask of its own dimensions; a channels-last image tensor by its permutation; a zero eps."""
    rng = np.random.default_rng(19)
    img = torch.from_numpy(rng.normal(size=(2, 24, 9, 11)).astype(np.float32)).cuda().contiguous(memory_format=torch.channels_last)
    x = img.permute(0, 2, 3, 1)
    mask = torch.from_numpy((rng.random((2, 9, 11)) < 0.3).astype(np.uint8)).cuda()
    y, _ = s2d.group_norm_fwd(x, None, None, 6, mask=mask, eps=0.0)
    torch.cuda.synchronize()
    ref = seq.group_norm(host(x).reshape(2, 99, 24), None, None, 6, 0.0, mask=mask.cpu().numpy().reshape(2, 99))
    close("y", y, ref["y"], "fp32")


def test_group_norm_past_32_bit_offsets(torch, s2d):
    N, P, C, G = 2, 2 ** 20 + 5, 1040, 4
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty((N, P, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    gamma, beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    y, stats = s2d.group_norm_fwd(x, gamma, beta, G)
    torch.cuda.synchronize()
    for n in range(N):
        for k in range(G):
            w = x[n, :, k * 260:(k + 1) * 260].float()
            assert abs(float(stats[n, k, 0]) - float(w.double().mean())) < 1e-5
            assert abs(float(stats[n, k, 1]) - 1.0) < 1e-3
    last = x[1, -7:].float().reshape(7, G, 260)
    want = ((last - stats[1, :, 0, None]) * stats[1, :, 1, None]).reshape(7, C)
    assert float((y[1, -7:].float() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 1e-5
    dx, dgamma, dbeta = s2d.group_norm_bwd(x, gamma, beta, G, stats, x)
    torch.cuda.synchronize()
    # dy = x: dv = x, so dx = rstd (x - mean x - xh mean(x xh)); with mean(x xh) = 1 / rstd (up to eps) that is about 0
    assert float(dx[1, -1000:].float().abs().max()) < 1e-2
    assert float((dbeta - x.float().sum((0, 1))).abs().max()) < 1.0


def chain_inputs(torch, rng, T, C, dtype):
    x, gates, dy = rows(torch, rng, (T, C), dtype), rows(torch, rng, (T, 2 * C), dtype), rows(torch, rng, (T, C), dtype)
    lam = torch.from_numpy(decays(rng, C)).cuda()
    gamma, beta = (torch.from_numpy((rng.normal(size=C) * 0.2 + m).astype(np.float32)).cuda() for m in (1.0, 0.0))
    return x, gates, dy, lam, gamma, beta


def chain(torch, s2d, x, gates, dy, lam, gamma, beta, off, G):
    """A recurrent layer: recurrence over packed sequences, then group norm with SiLU per token; and its backward pass."""
    C = x.shape[1]
    r, i = gates[:, :C], gates[:, C:]
    h, hT, saved = s2d.seq_recur_fwd(x, r, i, lam, offsets=off, want_final=True, want_saved=True)
    y, stats = s2d.group_norm_fwd(h[:, None], gamma, beta, G, act=s2d.ACT_SILU)
    dh, dgamma, dbeta = s2d.group_norm_bwd(h[:, None], gamma, beta, G, stats, dy[:, None], act=s2d.ACT_SILU)
    dgates = torch.empty_like(gates)
    dx, _, _, dlam, _ = s2d.seq_recur_bwd(x, r, i, lam, dh[:, 0], saved, offsets=off, out=(None, dgates[:, :C], dgates[:, C:]))
    return dict(h=h, hT=hT, y=y[:, 0], dh=dh[:, 0], dx=dx, dgates=dgates, dlam=dlam, dgamma=dgamma, dbeta=dbeta)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_recurrence_and_norm_in_a_row_match_the_oracle(torch, s2d, dtype):
    rng = np.random.default_rng(23)
    lens, C, G = [130, 1, 0, 261, 40], 160, 5
    T = sum(lens)
    v = chain_inputs(torch, rng, T, C, dtype)
    x, gates, dy, lam, gamma, beta = v
    off = torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device="cuda")
    got = chain(torch, s2d, *v, off, G)
    torch.cuda.synchronize()
    # each stage against the oracle on the tensors that this run handed it
    norm = seq.group_norm(host(got["h"])[:, None], host(gamma), host(beta), G, 1e-5, "silu", dy=host(dy)[:, None])
    rec = seq.recur(host(x), host(gates)[:, :C], host(gates)[:, C:], host(lam), spans_of("packed", lens), dh=host(got["dh"]))
    close("h", got["h"], rec["h"], dtype)
    close("y", got["y"], tuple(t[:, 0] for t in norm["y"]), dtype)
    close("dh", got["dh"], tuple(t[:, 0] for t in norm["dx"]), dtype)
    close("dx", got["dx"], rec["dx"], dtype)
    close("dr", got["dgates"][:, :C], rec["dr"], dtype)
    close("di", got["dgates"][:, C:], rec["di"], dtype)
    for name, ref in (("hT", rec["hT"]), ("dlam", rec["dlam"]), ("dgamma", norm["dgamma"]), ("dbeta", norm["dbeta"])):
        close(name, got[name], ref, "fp32")


@pytest.mark.parametrize("T,C,G", [(40, 64, 4), (5000, 256, 8)])
def test_captured_and_replayed(torch, s2d, T, C, G):
    """The layer's forward and backward, a grid's group norm and a decode step in one graph, replayed on new values between
    eager work; two graphs that share one memory pool."""
    rng = np.random.default_rng(29)
    off = torch.tensor([0, T // 3, T], dtype=torch.int32, device="cuda")
    still = [chain_inputs(torch, rng, T, C, "bf16") for _ in range(2)]
    grid = [rows(torch, rng, (2, T, C), "bf16") for _ in range(2)]
    state = [torch.zeros(8, C, device="cuda") for _ in range(2)]

    def work(k):
        out = chain(torch, s2d, *still[k], off, G)
        out["grid"], stats = s2d.group_norm_fwd(grid[k], None, None, G, act=s2d.ACT_GELU)
        out["dgrid"], _, _ = s2d.group_norm_bwd(grid[k], None, None, G, stats, grid[k], act=s2d.ACT_GELU)
        x, gates = still[k][0], still[k][1]
        out["step"] = s2d.seq_recur_step(x[:8], gates[:8, :C], gates[:8, C:], still[k][3], state[k])
        return out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in range(2):
            work(k)
    torch.cuda.current_stream().wait_stream(side)
    pool = torch.cuda.graph_pool_handle()
    graphs, outs = [], []
    for k in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, pool=pool):
            outs.append(work(k))
        graphs.append(gr)
    for turn in range(3):
        for k in range(2):
            for t, new in zip(still[k], chain_inputs(torch, rng, T, C, "bf16")):
                t.copy_(new)
            state[k].fill_(turn + 0.5)
            torch.cuda.synchronize()
            graphs[k].replay()
            torch.cuda.synchronize()
            got = {n: t.clone() for n, t in outs[k].items()}
            state[k].fill_(turn + 0.5)
            want = work(k)
            torch.cuda.synchronize()
            for n in want:
                assert torch.equal(got[n], want[n]), (turn, k, n)


def test_two_streams_at_once(torch, s2d):
    """The same calls on two streams side by side, long enough to overlap, give what each gives alone."""
    rng = np.random.default_rng(31)
    T, C, G = 20000, 512, 8
    off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    v = [chain_inputs(torch, rng, T, C, "bf16") for _ in range(2)]
    alone = [chain(torch, s2d, *v[k], off, G) for k in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [None, None]
    for turn in range(3):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                both[k] = chain(torch, s2d, *v[k], off, G)
    torch.cuda.synchronize()
    for k in range(2):
        for n in alone[k]:
            assert torch.equal(alone[k][n], both[k][n]), n


def test_binding_refusals(torch, s2d):
    x = torch.zeros(6, 8, device="cuda")
    lam = torch.zeros(8, device="cuda")
    off = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    ok = lambda **k: s2d.seq_recur_fwd(**{**dict(x=x, r=x, i=x, lam=lam), **k})
    ok()
    for bad, kind in ((dict(x=x.half()), TypeError), (dict(r=x.bfloat16()), ValueError), (dict(i=x[:5]), ValueError), (dict(lam=lam[:7]), ValueError),
                      (dict(lam=lam.double()), ValueError), (dict(offsets=off.long()), ValueError), (dict(offsets=off[:1]), ValueError),
                      (dict(lengths=off[:1]), ValueError), (dict(h0=torch.zeros(2, 8, device="cuda")), ValueError), (dict(r=x.cpu()), ValueError),
                      (dict(x=x.t().contiguous().t()), ValueError), (dict(r=x[:1].expand(6, 8)), ValueError), (dict(offsets=off.cpu()), ValueError),
                      (dict(x=x[:, None, None]), ValueError), (dict(lam=None), ValueError), (dict(x=lam), ValueError), (dict(scale="a"), TypeError)):
        with pytest.raises(kind):
            ok(**bad)
    for bad, code in ((dict(scale=0.0), -2), (dict(h=x), -2), (dict(x=x[None], r=x[None], i=x[None], offsets=None, scale=float("nan")), -2)):
        with pytest.raises(s2d.Scan2dError) as e:
            ok(**bad)
        assert e.value.code == code
    _, _, saved = ok(want_saved=True)
    with pytest.raises(ValueError):
        s2d.seq_recur_bwd(x, x, x, lam, x, None)
    with pytest.raises(ValueError):
        s2d.seq_recur_bwd(x, x, x, lam, x, saved, out=(None, None))
    with pytest.raises(s2d.Scan2dError) as e:
        s2d.seq_recur_bwd(x, x, x, lam, x, saved[:0])
    assert e.value.code in (-1, -5)
    with pytest.raises(ValueError):
        s2d.seq_recur_step(x, x, x, lam, torch.zeros(6, 8, device="cuda").bfloat16())
    with pytest.raises(s2d.Scan2dError):
        s2d.seq_recur_step(x, x, x, lam, torch.zeros(5, 8, device="cuda"))
    m = torch.zeros(2, 3, 8, device="cuda")
    for bad, kind in ((dict(groups=0), ValueError), (dict(groups=9), ValueError), (dict(gamma=lam[:4]), ValueError),
                      (dict(mask=torch.zeros(2, 4, dtype=torch.uint8, device="cuda")), ValueError),
                      (dict(mask=torch.zeros(2, 3, device="cuda")), ValueError), (dict(x=x), ValueError)):
        with pytest.raises(kind):
            s2d.group_norm_fwd(**{**dict(x=m, gamma=None, beta=None, groups=2), **bad})
    for bad, code in ((dict(groups=3), -2), (dict(act=7), -4), (dict(eps=-1.0), -2)):
        with pytest.raises(s2d.Scan2dError) as e:
            s2d.group_norm_fwd(**{**dict(x=m, gamma=None, beta=None, groups=2), **bad})
        assert e.value.code == code


@pytest.mark.parametrize("P", [1, 9, 4000])
@pytest.mark.parametrize("C,G,dtype", [(18, 3, "fp32"), (36, 3, "fp32"), (72, 3, "bf16"), (1194, 2, "bf16")])
def test_group_norm_infinite_gamma_stays_in_its_group(torch, s2d, P, C, G, dtype):
    """A weight that is infinite or NaN spoils its own group only: the others keep their bits."""
    rng = np.random.default_rng(P + C)
    N, D = (3, C // G)
    x, dy = (rows(torch, rng, (N, P, C), dtype) for _ in range(2))
    beta = torch.zeros(C, device="cuda")
    results = []
    for bad in (1.0, float("inf"), float("nan")):
        gamma = torch.ones(C, device="cuda")
        gamma[0] = gamma[D - 1] = gamma[C - D] = bad             # of the first and the last group
        if G == 2:
            gamma[C - D:] = 1.0                                  # two groups: the first only
        y, stats = s2d.group_norm_fwd(x, gamma, beta, G, act=s2d.ACT_SILU)
        results.append((y, stats, *s2d.group_norm_bwd(x, gamma, beta, G, stats, dy, act=s2d.ACT_SILU)))
    well = slice(D, 2 * D)
    for got in results[1:]:
        for a, b in zip(results[0], got):
            keep = (..., slice(1, 2), slice(None)) if a is results[0][1] else (..., well)
            assert torch.equal(a[keep], b[keep])


def test_group_norm_of_as_many_rows_as_there_may_be(torch, s2d):
    """2^31 - 4100 rows, as one item's positions and as items of one: the last rows are done too."""
    rows_, last = 2 ** 31 - 4100, 2 ** 23
    pattern = torch.tensor([1.0, 3.0, -2.0, 0.5, -0.5, 4.0], dtype=torch.bfloat16, device="cuda")      # whole patterns: the rows are a multiple of 6
    x = pattern.repeat(rows_ // 6 + 1)[:rows_].reshape(1, rows_, 1)
    y, stats = s2d.group_norm_fwd(x, None, None, 1)
    torch.cuda.synchronize()
    mean, var = 1.0, float(pattern.double().var(unbiased=False))
    # a lane joins its 2^13 rows four at a time, 2^11 roundings of 2^-24 of a mean (1) and of a sum of squares
    assert abs(float(stats[0, 0, 0]) - mean) < 2.0 ** -12 and abs(float(stats[0, 0, 1]) * var ** 0.5 - 1.0) < 2.0 ** -12
    tail = (x[0, -last:, 0].float() - stats[0, 0, 0]) * stats[0, 0, 1]
    assert float((y[0, -last:, 0].float() - tail).abs().max()) <= 2.0 ** -8 * 2.0
    dx, dgamma, _ = s2d.group_norm_bwd(x, torch.ones(1, device="cuda"), None, 1, stats, y)
    torch.cuda.synchronize()
    # dy = y: sum dv = 0, sum dv xh = the rows, so dx = 0 up to the rounding of y to bf16
    assert float(dx[0, -last:].float().abs().max()) <= 2.0 ** -7 * 2.0
    assert abs(float(dgamma[0]) / rows_ - 1.0) < 2.0 ** -7
    del y, dx
    x = x.reshape(rows_, 1, 1)
    gamma, beta = torch.ones(1, device="cuda"), torch.tensor([0.75], device="cuda")
    y, stats = s2d.group_norm_fwd(x, gamma, beta, 1, eps=1.0)
    torch.cuda.synchronize()
    assert torch.equal(stats[-last:, 0, 0], x[-last:, 0, 0].float()) and bool((stats[-last:, 0, 1] == 1.0).all())
    assert bool((y[-last:] == 0.75).all())
    dx, dgamma, dbeta = s2d.group_norm_bwd(x, gamma, beta, 1, stats, y, dx=y)
    torch.cuda.synchronize()
    assert bool((dx[-last:] == 0).all()) and abs(float(dbeta[0]) / rows_ - 0.75) < 1e-5 and float(dgamma[0]) == 0.0


@pytest.mark.parametrize("T", [256, 257, 1027, 5002])
def test_step_finds_a_slot_again_wherever_it_stands(torch, s2d, T):
    """Two rows of one slot at any distance, the table at any 4-byte address: as one call after the other."""
    rng = np.random.default_rng(T)
    C = 3
    x, r, i = (rows(torch, rng, (T, C), "fp32") for _ in range(3))
    lam = torch.from_numpy(decays(rng, C)).cuda()
    table = rng.permutation(T + 40).astype(np.int32)[:T]
    pairs = [(0, T - 1), (1, T // 2), (T // 3, T - 2), (T - 4, T - 3)]
    for a, b in pairs:
        table[b] = table[a]
    slots = torch.from_numpy(np.concatenate([[0], table]).astype(np.int32)).cuda()[1:]
    pool = torch.from_numpy(rng.normal(size=(T + 40, C)).astype(np.float32)).cuda()
    state, one = pool.clone(), pool.clone()
    h = s2d.seq_recur_step(x, r, i, lam, state, slots=slots)
    later = [b for _, b in pairs]
    early = [t for t in range(T) if t not in later]
    each = torch.empty_like(h)
    for part in (early, later):                              # no slot twice in either
        part = torch.tensor(part, device="cuda")
        each[part] = s2d.seq_recur_step(x[part], r[part], i[part], lam, one, slots=slots[part])
    torch.cuda.synchronize()
    assert torch.equal(state, one) and torch.equal(h, each)


@pytest.mark.parametrize("N,P,C,G,dtype,act,share,affine", [
    (1, 2500, 130, 2, "bf16", "silu", 0.5, True), (2, 6000, 516, 2, "fp32", "gelu", 0.3, True), (1, 3001, 1192, 2, "bf16", "none", 0.7, True),
    (1, 1500, 2600, 1, "bf16", "silu", 0.5, True), (2, 4100, 24, 1, "fp32", "silu", 0.9, False), (1, 9000, 7, 7, "fp32", "gelu", 0.5, True),
    (1, 5000, 3, 1, "bf16", "silu", 0.5, True), (2, 700, 1602, 2, "fp32", "silu", 0.5, True), (1, 20000, 64, 32, "bf16", "gelu", 0.99, True)])
def test_group_norm_with_runs_and_scattered_masked_positions(torch, s2d, N, P, C, G, dtype, act, share, affine):
    """Many positions of which a run and scattered ones are masked: NaN there, in place and not."""
    rng = np.random.default_rng(P + C)
    x, dy = rows(torch, rng, (N, P, C), dtype, 1.5), rows(torch, rng, (N, P, C), dtype)
    gamma, beta = (torch.from_numpy(v.astype(np.float32)).cuda() if affine else None
                   for v in (rng.normal(size=C) * 0.3 + 1, rng.normal(size=C) * 0.3))
    mask = (rng.random((N, P)) < share).astype(np.uint8)
    mask[0, P // 3:P // 3 + P // 4] = 255
    mask[-1, -3:] = [0, 1, 0]
    m = torch.from_numpy(mask).cuda()
    x[m != 0], dy[m != 0] = float("nan"), float("inf")
    code = {"none": s2d.ACT_NONE, "silu": s2d.ACT_SILU, "gelu": s2d.ACT_GELU}[act]
    param = lambda t: None if t is None else host(t)
    ref = seq.group_norm(host(x), param(gamma), param(beta), G, 1e-5, act, mask, host(dy))
    y, stats = s2d.group_norm_fwd(x, gamma, beta, G, act=code, mask=m)
    dx, dgamma, dbeta = s2d.group_norm_bwd(x, gamma, beta, G, stats, dy, act=code, mask=m)
    for name, got in dict(y=y, dx=dx).items():
        close(name, got, ref[name], dtype)
        assert bool((got[m != 0] == 0).all())
    close("stats", stats, ref["stats"], "fp32")
    if affine:
        close("dgamma", dgamma, ref["dgamma"], "fp32")
        close("dbeta", dbeta, ref["dbeta"], "fp32")
    assert torch.equal(s2d.group_norm_bwd(x, gamma, beta, G, stats, dy, act=code, mask=m, dx=dy)[0], dx)
    assert torch.equal(s2d.group_norm_fwd(x, gamma, beta, G, act=code, mask=m, y=x)[0], y)


@pytest.mark.parametrize("shape,one", [((4, 50, 8), (1,)), ((4, 50, 8), (0,)), ((4, 50, 8), (0, 1)), ((2, 3, 5, 8), (1,)), ((2, 3, 5, 8), (2,)),
                                       ((2, 3, 5, 8), (1, 2)), ((6, 8), (0,))])
def test_broadcast_rows_are_refused(torch, s2d, shape, one):
    """Tensors that have one row for all of a dimension, as each argument in turn, read or written: an error and no call."""
    x = torch.zeros(shape, device="cuda")
    lam = torch.zeros(8, device="cuda")
    flat = torch.zeros([1 if k in one else n for k, n in enumerate(shape)], device="cuda").expand(shape)
    calls = []
    if len(shape) <= 3:
        _, _, saved = s2d.seq_recur_fwd(x, x, x, lam, want_saved=True)
        calls += [(s2d.seq_recur_fwd, dict(x=x, r=x, i=x, lam=lam, h=torch.zeros_like(x)), ("x", "r", "i", "h")),
                  (s2d.seq_recur_bwd, dict(x=x, r=x, i=x, lam=lam, dh=x, saved=saved), ("x", "r", "i", "dh"))]
        for k in range(3):
            with pytest.raises(ValueError, match="rows at one stride"):
                s2d.seq_recur_bwd(x, x, x, lam, x, saved, out=tuple(flat if q == k else None for q in range(3)))
    if len(shape) == 2:
        calls.append((s2d.seq_recur_step, dict(x=x, r=x, i=x, lam=lam, state=torch.zeros(6, 8, device="cuda"), h=torch.zeros_like(x)), ("x", "r", "i", "h")))
    if len(shape) >= 3:
        _, stats = s2d.group_norm_fwd(x, None, None, 2)
        calls += [(s2d.group_norm_fwd, dict(x=x, gamma=None, beta=None, groups=2, y=torch.zeros_like(x)), ("x", "y")),
                  (s2d.group_norm_bwd, dict(x=x, gamma=None, beta=None, groups=2, stats=stats, dy=x, dx=torch.zeros_like(x)), ("x", "dy", "dx"))]
    for fn, kw, names in calls:
        fn(**kw)
        for name in names:
            with pytest.raises(ValueError, match="rows at one stride"):
                fn(**{**kw, name: flat})
    torch.cuda.synchronize()


@pytest.mark.parametrize("N,P,C,G,dtype,act", [
    # more items than workgroups: each takes several at once.  Groups in a workgroup's slab, many and one, rows that fill it and do not
    (4100, 9, 192, 32, "bf16", "silu"), (4100, 3, 512, 1, "fp32", "gelu"), (2500, 10, 160, 32, "fp32", "none"), (4099, 4, 512, 1, "bf16", "silu"),
    (5000, 2, 1024, 2, "bf16", "silu"), (2049, 6, 320, 1, "fp32", "silu"), (2300, 12, 160, 5, "bf16", "gelu"),
    # teams within a wavefront, and workgroups that take one item after the other
    (9000, 4, 64, 4, "bf16", "silu"), (40000, 3, 20, 5, "fp32", "silu"), (8200, 2, 516, 3, "bf16", "none"), (2100, 70, 160, 4, "bf16", "silu")])
def test_group_norm_of_many_masked_items_of_a_few_positions(torch, s2d, N, P, C, G, dtype, act):
    """Windows with masked positions, different numbers of them, many more than there are workgroups."""
    norm_case(torch, s2d, N, P, C, G, dtype, act, True, True, seed=N + C)


@pytest.mark.parametrize("where", ["r", "-r", "i", "x", "dh", "h0", "dhT"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("lens", [(16, 19, 40, 8), (50, 3, 160, 20, 1, 64), (1000, 608, 3, 996, 1403, 700)], ids=["one chunk", "chunks", "groups of chunks"])
def test_recurrence_nan_stays_in_its_sequence_forward_and_backward(torch, s2d, lens, dtype, where):
    """A NaN of either sign in one sequence, one to seven rows behind its first in different channels (among the rows of one
    wavefront, that is): the other sequences keep their bits in every output, and a channel without one keeps all of them."""
    rng = np.random.default_rng(len(lens))
    T, S, C = sum(lens), len(lens), 72
    ends = np.cumsum(lens)
    off = torch.tensor([0, *ends], dtype=torch.int32, device="cuda")
    lam = torch.from_numpy(decays(rng, C)).cuda()
    x, r, i, dh = (rows(torch, rng, (T, C), dtype) for _ in range(4))
    h0, dhT = (torch.from_numpy(rng.normal(size=(S, C)).astype(np.float32)).cuda() for _ in range(2))

    def once(x, r, i, dh, h0, dhT):
        h, hT, saved = s2d.seq_recur_fwd(x, r, i, lam, offsets=off, h0=h0, want_final=True, want_saved=True)
        dx, dr, di, dlam, dh0 = s2d.seq_recur_bwd(x, r, i, lam, dh, saved, offsets=off, h0=h0, dhT=dhT)
        torch.cuda.synchronize()
        return dict(h=h, dx=dx, dr=dr, di=di), dict(hT=hT, dh0=dh0), dlam

    clean = once(x, r, i, dh, h0, dhT)
    channels = torch.arange(1, C, device="cuda")                               # channel 0 has none
    for s in range(S):
        v = dict(x=x, r=r, i=i, dh=dh, h0=h0, dhT=dhT)
        name = where[-1] if where[0] == "-" else where
        t = v[name] = v[name].clone()
        nan = torch.tensor(float("nan"), device="cuda").to(t.dtype)
        nan = torch.copysign(nan, torch.tensor(-1.0 if where[0] == "-" else 1.0, device="cuda").to(t.dtype))
        if name in ("h0", "dhT"):
            t[s, 1:] = nan
        else:
            at = torch.clamp(int(ends[s]) - lens[s] + 1 + channels % 7, max=int(ends[s]) - 1)
            t[at, channels] = nan
        got = once(**v)
        others = torch.ones(T, dtype=torch.bool, device="cuda")
        others[int(ends[s]) - lens[s]:int(ends[s])] = False
        rest = [k for k in range(S) if k != s]
        for n in clean[0]:
            assert torch.equal(got[0][n][others], clean[0][n][others]), (n, s)
            assert torch.equal(got[0][n][:, 0], clean[0][n][:, 0]), (n, s)
        for n in clean[1]:
            assert torch.equal(got[1][n][rest], clean[1][n][rest]), (n, s)
            assert torch.equal(got[1][n][:, 0], clean[1][n][:, 0]), (n, s)
        assert torch.equal(got[2][:1], clean[2][:1]), s


@pytest.mark.parametrize("N,P,C,G", [(16384, 1, 4096, 1), (16384, 520, 256, 256), (5000, 81, 320, 1), (1700001, 1, 2049, 1)])
def test_group_norm_backward_of_many_items(torch, s2d, N, P, C, G):
    """As many items and channels as would need 2^32 threads in one launch of the kernels that join the items' sums (and fewer), and of the
    tiles themselves: the first and last items, and the parameters' sums of some channels, against the oracle."""
    g = torch.Generator(device="cuda").manual_seed(N + C)
    make = lambda: torch.empty((N, P, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    x, dy = make(), make()
    rng = np.random.default_rng(N)
    gamma, beta = (torch.from_numpy((rng.normal(size=C) * 0.2 + m).astype(np.float32)).cuda() for m in (1.0, 0.0))
    print(f"group norm backward N={N} P={P} C={C} G={G}", flush=True)
    y, stats = s2d.group_norm_fwd(x, gamma, beta, G)
    dx, dgamma, dbeta = s2d.group_norm_bwd(x, gamma, beta, G, stats, dy)
    torch.cuda.synchronize()
    for part in (slice(0, 3), slice(N // 2, N // 2 + 3), slice(N - 3, N)):
        ref = seq.group_norm(host(x[part]), host(gamma), host(beta), G, 1e-5, dy=host(dy[part]))
        for name, got in (("y", y), ("dx", dx)):
            close(name, got[part], ref[name], "bf16")
        close("stats", stats[part], ref["stats"], "fp32")
    # dbeta = sum dy, dgamma = sum dy xh: a sum over N P terms in at least 32 partial sums of which up to 72 are joined (the oracle's
    # count), and xh from the statistics with 4 roundings
    U = 2.0 ** -24
    for c in (0, 1, C // 2, C - 1):
        d, v = dy[:, :, c].double(), x[:, :, c].double()
        m, rs = (stats[:, c // (C // G), k].double()[:, None] for k in (0, 1))
        terms = d * (v - m) * rs
        slack = (N * P / 32 + 72) * U
        assert abs(float(dbeta[c]) - float(d.sum())) <= slack * float(d.abs().sum()), c
        assert abs(float(dgamma[c]) - float(terms.sum())) <= (slack + 4 * U) * float((d.abs() * (v.abs() + m.abs()) * rs).sum()), c


def test_recurrence_of_as_many_rows_as_there_may_be(torch, s2d):
    """2^31 - 4097 rows, whose chunks take several launches: rows at both ends and on both sides of every cut against the oracle."""
    T, C = 2 ** 31 - 4097, 1
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((T, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    lam = torch.zeros(C, device="cuda")                                        # scale 8: a state is forgotten within some ten tokens
    print(f"recurrence T={T} C={C}", flush=True)
    h, hT, saved = s2d.seq_recur_fwd(x, x, x, lam, want_final=True, want_saved=True)
    torch.cuda.synchronize()
    dx, dr, di, dlam, _ = s2d.seq_recur_bwd(x, x, x, lam, x, saved)
    torch.cuda.synchronize()
    most, chunks = (2 ** 32 - 1) // 768, -(-T // 96)                           # chunks of a launch backward; and below, forward
    cuts = [8388607 * 128, 2 * 8388607 * 128] + [(chunks - k * most) * 96 for k in range(1, 5)]
    for lo, hi in [(0, 500), (T - 500, T)] + [(c - 300, c + 300) for c in cuts if 300 <= c <= T - 300]:
        w = host(x[lo:hi])
        ref = seq.recur(w, w, w, host(lam), [(0, hi - lo)], dh=w)
        clear = slice(0 if lo == 0 else 200, hi - lo if hi == T else hi - lo - 200)      # behind 200 rows nothing of a cut is left
        for name, got in dict(h=h, dx=dx, dr=dr, di=di).items():
            close(name, got[lo:hi][clear], tuple(t[clear] for t in ref[name]), "bf16")
        if hi == T:
            close("hT", hT, ref["hT"], "fp32")
    # dlam from dr = q (1 - sigmoid(r)), each off by half a step, and the library's sums: a share of the chunks in a row, 64 of these
    total, size = 0.0, 0.0
    for lo in range(0, T, 2 ** 28):
        q = dr[lo:lo + 2 ** 28].double() / torch.sigmoid(-x[lo:lo + 2 ** 28].double())
        total, size = total + float(q.sum()), size + float(q.abs().sum())
    ratio = 0.5 / np.log(2.0)                                                  # sigmoid(0) / softplus(0)
    assert abs(float(dlam[0]) - total * ratio) <= (2.0 ** -8 + (chunks / 64 + 200) * 2.0 ** -24) * size * ratio


def test_recurrence_of_no_rows_with_many_states(torch, s2d):
    """2^32 states and more go through a call of no rows, forward and backward."""
    S, C = 2 ** 16 + 1, 2 ** 16
    x, lam = torch.empty((0, C), device="cuda"), torch.zeros(C, device="cuda")
    off = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    h0 = torch.empty((S, C), device="cuda").uniform_()
    _, hT, saved = s2d.seq_recur_fwd(x, x, x, lam, offsets=off, h0=h0, want_final=True, want_saved=True)
    torch.cuda.synchronize()
    assert all(torch.equal(hT[k:k + 4096], h0[k:k + 4096]) for k in range(0, S, 4096))
    del hT
    *_, dlam, dh0 = s2d.seq_recur_bwd(x, x, x, lam, x, saved, offsets=off, dhT=h0, want_dh0=True)
    torch.cuda.synchronize()
    assert all(torch.equal(dh0[k:k + 4096], h0[k:k + 4096]) for k in range(0, S, 4096)) and bool((dlam == 0).all())
    del dh0
    _, hT, _ = s2d.seq_recur_fwd(x, x, x, lam, offsets=off, want_final=True)
    torch.cuda.synchronize()
    assert all(not bool(hT[k:k + 4096].any()) for k in range(0, S, 4096))
