"""Operators on embedding tables against their formulas in float64: lookups and their gradient, tables in 4 bits and scores against
them, adjusted scores.  Tolerances count roundings: u is half a step of a type relative to the value (float32 2^-24, bfloat16 2^-8); a
float32 sum of k terms is off by at most k u times the sum of their magnitudes, whatever its order."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TINY = 1e-37                                        # results near the smallest normal number


def _t(name):
    import torch
    return torch.float32 if name == "f32" else torch.bfloat16


def _embed(dtype="f32", **kw):
    import paper_2307_12059_amd as kgc
    return kgc.Embed(dtype=dtype, **kw)


def _strided(x, extra, shift):
    """x as rows of a wider buffer of -77s, from an element offset on; the buffer too."""
    import torch
    n, d = x.shape
    buf = torch.full((n * (d + extra) + shift,), -77.0, dtype=x.dtype, device=x.device)
    view = buf[shift:].view(n, d + extra)[:, :d] if n else x
    view.copy_(x)
    return view, buf


def _close(got, want, tol, out):
    """got (device tensor) within tol (float64 array, float32 arithmetic) and the rounding of its type of want."""
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    bound = tol + U[out] * (np.abs(want) + tol) + TINY
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / bound)} bounds"


# ---- lookup ----
def _lookup_want(A, ia, sa, B=None, ib=None, sb=0.0):
    def rows(T, ids):
        T, ids = T.double().cpu().numpy(), ids.cpu().numpy()
        ok = (ids >= 0) & (ids < len(T))
        out = np.zeros((len(ids), T.shape[1]))
        out[ok] = T[ids[ok]]
        return out
    a = sa * rows(A, ia)
    b = sb * rows(B, ib) if B is not None else 0.0 * a
    return a + b, np.abs(a) + np.abs(b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,N,R,d", [(1, 1, 1, 1), (1, 5, 0, 3), (7, 3, 2, 4), (1000, 50, 7, 5), (513, 2000, 8, 32), (4099, 301, 18, 100),
                                     (65, 40, 3, 127), (300, 77, 5, 512), (33, 20, 4, 957), (20, 20, 4, 960)])
def test_lookup(n, N, R, d, dtype, out):
    import torch
    g = torch.Generator(device="cuda").manual_seed(n + d)
    A = torch.randn((N, d), generator=g, device="cuda").to(_t(dtype))
    triples = torch.randint(-2, N + 3, (n, 3), generator=g, device="cuda", dtype=torch.int32)      # some name no row
    e = _embed(dtype)
    sa, sb = 1.75, -0.3
    if R:
        B = torch.randn((R, d), generator=g, device="cuda").to(_t(dtype))
        got = e.lookup(A, triples[:, 0], B, triples[:, 2], sa=sa, sb=sb, out_dtype=_t(out))
        want, size = _lookup_want(A, triples[:, 0], sa, B, triples[:, 2], float(np.float32(sb)))
    else:
        got = e.lookup(A, triples[:, 0], sa=sa, out_dtype=_t(out))
        want, size = _lookup_want(A, triples[:, 0], sa)
    assert got.dtype == _t(out)
    _close(got, want, 3 * U["f32"] * size, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,extra,shift", [(100, 1, 0), (33, 2, 1), (64, 5, 3), (3, 1, 2)])
def test_lookup_of_strided_rows_leaves_what_lies_between_them(dtype, d, extra, shift):
    import torch
    g = torch.Generator(device="cuda").manual_seed(d)
    A, _ = _strided(torch.randn((90, d), generator=g, device="cuda").to(_t(dtype)), extra, shift)
    B, _ = _strided(torch.randn((9, d), generator=g, device="cuda").to(_t(dtype)), 2 * extra, 0)
    ids = torch.randint(0, 9, (2 * 211,), generator=g, device="cuda", dtype=torch.int32)[::2]
    out, buf = _strided(torch.zeros((211, d), device="cuda", dtype=_t(dtype)), extra, shift)
    e = _embed(dtype)
    assert e.lookup(A, ids, B, ids, out=out) is out
    want, size = _lookup_want(A, ids, 1.0, B, ids, 1.0)
    _close(out, want, 3 * U["f32"] * size, dtype)
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask[shift:].view(211, d + extra)[:, :d] = False
    assert (buf[mask] == -77).all()
    # one row again and again, as an expanded tensor has it
    same = e.lookup(A[5:6].expand(40, d), torch.arange(40, dtype=torch.int32, device="cuda"))
    assert torch.equal(same, A[5:6].expand(40, d))


def test_lookup_of_the_records_of_a_join_and_of_nothing():
    import torch
    import paper_2307_12059_amd as kgc
    g = torch.Generator(device="cuda").manual_seed(0)
    E, Rv = torch.randn((300, 16), generator=g, device="cuda"), torch.randn((4, 16), generator=g, device="cuda")
    j = kgc.Join(dtype="f32")
    got = j.join(E, Rv, 2, 3.0, cap=1 << 18, fetch=False)
    rec = got["out"][:got["count"]]
    assert got["count"] > 100
    e = _embed()
    q = e.lookup(E, rec[:, 0], Rv, rec[:, 1])
    dist = (q.double() - e.lookup(E, rec[:, 2]).double()).norm(dim=1)
    # coordinates of size up to 8 are off by 2^-24 of it each
    assert torch.allclose(dist, rec[:, 3].view(torch.float32).double(), rtol=1e-6, atol=16 * 8 * 2.0 ** -24)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert e.lookup(E, none).shape == (0, 16)
    two = torch.tensor([0, -1], dtype=torch.int32, device="cuda")
    assert (e.lookup(E[:0], two) == 0).all()
    assert torch.equal(e.lookup(E, two, Rv[:0], two)[0], E[0])
    # an infinity and a NaN stay where they are; a missing row is 0 whatever the scale
    E[3, 2], E[3, 5] = float("inf"), float("nan")
    x = e.lookup(E, torch.tensor([3, -1], dtype=torch.int32, device="cuda"), sa=2.0)
    assert x[0, 2] == float("inf") and torch.isnan(x[0, 5]) and torch.isfinite(x[0, [0, 1, 3, 4]]).all() and (x[1] == 0).all()
    nan = torch.full((1, 4), 1.0, device="cuda"); nan.view(torch.int32)[0, 1] = 0x7FFFFFFF
    low = e.lookup(nan, torch.zeros(1, dtype=torch.int32, device="cuda"), out_dtype=torch.bfloat16)
    assert torch.isnan(low[0, 1]) and (low[0, [0, 2, 3]] == 1).all()


# ---- its gradient ----
def _grad_want(G, ids, N, scale, before=None):
    G, ids = G.double().cpu().numpy(), ids.cpu().numpy()
    ok = (ids >= 0) & (ids < N)
    want, size = np.zeros((N, G.shape[1])), np.zeros((N, G.shape[1]))
    np.add.at(want, ids[ok], scale * G[ok])
    np.add.at(size, ids[ok], abs(scale) * np.abs(G[ok]))
    times = np.bincount(ids[ok], minlength=N)[:, None]
    if before is not None:
        before = before.double().cpu().numpy()
        want, size = want + before, size + np.abs(before)
    return want, (times + 3) * U["f32"] * size


GRADS = [(1, 1, 1), (1, 40, 7), (2, 1, 100), (64, 3, 5), (65, 100, 32), (1000, 17, 100), (1024, 9000, 33), (1025, 9, 64), (1300, 60000, 12),
         (4097, 2, 100), (5000, 700, 129), (9000, 300, 513), (3000, 5, 960), (20011, 2049, 31), (70001, 130, 20), (300007, 1, 16), (300007, 4099, 8), (4096, 5, 20), (12000, 2, 30), (9001, 40, 33), (30000, 140, 16), (30001, 44, 100), (8193, 4, 256), (70000, 20, 199), (9000, 12, 4), (20000, 9, 5), (10001, 400000, 6),
         (4096, 7000, 33), (8000, 700, 30), (8192, 2048, 100), (8192, 5, 40), (290001, 60000, 4), (280001, 1300000, 2), (265000, 5000000, 1)]


@pytest.mark.parametrize("n,N,d", GRADS)
@pytest.mark.parametrize("g_dtype,out", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_lookup_grad(n, N, d, g_dtype, out):
    import torch
    g = torch.Generator(device="cuda").manual_seed(n + N)
    G = torch.randn((n, d), generator=g, device="cuda").to(_t(g_dtype))
    ids = torch.randint(-1, N + 1, (n, 3), generator=g, device="cuda", dtype=torch.int32)[:, 1]
    e = _embed()
    first = e.lookup_grad(G, ids, N=N, scale=-0.5, out_dtype=_t(out))
    want, tol = _grad_want(G, ids, N, -0.5)
    _close(first, want, tol, out)
    assert torch.equal(first, e.lookup_grad(G, ids, N=N, scale=-0.5, out_dtype=_t(out)))          # bit for bit
    before = torch.randn((N, d), generator=g, device="cuda").to(_t(out))
    more = before.clone()
    assert e.lookup_grad(G, ids, out=more, scale=0.25, accumulate=True) is more
    want, tol = _grad_want(G, ids, N, 0.25, before)
    _close(more, want, tol, out)
    named = torch.zeros(N + 1, dtype=torch.bool, device="cuda")
    named[torch.where((ids >= 0) & (ids < N), ids, N).long()] = True
    assert torch.equal(more[~named[:N]], before[~named[:N]])


@pytest.mark.parametrize("n", [700, 9500, 150000])
@pytest.mark.parametrize("kind", ["hub", "sorted", "same", "none", "runs", "last"])
def test_lookup_grad_of_uneven_ids(n, kind):
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    N, d = 5000, 24
    ids = {"hub": lambda: torch.where(torch.rand(n, generator=g, device="cuda") < 0.9, 17, torch.randint(0, N, (n,), generator=g, device="cuda")),
           "sorted": lambda: torch.arange(n, device="cuda") % N,
           "same": lambda: torch.full((n,), N - 1, device="cuda"),
           "none": lambda: torch.full((n,), -1, device="cuda"),
           "runs": lambda: torch.arange(n, device="cuda") // 37,
           "last": lambda: torch.where(torch.arange(n, device="cuda") == n - 1, 0, 2 ** 31 - 1)}[kind]().to(torch.int32)
    G = torch.randn((n, d), generator=g, device="cuda")
    got = _embed().lookup_grad(G, ids, N=N)
    want, tol = _grad_want(G, ids, N, 1.0)
    _close(got, want, tol, "f32")


@pytest.mark.parametrize("n", [3501, 16384, 16385, 49152, 49153])
@pytest.mark.parametrize("N", [255, 257, 15000, 262144, 262145])
def test_lookup_grad_of_ids_that_one_launch_groups(n, N):
    """Around the sizes at which the grouping changes: uneven ids, padding among them, every stride, alone and added."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n + N)
    d = 6
    wide = torch.empty(n * 5, dtype=torch.int32, device="cuda")
    ids = (N ** torch.rand(n, generator=g, device="cuda", dtype=torch.float64)).to(torch.int32)           # small numbers most of all
    ids[torch.rand(n, generator=g, device="cuda") < 0.05] = -5
    ids[:3] = torch.tensor([N - 1, 0, N - 1])
    ids[n // 2:n // 2 + 1500] = N // 2                       # longer than a wave's share of the ids
    G = torch.randn((n, d), generator=g, device="cuda")
    want, tol = _grad_want(G, ids, N, 1.0)
    e, got = _embed(), []
    for step in (1, 2, 3, 4, 5):
        its = wide[:n * step].view(n, step)[:, step // 2]
        its.copy_(ids)
        assert its.stride(0) == step
        got.append(e.lookup_grad(G, its, N=N))
        _close(got[-1], want, tol, "f32")
        assert torch.equal(got[-1], e.lookup_grad(G, its, N=N))
        more = torch.ones((N, d), device="cuda")
        e.lookup_grad(G, its, out=more, accumulate=True)
        _close(more, *_grad_want(G, ids, N, 1.0, torch.ones((N, d))), "f32")


@pytest.mark.parametrize("n,N", [(300, 800), (5000, 800), (12000, 800), (12000, 20)])
def test_lookup_grad_of_strided_and_broadcast_gradients(n, N):
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    d = 45
    ids = torch.randint(0, N, (n,), generator=g, device="cuda", dtype=torch.int32)
    G, _ = _strided(torch.randn((n, d), generator=g, device="cuda"), 3, 1)
    e = _embed()
    for accumulate in (False, True):
        out, buf = _strided(torch.ones((N, d), device="cuda"), 7, 2)
        e.lookup_grad(G, ids, out=out, accumulate=accumulate)
        want, tol = _grad_want(G, ids, N, 1.0, torch.ones((N, d)) if accumulate else None)
        _close(out, want, tol, "f32")
        rest = torch.ones_like(buf, dtype=torch.bool)
        rest[2:].view(N, d + 7)[:, :d] = False
        assert (buf[rest] == -77).all()
    # the gradient of a sum over rows: one row for all
    row = torch.randn((1, d), generator=g, device="cuda").expand(n, d)
    got = e.lookup_grad(row, ids, N=N)
    want, tol = _grad_want(row, ids, N, 1.0)
    _close(got, want, tol, "f32")
    # one id for all, as an expanded tensor has it
    got = e.lookup_grad(G, ids[:1].expand(n), N=N)
    want, tol = _grad_want(G, ids[:1].expand(n), N, 1.0)
    _close(got, want, tol, "f32")


@pytest.mark.parametrize("n,N", [(300, 50), (9000, 50), (9000, 2000)])
def test_gradients_of_padding_reach_no_row(n, N):
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    G = torch.randn((n, 37), generator=g, device="cuda")
    ids = torch.randint(0, N, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[n // 2:] = torch.tensor([-1, N, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda").repeat(n)[:n - n // 2]
    G[n // 2:] = float("nan")
    want, tol = _grad_want(G[:n // 2], ids[:n // 2], N, 1.0)
    _close(_embed().lookup_grad(G, ids, N=N), want, tol, "f32")
    G[3, 5] = float("inf")                                  # one that names a row reaches this row's column alone
    got = _embed().lookup_grad(G, ids, N=N)
    bad = torch.zeros((N, 37), dtype=torch.bool, device="cuda"); bad[int(ids[3]), 5] = True
    assert torch.isinf(got[bad]).all() and torch.isfinite(got[~bad]).all()


def test_lookup_grad_of_nothing_clears_or_leaves():
    import torch
    e = _embed()
    none, G = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty((0, 6), device="cuda")
    assert (e.lookup_grad(G, none, N=5) == 0).all() and e.lookup_grad(G, none, N=0).shape == (0, 6)
    many = torch.zeros(9000, dtype=torch.int32, device="cuda")
    assert e.lookup_grad(torch.ones((9000, 6), device="cuda"), many, N=0).shape == (0, 6)
    kept = torch.ones((5, 6), device="cuda")
    e.lookup_grad(torch.ones((9000, 6), device="cuda"), many - 1, out=kept, accumulate=True)
    assert (kept == 1).all()
    assert (e.lookup_grad(G, none, out=kept, accumulate=True) == 1).all()
    assert (e.lookup_grad(G, none, out=kept) == 0).all()
    assert e.lookup_grad(torch.ones((3, 6), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), N=0).shape == (0, 6)


def test_lookup_grad_is_the_derivative_of_a_lookup():
    """Central differences of f(E, R) = sum(C * (E[h] + 2 R[r])) in float32: f is linear, so they are off by roundings only."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    E, R = torch.randn((40, 6), generator=g, device="cuda"), torch.randn((3, 6), generator=g, device="cuda")
    t = torch.stack([torch.randint(0, k, (90,), generator=g, device="cuda", dtype=torch.int32) for k in (40, 3)], 1)
    C = torch.randn((90, 6), generator=g, device="cuda")
    e = _embed()
    f = lambda: (C.double() * e.lookup(E, t[:, 0], R, t[:, 1], sb=2.0).double()).sum()
    for table, column, scale in ((E, 0, 1.0), (R, 1, 2.0)):
        grad = e.lookup_grad(C, t[:, column], N=table.shape[0], scale=scale)
        for v, k in ((0, 0), (2, 5), (1, 3)):
            was, h = table[v, k].clone(), 0.5
            table[v, k] = was + h; up = f()
            table[v, k] = was - h; down = f()
            table[v, k] = was
            # each of the 90 rows is off by 3 roundings of numbers below 16 either way, times |C| < 8
            assert abs(float((up - down) / (2 * h)) - float(grad[v, k])) <= 2 * 90 * 3 * 16 * 8 * U["f32"]


# ---- tables in 4 bits ----
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def _packed_want(W):
    """The values a packed table stands for, in float64."""
    W = W.float().cpu().numpy()
    N, d = W.shape
    out = np.zeros((N, d))
    for k in range(0, d, 32):
        w = W[:, k:k + 32]
        s = _bf16(np.abs(w).max(1, keepdims=True) / np.float32(6))
        away = np.abs(np.abs(w.astype(np.float64))[..., None] - LEVELS * s[..., None])
        best = away.min(-1, keepdims=True)
        first, last = (away == best).argmax(-1), 7 - (away == best)[..., ::-1].argmax(-1)
        pick = np.where(first % 2 == 0, first, last)
        out[:, k:k + 32] = np.sign(w) * LEVELS[pick] * s
    return out


def _unpacked(e, table):
    """The values again, as scores of unit vectors: one product each, exact in float32."""
    import torch
    return e.scores4(table, torch.eye(table.d, device="cuda")).t()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d", [(1, 1), (3, 31), (64, 32), (65, 33), (130, 100), (1000, 128), (77, 257), (70, 960)])
def test_pack4(N, d, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(N)
    W = torch.randn((N, d), generator=g, device="cuda")
    W = (W * torch.exp(3 * torch.randn((N, 1), generator=g, device="cuda"))).to(_t(dtype))
    W[0] = 0
    if N > 2 and d > 8:
        # middles between levels, exactly: the scale is 1
        W[1] = 0
        W[1, :9] = torch.tensor([6.0, 0.25, -0.75, 1.25, 1.75, -2.5, 3.5, -5.0, 0.2])
        W[2] = W[1] * 2.0 ** -120
    W, _ = _strided(W, 3, 1)
    e = _embed(dtype)
    table = e.pack4(W)
    want = _packed_want(W)
    got = _unpacked(e, table).double().cpu().numpy()
    assert np.array_equal(got, want)
    sq = (want ** 2).sum(1)
    assert np.all(np.abs(table.sq.double().cpu().numpy() - sq) <= U["f32"] * sq + 1e-45)


def test_pack4_of_what_is_not_finite_and_of_nothing():
    import torch
    e = _embed()
    W = torch.randn((70, 70), device="cuda")
    W[3, 40], W[66, 0] = float("inf"), float("nan")
    table = e.pack4(W)
    x = torch.zeros((2, 70), device="cuda"); x[0, 69] = 1
    y = e.scores4(table, x)
    bad = torch.zeros(70, dtype=torch.bool, device="cuda"); bad[[3, 66]] = True
    assert torch.isnan(y[:, bad]).all() and torch.isfinite(y[:, ~bad]).all() and torch.isnan(table.sq[bad]).all()
    empty = e.pack4(W[:0])
    assert e.scores4(empty, x).shape == (2, 0)
    assert e.scores4(e.pack4(W[:5]), x[:0]).shape == (0, 5)


@pytest.mark.parametrize("x_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,N,d", [(1, 1, 1), (1, 64, 32), (1, 65, 100), (2, 3000, 31), (15, 129, 200), (16, 127, 64), (17, 1001, 128), (33, 700, 512),
                                   (64, 512, 100), (65, 333, 960), (130, 200, 48), (5, 140001, 16)])
def test_scores4(n, N, d, x_dtype, out):
    import torch
    g = torch.Generator(device="cuda").manual_seed(n + N + d)
    W = torch.randn((N, d), generator=g, device="cuda")
    x = torch.randn((n, d), generator=g, device="cuda").to(_t(x_dtype))
    c = torch.randn(N, generator=g, device="cuda")
    x, _ = _strided(x, 3, 1)
    e = _embed()
    table = e.pack4(W)
    t, xd, cd = _packed_want(W), x.double().cpu().numpy(), c.double().cpu().numpy()
    y, buf = _strided(torch.zeros((n, N), device="cuda").to(_t(out)), 5, 3)
    e.scores4(table, x, alpha=2.0, beta=-0.5, c=c, out=y)
    want = 2.0 * xd @ t.T - 0.5 * cd
    size = 2.0 * np.abs(xd) @ np.abs(t).T + 0.5 * np.abs(cd)
    # at most d additions in the matrix pipes, which may cut off (2 u each), a rounding per group and piece, scale, alpha and c
    tol = (2 * d + 3 * (d // 32 + 1) + 6) * U["f32"] * size
    _close(y, want, tol, out)
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[3:].view(n, N + 5)[:, :N] = False
    assert (buf[rest] == -77).all()
    plain = e.scores4(table, x, out_dtype=_t(out))
    _close(plain, xd @ t.T, (2 * d + 3 * (d // 32 + 1) + 6) * U["f32"] * (np.abs(xd) @ np.abs(t).T), out)


def test_scores4_takes_all_of_a_float32_and_its_largest_numbers():
    import torch
    e = _embed()
    W = torch.zeros((64, 32), device="cuda"); W[:, 0] = 6.0
    table = e.pack4(W)                                      # scale 1, value 6
    x = torch.zeros((6, 32), device="cuda")
    x[0, 0], x[1, 0], x[2, 0] = 1 + 2.0 ** -23, 3.0e38 / 6, -(1 + 2.0 ** -12 + 2.0 ** -23)
    x[3, 0], x[4, 0], x[5, 0] = float("inf"), float("-inf"), float("nan")
    y = e.scores4(table, x)
    for k in range(3):
        want = 6.0 * float(x[k, 0])
        assert (y[k].double() - want).abs().max() <= 2 * U["f32"] * abs(want)
    assert torch.isinf(y[3]).all() and (y[3] > 0).all() and (y[4] < 0).all() and torch.isnan(y[5]).all()


# ---- adjusted scores ----
def _bits(keep):
    """Boolean masks as int32 words."""
    import torch
    m, N = keep.shape
    pad = np.zeros((m, (N + 31) // 32 * 32), dtype=np.uint64)
    pad[:, :N] = keep
    words = (pad.reshape(m, -1, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32)
    return torch.from_numpy(words.view(np.int32).copy()).cuda()


def _lists(lists):
    import torch
    off = np.zeros(len(lists) + 1, dtype=np.int64)
    off[1:] = np.cumsum([len(x) for x in lists])
    ids = np.concatenate([np.asarray(x, dtype=np.int32) for x in lists] + [np.empty(0, np.int32)])
    return torch.from_numpy(off).cuda(), torch.from_numpy(ids).cuda()


def _adjust_want(scores, bias=None, keep=None, known=None, seen=None, repeat=1.0, presence=0.0, frequency=0.0):
    x = scores.double().cpu().numpy().copy()
    n, N = x.shape
    size = np.abs(x)
    if bias is not None:
        x += bias.double().cpu().numpy()
        size += np.abs(bias.double().cpu().numpy())
    if seen is not None:
        for b in range(n):
            ids = np.asarray(seen[b], dtype=np.int64)
            k = np.bincount(ids[(ids >= 0) & (ids < N)], minlength=N)
            at = k > 0
            with np.errstate(invalid="ignore"):
                x[b, at] = np.where(x[b, at] > 0, x[b, at] / repeat, x[b, at] * repeat) - (presence + frequency * k[at])
            size[b, at] = size[b, at] * max(repeat, 1 / repeat) + abs(presence) + abs(frequency) * k[at]
    if keep is not None:
        x[~keep] = -np.inf
    if known is not None:
        for b in range(n):
            ids = np.asarray(known[b], dtype=np.int64)
            x[b, ids[(ids >= 0) & (ids < N)]] = -np.inf
    return x, size


def _same(got, want, size, dtype):
    got = got.double().cpu().numpy()
    out = np.isneginf(want)
    assert np.array_equal(np.isneginf(got), out)
    tol = 6 * U["f32"] * size[~out]
    assert np.all(np.abs(got[~out] - want[~out]) <= tol + U[dtype] * (np.abs(want[~out]) + tol) + TINY)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,N", [(1, 1), (3, 31), (2, 33), (1, 4096), (5, 4097), (4, 12289), (300, 50), (3, 262147)])
@pytest.mark.parametrize("parts", ["all", "bias", "masks", "known", "seen", "lists"])
def test_adjust(n, N, parts, dtype):
    import torch
    rng = np.random.default_rng(n * N)
    scores = torch.from_numpy(rng.standard_normal((n, N)).astype(np.float32)).cuda().to(_t(dtype))
    kw, want = {}, {}
    if parts in ("all", "bias"):
        kw["bias"] = want["bias"] = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).cuda()
    if parts in ("all", "masks"):
        masks = rng.random((4, N)) < 0.5
        masks[2] = False                                    # a row that nothing is allowed for
        row = rng.integers(-1, 6, n).astype(np.int32)       # some have no mask
        kw["allowed"], kw["mask_row"] = _bits(masks), torch.from_numpy(row).cuda()
        want["keep"] = np.stack([masks[r] if 0 <= r < 4 else np.ones(N, bool) for r in row])
    for name in ("known", "seen"):
        if parts in ("all", "lists", name):
            most = rng.integers(0, 400, n)
            lists = [rng.integers(-3, N + 3, k) for k in most]
            lists[n // 2] = np.empty(0, int)
            if n > 2:
                lists[n - 1] = rng.integers(0, min(N, 7), 5000)
            kw[name], want[name] = _lists(lists), lists
    if "seen" in kw:
        kw.update(repeat=1.3, presence=0.4, frequency=-0.01)
        want.update(repeat=float(np.float32(1.3)), presence=float(np.float32(0.4)), frequency=float(np.float32(-0.01)))
    e = _embed()
    wide, buf = _strided(scores, 3, 1)
    was = buf.clone()
    expect, size = _adjust_want(scores, **want)
    got = e.adjust(wide, **kw)
    _same(got, expect, size, dtype)
    assert torch.equal(buf, was)
    assert e.adjust(wide, out=wide, **kw) is wide           # in place: the same bits, nothing else touched
    assert torch.equal(wide, got)
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[1:].view(n, N + 3)[:, :N] = False
    assert (buf[rest] == -77).all()


def test_adjust_of_what_is_not_finite():
    import torch
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    s = torch.tensor([[nan, inf, -inf, low, 1.0, nan, -2.0, 3.0]], device="cuda")
    e = _embed()
    x = e.adjust(s, known=_lists([[0, 1, 4]]), seen=_lists([[1, 2, 2, 3, 5, 6, 7]]), repeat=2.0, presence=1.0)
    assert torch.isneginf(x[0, [0, 1, 2, 3, 4]]).all() and torch.isnan(x[0, 5]) and x[0, 6] == -5.0 and x[0, 7] == 0.5
    # a row without a single entity left, by a mask shared by all rows
    gone = e.adjust(torch.randn((3, 40), device="cuda"), allowed=torch.zeros((1, 2), dtype=torch.int32, device="cuda"))
    assert torch.isneginf(gone).all()
    # nothing to do: a copy, or nothing at all
    y = torch.randn((2, 9), device="cuda")
    assert torch.equal(e.adjust(y), y) and e.adjust(y, out=y) is y
    assert e.adjust(y[:0]).shape == (0, 9) and e.adjust(y[:, :0].contiguous()).shape == (2, 0)


def test_adjust_with_lists_longer_than_a_row():
    import torch
    rng = np.random.default_rng(8)
    scores = torch.from_numpy(rng.standard_normal((3, 9000)).astype(np.float32)).cuda()
    known = [rng.integers(0, 4000, 30000), [], rng.integers(-5, 9005, 1025)]
    seen = [[], rng.integers(0, 9000, 70001), np.full(65537, 8999)]
    want, size = _adjust_want(scores, known=known, seen=seen, presence=0.25, frequency=2.0 ** -10)
    e = _embed()
    for out in (None, scores):
        _same(e.adjust(scores, known=_lists(known), seen=_lists(seen), presence=0.25, frequency=2.0 ** -10, out=out), want, size, "f32")


def test_adjust_cuts_offsets_off_at_the_lists_end():
    import torch
    e = _embed()
    s = torch.zeros((3, 64), device="cuda")
    ids = torch.arange(10, dtype=torch.int32, device="cuda")
    off = torch.tensor([-5, 4, 2, 1 << 40], dtype=torch.int64, device="cuda")       # lists 0..3, none (it ends before it begins), 2..9
    for kw in ({"known": (off, ids)}, {"seen": (off, ids), "presence": float(2 ** 20)}):
        for out in (None, s.clone()):
            x = e.adjust(s if out is None else out, out=out, **kw) < -1
            assert x[0].nonzero()[:, 0].tolist() == [0, 1, 2, 3] and not x[1].any() and x[2].nonzero()[:, 0].tolist() == list(range(2, 10))


# ---- many shapes ----
@pytest.mark.parametrize("seed", range(10))
def test_seeded_sweep(seed):
    """Random sizes, types, strides and offsets of every operator."""
    import torch
    rng = np.random.default_rng(100 + seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    size = lambda lo, hi: int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))
    kind = lambda: str(rng.choice(["f32", "bf16"]))
    normal = lambda shape, t: torch.randn(shape, generator=g, device="cuda").to(_t(t))
    wide = lambda x: _strided(x, int(rng.integers(0, 9)), int(rng.integers(0, 8)))[0]

    def ids(n, N):
        x = rng.integers(-1, N + 1, n) if rng.random() < 0.5 else np.minimum(N - 1, np.exp(rng.uniform(0, np.log(N + 1), n)).astype(np.int64) - 1)
        return torch.from_numpy(np.repeat(x.astype(np.int32), 3)).cuda()[1::3] if rng.random() < 0.5 else torch.from_numpy(x.astype(np.int32)).cuda()

    for _ in range(12):
        n, N, d, dtype, out = size(1, 3000), size(1, 5000), size(1, 960), kind(), kind()
        print("lookup", seed, n, N, d, dtype, out, flush=True)
        e = _embed(dtype)
        A, B, i, j = wide(normal((N, d), dtype)), wide(normal((7, d), dtype)), ids(n, N), ids(n, 7)
        want, big = _lookup_want(A, i, -2.0, B, j, 0.5)
        _close(e.lookup(A, i, B, j, sa=-2.0, sb=0.5, out=wide(normal((n, d), out))), want, 3 * U["f32"] * big, out)

        n, N, d, dtype, out = size(1, 60000), size(1, 30000), size(1, 300), kind(), kind()
        print("grad", seed, n, N, d, dtype, out, flush=True)
        G, i, before = wide(normal((n, d), dtype)), ids(n, N), normal((N, d), out)
        accumulate = bool(rng.integers(0, 2))
        want, tol = _grad_want(G, i, N, 1.5, before if accumulate else None)
        _close(e.lookup_grad(G, i, out=wide(before.clone()), scale=1.5, accumulate=accumulate), want, tol, out)

        n, N, d, dtype, out = size(1, 300), size(1, 3000), size(1, 400), kind(), kind()
        print("scores", seed, n, N, d, dtype, out, flush=True)
        W, x, c = normal((N, d), "f32"), wide(normal((n, d), dtype)), normal((N,), "f32")
        t, xd, cd = _packed_want(W), x.double().cpu().numpy(), c.double().cpu().numpy()
        f = _embed("f32")
        y = f.scores4(f.pack4(wide(W)), x, alpha=-0.5, beta=3.0, c=c, out=wide(normal((n, N), out)))
        tol = (2 * d + 3 * (d // 32 + 1) + 6) * U["f32"] * (0.5 * np.abs(xd) @ np.abs(t).T + 3.0 * np.abs(cd))
        _close(y, -0.5 * xd @ t.T + 3.0 * cd, tol, out)

        n, N, dtype = size(1, 60), size(1, 20000), kind()
        print("adjust", seed, n, N, dtype, flush=True)
        kw, want = {}, {}
        if rng.random() < 0.5:
            kw["bias"] = want["bias"] = normal((N,), "f32")
        if rng.random() < 0.5:
            keep = rng.random((n, N)) < rng.random()
            kw["allowed"], want["keep"] = _bits(keep), keep
        for name in ("known", "seen"):
            if rng.random() < 0.5:
                lists = [rng.integers(-2, N + 2, rng.integers(0, size(1, 2000) + 1)) for _ in range(n)]
                kw[name], want[name] = _lists(lists), lists
        if "seen" in kw:
            kw.update(repeat=0.75, presence=-0.5, frequency=0.125)
            want.update(repeat=0.75, presence=-0.5, frequency=0.125)
        scores = wide(normal((n, N), dtype))
        expect, big = _adjust_want(scores, **want)
        _same(e.adjust(scores, out=scores if rng.random() < 0.5 else None, **kw), expect, big, dtype)


# ---- together ----
def test_queries_are_answered_from_a_packed_table():
    """pack, look up h + r, score, leave out what the graph holds and what the relation cannot lead to, take the ten best."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(11)
    N, R, d, n, k = 3000, 7, 100, 40, 10
    E, Rv = torch.randn((N, d), generator=g, device="cuda"), 0.3 * torch.randn((R, d), generator=g, device="cuda")
    q = torch.stack([torch.randint(0, m, (n,), generator=g, device="cuda", dtype=torch.int32) for m in (N, R)], 1)
    rng = np.random.default_rng(3)
    keep = rng.random((R, N)) < 0.5
    known = [rng.integers(0, N, rng.integers(0, 60)) for _ in range(n)]
    e = _embed()
    table = e.pack4(E)
    x = e.lookup(E, q[:, 0], Rv, q[:, 1])
    y = e.adjust(e.scores4(table, x, alpha=2.0, beta=-1.0, c=table.sq), allowed=_bits(keep), mask_row=q[:, 1].contiguous(), known=_lists(known))
    top = y.topk(k, dim=1).indices.cpu().numpy()
    W, h, r = _packed_want(E), q[:, 0].cpu().numpy(), q[:, 1].cpu().numpy()
    xd = E.double().cpu().numpy()[h] + Rv.double().cpu().numpy()[r]
    for b in range(n):
        dist = ((xd[b] - W) ** 2).sum(1)
        ok = keep[r[b]].copy()
        ok[known[b]] = False
        assert ok[top[b]].all()
        best = np.sort(dist[ok])[:k]
        # a score is off by the roundings of sums of about 300; the kth best by no more than two of those
        assert np.all(np.abs(np.sort(dist[top[b]]) - best) <= 4 * d * 2 * U["f32"] * 600)
    full = np.isfinite(y.cpu().numpy())
    assert np.array_equal(full.sum(1), [keep[r[b]].sum() - np.unique(known[b][keep[r[b]][known[b]]]).size for b in range(n)])


def test_a_training_step_follows_the_formula():
    """Squared TransE distances of a batch, their gradients, a step of descent on the tables in place: against float64."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    N, R, d, n, rate = 500, 6, 50, 2000, 2.0 ** -6
    E, Rv = torch.randn((N, d), generator=g, device="cuda"), torch.randn((R, d), generator=g, device="cuda")
    t = torch.stack([torch.randint(0, m, (n,), generator=g, device="cuda", dtype=torch.int32) for m in (N, R, N)], 1)
    E0, R0, tn = E.double().cpu().numpy(), Rv.double().cpu().numpy(), t.cpu().numpy()
    e = _embed()
    x = e.lookup(E, t[:, 0], Rv, t[:, 1]) - e.lookup(E, t[:, 2])
    e.lookup_grad(x, t[:, 0], out=E, scale=-2 * rate, accumulate=True)
    e.lookup_grad(x, t[:, 2], out=E, scale=2 * rate, accumulate=True)
    e.lookup_grad(x, t[:, 1], out=Rv, scale=-2 * rate, accumulate=True)
    res = E0[tn[:, 0]] + R0[tn[:, 1]] - E0[tn[:, 2]]
    wE, wR, sE, sR = E0.copy(), R0.copy(), np.abs(E0), np.abs(R0)
    np.add.at(wE, tn[:, 0], -2 * rate * res); np.add.at(wE, tn[:, 2], 2 * rate * res); np.add.at(wR, tn[:, 1], -2 * rate * res)
    size = 2 * rate * (np.abs(E0)[tn[:, 0]] + np.abs(R0)[tn[:, 1]] + np.abs(E0)[tn[:, 2]])
    for s, c in ((sE, 0), (sE, 2), (sR, 1)):
        np.add.at(s, tn[:, c], size)
    times = lambda c, m: np.bincount(tn[:, c], minlength=m)[:, None]
    _close(E, wE, (times(0, N) + times(2, N) + 8) * U["f32"] * sE, "f32")
    _close(Rv, wR, (times(1, R) + 8) * U["f32"] * sR, "f32")


def test_calls_follow_the_current_stream():
    import torch
    e = _embed()
    g = torch.Generator(device="cuda").manual_seed(1)
    E = torch.randn((20000, 64), generator=g, device="cuda")
    ids = torch.randint(0, 20000, (200000,), generator=g, device="cuda", dtype=torch.int32)
    want = e.lookup(E, ids)
    grad = e.lookup_grad(want, ids, N=20000)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in sides * 2:                                     # two streams in turn, each with workspaces of its own
        with torch.cuda.stream(s):
            x = e.lookup(E, ids)
            got.append((x, e.lookup_grad(x, ids, N=20000)))
    torch.cuda.synchronize()
    for x, y in got:
        assert torch.equal(x, want) and torch.equal(y, grad)
    assert torch.equal(e.lookup(E, ids), want)              # and back on the first one


def test_closed_handles_are_used_again():
    import torch
    e = _embed()
    handle, x = e.handle, torch.arange(12.0, device="cuda").view(3, 4)
    with pytest.raises(RuntimeError):
        e.adjust(x, repeat=-1.0)
    e.close(); e.close()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        f = _embed()
        assert f.handle == handle                           # on another stream, without the message of its last failure in the way
        got = f.lookup(x, torch.tensor([2], dtype=torch.int32, device="cuda"))
    side.synchronize()
    assert torch.equal(got, x[2:])
    assert _embed("bf16").handle != handle and _embed(max_d=8).handle != handle
    f.close()


def test_captured_calls_replay():
    """Two graphs of the same calls on one handle, replayed in turn with eager calls and new inputs between."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    N, d, n = 6000, 900, 9000                               # (queries this long need more LDS than a launch gets unasked)
    E = torch.randn((N, d), generator=g, device="cuda")
    e = _embed()
    table = e.pack4(E)

    def step(ids, known):
        x = e.lookup(E, ids)
        y = e.adjust(e.scores4(table, x[:20], alpha=2.0, beta=-1.0, c=table.sq), known=known, seen=known, presence=1.0)
        return x, y, e.lookup_grad(x, ids, N=N), e.lookup_grad(x[:500], ids[:500], N=N)

    inputs = [torch.randint(0, N, (n,), generator=g, device="cuda", dtype=torch.int32) for _ in range(2)]
    known = _lists([[3, 4, 5000 + b] for b in range(20)])
    graphs = []
    for ids in inputs:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(ids, known)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step(ids, known)
        graphs.append((graph, outs))
    for turn in range(4):
        for ids, (graph, outs) in zip(inputs, graphs):
            ids.copy_(torch.randint(0, N, (n,), generator=g, device="cuda", dtype=torch.int32))
            want = step(ids, known)
            for o in outs:
                o.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b), turn


def test_rows_past_two_to_the_31_elements():
    """A table and scores whose last rows lie more than 2^31 elements from the first."""
    import torch
    N, d = 16_800_000, 128                                  # 2,150,400,000 elements
    e = _embed("bf16")
    g = torch.Generator(device="cuda").manual_seed(9)
    A = torch.empty((N, d), dtype=torch.bfloat16, device="cuda")
    A[-300:] = torch.randn((300, d), generator=g, device="cuda").to(torch.bfloat16)
    ids = (N - 1 - torch.randint(0, 300, (6000,), generator=g, device="cuda")).to(torch.int32)
    rows = A[ids.long()]
    assert torch.equal(e.lookup(A, ids), rows)
    before = A[-300:].clone()
    for n in (6000, 200):                                   # with the sort, and without
        A[-300:] = before
        e.lookup_grad(rows[:n], ids[:n], out=A, scale=-0.5, accumulate=True)
        want, tol = _grad_want(rows[:n], ids[:n] - (N - 300), 300, -0.5, before)
        _close(A[-300:], want, tol, "bf16")
    del A, rows
    table = e.pack4(torch.randn((70, 32), generator=g, device="cuda").to(torch.bfloat16))
    wide = torch.empty((3, 1 << 30), device="cuda")         # rows 2^30 elements apart
    x = torch.randn((3, 32), generator=g, device="cuda")
    far = wide[:, :70]
    assert torch.equal(e.scores4(table, x, out=far), e.scores4(table, x))
    known = _lists([[1], [2, 3], [69]])
    want = e.adjust(e.scores4(table, x), known=known, seen=known, presence=1.0)
    assert torch.equal(e.adjust(far, known=known, seen=known, presence=1.0, out=far), want)


# ---- refusals ----
def test_tensors_that_do_not_fit_are_refused():
    import torch
    e = _embed()
    E, ids = torch.randn((10, 8), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    G = torch.randn((4, 8), device="cuda")
    table = e.pack4(E)
    bad = [lambda: e.lookup(E.cpu(), ids), lambda: e.lookup(E.bfloat16(), ids), lambda: e.lookup(E.t(), ids), lambda: e.lookup(E[0], ids),
           lambda: e.lookup(E, ids.long()), lambda: e.lookup(E, ids, E[:, :4], ids), lambda: e.lookup(E, ids, E, ids[:2]),
           lambda: e.lookup(E, ids, E), lambda: e.lookup(E, ids, out=torch.empty((3, 8), device="cuda")),
           lambda: e.lookup(E, ids, out_dtype=torch.float16), lambda: e.lookup(E, ids, out=torch.empty((4, 9), device="cuda")),
           lambda: e.lookup_grad(G, ids[:3], N=5), lambda: e.lookup_grad(G, ids), lambda: e.lookup_grad(G, ids, N=5, accumulate=True),
           lambda: e.lookup_grad(G.half(), ids, N=5), lambda: e.lookup_grad(G[:, :1].expand(4, 8), ids, N=5),
           lambda: e.scores4(table, G[:, :7].contiguous()), lambda: e.scores4(table, G, c=torch.zeros(9, device="cuda")),
           lambda: e.scores4(table, G, out=torch.empty((4, 9), device="cuda")), lambda: e.adjust(G.long()),
           lambda: e.adjust(G, bias=torch.zeros(7, device="cuda")), lambda: e.adjust(G, allowed=torch.zeros((1, 2), dtype=torch.int32, device="cuda")),
           lambda: e.adjust(G, known=(torch.zeros(4, dtype=torch.int64, device="cuda"), ids)),
           lambda: e.adjust(G, known=(torch.zeros(5, dtype=torch.int32, device="cuda"), ids)),
           lambda: e.adjust(G, out=torch.empty((4, 8), dtype=torch.bfloat16, device="cuda"))]
    for k, call in enumerate(bad):
        with pytest.raises((ValueError, KeyError)):
            call()
            pytest.fail(f"call {k} was not refused")
    refused = [lambda: e.lookup(E, ids, out=E[:4]), lambda: e.lookup(E, ids, E, ids, out=E[2:6]), lambda: e.lookup_grad(E[:4], ids, out=E),
               lambda: e.adjust(E[:5], out=E[1:6]), lambda: e.adjust(E, repeat=0.0), lambda: e.adjust(E, repeat=float("inf")),
               lambda: e.adjust(E, presence=float("nan")), lambda: e.adjust(E, mask_row=torch.zeros(10, dtype=torch.int32, device="cuda")),
               lambda: e.adjust(E, allowed=torch.zeros((3, 1), dtype=torch.int32, device="cuda")),
               lambda: _embed(max_d=4).lookup(E, ids), lambda: e.lookup_grad(torch.ones((4, 961), device="cuda"), ids, N=5)]
    for k, call in enumerate(refused):
        with pytest.raises(RuntimeError, match="code -1"):
            call()
            pytest.fail(f"call {k} was not refused")
    assert torch.equal(e.lookup(E, ids), E[ids.long()])     # the handle is as good as before
    e.close()
    with pytest.raises(RuntimeError, match="closed"):
        e.lookup(E, ids)


def test_raw_arguments_out_of_range_are_refused():
    import torch
    import paper_2307_12059_amd as kgc
    e = _embed()
    h = e.handle
    x = torch.zeros(4096, device="cuda")
    p, q, ids = x.data_ptr(), x.data_ptr() + 8192, torch.zeros(64, dtype=torch.int32, device="cuda").data_ptr()
    good = dict(A=p, Na=8, lda=8, ia=ids, sia=1, sa=1.0, B=0, Nb=0, ldb=0, ib=0, sib=0, sb=0.0, n=4, d=8, out=q, ldo=8, t=0)
    assert kgc.kgc_lookup(h, *good.values()) == kgc.KGC_OK
    for k, v in (("A", 0), ("A", p + 2), ("Na", -1), ("Na", 1 << 40), ("lda", -1), ("lda", 1 << 40), ("ia", 0), ("ia", ids + 1), ("sia", -1),
                 ("B", q), ("ib", ids), ("n", -1), ("n", 1 << 40), ("d", 0), ("d", 961), ("out", 0), ("out", q + 1), ("out", p), ("ldo", 7), ("t", 2)):
        assert kgc.kgc_lookup(h, *{**good, **{"Nb": 4, "ldb": 8, "sib": 1} , k: v}.values()) == kgc.KGC_E_INVALID, (k, v)
        assert kgc.kgc_last_error(h)
    assert kgc.kgc_lookup(None, *good.values()) == kgc.KGC_E_INVALID
    size = kgc.kgc_lookup_grad_bytes(20000, 8, 8)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    many = torch.zeros(20000, dtype=torch.int32, device="cuda")
    G = torch.zeros((20000, 8), device="cuda")
    good = dict(G=G.data_ptr(), gt=0, ldg=8, ids=many.data_ptr(), sid=1, n=20000, d=8, scale=1.0, acc=0, dW=p, wt=0, N=8, ldw=8, work=work.data_ptr(), size=size)
    assert kgc.kgc_lookup_grad(h, *good.values()) == kgc.KGC_OK
    for k, v in (("G", 0), ("gt", 3), ("ldg", -1), ("ids", 0), ("sid", -1), ("n", -1), ("d", 0), ("acc", 2), ("dW", 0), ("dW", p + 1), ("wt", -1), ("N", -1),
                 ("ldw", 7), ("work", 0), ("work", work.data_ptr() + 8), ("work", G.data_ptr()), ("size", size - 1)):
        assert kgc.kgc_lookup_grad(h, *{**good, k: v}.values()) == kgc.KGC_E_INVALID, (k, v)
    table = torch.empty(kgc.kgc_table4_bytes(64, 8), dtype=torch.uint8, device="cuda")
    good = dict(W=p, N=64, ldw=8, d=8, t=table.data_ptr(), size=table.numel(), sq=0)
    assert kgc.kgc_pack4(h, *good.values()) == kgc.KGC_OK
    for k, v in (("W", 0), ("N", -1), ("ldw", -1), ("d", 0), ("t", 0), ("t", table.data_ptr() + 4), ("size", table.numel() - 1), ("sq", p), ("sq", 2)):
        assert kgc.kgc_pack4(h, *{**good, k: v}.values()) == kgc.KGC_E_INVALID, (k, v)
    y = torch.zeros((2, 64), device="cuda")
    good = dict(t=table.data_ptr(), N=64, d=8, x=p, xt=0, ldx=8, n=2, alpha=1.0, c=0, beta=0.0, y=y.data_ptr(), yt=0, ldy=64)
    assert kgc.kgc_scores4(h, *good.values()) == kgc.KGC_OK
    for k, v in (("t", 0), ("t", table.data_ptr() + 8), ("N", -1), ("d", 961), ("x", 0), ("xt", 2), ("ldx", -1), ("n", -1), ("n", 1 << 21), ("c", 2), ("y", 0), ("y", p),
                 ("yt", 5), ("ldy", 63)):
        assert kgc.kgc_scores4(h, *{**good, k: v}.values()) == kgc.KGC_E_INVALID, (k, v)

    def adjust(**kw):
        j = kgc.kgc_adjustment(scores=y.data_ptr(), out=y.data_ptr(), n=2, N=64, ld_scores=64, ld_out=64, repeat=1.0)
        for k, v in kw.items():
            setattr(j, k, v)
        return kgc.kgc_adjust(h, j)
    assert adjust() == kgc.KGC_OK
    for kw in (dict(scores=0), dict(out=0), dict(out=y.data_ptr() + 4), dict(n=-1), dict(N=-1), dict(ld_scores=-1), dict(ld_out=63), dict(ld_scores=65), dict(dtype=2), dict(reserved=1),
               dict(allowed=ids, masks=0), dict(allowed=ids, masks=3), dict(mask_row=ids), dict(known_ids=ids), dict(known_count=3), dict(seen_offsets=p, seen_count=4),
               dict(seen_offsets=p + 4), dict(known_offsets=p, known_ids=ids, known_count=-1), dict(repeat=-1.0), dict(frequency=float("inf")), dict(bias=y.data_ptr())):
        assert adjust(**kw) == kgc.KGC_E_INVALID, kw
    assert kgc.load_library().kgc_adjust(h, None) == kgc.KGC_E_INVALID
    assert kgc.kgc_set_stream(None, 0) == kgc.KGC_E_INVALID
    torch.cuda.synchronize()
