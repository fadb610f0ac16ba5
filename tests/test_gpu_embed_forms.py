"""The operators on embedding tables form by form: every way that a gradient of a lookup takes, at the borders between them, what holds on all of
them, and what the binding tells torch.  Gradients here are whole numbers whose sums a float32 holds exactly, so that a sum is right or wrong whatever
its order; a bfloat16 result is off by its one rounding."""
import numpy as np
import pytest

from tests.embed_plan import plan
from tests.test_gpu_embed import _adjust_want, _close, _embed, _lists, _same, _strided, _t

pytestmark = pytest.mark.gpu


def _whole(shape, g, dtype="f32"):
    import torch
    return torch.randint(-8, 9, shape, generator=g, device="cuda").to(_t(dtype))


def _sums(G, ids, N, before=None):
    """The sums in float64, and which rows are named."""
    G, ids = G.double().cpu().numpy(), ids.cpu().numpy()
    ok = (ids >= 0) & (ids < N)
    want = np.zeros((N, G.shape[1])) if before is None else before.double().cpu().numpy().copy()
    np.add.at(want, ids[ok], G[ok])
    return want, np.bincount(ids[ok], minlength=N) > 0


def _some_ids(n, N, g):
    """Small numbers most of all, some that name no row, one long run."""
    import torch
    ids = (N ** torch.rand(n, generator=g, device="cuda", dtype=torch.float64)).to(torch.int32) - 1
    ids[torch.rand(n, generator=g, device="cuda") < 0.05] = -7
    ids[:2] = torch.tensor([N - 1, N], dtype=torch.int32)
    ids[n // 2:n // 2 + min(1500, n // 4)] = N // 2
    return ids


# form, and what of it a size is for
FORMS = [(9000, 3000, 300, dict(form="once", vectors=2)), (9000, 3000, 512, dict(form="once", vectors=2)), (60000, 3000, 300, dict(form="sort", vectors=2)),
         (20000, 3000, 200, dict(form="once", vectors=1, lanes=64)), (60000, 900, 256, dict(form="sort", vectors=1, lanes=64)),
         (9001, 2500, 957, dict(form="once", vectors=4)), (60000, 700, 700, dict(form="sort", vectors=4)),
         (600000, 5000, 8, dict(form="sort", chunk=256, tile=4096, scanned=True)), (600000, 5000, 130, dict(form="sort", chunk=256, lanes=64)),
         (530000, 40, 300, dict(form="sort", chunk=256, passes=1)), (300000, 300000, 36, dict(form="sort", passes=2, tile=4096)),
         (200000, 3000, 40, dict(form="sort", tile=1024)), (120000, 500, 80, dict(form="sort", passes=1, tile=1024)),
         (70000, 600000, 5, dict(form="sort", passes=3)), (50000, 3, 257, dict(form="sort", tile=512, passes=1)),
         (300000, 30, 128, dict(form="table", lanes=32)), (100000, 18, 256, dict(form="table", lanes=64)), (50000, 500, 4, dict(form="table", lanes=16)),
         (3500, 4097, 20, dict(form="few", by_row=False)), (3000, 2999, 70, dict(form="few", by_row=True)), (8192, 2048, 300, dict(form="few", by_row=True))]


@pytest.mark.parametrize("n,N,d,what", FORMS)
@pytest.mark.parametrize("g_dtype,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
def test_every_form_of_the_gradient(n, N, d, what, g_dtype, out):
    import torch
    p = plan(n, N, d)
    assert {k: getattr(p, k) for k in what} == what
    g = torch.Generator(device="cuda").manual_seed(n + N + d)
    G, ids = _whole((n, d), g, g_dtype), _some_ids(n, N, g)
    e = _embed()
    _close(e.lookup_grad(G, ids, N=N, out_dtype=_t(out)), _sums(G, ids, N)[0], 0.0, out)
    before = _whole((N, d), g, out)
    want, named = _sums(G, ids, N, before)
    more = before.clone()
    e.lookup_grad(G, ids, out=more, accumulate=True)
    _close(more, want, 0.0, out)
    assert torch.equal(more[torch.from_numpy(~named).cuda()], before[torch.from_numpy(~named).cuda()])


@pytest.mark.parametrize("hub", [0.0, 0.6, 1.0])
def test_gradient_of_millions_of_ids(hub):
    """Joining waves that take several chunks; a sum of thousands of parts among them."""
    import torch
    n, N, d = 4_300_001, 5000, 4
    p = plan(n, N, d)
    assert p.form == "sort" and p.per_wave == 2
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, N, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand(n, generator=g, device="cuda") < hub] = 17
    G = torch.randint(-2, 3, (n, d), generator=g, device="cuda").float()
    _close(_embed().lookup_grad(G, ids, N=N), _sums(G, ids, N)[0], 0.0, "f32")


@pytest.mark.parametrize("n", [3501, 8193, 16384, 16385, 49152, 49153])
@pytest.mark.parametrize("N", [255, 256, 257, 511, 512, 513, 245760, 245761, 262144, 262145])
def test_ids_at_the_borders_of_the_grouping(n, N):
    """Rows too long for the sums in the LDS, so that small tables are grouped too."""
    import torch
    d = 100 if N < 1000 else 2
    p = plan(n, N, d)
    few = n == 3501 and N < 800
    assert p.form == ("few" if few else "once" if n <= (16384 if N < 512 else 49152) and N <= 262144 and not (n > 47104 and N > 245760) else "sort")
    g = torch.Generator(device="cuda").manual_seed(n + N)
    G, ids = _whole((n, d), g), _some_ids(n, N, g)
    e = _embed()
    want = _sums(G, ids, N)[0]
    for step in (1, 3, 4, 5):
        wide = torch.full((n, step), -1, dtype=torch.int32, device="cuda")
        wide[:, step // 2] = ids
        _close(e.lookup_grad(G, wide[:, step // 2], N=N), want, 0.0, "f32")


@pytest.mark.parametrize("n,N,d,form", [(3000, 5000, 33, "few"), (8000, 1500, 33, "few"), (20000, 40, 33, "table"), (5000, 1300, 33, "once"),
                                        (40000, 3000, 130, "once"), (49152, 262144, 7, "sort"), (60000, 3000, 130, "sort"), (300007, 20000, 16, "sort")])
def test_sums_do_not_depend_on_strides(n, N, d, form):
    """The same numbers in other places, or added to zeros: the same bits."""
    import torch
    assert plan(n, N, d).form == form
    g = torch.Generator(device="cuda").manual_seed(n)
    G, ids = torch.randn((n, d), generator=g, device="cuda"), _some_ids(n, N, g)
    e = _embed()
    want = e.lookup_grad(G, ids, N=N)
    for step in (2, 4, 5, 8, 33):
        wide = torch.full((n, step), 3, dtype=torch.int32, device="cuda")
        wide[:, step - 1] = ids
        assert torch.equal(e.lookup_grad(G, wide[:, step - 1], N=N), want), step
    assert torch.equal(e.lookup_grad(_strided(G, 3, 1)[0], ids, N=N), want)
    out, _ = _strided(torch.zeros((N, d), device="cuda"), 5, 2)
    assert torch.equal(e.lookup_grad(G, ids, out=out, accumulate=True), want)


@pytest.mark.parametrize("n,N,d,form", [(200, 900, 20, "few"), (3000, 6000, 20, "few"), (8000, 1000, 3, "few"), (20000, 40, 36, "table"), (50000, 30, 100, "table"),
                                        (5000, 1300, 24, "once"), (60000, 3000, 24, "sort"), (60000, 3000, 2, "sort")])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_rows_that_no_id_names_are_zero_whatever_the_scale(n, N, d, form, out):
    import torch
    assert plan(n, N, d).form == form
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(0, max(1, N // 2), (n,), generator=g, device="cuda", dtype=torch.int32) * 2
    ids[::7] = -1
    G = torch.ones((n, d), device="cuda")
    named = torch.from_numpy(_sums(G, ids, N)[1]).cuda()
    e = _embed()
    for scale in (-1.0, float("inf"), float("nan")):
        for wide in (False, True):
            got, _ = _strided(torch.full((N, d), 5.0, device="cuda").to(_t(out)), 3 if wide else 0, 1)
            e.lookup_grad(G, ids, out=got, scale=scale)
            assert (got[~named] == 0).all() and not torch.signbit(got[~named]).any(), scale
            assert torch.isnan(got[named]).all() if scale != scale else torch.equal(torch.isinf(got[named]).any(), torch.tensor(scale > 1, device="cuda"))


def test_known_answers_of_long_lists_leave_in_place():
    """Lists alone, in place, of which several workgroups take a part each."""
    import torch
    rng = np.random.default_rng(2)
    n, N = 5, 30011
    known = [rng.integers(-3, N + 3, k) for k in (9000, 0, 40000, 3001, 1)]
    assert sum(map(len, known)) // n >= 2 * 1024
    for dtype in ("f32", "bf16"):
        scores = torch.from_numpy(rng.standard_normal((n, N)).astype(np.float32)).cuda().to(_t(dtype))
        want, size = _adjust_want(scores, known=known)
        wide, buf = _strided(scores, 5, 3)
        e = _embed()
        assert e.adjust(wide, known=_lists(known), out=wide) is wide
        _same(wide, want, size, dtype)
        rest = torch.ones_like(buf, dtype=torch.bool)
        rest[3:].view(n, N + 5)[:, :N] = False
        assert (buf[rest] == -77).all()


def test_queries_that_a_group_of_dimensions_can_hold():
    """The 32 products of a group are added before its scale: 32 x 6 x |x| has to stay a float32, however small the scale is."""
    import torch
    W = torch.full((65, 64), 6.0 * 2.0 ** -100, device="cuda")
    e = _embed()
    x = torch.full((1, 64), 1.7e36, device="cuda")
    y = e.scores4(e.pack4(W), x)
    want = 64 * 6.0 * 2.0 ** -100 * float(x[0, 0])
    # 64 additions in the matrix pipes, which may cut off (2 u each), one more for the two groups
    assert torch.isfinite(y).all() and (y.double() - want).abs().max() <= (2 * 64 + 8) * 2.0 ** -24 * want


def test_torch_is_told_of_what_is_written():
    """Outputs that a caller gave count as changed: a gradient that needs their old values is refused."""
    import torch
    e = _embed()
    ids = torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
    table = e.pack4(torch.ones((4, 4), device="cuda"))
    E = torch.ones((3, 4), device="cuda")
    calls = {"lookup": lambda out: e.lookup(E, ids, out=out), "lookup_grad": lambda out: e.lookup_grad(E, ids, out=out),
             "scores4": lambda out: e.scores4(table, E, out=out), "adjust": lambda out: e.adjust(E, out=out)}
    for name, call in calls.items():
        leaf = torch.ones((3, 4), device="cuda", requires_grad=True)
        x = leaf * 2
        y = (x * x).sum()                                   # keeps x
        before = x._version
        call(x.detach())
        assert x._version > before, name
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    with torch.inference_mode():
        x = torch.empty((3, 4), device="cuda")              # (has no count of changes)
        assert torch.equal(e.lookup(E, ids, out=x), E)


def test_a_table_whose_bytes_do_not_fit_its_sizes_is_refused():
    import torch
    import paper_2307_12059_amd as kgc
    e = _embed()
    x = torch.zeros((2, 40), device="cuda")
    t = e.pack4(torch.ones((130, 40), device="cuda"))
    assert torch.equal(e.scores4(kgc.Table4(t.data.clone(), t.N, t.d, None), x), e.scores4(t, x))
    for data, N, d in ((t.data[:-16], 130, 40), (t.data, 193, 40), (t.data, 130, 65), (t.data[:0], 130, 40), (t.data.view(torch.int32), 130, 40),
                       (torch.stack((t.data, t.data), 1)[:, 0], 130, 40), (t.data.cpu(), 130, 40)):
        with pytest.raises(ValueError):
            e.scores4(kgc.Table4(data, N, d, None), torch.zeros((2, d), device="cuda"))


def test_a_join_over_blocks_goes_on_after_operators_and_on_another_stream():
    """They leave what the handle keeps of it, and a join has ended when its call returns."""
    import torch
    import paper_2307_12059_amd as kgc
    import ctypes
    g = torch.Generator(device="cuda").manual_seed(3)
    E, Rv = torch.randn((1500, 16), generator=g, device="cuda"), torch.randn((3, 16), generator=g, device="cuda")
    j = kgc.Join(dtype="f32", prune=kgc.KGC_PRUNE_ON)
    whole = j.join(E, Rv, 2, 3.0, cap=1 << 20)
    assert whole["count"] > 1000
    lib, out, ids = kgc.load_library(), torch.empty((1 << 20, 4), dtype=torch.int32, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda")
    rows = torch.empty((9, 16), device="cuda")
    cursor, seen, streams = kgc.kgc_cursor(), [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    cap = int(whole["count"]) // 3 + 1
    for turn in range(100):
        count = ctypes.c_uint64()
        rc = lib.kgc_join_blocks(j.handle, E.data_ptr(), 1500, 16, Rv.data_ptr(), 3, 2, 3.0, 512, 1, ctypes.byref(cursor), out.data_ptr(), cap, ctypes.byref(count))
        assert rc in (kgc.KGC_OK, kgc.KGC_OVERFLOW) and count.value > 0
        seen.append(out[:count.value, :3].cpu().numpy().copy())
        if rc == kgc.KGC_OK:
            break
        assert kgc.kgc_set_stream(j.handle, streams[turn % 2].cuda_stream) == kgc.KGC_OK
        assert kgc.kgc_lookup(j.handle, E.data_ptr(), 1500, 16, ids.data_ptr(), 1, 1.0, 0, 0, 0, 0, 0, 0.0, 9, 16, rows.data_ptr(), 16, 0) == kgc.KGC_OK
    torch.cuda.synchronize()
    assert turn > 0 and torch.equal(rows, E[:1].expand(9, 16))
    got = np.concatenate(seen)
    assert len(np.unique(got, axis=0)) == len(got) == whole["count"]
