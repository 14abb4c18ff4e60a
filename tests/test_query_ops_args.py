"""Refusals of the query-side operators: answered on the host, before anything is enqueued, so they need
no GPU (the addresses below are never read)."""
import ctypes as C

import pytest
import torch

from paper_2601_07183_amd import binding

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -4, -5
P = 1 << 20                                     # an aligned address


def projection(**kw):
    p = binding._Projection(d_in=64, d_out=32, rank=8, n_adapters=3, dtype=0, W=P, A=P, B=P, scale=None)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def table(**kw):
    t = binding._Table(vectors=P, ld=64, V=1000, d=64, dtype=0, scale=1.0, d_live=None, ld_live=0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def project(p, x=P, ldx=64, n=4, ad=P, y=P, ldy=32, yt=0, ws=P, nw=1 << 40):
    lib = binding.load()
    return lib.rairs_project(C.byref(p) if p else None, C.c_void_p(x), C.c_int64(ldx), C.c_int64(n), C.c_void_p(ad), C.c_void_p(y),
                             C.c_int64(ldy), C.c_int(yt), C.c_void_p(ws), C.c_size_t(nw), None)


def project_backward(p, x=P, ldx=64, n=4, ad=P, dy=P, lddy=32, dx=P, lddx=64, da=P, db=P, ws=P, nw=1 << 40):
    lib = binding.load()
    return lib.rairs_project_backward(C.byref(p), C.c_void_p(x), C.c_int64(ldx), C.c_int64(n), C.c_void_p(ad), C.c_void_p(dy),
                                      C.c_int64(lddy), C.c_void_p(dx), C.c_int64(lddx), C.c_void_p(da), C.c_void_p(db), C.c_void_p(ws),
                                      C.c_size_t(nw), None)


def logprob(t, q=P, ldq=64, qt=0, n=4, tg=P, lp=P, lse=P, h=None, top=0, ids=None, tlp=None, ws=P, nw=1 << 40):
    lib = binding.load()
    return lib.rairs_logprob(C.byref(t) if t else None, C.c_void_p(q), C.c_int64(ldq), C.c_int(qt), C.c_int64(n), C.c_void_p(tg),
                             C.c_void_p(lp), C.c_void_p(lse), C.c_void_p(h), C.c_int(top), C.c_void_p(ids), C.c_void_p(tlp),
                             C.c_void_p(ws), C.c_size_t(nw), None)


def logprob_backward(t, q=P, ldq=64, qt=0, n=4, tg=P, lse=P, h=None, da=P, db=None, dq=P, lddq=64, dt=None, lddt=64, ws=P, nw=1 << 40):
    lib = binding.load()
    return lib.rairs_logprob_backward(C.byref(t), C.c_void_p(q), C.c_int64(ldq), C.c_int(qt), C.c_int64(n), C.c_void_p(tg),
                                      C.c_void_p(lse), C.c_void_p(h), C.c_void_p(da), C.c_void_p(db), C.c_void_p(dq), C.c_int64(lddq),
                                      C.c_void_p(dt), C.c_int64(lddt), C.c_void_p(ws), C.c_size_t(nw), None)


def message():
    return binding.load().rairs_last_error().decode()


@pytest.mark.parametrize("change,code,says", [
    (dict(dtype=2), EINVAL, "type"), (dict(d_in=0), EINVAL, "shape"), (dict(d_out=-1), EINVAL, "shape"),
    (dict(d_in=20_000), EUNSUPPORTED, "limit"), (dict(n_adapters=-1), EINVAL, "n_adapters"),
    (dict(n_adapters=5000), EUNSUPPORTED, "n_adapters"), (dict(rank=0), EINVAL, "rank"), (dict(rank=129), EUNSUPPORTED, "rank"),
    (dict(W=None), EINVAL, "W"), (dict(A=None), EINVAL, "A"), (dict(B=None), EINVAL, "B"), (dict(W=P + 2), EINVAL, "aligned"),
])
def test_a_projection_that_cannot_be(change, code, says):
    for call in (project, project_backward):
        assert call(projection(**change)) == code and says in message()
    if not {"W", "A", "B"} & set(change):
        lib = binding.load()
        assert lib.rairs_project_workspace_bytes(C.byref(projection(**change)), C.c_int64(100)) == 0
        assert lib.rairs_project_backward_workspace_bytes(C.byref(projection(**change)), C.c_int64(100)) == 0


@pytest.mark.parametrize("kw,code,says", [
    (dict(n=-1), EINVAL, "negative"), (dict(n=1 << 25), EUNSUPPORTED, "limit"), (dict(x=None), EINVAL, "d_x"), (dict(y=None), EINVAL, "d_y"),
    (dict(ldx=63), EINVAL, "stride"), (dict(ldy=31), EINVAL, "stride"), (dict(x=P + 1), EINVAL, "aligned"), (dict(yt=1), EINVAL, "output type"),
    (dict(n=20, ws=None), EWORKSPACE, "workspace"), (dict(n=20, nw=4), EWORKSPACE, "needed"), (dict(n=20, ws=P + 16), EINVAL, "256-byte"),
    (dict(ldx=1 << 40), EUNSUPPORTED, "stride"),
])
def test_project_refuses(kw, code, says):
    assert project(projection(), **kw) == code and says in message()
    assert project(None) == EINVAL


@pytest.mark.parametrize("kw,code,says", [
    (dict(n=-1), EINVAL, "negative"), (dict(dy=None), EINVAL, "d_dy"), (dict(lddy=1), EINVAL, "stride"), (dict(x=None), EINVAL, "d_x"),
    (dict(lddx=5), EINVAL, "stride"), (dict(da=None), EINVAL, "both"), (dict(db=None), EINVAL, "both"), (dict(db=P + 1), EINVAL, "aligned"),
    (dict(nw=100), EWORKSPACE, "needed"), (dict(ws=None), EWORKSPACE, "NULL"),
])
def test_project_backward_refuses(kw, code, says):
    assert project_backward(projection(), **kw) == code and says in message()
    assert project_backward(projection(n_adapters=0)) == EINVAL and "no adapters" in message()


@pytest.mark.parametrize("change,code,says", [
    (dict(dtype=3), EINVAL, "type"), (dict(dtype=1), EINVAL, "queries of type"), (dict(d=0), EINVAL, "d="), (dict(V=0), EINVAL, "row"),
    (dict(d=20_000, ld=20_000), EUNSUPPORTED, "limit"), (dict(V=1 << 31), EUNSUPPORTED, "V="), (dict(scale=0.0), EINVAL, "scale"),
    (dict(scale=-1.0), EINVAL, "scale"), (dict(scale=float("inf")), EINVAL, "scale"), (dict(scale=1e-31), EINVAL, "scale"), (dict(scale=2e30), EINVAL, "scale"), (dict(scale=float("nan")), EINVAL, "scale"),
    (dict(ld_live=31, d_live=P), EINVAL, "ld_live"), (dict(ld_live=-1), EINVAL, "ld_live"), (dict(ld_live=40), EINVAL, "without a mask"),
    (dict(vectors=None), EINVAL, "vectors"), (dict(ld=63), EINVAL, "stride"),
])
def test_a_table_that_cannot_be(change, code, says):
    for call in (logprob, logprob_backward):
        assert call(table(**change)) == code and says in message()


@pytest.mark.parametrize("kw,code,says", [
    (dict(n=-1), EINVAL, "negative"), (dict(q=None), EINVAL, "d_q"), (dict(ldq=10), EINVAL, "stride"), (dict(tg=None), EINVAL, "null"),
    (dict(lp=None), EINVAL, "null"), (dict(lse=None), EINVAL, "null"), (dict(top=-1), EINVAL, "top"), (dict(top=65), EUNSUPPORTED, "top"),
    (dict(top=3), EINVAL, "room"), (dict(nw=8), EWORKSPACE, "needed"), (dict(ws=P + 8), EINVAL, "256-byte"), (dict(qt=1), EINVAL, "queries"),
])
def test_logprob_refuses(kw, code, says):
    assert logprob(table(), **kw) == code and says in message()
    assert logprob(None) == EINVAL


@pytest.mark.parametrize("kw,code,says", [
    (dict(n=(1 << 20) + 1), EUNSUPPORTED, "gradient"),
    (dict(n=-1), EINVAL, "negative"), (dict(q=None), EINVAL, "d_q"), (dict(tg=None), EINVAL, "null"), (dict(da=None), EINVAL, "null"),
    (dict(lse=None), EINVAL, "null"), (dict(db=P), EINVAL, "d_entropy"), (dict(lddq=1), EINVAL, "stride"), (dict(dt=P, lddt=1), EINVAL, "stride"),
    (dict(nw=8), EWORKSPACE, "needed"),
])
def test_logprob_backward_refuses(kw, code, says):
    assert logprob_backward(table(), **kw) == code and says in message()
    assert logprob_backward(table(dtype=2, ld=64), dt=P) == EINVAL and "bytes has no gradient" in message()


def test_an_empty_batch_is_a_no_op():
    assert project(projection(), x=None, n=0, ad=None, y=None, ws=None, nw=0) == 0
    assert logprob(table(), q=None, n=0, tg=None, lp=None, lse=None, ws=None, nw=0) == 0
    assert logprob_backward(table(), q=None, n=0, tg=None, lse=None, da=None, dq=None, ws=None, nw=0) == 0


def test_workspaces_grow_with_the_batch():
    lib = binding.load()
    p, t = projection(), table()
    sizes = [[lib.rairs_project_workspace_bytes(C.byref(p), C.c_int64(n)) for n in (65, 1000, 5000)],
             [lib.rairs_project_backward_workspace_bytes(C.byref(p), C.c_int64(n)) for n in (1, 65, 1000, 5000)],
             [lib.rairs_logprob_workspace_bytes(C.byref(t), C.c_int64(n), C.c_int(0), C.c_int(10)) for n in (1, 64)],
             [lib.rairs_logprob_workspace_bytes(C.byref(t), C.c_int64(n), C.c_int(0), C.c_int(10)) for n in (65, 500, 5000)]]
    for s in sizes:
        assert all(0 < a < b for a, b in zip(s, s[1:])), s


def test_projected_search_refuses_without_a_handle():
    lib = binding.load()
    assert lib.rairs_search_projected(None, C.byref(projection()), C.c_void_p(P), C.c_int64(64), C.c_int64(1), None, C.c_void_p(P), 1, 1, 1,
                                      C.c_void_p(P), C.c_void_p(P), C.c_void_p(P), C.c_size_t(1 << 30), None) == EINVAL
    assert lib.rairs_index_table(None, None) == EINVAL


def test_the_binding_checks_its_tensors():
    w = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        binding.Projection(w)                                        # not on a device
    with pytest.raises(TypeError):
        binding.Projection(w.to(torch.float16))
    with pytest.raises(ValueError):
        binding.Projection(w, A=torch.zeros(1, 2, 8))
    with pytest.raises(TypeError):
        binding.logprob(torch.zeros(2, 8), torch.zeros(5, 8), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError):
        binding.logprob(torch.zeros(2, 8), torch.zeros(5, 8, dtype=torch.float16), torch.zeros(2, dtype=torch.int64))


class NoDevice:
    """Stands in for a call's device and stream where only the allocation of its results is looked at."""

    def __init__(self, *_):
        pass

    def __enter__(self):
        return C.c_void_p(0)

    def __exit__(self, *_):
        return False


class NoLibrary:
    def __getattr__(self, name):
        return lambda *_: 0


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64, torch.float32])
def test_results_of_logprob_are_fp32_whatever_the_default_type_is(default, monkeypatch):
    # the kernels write four bytes a value
    monkeypatch.setattr(binding, "load", NoLibrary)
    monkeypatch.setattr(binding, "_On", NoDevice)
    monkeypatch.setattr(binding, "_rows", lambda *_: (C.c_void_p(0), C.c_int64(8)))
    monkeypatch.setattr(binding, "_vec", lambda *_: C.c_void_p(0))
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        r = binding.logprob(torch.zeros(3, 8, dtype=torch.float32), torch.zeros(5, 8, dtype=torch.float32), torch.zeros(3, dtype=torch.int64), top=2)
    finally:
        torch.set_default_dtype(before)
    assert [x.dtype for x in r] == [torch.float32] * 3 + [torch.int64, torch.float32]
    assert [tuple(x.shape) for x in r] == [(3,), (3,), (3,), (3, 2), (3, 2)]


def test_a_table_whose_last_tile_does_not_end_within_an_int_is_refused():
    # tiles have up to 256 rows, and a tile's end is compared with V
    lib = binding.load()
    for v, code in ((2 ** 31 - 256, EWORKSPACE), (2 ** 31 - 255, EUNSUPPORTED), (2 ** 31 - 65, EUNSUPPORTED)):
        for call in (logprob, logprob_backward):
            assert call(table(V=v), ws=None) == code, v
        assert (lib.rairs_logprob_workspace_bytes(C.byref(table(V=v)), C.c_int64(4), C.c_int(0), C.c_int(0)) > 0) == (code == EWORKSPACE)


def test_workspaces_do_not_grow_with_the_product_of_batch_and_table():
    # what is held for every pair of a query and a row (or 16 of them) is bounded by parts; what is left are the pieces of
    # the table (6 bytes a value of fp32, 2 of others; backward up to 8 GB at a time), of the queries and of a few gradients
    lib = binding.load()
    GB = 1 << 30
    for dtype, piece in ((0, 6), (1, 2), (2, 2)):
        for v, d in ((1_000_000, 64), (1_000_000, 1024), (100_000, 4096), (20_000_000, 64)):
            t = table(V=v, d=d, ld=d, dtype=dtype)
            qt = 0 if dtype == 2 else dtype
            for n in (1, 16, 65, 10_000, 1 << 20):
                fwd = lib.rairs_logprob_workspace_bytes(C.byref(t), C.c_int64(n), C.c_int(qt), C.c_int(50))
                rows = 6 * n * d if qt == 0 else 2 * n * d
                assert 0 < fwd <= 9 * GB + (piece * v * d if n > 64 else 0) + 2 * rows, (dtype, v, d, n, fwd / GB)
                for grad in (0, 1):
                    if grad and dtype == 2:
                        continue
                    back = lib.rairs_logprob_backward_workspace_bytes(C.byref(t), C.c_int64(n), C.c_int(qt), C.c_int(grad))
                    # sums of dq in at most 8 parts of a large batch, or of a small one for a few thousand workgroups
                    sums = max(8 * 4 * n * d, GB)
                    parts = 16 * n * (v // 256 // 16 + 64) if qt == 0 else 0
                    assert 0 < back <= 17 * GB + 3 * rows + sums + parts, (dtype, v, d, n, grad, back / GB)


def test_workspaces_of_projections_grow_with_the_adapters_that_a_batch_can_have():
    # 300 rows have at most 300 adapters, however many there are
    lib = binding.load()
    for dtype in (0, 1):
        for f in (lib.rairs_project_workspace_bytes, lib.rairs_project_backward_workspace_bytes):
            few, many = (f(C.byref(projection(d_in=1024, d_out=4096, rank=16, n_adapters=na, dtype=dtype)), C.c_int64(300)) for na in (300, 4096))
            assert 0 < few <= many <= few + (1 << 20), (dtype, few, many)
