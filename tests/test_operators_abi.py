"""The operators around the recurrent layers without a GPU: every bad argument
is refused on the host, before any launch, and the sizes of the workspaces."""
import pytest

from paper_1907_13257_amd import StackLayer
from paper_1907_13257_amd import lstm355 as L

A = 1 << 20   # a 16-byte aligned stand-in address; validation fails before any use
BIG = 1 << 60
BAD, OK = L.LSTM_ERR_INVALID_ARG, L.LSTM_OK


@pytest.fixture(scope="module")
def lib():
    return L.load_library()


def changed(args, **kw):
    a = dict(args)
    assert not set(kw) - set(a), kw
    a.update(kw)
    return list(a.values())


EMBED = dict(dtype=1, N=6, V=10, D=16, ids=A, table=A, scale=1.0, out=A, ldo=0, stream=None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(N=-1), dict(N=1 << 31), dict(V=0), dict(V=1 << 31), dict(D=0), dict(D=12), dict(ldo=8),
    dict(ldo=20), dict(ids=None), dict(table=None), dict(out=None), dict(ids=A + 4), dict(table=A + 2), dict(out=A + 2),
])
def test_embed_forward_refuses(lib, kw):
    assert lib.lstm_embed_forward(*changed(EMBED, **kw)) == BAD


EMBED_BWD = dict(dtype=1, N=6, V=10, D=16, ids=A, dout=A, ldo=0, scale=1.0, dtable=A, accumulate=0, ws=A, wb=BIG,
                 stream=None)


@pytest.mark.parametrize("kw", [
    dict(dtype=-1), dict(N=-1), dict(V=0), dict(D=4), dict(ldo=8), dict(accumulate=2), dict(ids=None), dict(dout=None),
    dict(dtable=None), dict(ws=None), dict(ws=A + 4), dict(dtable=A + 4), dict(dout=A + 2), dict(ids=A + 4),
])
def test_embed_backward_refuses(lib, kw):
    assert lib.lstm_embed_backward(*changed(EMBED_BWD, **kw)) == BAD


def test_embed_without_tokens(lib):
    assert lib.lstm_embed_forward(*changed(EMBED, N=0, ids=None, table=None, out=None)) == OK
    assert lib.lstm_embed_backward(*changed(EMBED_BWD, N=0, ids=None, dout=None, dtable=None, accumulate=1, ws=None,
                                            wb=0)) == OK
    assert lib.lstm_embed_backward(*changed(EMBED_BWD, N=0, dtable=None)) == BAD   # there is a gradient to clear


NORM = dict(dtype=1, rows=5, D=16, x=A, ldx=0, res=A, ldr=0, g=A, eps=1e-5, sum=A, y=A, ldy=0, stream=None)
NORM8 = dict(dtype=1, rows=5, D=16, x=A, ldx=0, res=A, ldr=0, g=A, eps=1e-5, sum=A, y8=A, scale=A, stream=None)
NORM_BWD = dict(dtype=1, rows=5, D=16, dy=A, ldy=0, dsum=A, sum=A, ldr=0, g=A, eps=1e-5, dx=2 * A, ldx=0, dg=A,
                accumulate=0, ws=A, wb=BIG, stream=None)
NORM_COMMON = [dict(dtype=7), dict(rows=-1), dict(D=0), dict(D=20), dict(eps=-1.0), dict(eps=float("nan")),
               dict(ldr=12), dict(ldx=8), dict(g=None), dict(g=A + 2), dict(sum=A + 2)]


@pytest.mark.parametrize("kw", NORM_COMMON + [dict(x=None), dict(y=None), dict(sum=None), dict(ldy=8), dict(res=A + 2),
                                              dict(ldx=24)])   # the last: sum in place of an x of another stride
def test_add_norm_refuses(lib, kw):
    assert lib.lstm_add_norm(*changed(NORM, **kw)) == BAD


@pytest.mark.parametrize("kw", NORM_COMMON + [dict(y8=None), dict(scale=None), dict(scale=A + 2), dict(y8=A + 8)])
def test_add_norm_q8_refuses(lib, kw):
    assert lib.lstm_add_norm_q8(*changed(NORM8, **kw)) == BAD


@pytest.mark.parametrize("kw", NORM_COMMON + [
    dict(dy=None), dict(sum=None), dict(dx=None), dict(dg=None), dict(accumulate=3), dict(ws=None), dict(ldy=8),
    dict(dx=A, ldx=24), dict(dx=A, dsum=None, sum=2 * A, ldx=24), dict(dg=A + 8)])
def test_add_norm_backward_refuses(lib, kw):
    assert lib.lstm_add_norm_backward(*changed(NORM_BWD, **kw)) == BAD


def test_add_norm_limits(lib):
    for fn, args in ((lib.lstm_add_norm, NORM), (lib.lstm_add_norm_q8, NORM8),
                     (lib.lstm_add_norm_backward, NORM_BWD)):
        assert fn(*changed(args, D=16384 + 8)) == L.LSTM_ERR_UNSUPPORTED
    assert lib.lstm_add_norm(*changed(NORM, rows=0)) == OK
    assert lib.lstm_add_norm_q8(*changed(NORM8, rows=0)) == OK
    assert lib.lstm_add_norm_backward(*changed(NORM_BWD, rows=0, accumulate=1)) == OK


DESC = dict(T=9, B=2, N=3, K=16, M=24, dtype="bf16", scale=0.25, ldq=0, ldk=0, ldv=0, ldo=0)
BAD_DESC = [dict(T=0), dict(B=0), dict(N=0), dict(K=0), dict(K=12), dict(K=264), dict(M=4), dict(M=264), dict(ldq=40),
            dict(ldq=52), dict(ldk=40), dict(ldv=64), dict(ldo=64), dict(scale=float("nan")), dict(B=1 << 21, N=4),
            dict(T=1 << 20, B=1 << 12)]


def linattn_calls(lib, d, **kw):
    ref = None if d is None else L.ctypes.byref(d)
    p = dict(q=A, k=A, v=A, decay=A, lengths=None, S0=A, o=A, ST=A, d_o=A, dST=A, dq=A, dk=A, dv=A, dS0=A, ws=A, wb=BIG)
    p.update(kw)
    fwd = lib.lstm_linattn_forward(ref, p["q"], p["k"], p["v"], p["decay"], p["lengths"], p["S0"], p["o"], p["ST"],
                                   p["ws"], p["wb"], None)
    bwd = lib.lstm_linattn_backward(ref, p["d_o"], p["q"], p["k"], p["v"], p["decay"], p["lengths"], p["S0"], p["dST"],
                                    p["dq"], p["dk"], p["dv"], p["dS0"], p["ws"], p["wb"], None)
    step = lib.lstm_linattn_step(ref, p["q"], p["k"], p["v"], p["decay"], p["lengths"], p["S0"], p["ST"], p["o"], None)
    return fwd, bwd, step


@pytest.mark.parametrize("kw", BAD_DESC)
def test_linattn_refuses_descriptors(lib, kw):
    d = L.lstm_linattn_desc(**dict(DESC, **kw))
    assert linattn_calls(lib, d) == (BAD, BAD, BAD)
    assert L.lstm_linattn_workspace_size(d) == 0


@pytest.mark.parametrize("kw,calls", [
    (dict(q=None), "fbs"), (dict(k=None), "fbs"), (dict(v=None), "fbs"), (dict(decay=None), "fbs"),
    (dict(q=A + 2), "fbs"), (dict(decay=A + 2), "fbs"), (dict(lengths=A + 2), "fbs"), (dict(o=None), "fs"),
    (dict(S0=A + 4), "fbs"), (dict(ST=A + 8), "fs"), (dict(d_o=None), "b"), (dict(dST=A + 4), "b"),
    (dict(dq=A + 2), "b"), (dict(dk=A + 2), "b"), (dict(dv=A + 2), "b"), (dict(dS0=A + 4), "b"),
])
def test_linattn_refuses_pointers(lib, kw, calls):
    d = L.lstm_linattn_desc(**dict(DESC, T=1))
    got = dict(zip("fbs", linattn_calls(lib, d, **kw)))
    assert all(got[c] == BAD for c in calls), got


def test_linattn_refuses_the_rest(lib):
    assert linattn_calls(lib, None) == (BAD, BAD, BAD)
    d = L.lstm_linattn_desc(**DESC)
    d.dtype = 5
    assert linattn_calls(lib, d) == (BAD, BAD, BAD)
    many = L.lstm_linattn_desc(**DESC)
    assert lib.lstm_linattn_step(L.ctypes.byref(many), A, A, A, A, None, A, A, A, None) == BAD   # nine tokens
    assert "one token" in L.lstm_last_error_detail()


def test_short_workspaces(lib):
    need = L.lstm_embed_workspace_size(6, 10, 16)
    assert need > 0
    assert lib.lstm_embed_backward(*changed(EMBED_BWD, wb=need - 1)) == L.LSTM_ERR_WORKSPACE
    need = L.lstm_add_norm_workspace_size(5, 16)
    assert need > 0
    assert lib.lstm_add_norm_backward(*changed(NORM_BWD, wb=need - 1)) == L.LSTM_ERR_WORKSPACE
    d = L.lstm_linattn_desc(**dict(DESC, T=5000))
    need = L.lstm_linattn_workspace_size(d)
    if need:
        assert linattn_calls(lib, d, wb=need - 1)[:2] == (L.LSTM_ERR_WORKSPACE,) * 2
    # sizes that do not exist have no workspace
    assert L.lstm_embed_workspace_size(6, 10, 12) == 0 and L.lstm_add_norm_workspace_size(5, 20) == 0


def test_bindings_refuse_types(lib):
    with pytest.raises(ValueError):
        L.lstm_linattn_desc(4, 1, 1, 8, 8, dtype="f16")
    with pytest.raises(ValueError):
        StackLayer(16, 16, norm=True)   # a norm without a residual
