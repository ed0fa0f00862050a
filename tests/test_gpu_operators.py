"""The operators around the recurrent layers on the GPU against their
definitions in 64 bits: embedding, residual norm, linear attention.

Tolerances count roundings.  u = 2^-24 is half a step of fp32, H that of the
storage type (bf16: 2^-8).  A sum of fp32 terms whose every term passes d
roundings is off by at most d u times the sum of the terms' sizes, which the
references compute beside the values (`size`); storing the result adds H of
the result.  So each check is |got - ref| <= H |ref| + d u size, element by
element, with d stated where it is used."""
import numpy as np
import pytest

from _gpu_helpers import TOL, announce, normwise

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def td(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype="bf16", scale=1.0):
    return (scale * torch.randn(*shape, generator=g, dtype=torch.float64)).to(td(dtype))


def close(got, ref, size, d, dtype, label, least=1e-30):
    """|got - ref| <= H |ref| + d u size + least"""
    got, ref, size = got.detach().double().cpu(), ref.double(), size.double()
    assert got.shape == ref.shape, (label, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{label}: not finite"
    limit = HALF[dtype] * ref.abs() + d * U * size + least
    worst = float(((got - ref).abs() / limit).max()) if got.numel() else 0.0
    announce(f"{label}: {worst:.3f} of the bound")
    assert worst <= 1.0, f"{label}: {worst} times the bound"


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
EMBED_CASES = [   # N, V, D, dtype, ldo, ids
    (1, 1, 8, "bf16", 0, "uniform"),
    (1, 7, 8, "f32", 16, "padding"),         # nothing but padding
    (15, 4, 24, "bf16", 0, "uniform"),       # less than a run
    (16, 3, 1032, "f32", 0, "one"),          # one run of one row
    (17, 5, 40, "bf16", 48, "one"),          # a row over two runs
    (1000, 3, 72, "bf16", 0, "uniform"),     # long rows over many runs
    (1023, 2048, 64, "f32", 0, "mixed"),     # two digits
    (1025, 2047, 8, "bf16", 0, "mixed"),     # one digit
    (6400, 32000, 1024, "bf16", 0, "zipf"),
    (5000, 300, 136, "f32", 0, "zipf"),
    (8192, 40, 16, "f32", 0, "zipf"),        # the most tokens that are ranked outright
    (8193, 40, 16, "f32", 0, "zipf"),        # the fewest that are not
    (9001, 5000000, 8, "bf16", 0, "mixed"),  # three digits
    (70001, 1000, 24, "bf16", 0, "zipf"),    # a row of some ten thousand tokens
    (300000, 100003, 8, "f32", 0, "mixed"),  # blocks of several tiles
]


def tokens(g, N, V, kind):
    if kind == "padding":
        return torch.full((N,), -1, dtype=torch.int64)
    if kind == "one":
        return torch.full((N,), V - 1, dtype=torch.int64)
    if kind == "zipf":
        ids = torch.exp(torch.rand(N, generator=g) * np.log(V + 1)).long().clamp(1, V) - 1
    else:
        ids = torch.randint(0, V, (N,), generator=g)
    if kind == "mixed":   # tokens outside the table on both sides, also far outside
        bad = torch.tensor([-1, -2 ** 40, V, V + 1, 2 ** 33, 2 ** 62])
        at = torch.rand(N, generator=g) < 0.2
        ids = torch.where(at, bad[torch.randint(0, 6, (N,), generator=g)], ids)
    return ids


def embed_reference(ids, table, dout, scale, V):
    inside = (ids >= 0) & (ids < V)
    at = torch.where(inside, ids, 0)
    out = torch.where(inside[:, None], (np.float32(scale) * table.float()[at]), 0.0).to(table.dtype)
    g = torch.zeros(V, table.shape[1], dtype=torch.float64)
    size = torch.zeros_like(g)
    rows = dout.double()[inside]
    g.index_add_(0, ids[inside], rows)
    size.index_add_(0, ids[inside], rows.abs())
    count = torch.bincount(ids[inside], minlength=V)
    return out, scale * g, scale * size, count


@pytest.mark.parametrize("N,V,D,dtype,ldo,kind", EMBED_CASES)
def test_embedding(N, V, D, dtype, ldo, kind):
    from paper_1907_13257_amd import Embedding
    label = f"embed N{N} V{V} D{D} {dtype} {kind}"
    announce(label)
    g = gen(N + V)
    scale = 1.5
    ids, table, dout = tokens(g, N, V, kind), normal(g, V, D, dtype=dtype), normal(g, N, D, dtype=dtype)
    ld = ldo or D
    E = Embedding(N, V, D, dtype, scale, ldo)
    dev_ids, dev_table = ids.cuda(), table.cuda()
    out = torch.full((N, ld), 7.0, dtype=td(dtype), device="cuda")
    dev_dout = torch.full((N, ld), float("nan"), dtype=td(dtype), device="cuda")
    dev_dout[:, :D] = dout.cuda()
    E.forward(dev_ids, dev_table, out[:, :D])
    ref, grad, size, count = embed_reference(ids, table, dout, scale, V)
    assert torch.equal(out[:, :D].cpu(), ref), label
    assert (out[:, D:] == 7.0).all()
    # overwrite: rows that no token picks become zeros
    dtable = torch.full((V, D), float("nan"), device="cuda")
    E.backward(dev_ids, dev_dout[:, :D], dtable)
    roundings = (count + 4).double()[:, None]   # the additions of a row, then scale, store
    close(dtable, grad, size * roundings, 1, "f32", label)
    assert (dtable[(count == 0).cuda()] == 0).all()
    again = torch.full((V, D), float("nan"), device="cuda")
    E.backward(dev_ids, dev_dout[:, :D], again)
    assert torch.equal(again, dtable), "equal inputs, other bits"
    # accumulate: what was there stays where no token picks, also a NaN
    base = torch.randn(V, D, generator=g)
    base[count == 0] = float("nan")
    acc = base.cuda()
    E.backward(dev_ids, dev_dout[:, :D], acc, accumulate=True)
    met = (count > 0)
    assert torch.equal(acc[~met.cuda()].isnan(), torch.ones_like(acc[~met.cuda()], dtype=torch.bool))
    if met.any():
        close(acc[met.cuda()], (base.double() + grad)[met], (size * roundings + base.abs() * 2)[met], 1, "f32",
              label + " accumulated")


def test_embedding_without_tokens():
    from paper_1907_13257_amd import Embedding
    E = Embedding(0, 9, 16)
    ids = torch.zeros(0, dtype=torch.int64, device="cuda")
    none = torch.zeros(0, 16, dtype=torch.bfloat16, device="cuda")
    E.forward(ids, torch.ones(9, 16, dtype=torch.bfloat16, device="cuda"), none)
    dtable = torch.ones(9, 16, device="cuda")
    E.backward(ids, none, dtable, accumulate=True)
    assert (dtable == 1).all()
    E.backward(ids, none, dtable)
    assert (dtable == 0).all()


def test_embedding_beyond_32_bit_offsets():
    """A table of more than 2^32 elements: its last rows are read and written."""
    from paper_1907_13257_amd import Embedding
    V, D, N = (1 << 22) + 3, 1032, 5
    table = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 2, V - 1, V], device="cuda")
    table[V - 1], table[V - 2], table[0] = 3.0, 2.0, 1.0
    E = Embedding(N, V, D, scale=2.0)
    out = torch.empty(N, D, dtype=torch.bfloat16, device="cuda")
    E.forward(ids, table, out)
    assert out[:, 5].tolist() == [6.0, 2.0, 4.0, 6.0, 0.0]
    del table
    dtable = torch.full((V, D), float("nan"), device="cuda")
    E.backward(ids, out, dtable)
    assert dtable[[0, V - 2, V - 1], 1031].tolist() == [4.0, 8.0, 24.0]
    dtable[[0, V - 2, V - 1]] = 0.0
    assert not dtable.any()


# ---------------------------------------------------------------------------
# residual norm
# ---------------------------------------------------------------------------
NORM_CASES = [   # rows, D, dtype, extra columns between rows, residual, scale of the rows
    (1, 8, "bf16", 0, True, 1.0),
    (3, 8, "f32", 8, True, 1e-4),       # eps counts
    (5, 520, "bf16", 16, True, 1.0),    # one vector past a wave
    (64, 512, "f32", 0, False, 100.0),
    (1025, 72, "bf16", 0, True, 1.0),   # more rows than partial sums
    (5001, 264, "f32", 0, True, 1.0),
    (7, 1024, "bf16", 0, False, 1.0),
    (37, 2048, "bf16", 0, True, 1.0),   # the widest and the narrowest row of a number of waves
    (19, 1024, "f32", 8, False, 1.0),
    (33, 2056, "bf16", 0, True, 1.0),
    (9, 4104, "f32", 0, True, 1.0),
    (21, 8192, "bf16", 8, True, 1.0),
    (4, 16384, "bf16", 0, True, 1.0),
    (3, 16384, "f32", 0, True, 1.0),
]
EPS = 1e-5


def norm_reference(x, res, g, dy, dsum):
    s = x if res is None else (x.float() + res.float()).to(x.dtype)
    S, G, D = s.double(), g.double(), s.shape[1]
    rho = 1 / torch.sqrt((S * S).mean(1, keepdim=True) + EPS)
    y = S * rho * G
    up = dy.double() * G
    mean = (up * S).mean(1, keepdim=True)
    dx = rho * up - S * rho ** 3 * mean
    dx_size = rho * up.abs() + S.abs() * rho ** 3 * (up * S).abs().mean(1, keepdim=True)
    if dsum is not None:
        dx = dx + dsum.double()
        dx_size = dx_size + dsum.double().abs()
    per = dy.double() * S * rho
    return dict(sum=s, y=y, dx=dx, dx_size=dx_size, dg=per.sum(0), dg_size=per.abs().sum(0))


def strided(t, extra, fill=None):
    """t on the GPU in rows `extra` elements further apart."""
    rows, D = t.shape
    buf = torch.full((rows, D + extra), float("nan") if fill is None else fill, dtype=t.dtype, device="cuda")
    buf[:, :D] = t.cuda()
    return buf[:, :D]


# a row's sum has at most 32 terms per thread, then 6 + 16 from the other lanes
# and waves; the mean, the root, its reciprocal and the products add less than 10
NORM_D = 64


@pytest.mark.parametrize("rows,D,dtype,extra,residual,scale", NORM_CASES)
def test_add_norm(rows, D, dtype, extra, residual, scale):
    from paper_1907_13257_amd import AddNorm
    label = f"norm rows{rows} D{D} {dtype} ld+{extra}"
    announce(label)
    r = gen(rows + D)
    x, dy = normal(r, rows, D, dtype=dtype, scale=scale), normal(r, rows, D, dtype=dtype)
    res = normal(r, rows, D, dtype=dtype, scale=scale) if residual else None
    dsum = normal(r, rows, D, dtype=dtype) if residual else None
    g = normal(r, D, dtype=dtype)
    ref = norm_reference(x, res, g, dy, dsum)
    ld = D + extra
    op = AddNorm(rows, D, dtype, EPS, ld, ld, ld)
    dx_, dg = strided(torch.zeros_like(x), extra), torch.full((D,), float("nan"), device="cuda")
    s_, y_ = strided(torch.zeros_like(x), extra, 7.0), strided(torch.zeros_like(x), extra, 7.0)
    X, R, G = strided(x, extra), None if res is None else strided(res, extra), g.cuda()
    op.forward(X, R, G, s_, y_)
    assert torch.equal(s_.cpu(), ref["sum"]), label
    close(y_, ref["y"], ref["y"].abs(), NORM_D, dtype, label + " y")
    if extra:
        assert (y_.as_strided((rows, extra), (ld, 1), D) == 7.0).all()
    DY, DS = strided(dy, extra), None if dsum is None else strided(dsum, extra)
    op.backward(DY, DS, s_, G, dx_, dg)
    close(dx_, ref["dx"], ref["dx_size"], 3 * NORM_D, dtype, label + " dx")
    close(dg, ref["dg"], ref["dg_size"], NORM_D + min(rows, 1024) + rows // 1024 + 8, "f32", label + " dg")
    # adding to dg, and the gradient in place of dsum
    acc = torch.ones(D, device="cuda")
    if DS is not None:
        op.backward(DY, DS, s_, G, DS, acc, accumulate=True)
        assert torch.equal(DS, dx_)
        assert torch.equal(acc, 1 + dg)
    # the sum in the residual's place
    if R is not None:
        op.forward(X, R, G, R, y_)
        assert torch.equal(R, s_)


@pytest.mark.parametrize("rows,D,dtype,extra,residual,scale", NORM_CASES)
def test_add_norm_q8(rows, D, dtype, extra, residual, scale):
    from paper_1907_13257_amd import AddNorm
    label = f"norm 8 bits rows{rows} D{D} {dtype}"
    announce(label)
    r = gen(rows + D + 1)
    x, g = normal(r, rows, D, dtype=dtype, scale=scale), normal(r, D, dtype=dtype)
    res = normal(r, rows, D, dtype=dtype, scale=scale) if residual else None
    if rows > 2:   # a row of zeros
        x[1] = 0
        if res is not None:
            res[1] = 0
    ref = norm_reference(x, res, g, torch.zeros_like(x), None)
    ld = D + extra
    op = AddNorm(rows, D, dtype, EPS, ld, ld)
    s_ = strided(torch.zeros_like(x), extra)
    y8 = torch.zeros(rows, D, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.full((rows,), float("nan"), device="cuda")
    op.forward_q8(strided(x, extra), None if res is None else strided(res, extra), g.cuda(), s_, y8, scales)
    assert torch.equal(s_.cpu(), ref["sum"])
    rowmax = ref["y"].abs().amax(1)
    close(scales, rowmax / 448, rowmax / 448, NORM_D, "f32", label + " scales")
    got = y8.cpu().double() * scales.cpu().double()[:, None]
    # half a step of e4m3 (2^-4 of the value, or half of the smallest step 2^-9), and the fp32 roundings before it
    limit = 2.0 ** -4 * ref["y"].abs() + (rowmax / 448)[:, None] * 2.0 ** -10 + 4 * NORM_D * U * ref["y"].abs()
    assert torch.isfinite(got).all()
    assert ((got - ref["y"]).abs() <= limit).all(), label
    # the largest value of a row is 448 steps
    some = rowmax > 0
    assert (y8.cpu().double().abs().amax(1)[some] == 448).all()
    assert (scales.cpu()[~some] == 0).all() and not y8.cpu().double()[~some].any()


def test_add_norm_no_rows():
    from paper_1907_13257_amd import AddNorm
    op = AddNorm(0, 16)
    e = torch.zeros(0, 16, dtype=torch.bfloat16, device="cuda")
    g, dg = torch.ones(16, dtype=torch.bfloat16, device="cuda"), torch.ones(16, device="cuda")
    op.forward(e, e, g, e, e)
    op.backward(e, None, e, g, e, dg, accumulate=True)
    assert (dg == 1).all()
    op.backward(e, None, e, g, e, dg)
    assert (dg == 0).all()


def test_add_norm_formula_by_differences():
    """The 64-bit gradient the kernels are held to, against differences."""
    r = gen(3)
    x, res, g, dy, ds = (torch.randn(*s, generator=r, dtype=torch.float64) for s in ((4, 16), (4, 16), (16,), (4, 16), (4, 16)))

    def loss(x, g):
        s = x + res
        return float((dy * s * g / torch.sqrt((s * s).mean(1, keepdim=True) + EPS) + ds * s).sum())

    ref = norm_reference(x + res, None, g, dy, ds)
    for name, t in (("dx", x), ("dg", g)):
        d = torch.randn(t.shape, generator=r, dtype=torch.float64)
        e = 1e-6
        got = [loss(x + k * e * d, g) if name == "dx" else loss(x, g + k * e * d) for k in (1, -1)]
        want = float((ref[name] * d).sum())
        # central differences of an O(1) smooth function: e^2 from the cubic term, 2^-53 / e from rounding
        assert abs((got[0] - got[1]) / (2 * e) - want) < 1e-7 * (1 + abs(want))


# ---------------------------------------------------------------------------
# linear attention
# ---------------------------------------------------------------------------
LINATTN_CASES = [   # T, B, N, K, M, dtype, lengths, states, fused
    (1, 1, 1, 8, 8, "bf16", None, False, False),
    (1, 3, 2, 64, 64, "f32", None, True, False),
    (2, 1, 1, 16, 8, "f32", None, True, True),
    (15, 2, 2, 32, 48, "bf16", None, True, False),
    (16, 1, 3, 64, 64, "bf16", None, False, True),
    (63, 2, 1, 40, 72, "bf16", "ragged", True, True),
    (64, 1, 2, 128, 128, "bf16", None, True, False),
    (65, 2, 2, 64, 64, "bf16", "ragged", False, True),
    (129, 1, 2, 128, 64, "f32", "ragged", True, True),
    (100, 3, 2, 24, 136, "f32", None, False, False),
    (200, 1, 1, 256, 256, "bf16", None, True, False),
    (130, 2, 1, 256, 8, "f32", "ragged", True, True),
    (97, 1, 2, 8, 256, "bf16", None, True, True),
    (333, 2, 3, 40, 72, "f32", "ragged", True, False),
    (1000, 1, 2, 64, 64, "bf16", "ragged", True, True),    # few heads, long: split
    (1500, 2, 1, 128, 128, "bf16", None, True, True),
    (2100, 1, 1, 16, 32, "f32", "ragged", True, False),
    (50, 40, 16, 64, 64, "bf16", "ragged", False, True),   # many heads
    # every padded width, in both sizes of a wave's columns, and key and value
    # widths far apart (one launch pads them to the wider)
    (70, 2, 2, 96, 80, "bf16", "ragged", True, False),
    (70, 1, 2, 96, 96, "f32", None, True, True),
    (100, 2, 1, 160, 136, "bf16", None, True, True),
    (50, 1, 2, 160, 160, "f32", "ragged", True, False),
    (66, 1, 1, 192, 24, "bf16", None, True, False),
    (40, 2, 1, 184, 192, "f32", None, False, False),
    (130, 1, 2, 224, 40, "bf16", "ragged", True, True),
    (35, 1, 1, 8, 224, "f32", None, True, False),
    (90, 1, 1, 248, 232, "f32", "ragged", True, True),
    (34, 70, 16, 128, 96, "bf16", "ragged", True, False),
    (20, 70, 16, 96, 112, "f32", None, True, True),
    (17, 70, 16, 24, 32, "bf16", None, False, False),
    (33, 70, 16, 16, 24, "f32", "ragged", True, False),
    (400, 3, 8, 128, 128, "bf16", "ragged", True, True),   # parts joined by their blocks
    (3000, 1, 1, 40, 256, "bf16", None, True, False),      # and by a launch of its own
]


def linattn_case(T, B, N, K, M, dtype, lengths, states, decay=None, seed=0):
    g = gen(seed + T * 7 + K)
    c = dict(q=normal(g, T, B, N * K, dtype=dtype), k=normal(g, T, B, N * K, dtype=dtype),
             v=normal(g, T, B, N * M, dtype=dtype), do=normal(g, T, B, N * M, dtype=dtype))
    if decay is None:
        decay = 1 - torch.exp2(-1 - 8 * torch.rand(N, generator=g))
    c["decay"] = torch.as_tensor(decay, dtype=torch.float32)
    c["lengths"] = None
    if lengths is not None:
        c["lengths"] = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
        c["lengths"][B - 1] = T
    c["S0"] = normal(g, B, N, K, M, dtype="f32", scale=2.0) if states else None
    c["dST"] = normal(g, B, N, K, M, dtype="f32") if states else None
    return c


def linattn_reference(c, T, B, N, K, M, scale):
    """Token by token in 64 bits; with each value the sum of its terms' sizes."""
    lam = c["decay"].double().view(1, N, 1, 1)
    length = torch.full((B,), T) if c["lengths"] is None else c["lengths"].clamp(0, T)
    alive = length.view(B, 1, 1, 1)
    zero = torch.zeros(B, N, K, M, dtype=torch.float64)

    def run(f):
        q, k, v, do = (torch.where((torch.arange(T).view(T, 1) < length)[:, :, None, None],
                                   f(c[n].double()).view(T, B, N, -1), 0.0) for n in ("q", "k", "v", "do"))
        S = zero if c["S0"] is None else f(c["S0"].double())
        G = zero if c["dST"] is None else f(c["dST"].double())
        out = dict(o=torch.zeros(T, B, N, M).double(), dq=torch.zeros(T, B, N, K).double(),
                   dk=torch.zeros(T, B, N, K).double(), dv=torch.zeros(T, B, N, M).double())
        for t in range(T):
            on = alive > t
            S = torch.where(on, lam * S + k[t].unsqueeze(3) * v[t].unsqueeze(2), S)
            out["o"][t] = torch.where(on[..., 0], scale * (q[t].unsqueeze(3) * S).sum(2), 0.0)
            out["dq"][t] = torch.where(on[..., 0], scale * (S * do[t].unsqueeze(2)).sum(3), 0.0)
        out["ST"] = S
        for t in range(T - 1, -1, -1):
            on = alive > t
            Gt = G + scale * q[t].unsqueeze(3) * do[t].unsqueeze(2)
            out["dk"][t] = torch.where(on[..., 0], (Gt * v[t].unsqueeze(2)).sum(3), 0.0)
            out["dv"][t] = torch.where(on[..., 0], (Gt * k[t].unsqueeze(3)).sum(2), 0.0)
            G = torch.where(on, lam * Gt, G)
        out["dS0"] = G
        return {n: x if x.shape[0] == B and x.dim() == 4 and n in ("ST", "dS0") else x.reshape(T, B, -1)
                for n, x in out.items()}

    return run(lambda x: x), run(lambda x: x.abs())


def linattn_roundings(c, T, K, M):
    """Roundings of a term of an fp32 result: the products' sums (K + M and T
    terms one after another), a few factors, and the power of the decay: an
    exponent e is off by |e| u, which changes the power by |e| u of itself
    (2^-160 and smaller powers are zero)."""
    far = min(160.0, T * float((-torch.log2(c["decay"].double())).max()))
    return K + M + T + 16 + 2 * far


# In bf16 storage the matrix products take fp32 factors (states, sums of a
# chunk, decayed rows) as two bf16 parts: what is left out is 2^-16 of a factor,
# 2^-8 of UPLUS u; a term passes two such factors at most
SPLIT = 2 * 2.0 ** -16 / U


def device_buffers(c, T, B, N, K, M, dtype, fused, poison=True):
    """The case on the GPU; with fused, q, k and v (and their gradients) are
    columns of one buffer.  Rows behind a sequence's end hold NaN."""
    d = {n: (None if x is None else x.cuda()) for n, x in c.items()}
    if c["lengths"] is not None and poison:
        dead = (torch.arange(T).view(T, 1) >= c["lengths"].clamp(0, T)).cuda()
        for n in ("q", "k", "v", "do"):
            d[n][dead] = float("nan")

    def three(make):
        if not fused:
            return make(N * K), make(N * K), make(N * M)
        b = make(N * (2 * K + M))
        return b[:, :, :N * K], b[:, :, N * K:2 * N * K], b[:, :, 2 * N * K:]

    q, k, v = three(lambda w: torch.empty(T, B, w, dtype=td(dtype), device="cuda"))
    for to, n in ((q, "q"), (k, "k"), (v, "v")):
        to.copy_(d[n])
    d.update(q=q, k=k, v=v)
    d["dq"], d["dk"], d["dv"] = three(lambda w: torch.full((T, B, w), float("nan"), dtype=td(dtype), device="cuda"))
    d["o"] = torch.full((T, B, N * M), float("nan"), dtype=td(dtype), device="cuda")
    d["ST"], d["dS0"] = (torch.full((B, N, K, M), float("nan"), device="cuda") for _ in range(2))
    return d


def make_linattn(T, B, N, K, M, dtype, fused, scale=None):
    from paper_1907_13257_amd import LinearAttention
    ld = N * (2 * K + M) if fused else 0
    return LinearAttention(T, B, N, K, M, dtype, scale, ldq=ld, ldk=ld, ldv=ld)


def run_linattn(op, d):
    op.forward(d["q"], d["k"], d["v"], d["decay"], d["o"], d["lengths"], d["S0"], d["ST"])
    op.backward(d["do"], d["q"], d["k"], d["v"], d["decay"], d["dq"], d["dk"], d["dv"], d["lengths"], d["S0"], d["dST"],
                d["dS0"])
    return {n: d[n] for n in ("o", "ST", "dq", "dk", "dv", "dS0")}


def check_linattn(got, c, T, B, N, K, M, dtype, scale, label):
    ref, size = linattn_reference(c, T, B, N, K, M, scale)
    r = linattn_roundings(c, T, K, M)
    for n in got:
        state = n in ("ST", "dS0")
        # fp32 states of bf16 rows: three bf16 parts, 2^-24 of a factor left out
        d = r if dtype == "f32" else r + (4 if state else SPLIT)
        close(got[n], ref[n], size[n], d, "f32" if state else dtype, f"{label} {n}")


@pytest.mark.parametrize("T,B,N,K,M,dtype,lengths,states,fused", LINATTN_CASES)
def test_linattn(T, B, N, K, M, dtype, lengths, states, fused):
    label = f"linattn T{T} B{B} N{N} K{K} M{M} {dtype} {lengths} states{int(states)} fused{int(fused)}"
    announce(label)
    c = linattn_case(T, B, N, K, M, dtype, lengths, states)
    op = make_linattn(T, B, N, K, M, dtype, fused)
    d = device_buffers(c, T, B, N, K, M, dtype, fused)
    got = run_linattn(op, d)
    check_linattn(got, c, T, B, N, K, M, dtype, K ** -0.5, label)
    first = {n: x.clone() for n, x in got.items()}
    for x in got.values():
        x.fill_(float("nan"))
    again = run_linattn(op, d)
    for n in first:
        assert torch.equal(again[n], first[n]), f"{label}: {n} in other bits"


@pytest.mark.parametrize("T,B,N,K,M,dtype", [
    (700, 13, 21, 16, 24, "bf16"),    # parts of 8 chunks, 819 of them
    (350, 13, 21, 24, 16, "f32"),
    (1010, 5, 7, 136, 8, "bf16"),     # two blocks to a head's columns
    (505, 7, 5, 8, 144, "f32"),
    (300, 17, 61, 32, 16, "bf16"),    # not split, 1037 heads
])
def test_linattn_blocks_of_many_chunks(T, B, N, K, M, dtype):
    """Long blocks, launched with those that read the same rows beside them,
    their number no multiple of eight; and each gradient by itself, in the same
    bits."""
    label = f"linattn long blocks T{T} B{B} N{N} K{K} M{M} {dtype}"
    announce(label)
    c = linattn_case(T, B, N, K, M, dtype, "ragged", True)
    op = make_linattn(T, B, N, K, M, dtype, True)
    d = device_buffers(c, T, B, N, K, M, dtype, True)
    got = run_linattn(op, d)
    check_linattn(got, c, T, B, N, K, M, dtype, K ** -0.5, label)
    for n in ("dq", "dk", "dv", "dS0"):
        whole = got[n].clone()
        got[n].fill_(float("nan"))
        only = [d[m] if m == n else None for m in ("dq", "dk", "dv", "dS0")]
        op.backward(d["do"], d["q"], d["k"], d["v"], d["decay"], *only[:3], d["lengths"], d["S0"], d["dST"], only[3])
        assert torch.equal(got[n], whole), f"{label}: {n} alone in other bits"


@pytest.mark.parametrize("decay", [1.0, 0.0, 0.5, 1 - 2.0 ** -14, 2.0 ** -40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linattn_decays(decay, dtype):
    """No decay, no memory at all, powers that vanish, and a decay whose log2
    in 32 bits would lose its digits."""
    T, B, N, K, M = 300, 2, 1, 32, 16
    c = linattn_case(T, B, N, K, M, dtype, "ragged", True, decay=[decay])
    if decay == 0.0:
        c["decay"] = torch.tensor([0.0])
    op = make_linattn(T, B, N, K, M, dtype, False)
    got = run_linattn(op, device_buffers(c, T, B, N, K, M, dtype, False))
    ref = dict(c)
    check_linattn(got, ref, T, B, N, K, M, dtype, K ** -0.5, f"decay {decay} {dtype}")


def test_linattn_lengths_out_of_range_and_empty():
    """Lengths below 0 count as 0, above T as T; a batch of nothing."""
    T, B, N, K, M = 20, 4, 2, 16, 24
    c = linattn_case(T, B, N, K, M, "f32", "ragged", True)
    c["lengths"] = torch.tensor([-5, 10 ** 9, 0, 7], dtype=torch.int32)
    op = make_linattn(T, B, N, K, M, "f32", False)
    got = run_linattn(op, device_buffers(c, T, B, N, K, M, "f32", False))
    check_linattn(got, c, T, B, N, K, M, "f32", K ** -0.5, "odd lengths")
    c["lengths"] = torch.zeros(B, dtype=torch.int32)
    got = run_linattn(op, device_buffers(c, T, B, N, K, M, "f32", False))
    assert torch.equal(got["ST"].cpu(), c["S0"]) and torch.equal(got["dS0"].cpu(), c["dST"])
    assert not any(got[n].any() for n in ("o", "dq", "dk", "dv"))


def test_linattn_only_what_is_wanted():
    """Each gradient alone equals the one of the full call; states in place."""
    T, B, N, K, M = 150, 2, 2, 64, 32
    c = linattn_case(T, B, N, K, M, "bf16", "ragged", True)
    op = make_linattn(T, B, N, K, M, "bf16", False)
    d = device_buffers(c, T, B, N, K, M, "bf16", False)
    want = {n: x.clone() for n, x in run_linattn(op, d).items()}
    for n in ("dq", "dk", "dv", "dS0"):
        buf = torch.full_like(want[n], float("nan"))
        args = {m: (buf if m == n else None) for m in ("dq", "dk", "dv", "dS0")}
        op.backward(d["do"], d["q"], d["k"], d["v"], d["decay"], args["dq"], args["dk"], args["dv"], d["lengths"],
                    d["S0"], d["dST"], args["dS0"])
        assert torch.equal(buf, want[n]), n
    S = d["S0"].clone()
    op.forward(d["q"], d["k"], d["v"], d["decay"], d["o"], d["lengths"], S, S)
    assert torch.equal(S, want["ST"]) and torch.equal(d["o"], want["o"])
    G = d["dST"].clone()
    op.backward(d["do"], d["q"], d["k"], d["v"], d["decay"], d["dq"], d["dk"], d["dv"], d["lengths"], d["S0"], G, G)
    assert torch.equal(G, want["dS0"]) and torch.equal(d["dv"], want["dv"])


@pytest.mark.parametrize("B,N,K,M,dtype", [(1, 1, 8, 8, "bf16"), (3, 2, 64, 64, "bf16"), (2, 3, 40, 72, "f32"),
                                           (5, 2, 256, 256, "bf16"), (70, 16, 128, 128, "bf16"), (2, 1, 256, 8, "f32"),
                                           (2, 2, 8, 256, "f32")])
@pytest.mark.parametrize("inplace", [False, True])
def test_linattn_step(B, N, K, M, dtype, inplace):
    """Single tokens, states in a second buffer or in place; a row of length 0
    keeps its state."""
    label = f"step B{B} N{N} K{K} M{M} {dtype}"
    announce(label)
    c = linattn_case(1, B, N, K, M, dtype, "ragged", True)
    if B > 1:
        c["lengths"][0] = 0
    op = make_linattn(1, B, N, K, M, dtype, False)
    d = device_buffers(c, 1, B, N, K, M, dtype, False)
    out = d["S0"] if inplace else d["ST"]
    op.step(d["q"], d["k"], d["v"], d["decay"], d["S0"], out, d["o"], d["lengths"])
    check_linattn(dict(o=d["o"], ST=out), c, 1, B, N, K, M, dtype, K ** -0.5, label)
    if B > 1:
        assert torch.equal(out[0].cpu(), c["S0"][0])


def test_linattn_prompt_then_steps():
    """A prompt's final states, carried by single tokens, give the outputs of
    the whole sequence."""
    T, P, B, N, K, M = 90, 77, 3, 2, 64, 48
    c = linattn_case(T, B, N, K, M, "bf16", None, True)
    d = device_buffers(c, T, B, N, K, M, "bf16", False)
    prompt, step = make_linattn(P, B, N, K, M, "bf16", False), make_linattn(1, B, N, K, M, "bf16", False)
    S = d["S0"]
    prompt.forward(d["q"][:P], d["k"][:P], d["v"][:P], d["decay"], d["o"][:P], S0=S, ST=S)
    for t in range(P, T):
        step.step(d["q"][t], d["k"][t], d["v"][t], d["decay"], S, S, d["o"][t])
    check_linattn(dict(o=d["o"], ST=S), c, T, B, N, K, M, "bf16", K ** -0.5, "prompt and steps")


def test_linattn_gradients_by_differences():
    """The outputs are linear in each of q, k, v and S0, so differences of the
    forward's loss are exact but for rounding."""
    T, B, N, K, M = 70, 2, 2, 16, 24
    c = linattn_case(T, B, N, K, M, "f32", "ragged", True)
    op = make_linattn(T, B, N, K, M, "f32", False)
    d = device_buffers(c, T, B, N, K, M, "f32", False, poison=False)
    got = {n: x.clone() for n, x in run_linattn(op, d).items()}

    def terms(**kw):
        a = {n: kw.get(n, d[n]) for n in ("q", "k", "v", "S0")}
        op.forward(a["q"], a["k"], a["v"], d["decay"], d["o"], d["lengths"], a["S0"], d["ST"])
        parts = [(d["do"].double() * d["o"].double()), (d["dST"].double() * d["ST"].double())]
        return sum(float(p.sum()) for p in parts), sum(float(p.abs().sum()) for p in parts)

    g = gen(5)
    live = torch.arange(T).view(T, 1) < c["lengths"]
    for n, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("S0", "dS0")):
        dirn = torch.randn(c[n].shape, generator=g)
        if n != "S0":
            dirn = torch.where(live[:, :, None], dirn, 0.0)
        up, su = terms(**{n: d[n] + dirn.cuda()})
        down, sd = terms(**{n: d[n] - dirn.cuda()})
        want = float((got[grad].double() * dirn.cuda().double()).sum())
        size = float((got[grad].double() * dirn.cuda().double()).abs().sum())
        # each loss is a sum whose terms pass the forward's roundings, the gradient the backward's
        limit = linattn_roundings(c, T, K, M) * U * (su + sd + size)
        announce(f"differences of {n}: {abs((up - down) / 2 - want):.2e} of {limit:.2e}")
        assert abs((up - down) / 2 - want) <= limit


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linattn_keeps_what_is_not_finite_to_its_head(dtype):
    """A NaN and an infinity in one head of one row leave every other head and
    row as they are, bit for bit, in both directions."""
    T, B, N, K, M = 100, 2, 3, 32, 48
    c = linattn_case(T, B, N, K, M, dtype, None, True)
    op = make_linattn(T, B, N, K, M, dtype, False)
    want = {n: x.clone() for n, x in run_linattn(op, device_buffers(c, T, B, N, K, M, dtype, False)).items()}
    d = device_buffers(c, T, B, N, K, M, dtype, False)
    d["k"][50, 1, 2 * K + 3] = float("nan")
    d["v"][60, 1, 2 * M + 5] = float("inf")
    got = run_linattn(op, d)
    for n, x in got.items():
        if n in ("ST", "dS0"):
            x, w = x.reshape(B * N, -1), want[n].reshape(B * N, -1)
        else:
            x, w = (t.view(T, B * N, -1).transpose(0, 1) for t in (x, want[n]))
        assert torch.equal(x[:B * N - 1], w[:B * N - 1]), n
    assert torch.equal(got["o"][:32, 1], want["o"][:32, 1])   # more than a chunk before it
    assert got["o"][50:, 1, 2 * M:].isnan().any()


def test_linattn_beyond_32_bit_offsets():
    """Rows more than 2^32 elements apart from the first."""
    T, B, N, K, M, ld = 70000, 4, 1, 8, 8, 16384
    from paper_1907_13257_amd import LinearAttention
    buf = torch.zeros(T, B, ld, dtype=torch.bfloat16, device="cuda")
    assert buf.numel() > 1 << 32
    g = gen(1)
    c = linattn_case(200, B, N, K, M, "bf16", None, False, decay=[0.5])
    # nothing but the last 200 tokens
    for n, at in (("q", 0), ("k", 8), ("v", 16)):
        buf[T - 200:, :, at:at + 8] = c[n].cuda()
    op = LinearAttention(T, B, N, K, M, ldq=ld, ldk=ld, ldv=ld, ldo=ld)
    ST = torch.empty(B, N, K, M, device="cuda")
    op.forward(buf[:, :, 0:8], buf[:, :, 8:16], buf[:, :, 16:24], torch.tensor([0.5], device="cuda"), buf[:, :, 24:32],
               ST=ST)
    check_linattn(dict(o=buf[T - 200:, :, 24:32].clone(), ST=ST), c, 200, B, N, K, M, "bf16", K ** -0.5, "far rows")
    assert not buf[:T - 200, :, 24:32].any()


# ---------------------------------------------------------------------------
# streams, graphs, devices
# ---------------------------------------------------------------------------
def everything():
    """One call of every entry point on its own buffers: a function that runs
    them, and its outputs."""
    from paper_1907_13257_amd import AddNorm, Embedding
    g = gen(11)
    T, B, N, K, M, V, D = 70, 2, 2, 32, 32, 50, 64
    c = linattn_case(T, B, N, K, M, "bf16", "ragged", True)
    d = device_buffers(c, T, B, N, K, M, "bf16", False)
    op = make_linattn(T, B, N, K, M, "bf16", False)
    one = make_linattn(1, B, N, K, M, "bf16", False)
    E, norm = Embedding(T * B, V, D, scale=2.0), AddNorm(T * B, D)
    ids, table = torch.randint(-1, V, (T, B), generator=g).cuda(), normal(g, V, D).cuda()
    gain, res = normal(g, D).cuda(), normal(g, T, B, D).cuda()
    x, s, y, dx = (torch.empty(T, B, D, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    y8, scales = torch.empty(T * B, D, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(T * B, device="cuda")
    dg, dtable = torch.empty(D, device="cuda"), torch.empty(V, D, device="cuda")
    S1, o1 = torch.empty_like(d["ST"]), torch.empty(B, N * M, dtype=torch.bfloat16, device="cuda")

    def run():
        E.forward(ids, table, x)
        norm.forward(x, res, gain, s, y)
        norm.forward_q8(x, res, gain, s, y8, scales)
        norm.backward(y, res, s, gain, dx, dg)
        E.backward(ids, dx, dtable)
        E.backward(ids, dx, dtable, accumulate=True)
        run_linattn(op, d)
        one.step(d["q"][0], d["k"][0], d["v"][0], d["decay"], d["S0"], S1, o1, d["lengths"])

    outs = dict(x=x, s=s, y=y, y8=y8.view(torch.uint8), scales=scales, dx=dx, dg=dg, dtable=dtable, S1=S1, o1=o1,
                **{n: d[n] for n in ("o", "ST", "dq", "dk", "dv", "dS0")})
    inputs = dict(ids=ids, table=table, res=res, q=d["q"], do=d["do"], S0=d["S0"])
    return run, outs, inputs


def clear(outs):
    for t in outs.values():
        t.fill_(1)


def test_on_another_stream():
    run, outs, _ = everything()
    run()
    want = {n: t.clone() for n, t in outs.items()}
    clear(outs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    for n in outs:
        assert torch.equal(outs[n].contiguous().view(torch.uint8), want[n].contiguous().view(torch.uint8)), n


def test_captured_and_replayed():
    """Captured once, replayed with other inputs between eager work: every
    replay equals the eager run on the same inputs."""
    run, outs, inputs = everything()
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(4):
        inputs["ids"].copy_(inputs["ids"].roll(3 * k + 1, 0))
        for n in ("table", "res"):
            inputs[n].mul_(-0.5)
        inputs["S0"].add_(1)
        clear(outs)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in outs.items()}
        clear(outs)
        run()
        for n in outs:
            a, b = got[n].view(torch.uint8), outs[n].contiguous().view(torch.uint8)
            assert torch.equal(a, b), (k, n)


def test_two_graphs_and_eager_calls_do_not_share_scratch():
    """Objects own their workspaces: graphs of two objects replayed at the same
    time on two streams give what each gives alone."""
    runs = [everything() for _ in range(2)]
    runs[1][2]["ids"].copy_(runs[1][2]["ids"].flip(0))
    runs[1][2]["S0"].mul_(3)
    want, graphs = [], []
    for run, outs, _ in runs:
        run()
        want.append({n: t.clone() for n, t in outs.items()})
    torch.cuda.synchronize()
    for run, outs, _ in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append(graph)
        clear(outs)
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, graph in zip(streams, graphs):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for (run, outs, _), w in zip(runs, want):
        for n in outs:
            assert torch.equal(outs[n].contiguous().view(torch.uint8), w[n].contiguous().view(torch.uint8)), n


def test_bindings_refuse_wrong_tensors():
    from paper_1907_13257_amd import AddNorm, Embedding
    E, norm = Embedding(6, 10, 16), AddNorm(6, 16)
    op = make_linattn(5, 2, 2, 16, 8, "bf16", False)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    ids = torch.zeros(6, dtype=torch.int64, device="cuda")
    bad = [
        lambda: E.forward(ids.int(), bf(10, 16), bf(6, 16)),             # 32-bit tokens
        lambda: E.forward(ids, bf(9, 16), bf(6, 16)),                    # a shorter table
        lambda: E.forward(ids, bf(10, 16), bf(6, 32)[:, :16]),           # another stride
        lambda: E.forward(ids, bf(10, 16), torch.zeros(6, 16, device="cuda")),
        lambda: E.forward(ids.cpu(), bf(10, 16), bf(6, 16)),
        lambda: E.backward(ids, bf(6, 16), bf(10, 16)),                  # the gradient is fp32
        lambda: norm.forward(bf(6, 16), bf(5, 16), bf(16), bf(6, 16), bf(6, 16)),
        lambda: norm.forward(bf(6, 16), bf(6, 16), bf(8), bf(6, 16), bf(6, 16)),
        lambda: norm.forward(bf(6, 16), None, bf(16), None, None),
        lambda: op.forward(bf(5, 2, 32), bf(5, 2, 32), bf(5, 2, 16), torch.ones(2, device="cuda"), bf(5, 2, 16),
                           lengths=torch.ones(2, dtype=torch.int64, device="cuda")),
        lambda: op.forward(bf(2, 5, 32).transpose(0, 1), bf(5, 2, 32), bf(5, 2, 16), torch.ones(2, device="cuda"),
                           bf(5, 2, 16)),                                # batch-major
        lambda: op.forward(bf(5, 2, 32), bf(5, 2, 32), bf(5, 2, 16), torch.ones(2, device="cuda"), bf(5, 2, 16),
                           S0=torch.zeros(2, 2, 8, 16, device="cuda").transpose(2, 3)),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was accepted")


# ---------------------------------------------------------------------------
# together: tokens -> embedding -> LSTM layers with norms -> linear attention
# ---------------------------------------------------------------------------
def lstm_reference(x, W, R, b):
    """One LSTM layer in 64 bits, gates in the order i, f, g, o."""
    T, B, _ = x.shape
    H = R.shape[1]
    h = c = torch.zeros(B, H, dtype=torch.float64)
    ys = []
    for t in range(T):
        i, f, g, o = (x[t] @ W.t() + h @ R.t() + b).split(H, 1)
        c = torch.sigmoid(f) * c + torch.sigmoid(i) * torch.tanh(g)
        h = torch.sigmoid(o) * torch.tanh(c)
        ys.append(h)
    return torch.stack(ys)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["norms", "mixed"])
def test_stack_with_embedding_and_norms(dtype, layout):
    """Embedding, LSTM layers whose residual sums are normed, and a layer of
    linear attention on top, forward and backward, against the same network in
    64 bits differentiated by torch; the tolerances are the LSTM stack's."""
    from paper_1907_13257_amd import Stack, StackLayer
    T, B, H, V, scale = 12, 5, 64, 37, 3.0
    N, K = 2, 32
    kinds = {"norms": [dict(residual=True, norm=True)] * 3,
             "mixed": [dict(), dict(residual=True, norm=True), dict(residual=True), dict(residual=True, norm=True),
                       dict()]}[layout]
    g = gen(23)
    layers = [StackLayer(H, H, **kw) for kw in kinds]
    params = []
    for kw in kinds:
        p = dict(W=normal(g, 4 * H, H, dtype=dtype, scale=0.1), R=normal(g, 4 * H, H, dtype=dtype, scale=0.1),
                 b=normal(g, 4 * H, dtype="f32", scale=0.1))
        if kw.get("norm"):
            p["g"] = normal(g, H, dtype=dtype, scale=0.3) + 1
        params.append(p)
    table = normal(g, V, H, dtype=dtype, scale=0.3)
    ids = torch.randint(-1, V, (T, B), generator=g)
    dout = normal(g, T, B, H, dtype=dtype)
    decay = torch.tensor([0.9, 0.5])

    # the same network in 64 bits
    leaves = {}

    def leaf(name, t):
        leaves[name] = t.double().requires_grad_(True)
        return leaves[name]

    tab = leaf("table", table)
    x = torch.where((ids >= 0)[:, :, None], scale * tab[ids.clamp(min=0)], 0.0)
    cur = carry = x
    for li, (kw, p) in enumerate(zip(kinds, params)):
        y = lstm_reference(cur, leaf(f"W{li}", p["W"]), leaf(f"R{li}", p["R"]), leaf(f"b{li}", p["b"]))
        if kw.get("residual"):
            y = y + carry
        cur = carry = y
        if kw.get("norm"):
            cur = y / torch.sqrt((y * y).mean(2, keepdim=True) + 1e-5) * leaf(f"g{li}", p["g"])
    S = torch.zeros(B, N, K, K, dtype=torch.float64)
    outs = []
    for t in range(T):
        h = cur[t].view(B, N, K)
        S = decay.double().view(1, N, 1, 1) * S + h.unsqueeze(3) * h.unsqueeze(2)
        outs.append((K ** -0.5 * (h.unsqueeze(3) * S).sum(2)).reshape(B, N * K))
    out = torch.stack(outs)
    out.backward(dout.double())

    stack = Stack(T, B, layers, dtype, vocab=V, embed_scale=scale)
    dev = [[{n: t.cuda() for n, t in p.items()}] for p in params]
    grads, dtable = stack.alloc_grads(dev), torch.full((V, H), float("nan"), device="cuda")
    attn = make_linattn(T, B, N, K, K, dtype, False)
    dev_ids, dec = ids.cuda(), decay.cuda()
    h = stack.forward(dev_ids, dev, table=table.cuda())
    o, dq, dk, dv = (torch.empty(T, B, H, dtype=td(dtype), device="cuda") for _ in range(4))
    attn.forward(h, h, h, dec, o)
    attn.backward(dout.cuda(), h, h, h, dec, dq, dk, dv)
    stack.backward((dq.float() + dk.float() + dv.float()).to(td(dtype)), dev, grads, dtable=dtable)
    assert stack.check() == 0
    errs = {"out": (normwise(o.double().cpu(), out.detach()), "out")}
    errs["table"] = (normwise(dtable.double().cpu(), leaves["table"].grad), "grad")
    for li, gl in enumerate(grads):
        for n, t in gl[0].items():
            errs[f"{n}{li}"] = (normwise(t.double().cpu(), leaves[f"{n[1:]}{li}"].grad), "grad")
    announce(f"stack {layout} {dtype}: " + ", ".join(f"{k}={v:.1e}" for k, (v, _) in errs.items()))
    bad = {k: v for k, (v, kind) in errs.items() if not v <= TOL[dtype][kind]}
    assert not bad, bad
    # gradients of a second mini-batch are added
    before = dtable.clone()
    stack.forward(dev_ids, dev, table=table.cuda())
    stack.backward((dq.float() + dk.float() + dv.float()).to(td(dtype)), dev, grads, accumulate=True, dtable=dtable)
    assert normwise(dtable.double().cpu(), 2 * before.double().cpu()) < 1e-6
