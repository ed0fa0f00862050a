"""The operators around the recurrent layers at the edges of their ranges, on
the GPU: sums whose terms cancel, rows of very small and very large values,
sequences that are split, and the less travelled ways through a stack.

Tolerances are those of test_gpu_operators: half a step of the storage type of
the result, and d half steps of fp32 of the sum of its terms' sizes, d counted
where it is used."""
import pytest

from _gpu_helpers import announce
import test_gpu_operators as basic
from test_gpu_operators import (U, check_linattn, close, device_buffers, gen, linattn_case, make_linattn, normal,
                                run_linattn)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# ---------------------------------------------------------------------------
# linear attention in bf16: factors that are fp32 values keep their 24 bits
# ---------------------------------------------------------------------------
def bf16(x):
    return x.to(torch.bfloat16).double()


def cancelling(x):
    """bf16 values c, d with x - c - d of at most 2^-17 of x."""
    c = bf16(x)
    return c, bf16(x - c)


def test_linattn_states_enter_with_all_their_bits():
    """o = q S of two rows that cancel to a few of their last bits: what is left
    shows every bit the product takes of the state."""
    B, N, K, M = 16, 4, 8, 16
    g = gen(41)
    S0 = torch.zeros(B, N, K, M)
    S0[:, :, 2] = 1 + torch.rand(B, N, M, generator=g)
    S0[:, :, 5] = (S0[:, :, 2].double() * (1 + 2.0 ** -13 * torch.rand(B, N, M, generator=g).double())).float()
    q = torch.zeros(1, B, N, K)
    q[..., 2], q[..., 5] = 1, -1
    zero = torch.zeros(1, B, N * M, dtype=torch.bfloat16, device="cuda")
    o, decay = torch.empty_like(zero), torch.ones(N, device="cuda")
    op = make_linattn(1, B, N, K, M, "bf16", False, 1.0)
    op.forward(q.to(torch.bfloat16).reshape(1, B, N * K).cuda(), torch.zeros(1, B, N * K, dtype=torch.bfloat16, device="cuda"),
               zero, decay, o, S0=S0.cuda())
    ref = (S0[:, :, 2].double() - S0[:, :, 5].double()).reshape(1, B, N * M)
    size = (S0[:, :, 2].double() + S0[:, :, 5].double()).reshape(1, B, N * M)
    # each state's three parts and the zeros' sum: six additions at most, and the two factors of 1
    close(o, ref, size, 8, "bf16", "cancelling states")


def test_linattn_sums_of_a_chunk_enter_with_all_their_bits():
    """Token 2 sees tokens 0, 1 and 1's copy with values that cancel all but
    2^-17 of the sum."""
    B, N, K, M = 32, 4, 8, 8
    g = gen(42)
    q, k = torch.zeros(3, B, N, K), torch.zeros(3, B, N, K)
    q[2] = 1 + torch.rand(B, N, K, generator=g)
    k[0], k[1] = 1 + torch.rand(B, N, K, generator=g), 1 + torch.rand(B, N, K, generator=g)
    k[2] = k[1]
    q, k = bf16(q), bf16(k)
    p0, p1 = (q[2] * k[0]).sum(-1), (q[2] * k[1]).sum(-1)
    c, d = cancelling(p0 / p1)
    v = torch.stack([torch.ones_like(c), -c, -d]).unsqueeze(-1).expand(3, B, N, M)
    ref = (p0 - p1 * c - p1 * d).unsqueeze(-1).expand(B, N, M).reshape(B, N * M)
    size = (p0 + p1 * c + p1 * d.abs()).unsqueeze(-1).expand(B, N, M).reshape(B, N * M)
    op = make_linattn(3, B, N, K, M, "bf16", False, 1.0)
    to = lambda t: t.to(torch.bfloat16).reshape(3, B, -1).cuda()   # noqa: E731
    o = torch.empty(3, B, N * M, dtype=torch.bfloat16, device="cuda")
    op.forward(to(q), to(k), to(v), torch.ones(N, device="cuda"), o)
    # a product of K terms, its factor, three tokens of three parts
    close(o[2], ref, size, K + 2 + 9, "bf16", "cancelling sums of a chunk")


@pytest.mark.parametrize("states", [False, True])
def test_linattn_decayed_rows_enter_with_all_their_bits(states):
    """Token 32 sees the state behind the first chunk, to which tokens 0, 1 and
    2 gave values that cancel all but 2^-17; also when no state is given or
    wanted."""
    T, B, N, K, M = 33, 4, 64, 8, 8
    g = gen(43)
    lam = (0.9 + 0.1 * torch.rand(N, generator=g)).float()
    L = lam.double()
    q, k, v = (torch.zeros(T, B, N, K, dtype=torch.float64) for _ in range(3))
    q[T - 1, ..., 3] = 1
    k[:3, ..., 3] = 1
    c = bf16(L)
    d = bf16((L - c) * L)
    v[0], v[1], v[2] = 1.0, -c.view(N, 1), -d.view(N, 1)
    p = [L ** (T - 1 - t) for t in range(3)]
    ref = (p[0] - p[1] * c - p[2] * d).view(1, N, 1).expand(B, N, M).reshape(B, N * M)
    size = (p[0] + p[1] * c + p[2] * d.abs()).view(1, N, 1).expand(B, N, M).reshape(B, N * M)
    op = make_linattn(T, B, N, K, M, "bf16", False, 1.0)
    to = lambda t: t.to(torch.bfloat16).reshape(T, B, -1).cuda()   # noqa: E731
    o = torch.empty(T, B, N * M, dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(B, N, K, M, device="cuda")
    op.forward(to(q), to(k), to(v), lam.cuda(), o, S0=zero if states else None, ST=zero if states else None)
    # powers of the decay of up to 2^-5 (three of them, off by 2 * 5 u each and a step for the
    # exponential), their quotient, three tokens of three parts, the state's factor and the product
    close(o[T - 1], ref, size, 3 * 11 + 2 + 9 + 4, "bf16", f"cancelling rows states{int(states)}")


@pytest.mark.parametrize("T,B,N,K,M", [(100, 2, 3, 64, 64), (700, 2, 2, 128, 72)])
def test_linattn_results_do_not_depend_on_the_states_wanted(T, B, N, K, M):
    """The same rows in the same bits with and without a state in the call."""
    c = linattn_case(T, B, N, K, M, "bf16", "ragged", True)
    c["S0"].zero_()
    c["dST"].zero_()
    op = make_linattn(T, B, N, K, M, "bf16", True)
    d = device_buffers(c, T, B, N, K, M, "bf16", True)
    want = {n: x.clone() for n, x in run_linattn(op, d).items()}
    d.update(S0=None, ST=None, dST=None, dS0=None)
    run_linattn(op, d)
    for n in ("o", "dq", "dk", "dv"):
        assert torch.equal(d[n], want[n]), n


# ---------------------------------------------------------------------------
# residual norm: rows far from 1
# ---------------------------------------------------------------------------
STEPS = 64   # roundings of a row's sum, its root and the products around it (as in test_gpu_operators)


def norm_definition(s, g, eps):
    S, G = s.double(), g.double()
    return S / torch.sqrt((S * S).mean(1, keepdim=True) + eps) * G


def check_q8(y8, scales, y, label):
    """The bytes and scales of rows whose definition is y."""
    top = y.abs().amax(1)
    want = top / 448
    scales, steps = scales.cpu().double(), y8.cpu().double()
    assert torch.isfinite(scales).all() and torch.isfinite(steps).all(), label
    # fp32 roundings, and half of fp32's smallest step where the scale is below the normal numbers
    assert ((scales - want).abs() <= 2 * STEPS * U * want + 2.0 ** -150).all(), (label, scales, want)
    at = y / torch.where(top > 0, want, 1.0)[:, None]
    # half a step of e4m3 (2^-4 of the value, or half of the smallest step 2^-9) and the fp32 roundings before it
    assert ((steps - at).abs() <= (2.0 ** -4 + 4 * STEPS * U) * at.abs() + 2.0 ** -10).all(), label
    announce(f"{label}: scales to {float(((scales - want).abs() / want.clamp(min=1e-300)).max()):.1e}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [16, 520, 2056, 16384])
@pytest.mark.parametrize("residual", [False, True])
def test_add_norm_q8_of_tiny_rows(dtype, D, residual):
    """Largest values of a row around the smallest normal number, and around
    448 over the largest one, where a quotient taken outright overflows; with
    zeros among them, a row of zeros, and an ordinary row."""
    from paper_1907_13257_amd import AddNorm
    tops = [2e-38, 1.3e-37, 1e-36, 1.4e-36, 2e-36, 1e-30, 5e-20, 1e-39, 3e-42, 0.0, 1.0]
    if dtype == "f32":
        tops += [7e-45, 1.5e-45]
    g = gen(D)
    x = (torch.tensor(tops, dtype=torch.float64)[:, None] * (2 * torch.rand(len(tops), D, generator=g) - 1)).to(
        normal(g, 1, dtype=dtype).dtype)
    x[:, 3] = 0
    x[:, 5] = torch.tensor(tops).to(x.dtype)   # the largest of its row
    gain = (0.5 + torch.rand(D, generator=g)).to(x.dtype)
    gain[5] = 2
    rows = len(tops)
    op = AddNorm(rows, D, dtype)
    y8 = torch.zeros(rows, D, dtype=torch.float8_e4m3fn, device="cuda")
    scales, s_ = torch.full((rows,), float("nan"), device="cuda"), torch.empty_like(x).cuda()
    res = torch.zeros_like(x).cuda() if residual else None
    op.forward_q8(x.cuda(), res, gain.cuda(), s_ if residual else None, y8, scales)
    check_q8(y8, scales, norm_definition(x, gain, 1e-5), f"8 bits of tiny rows D{D} {dtype}")
    if residual:
        assert torch.equal(s_.cpu(), x)
        # the sum in the residual's place
        op.forward_q8(x.cuda(), res, gain.cuda(), res, y8, scales)
        check_q8(y8, scales, norm_definition(x, gain, 1e-5), f"8 bits of tiny rows in place D{D} {dtype}")


def test_add_norm_q8_shows_what_is_not_a_number():
    """A NaN among zeros, an infinity, a NaN among ordinary values: the row's
    values by bytes and scale are no numbers, other rows stay as they are."""
    from paper_1907_13257_amd import AddNorm
    D = 72
    x = torch.randn(5, D, generator=gen(9))
    x[1] = 0
    x[1, 7], x[2, 7], x[3, 7] = float("nan"), float("inf"), float("nan")
    gain = torch.ones(D)
    op = AddNorm(5, D, "f32")
    y8, scales = torch.zeros(5, D, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(5, device="cuda")
    op.forward_q8(x.cuda(), None, gain.cuda(), None, y8, scales)
    y = y8.float().cpu() * scales.cpu()[:, None]
    assert y[1].isnan().all() and y[2].isnan().all() and y[3].isnan().all()
    check_q8(y8[::4], scales[::4], norm_definition(x[::4], gain, 1e-5), "rows beside them")


def norm_gradient(s, g, dy, dsum, eps):
    """The definition's gradients in 64 bits and their terms' sizes."""
    S, G, DY = s.double(), g.double(), dy.double()
    root = torch.sqrt((S * S).mean(1, keepdim=True) + eps)
    unit, up = S / root, DY * G
    dx = (up - unit * (up * unit).mean(1, keepdim=True)) / root
    size = (up.abs() + unit.abs() * (up * unit).abs().mean(1, keepdim=True)) / root
    if dsum is not None:
        dx, size = dx + dsum.double(), size + dsum.double().abs()
    return dx, size, (DY * unit).sum(0), (DY * unit).abs().sum(0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 1024, 4104])
@pytest.mark.parametrize("scale,eps", [(1e12, 1e-5), (1e14, 1e-5), (1e17, 1e-5), (1e17, 0.0), (1e-12, 0.0),
                                       (1e-14, 0.0), (1e-16, 0.0), (1e-16, 1e-5)])
def test_add_norm_gradient_of_rows_far_from_one(dtype, D, scale, eps):
    """The norm's projection term counts at every size of a row; dsum at the
    size of the rest, or none."""
    from paper_1907_13257_amd import AddNorm
    g = gen(D)
    rows = 7
    s, dy, gain = normal(g, rows, D, dtype=dtype, scale=scale), normal(g, rows, D, dtype=dtype), normal(g, D, dtype=dtype)
    s[3] = s[3].abs() + scale   # a mean far from zero: dy's projection is large
    dy[3] = gain.sign() * dy[3].abs()
    op = AddNorm(rows, D, dtype, eps)
    for dsum in (None, normal(g, rows, D, dtype=dtype, scale=1 / max(scale, eps ** 0.5))):
        dx, dg = torch.full_like(s, float("nan")).cuda(), torch.full((D,), float("nan"), device="cuda")
        op.backward(dy.cuda(), None if dsum is None else dsum.cuda(), s.cuda(), gain.cuda(), dx, dg)
        rdx, size, rdg, gsize = norm_gradient(s, gain, dy, dsum, eps)
        label = f"norm's gradient at {scale} eps {eps} D{D} {dtype}"
        close(dx, rdx, size, 3 * STEPS, dtype, label + " dx")
        close(dg, rdg, gsize, STEPS + rows + 8, "f32", label + " dg")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [8, 512, 1024, 2048, 4104, 8192, 16384])
@pytest.mark.parametrize("scale,eps", [(1e18, 1e-5), (1e-17, 0.0)])
def test_add_norm_at_the_ends_of_its_range(dtype, D, scale, eps):
    """Rows throughout of the largest and of the smallest stated size, forward,
    to 8 bits and backward."""
    from paper_1907_13257_amd import AddNorm
    g = gen(D + 1)
    rows = 3
    t = normal(g, 1, dtype=dtype).dtype
    size = torch.full((rows, D), scale, dtype=torch.float64)
    size = torch.where(size.to(t).double() > 1e18, torch.nextafter(size.to(t), torch.zeros(1, dtype=t)).double(), size)
    s = (size * torch.where(torch.rand(rows, D, generator=g) < 0.5, -1.0, 1.0)).to(t)
    gain, dy = normal(g, D, dtype=dtype), normal(g, rows, D, dtype=dtype)
    label = f"norm at {scale} D{D} {dtype}"
    op = AddNorm(rows, D, dtype, eps)
    y = torch.empty_like(s).cuda()
    op.forward(s.cuda(), None, gain.cuda(), None, y)
    ref = norm_definition(s, gain, eps)
    close(y, ref, ref.abs(), STEPS, dtype, label + " y")
    y8, scales = torch.zeros(rows, D, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(rows, device="cuda")
    op.forward_q8(s.cuda(), None, gain.cuda(), None, y8, scales)
    check_q8(y8, scales, ref, label + " 8 bits")
    dx, dg = torch.full_like(s, float("nan")).cuda(), torch.full((D,), float("nan"), device="cuda")
    op.backward(dy.cuda(), None, s.cuda(), gain.cuda(), dx, dg)
    rdx, dsize, rdg, gsize = norm_gradient(s, gain, dy, None, eps)
    close(dx, rdx, dsize, 3 * STEPS, dtype, label + " dx")
    close(dg, rdg, gsize, STEPS + rows + 8, "f32", label + " dg")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 3, 512])
def test_linattn_long_memories(N, dtype):
    """Heads that remember 32768 to 65536 tokens: the state of a sequence of
    several times that, forwards and backwards; split into 2048 parts of a few
    chunks, and (many heads) into 4 of thousands."""
    T, K, M, some = 1 << 18, 8, 8, 64
    g = torch.Generator(device="cuda").manual_seed(N)
    lam = (1 - 2.0 ** -16 * (1 + (torch.arange(N) * 37 % 64) / 64)).float()
    t = normal(gen(0), 1, dtype=dtype).dtype
    k, v = ((0.5 + torch.rand(T, 1, N * w, generator=g, device="cuda")).to(t) for w in (K, M))
    L = lam[:some].double().cuda()
    age = torch.arange(T, dtype=torch.float64, device="cuda").flip(0)
    weight = torch.exp(torch.log(L)[:, None] * age)                              # [N][T]
    a, b = (x[:, 0, :some * w].double().view(T, -1, w).permute(1, 0, 2).contiguous() for x, w in ((k, K), (v, M)))
    ref = torch.matmul((a * weight[..., None]).transpose(1, 2).contiguous(), b)  # [N][K][M]
    # backwards the first token's state is decay^(t+1) of token t's product
    back = torch.matmul((a * (weight.flip(1) * L[:, None])[..., None]).transpose(1, 2).contiguous(), b)
    op = make_linattn(T, 1, N, K, M, dtype, False, 1.0)
    o = torch.empty(T, 1, N * M, dtype=t, device="cuda")
    ST, dS0 = (torch.empty(1, N, K, M, device="cuda") for _ in range(2))
    op.forward(k, k, v, lam.cuda(), o, ST=ST)
    op.backward(v, k, k, v, lam.cuda(), None, None, None, dS0=dS0)
    # a state takes three roundings a chunk (16 or 32 tokens) that have no common sign: over the 65536
    # tokens it remembers a walk of 3 * 4096 steps of up to u, 64 u in the mean square; six of them,
    # and the powers' own errors, 20 u
    for got, want, n in ((ST, ref, "ST"), (dS0, back, "dS0")):
        close(got[0, :some], want.cpu(), want.cpu(), 6 * 64 + 20, "f32", f"long memory N{N} {dtype} {n}")


# ---------------------------------------------------------------------------
# linear attention, sequences that are split: the only calls with a workspace
# ---------------------------------------------------------------------------
SPLIT_CASES = [   # T, dtype, parts of a sequence, forward and backward alike
    (320, "bf16", 3),     # joined by their blocks
    (160, "f32", 3),
    (700, "bf16", 6),     # and by a launch of their own
    (350, "f32", 6),
]


class SplitCase:
    """Forward and backward of a split call on its own buffers; the workspace
    says that it is split, and into how many parts."""

    def __init__(self, T, dtype, parts, lengths="ragged", B=3, N=2, K=32, M=40, seed=0):
        self.shape = T, B, N, K, M, dtype
        self.c = linattn_case(T, B, N, K, M, dtype, lengths, True, seed=seed)
        self.d = device_buffers(self.c, T, B, N, K, M, dtype, True, poison=False)
        self.op = make_linattn(T, B, N, K, M, dtype, True)
        assert self.op.ws_bytes == 2 * parts * B * N * K * M * 4

    def run(self):
        return run_linattn(self.op, self.d)

    def check(self, got, label):
        T, B, N, K, M, dtype = self.shape
        check_linattn(got, self.c, T, B, N, K, M, dtype, K ** -0.5, label)

    def outs(self):
        return {n: self.d[n] for n in ("o", "ST", "dq", "dk", "dv", "dS0")}

    def clear(self):
        for t in list(self.outs().values()) + [self.op.workspace]:
            t.fill_(1)


def same(got, want, label=""):
    for n in want:
        assert torch.equal(got[n], want[n]), (label, n)


def copies(tensors):
    return {n: t.clone() for n, t in tensors.items()}


@pytest.mark.parametrize("T,dtype,parts", SPLIT_CASES)
def test_linattn_split_states_in_place(T, dtype, parts):
    """Final states over initial ones, and each gradient alone, in the bits of
    the call with everything apart: the first states are read from the
    workspace, since another block may have replaced them."""
    s = SplitCase(T, dtype, parts)
    d = s.d
    want = copies(s.run())
    s.check(want, f"split T{T} {dtype}")
    for n in ("dq", "dk", "dv", "dS0"):
        s.clear()
        only = [d[m] if m == n else None for m in ("dq", "dk", "dv", "dS0")]
        s.op.backward(d["do"], d["q"], d["k"], d["v"], d["decay"], *only[:3], d["lengths"], d["S0"], d["dST"], only[3])
        assert torch.equal(d[n], want[n]), n
    S, G = d["S0"].clone(), d["dST"].clone()
    s.clear()
    s.op.forward(d["q"], d["k"], d["v"], d["decay"], d["o"], d["lengths"], S, S)
    assert torch.equal(S, want["ST"]) and torch.equal(d["o"], want["o"])
    s.op.backward(d["do"], d["q"], d["k"], d["v"], d["decay"], d["dq"], d["dk"], d["dv"], d["lengths"], d["S0"], G, G)
    same(dict(dq=d["dq"], dk=d["dk"], dv=d["dv"], dS0=G), {n: want[n] for n in ("dq", "dk", "dv", "dS0")})


@pytest.mark.parametrize("T,dtype,parts", SPLIT_CASES)
def test_linattn_split_lengths_at_the_parts_ends(T, dtype, parts):
    """Sequences that end where a part does, one token before and after, in the
    first part, and not at all; rows behind the end hold NaN and get zeros."""
    chunk = 32 if dtype == "bf16" else 16
    part = ((T + chunk - 1) // chunk + parts - 1) // parts * chunk
    lengths = torch.tensor([0, 1, part - 1, part, part + 1, 2 * part, 2 * part + 1, T - 1, T], dtype=torch.int32)
    B, N, K, M = len(lengths), 1, 16, 24
    c = linattn_case(T, B, N, K, M, dtype, "ragged", True)
    c["lengths"] = lengths
    op = make_linattn(T, B, N, K, M, dtype, False)
    assert op.ws_bytes == 2 * parts * B * N * K * M * 4
    op.workspace.fill_(255)   # NaN: nothing is read that was not written
    d = device_buffers(c, T, B, N, K, M, dtype, False)
    check_linattn(run_linattn(op, d), c, T, B, N, K, M, dtype, K ** -0.5, f"ends of parts T{T} {dtype}")
    assert torch.equal(d["ST"][0].cpu(), c["S0"][0]) and torch.equal(d["dS0"][0].cpu(), c["dST"][0])
    for n in ("o", "dq", "dk", "dv"):
        for b in range(B):
            assert not d[n][int(lengths[b]):, b].any(), (n, b)


@pytest.mark.parametrize("T,dtype,parts", SPLIT_CASES)
def test_linattn_split_on_another_stream(T, dtype, parts):
    s = SplitCase(T, dtype, parts)
    want = copies(s.run())
    s.clear()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    same(s.outs(), want)


@pytest.mark.parametrize("T,dtype,parts", SPLIT_CASES)
def test_linattn_split_captured_and_replayed(T, dtype, parts):
    """Captured once, replayed with other inputs and lengths between eager runs."""
    s = SplitCase(T, dtype, parts)
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for k in range(4):
        s.d["q"].mul_(-0.5)
        s.d["S0"].add_(1)
        s.d["lengths"].copy_(s.d["lengths"].roll(1))
        s.clear()
        graph.replay()
        torch.cuda.synchronize()
        got = copies(s.outs())
        s.clear()
        same(got, s.run(), k)


@pytest.mark.parametrize("T,dtype,parts", SPLIT_CASES)
def test_linattn_split_graphs_and_eager_calls_at_once(T, dtype, parts):
    """Two objects' graphs on two streams beside a third's eager calls: each has
    its own workspace, and gives what it gives alone."""
    cases = [SplitCase(T, dtype, parts, seed=k) for k in range(3)]
    want, graphs = [], []
    for s in cases:
        want.append(copies(s.run()))
    torch.cuda.synchronize()
    for s in cases[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run()
        graphs.append(graph)
        s.clear()
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, graph in zip(streams, graphs):
            with torch.cuda.stream(st):
                graph.replay()
        cases[2].run()
    torch.cuda.synchronize()
    for k, s in enumerate(cases):
        same(s.outs(), want[k], k)


@pytest.mark.parametrize("T,dtype,parts", SPLIT_CASES)
def test_linattn_split_prompt_then_steps(T, dtype, parts):
    """A split prompt whose final states replace the first ones, then single
    tokens: the outputs of the whole sequence."""
    B, N, K, M, more = 3, 2, 32, 40, 5
    c = linattn_case(T + more, B, N, K, M, dtype, None, True)
    d = device_buffers(c, T + more, B, N, K, M, dtype, False)
    prompt, step = make_linattn(T, B, N, K, M, dtype, False), make_linattn(1, B, N, K, M, dtype, False)
    assert prompt.ws_bytes == 2 * parts * B * N * K * M * 4
    S = d["S0"]
    prompt.forward(d["q"][:T], d["k"][:T], d["v"][:T], d["decay"], d["o"][:T], S0=S, ST=S)
    for t in range(T, T + more):
        step.step(d["q"][t], d["k"][t], d["v"][t], d["decay"], S, S, d["o"][t])
    check_linattn(dict(o=d["o"], ST=S), c, T + more, B, N, K, M, dtype, K ** -0.5, f"split prompt and steps T{T} {dtype}")


# ---------------------------------------------------------------------------
# embedding: the widest digits of the sort
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("N,V,D,dtype", [
    (9001, 2047, 8, "bf16"),           # one digit of eleven bits: every thread has two counters
    (9001, 2048, 8, "f32"),            # the first rows that need a second digit
    (9001, 1 << 21, 8, "bf16"),        # two digits of eleven bits
    (70001, (1 << 22) - 1, 8, "f32"),  # the last rows that two digits reach
    (9001, 1 << 22, 8, "bf16"),        # and the first that need three
])
def test_embedding_sorted_by_wide_digits(N, V, D, dtype):
    basic.test_embedding(N, V, D, dtype, 0, "mixed")


# ---------------------------------------------------------------------------
# stacks: an embedding below the layer wavefront; norms on other kinds of layers
# ---------------------------------------------------------------------------
def test_embedding_below_a_wavefront_stack():
    """The layer wavefront takes an embedding's rows as it takes any input: the
    same bits as the stack without an embedding on those rows, and the table's
    gradient of its input gradient, over two mini-batches."""
    from paper_1907_13257_amd import Embedding, Stack, StackLayer
    T, B, H, V, scale = 6, 16, 1024, 50, 2.0
    g = gen(51)
    layers = [StackLayer(H, H), StackLayer(H, H, residual=True), StackLayer(H, H, residual=True)]
    params = [[dict(W=normal(g, 4 * H, H, scale=0.05).cuda(), R=normal(g, 4 * H, H, scale=0.05).cuda(),
                    b=normal(g, 4 * H, dtype="f32", scale=0.05).cuda())] for _ in layers]
    table, dout = normal(g, V, H, scale=0.5).cuda(), normal(g, T, B, H).cuda()
    whole, plain = Stack(T, B, layers, vocab=V, embed_scale=scale), Stack(T, B, layers)
    E = Embedding(T * B, V, H, scale=scale)
    rows = torch.empty(T, B, H, dtype=torch.bfloat16, device="cuda")
    grads, want = whole.alloc_grads(params), plain.alloc_grads(params)
    dtable, wtable = (torch.full((V, H), float("nan"), device="cuda") for _ in range(2))
    for k in range(2):
        ids = torch.randint(-1, V, (T, B), generator=g).cuda()
        out = whole.forward(ids, params, table=table)
        dx = whole.backward(dout, params, grads, accumulate=k > 0, dtable=dtable)
        assert whole.last_forward == whole.last_backward == "wavefront"
        E.forward(ids, table, rows)
        assert torch.equal(plain.forward(rows, params), out)
        assert plain.last_forward == "wavefront"
        assert torch.equal(plain.backward(dout, params, want, accumulate=k > 0), dx)
        E.backward(ids, dx, wtable, accumulate=k > 0)
        assert whole.check() == plain.check() == 0
    assert torch.equal(dtable, wtable) and dtable.any()
    for a, b in zip(grads, want):
        for n in a[0]:
            assert torch.equal(a[0][n], b[0][n]), n


def lstm_definition(x, p, reverse):
    """One direction of an LSTM or LSTMP layer in 64 bits, gates in the order i, f, g, o."""
    T, B, _ = x.shape
    H = p["R"].shape[0] // 4
    c = torch.zeros(B, H, dtype=torch.float64)
    h = torch.zeros(B, p["R"].shape[1], dtype=torch.float64)
    ys = [None] * T
    for t in reversed(range(T)) if reverse else range(T):
        i, f, z, o = (x[t] @ p["W"].t() + h @ p["R"].t() + p["b"]).split(H, 1)
        c = torch.sigmoid(f) * c + torch.sigmoid(i) * torch.tanh(z)
        h = torch.sigmoid(o) * torch.tanh(c)
        if "P" in p:
            h = h @ p["P"].t()
        ys[t] = h
    return torch.stack(ys)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norms_on_bidirectional_and_projected_layers(dtype):
    """Norms on a bidirectional layer, a projected one and one that is both,
    with a residual layer without a norm among them; against the same network
    in 64 bits differentiated by torch, with the LSTM stack's tolerances."""
    from _gpu_helpers import TOL, normwise
    from paper_1907_13257_amd import Stack, StackLayer
    T, B, W, V, eps = 9, 5, 64, 31, 1e-3
    kinds = [dict(H=32, bidirectional=True, residual=True, norm=True), dict(H=96, Hp=64, residual=True, norm=True),
             dict(H=64, residual=True), dict(H=48, Hp=32, bidirectional=True, residual=True, norm=True), dict(H=64)]
    g = gen(61)
    layers = [StackLayer(W, **kw) for kw in kinds]
    params = []
    for L in layers:
        dirs = []
        for d in range(2 if L.bidirectional else 1):
            p = dict(W=normal(g, 4 * L.H, W, dtype=dtype, scale=0.1), R=normal(g, 4 * L.H, L.Hr, dtype=dtype, scale=0.1),
                     b=normal(g, 4 * L.H, dtype="f32", scale=0.1))
            if L.Hp:
                p["P"] = normal(g, L.Hp, L.H, dtype=dtype, scale=0.2)
            if L.norm and d == 0:
                p["g"] = normal(g, W, dtype=dtype, scale=0.3) + 1
            dirs.append(p)
        params.append(dirs)
    table, dout = normal(g, V, W, dtype=dtype, scale=0.5), normal(g, T, B, W, dtype=dtype)
    ids = torch.randint(-1, V, (T, B), generator=g)

    leaves = [[{n: t.double().requires_grad_(True) for n, t in p.items()} for p in dirs] for dirs in params]
    tab = table.double().requires_grad_(True)
    cur = carry = torch.where((ids >= 0)[:, :, None], tab[ids.clamp(min=0)], 0.0)
    for L, dirs in zip(layers, leaves):
        y = torch.cat([lstm_definition(cur, p, d == 1) for d, p in enumerate(dirs)], 2)
        y = y + carry if L.residual else y
        cur = carry = y
        if L.norm:
            cur = y / torch.sqrt((y * y).mean(2, keepdim=True) + eps) * dirs[0]["g"]
    cur.backward(dout.double())

    stack = Stack(T, B, layers, dtype, vocab=V, eps=eps)
    dev = [[{n: t.cuda() for n, t in p.items()} for p in dirs] for dirs in params]
    grads, dtable = stack.alloc_grads(dev), torch.full((V, W), float("nan"), device="cuda")
    out = stack.forward(ids.cuda(), dev, table=table.cuda())
    stack.backward(dout.cuda(), dev, grads, dtable=dtable)
    assert stack.check() == 0 and stack.last_forward == "layers"
    errs = {"out": (normwise(out.double().cpu(), cur.detach()), "out"),
            "table": (normwise(dtable.double().cpu(), tab.grad), "grad")}
    for li, dirs in enumerate(grads):
        for d, gd in enumerate(dirs):
            for n, t in gd.items():
                errs[f"{n}{li}.{d}"] = (normwise(t.double().cpu(), leaves[li][d][n[1:]].grad), "grad")
    assert {n for n in errs if n.startswith("dg")} == {"dg0.0", "dg1.0", "dg3.0"}
    announce(f"norms on other layers {dtype}: " + ", ".join(f"{k}={v:.1e}" for k, (v, _) in errs.items()))
    bad = {k: v for k, (v, kind) in errs.items() if not v <= TOL[dtype][kind]}
    assert not bad, bad


@pytest.mark.parametrize("T,B,N,K,M,dtype,lengths,states,fused", [
    (100, 2, 2, 128, 144, "bf16", "ragged", True, True),   # keys of 97 .. 128 with values wider than 128
    (70, 1, 2, 88, 136, "bf16", None, True, False),
    (70, 1, 2, 120, 136, "f32", "ragged", True, False),
    (90, 2, 1, 96, 200, "f32", None, False, True),
    (200, 2, 2, 72, 64, "bf16", "ragged", True, False),    # few heads on both sides of 64 and of 80
    (200, 2, 2, 64, 64, "bf16", "ragged", True, False),
    (100, 2, 2, 80, 64, "f32", "ragged", True, False),
    (100, 2, 2, 64, 88, "f32", "ragged", True, False),
    (100, 2, 2, 128, 128, "f32", "ragged", True, True),
])
def test_linattn_widths_around_the_waves_columns(T, B, N, K, M, dtype, lengths, states, fused):
    basic.test_linattn(T, B, N, K, M, dtype, lengths, states, fused)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linattn_wide_heads_captured(dtype):
    """The widest heads, whose blocks ask for more shared memory than a launch
    has by default: captured as their first call on these sizes, then replayed."""
    T, B, N, K, M = 75, 2, 1, 256, 248
    c = linattn_case(T, B, N, K, M, dtype, "ragged", True)
    d = device_buffers(c, T, B, N, K, M, dtype, False)
    op = make_linattn(T, B, N, K, M, dtype, False)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_linattn(op, d)
    for _ in range(3):
        for n in ("o", "ST", "dq", "dk", "dv", "dS0"):
            d[n].fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        check_linattn({n: d[n] for n in ("o", "ST", "dq", "dk", "dv", "dS0")}, c, T, B, N, K, M, dtype, K ** -0.5,
                      f"captured wide heads {dtype}")


# ---------------------------------------------------------------------------
# strides of their own for every tensor, and every output in an input's place
# that the calls allow
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [72, 2056])
def test_add_norm_strides_and_places(dtype, D):
    from paper_1907_13257_amd import AddNorm
    g = gen(D)
    rows, eps = 9, 1e-5
    x, res, dy, dsum = (normal(g, rows, D, dtype=dtype) for _ in range(4))
    gain = normal(g, D, dtype=dtype)
    dense = AddNorm(rows, D, dtype, eps)
    s, y, dx = (torch.empty_like(x).cuda() for _ in range(3))
    dg = torch.empty(D, device="cuda")
    G = gain.cuda()
    dense.forward(x.cuda(), res.cuda(), G, s, y)
    dense.backward(dy.cuda(), dsum.cuda(), s, G, dx, dg)
    ref = norm_definition(s.cpu(), gain, eps)
    close(y, ref, ref.abs(), STEPS, dtype, f"norm D{D} {dtype}")
    # ldx, ldr and ldy all different; what lies between the rows stays
    op = AddNorm(rows, D, dtype, eps, D + 8, D + 16, D + 40)
    at = lambda t, extra: basic.strided(t, extra, 7.0)   # noqa: E731
    s2, y2, dx2, dg2 = at(x, 16), at(x, 40), at(x, 8), torch.empty(D, device="cuda")
    op.forward(at(x, 8), at(res, 16), G, s2, y2)
    op.backward(at(dy, 40), at(dsum, 16), s2, G, dx2, dg2)
    for got, want, extra in ((s2, s, 16), (y2, y, 40), (dx2, dx, 8)):
        assert torch.equal(got, want)
        between = got.as_strided((rows, extra), (D + extra, 1), D)
        assert (between == 7.0).all()
    assert torch.equal(dg2, dg)
    # the sum in x's place; the gradient in dy's, the sum's and dsum's
    X = x.cuda()
    dense.forward(X, res.cuda(), G, X, y2 := torch.empty_like(X))
    assert torch.equal(X, s) and torch.equal(y2, y)
    for place in ("dy", "dsum", "sum"):
        t = dict(dy=dy.cuda(), dsum=dsum.cuda(), sum=s.clone())
        dense.backward(t["dy"], t["dsum"], t["sum"], G, t[place], dg2)
        assert torch.equal(t[place], dx) and torch.equal(dg2, dg), place


@pytest.mark.parametrize("T,dtype", [(75, "bf16"), (700, "bf16"), (75, "f32")])
def test_linattn_strides(T, dtype):
    """q, k, v and o in rows of four different strides: the dense call's bits,
    and nothing between the rows is touched."""
    from paper_1907_13257_amd import LinearAttention
    B, N, K, M = 2, 3, 24, 40
    c = linattn_case(T, B, N, K, M, dtype, "ragged", True)
    d = device_buffers(c, T, B, N, K, M, dtype, False)
    want = copies(run_linattn(make_linattn(T, B, N, K, M, dtype, False), d))
    extra = dict(q=8, k=24, v=56, o=16)
    ld = {n: N * w + extra[n] for n, w in (("q", K), ("k", K), ("v", M), ("o", M))}
    op = LinearAttention(T, B, N, K, M, dtype, ldq=ld["q"], ldk=ld["k"], ldv=ld["v"], ldo=ld["o"])

    def spread(t, n):
        buf = torch.full((T, B, ld[n]), 7.0, dtype=t.dtype, device="cuda")
        buf[:, :, :t.shape[2]] = t
        return buf[:, :, :t.shape[2]]

    e = dict(d, **{n: spread(d[n], n if n in ld else "o") for n in ("q", "k", "v", "do")})
    for n in ("o", "dq", "dk", "dv"):
        e[n] = spread(torch.zeros_like(d[n]), n[-1])
    e["ST"], e["dS0"] = torch.empty_like(d["ST"]), torch.empty_like(d["dS0"])
    same(run_linattn(op, e), want)
    for n in ("o", "dq", "dk", "dv"):
        assert (e[n].as_strided((T, B, extra[n[-1]]), (B * ld[n[-1]], ld[n[-1]], 1), e[n].shape[2]) == 7.0).all(), n
