"""The operators around the recurrent layers at the edges of their ranges, on
the GPU: sums whose terms cancel, rows of very small and very large values,
sequences that are split, and the less travelled ways through a stack.

Tolerances are those of test_gpu_operators: half a step of the storage type of
the result, and d half steps of fp32 of the sum of its terms' sizes, d counted
where it is used."""
import numpy as np
import pytest

from _gpu_helpers import announce
from test_gpu_operators import U, close, device_buffers, gen, linattn_case, make_linattn, normal, run_linattn

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
