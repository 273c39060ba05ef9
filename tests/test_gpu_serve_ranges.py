"""Linear attention and 8-bit products where lengths, decays and scales are at
the ends of their ranges, on the GPU, against 64-bit implementations."""
import pytest

import serve_reference as ref
from paper_2606_09905_amd import qx

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [BF16, F16, F32]


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


# ---------------------------------------------------------------------------
# rows behind the end
# ---------------------------------------------------------------------------
def _dirty(*sizes):
    """Blocks of these many bytes, full of NaN, back with the allocator."""
    torch.cuda.synchronize()
    blocks = [torch.full((n // 4 + 1,), float("nan"), device="cuda") for n in sizes for _ in range(4)]
    del blocks


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("L", [40, 600])        # one segment, and several
@pytest.mark.parametrize("side", [False, True])
def test_rows_behind_the_end_of_a_result_made_by_the_call_are_zeros(dtype, L, side):
    B, H, d = 4, 2, 64
    g = gen(L)
    q, k, v, do = (normal(g, B, H, L, d, dtype=dtype) for _ in range(4))
    ld = torch.tensor([-0.1, -0.01], device="cuda")
    n = [L, 0, 1, L - 3]
    lens = torch.tensor(n, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream() if side else None
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        _dirty(B * H * L * d * q.element_size(), B * H * d * d * 4)
    out, _ = qx.lin_attn(q, k, v, ld, lens=lens, stream=stream)
    with torch.cuda.stream(stream):
        _dirty(B * H * L * d * q.element_size(), B * H * d * d * 4)
    grads = qx.lin_attn_backward(q, k, v, do, ld, lens=lens, stream=stream)[:3]
    torch.cuda.synchronize()
    for t in (out, *grads):
        for b in range(B):
            assert (t[b, :, n[b]:] == 0).all() and torch.isfinite(t[b, :, :n[b]]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("L,dk,dv", [(40, 64, 64), (600, 64, 64), (530, 33, 100), (70, 256, 8)])
def test_rows_behind_the_end_of_a_callers_gradients_stay(dtype, L, dk, dv):
    B, H = 4, 2
    g = gen(L + dk)
    q, k, v, do = (normal(g, B, H, L, d, dtype=dtype) for d in (dk, dk, dv, dv))
    ld = torch.tensor([-0.1, -0.01], device="cuda")
    n = [L, 0, 1, L - 3]
    lens = torch.tensor(n, dtype=torch.int32, device="cuda")
    out = [torch.full_like(t, 7.0) for t in (q, k, v)]
    got = qx.lin_attn_backward(q, k, v, do, ld, scale=0.2, lens=lens, out=out)[:3]
    want = ref.lin_attn_backward(q, k, v, do, ld, 0.2, lens=n)[:3]
    for t, w in zip(got, want):
        for b in range(B):
            assert (t[b, :, n[b]:] == 7).all()
            assert ref.norm_error(t[b, :, :n[b]], w[b, :, :n[b]]) <= ref.norm_tolerance(dtype)


# ---------------------------------------------------------------------------
# scales
# ---------------------------------------------------------------------------
# one launch, rows kernels, and tiles of aligned and of unaligned rows, in every tile size
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N,K", [(2, 40, 300), (12, 70, 2048), (20, 2100, 160), (70, 130, 128), (70, 130, 77),
                                   (600, 9000, 256), (4096, 4200, 64), (4096, 4200, 65)])
def test_large_rows_and_small_weights(dtype, M, N, K):
    """A product with one scale may pass the range of float32 where the result does not."""
    g = gen(M + K)
    x = normal(g, M, K, dtype=dtype)
    w = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int32).to(torch.int8).cuda()
    sw = torch.rand(N, generator=g).cuda() * 1e-3
    bias = normal(g, N)
    plain = qx.linear_i8(x, w, sw, bias=bias)
    rows = torch.arange(0, M, 3, device="cuda")
    big = x.clone()
    big[rows] = (x[rows].float() * 3e37 / x[rows].float().abs().amax(1, keepdim=True)).to(dtype)
    if M > 10:
        big[4, 1] = float("nan")
    y = qx.linear_i8(big, w, sw, bias=bias)
    a, sa = qx.quantize_rows_i8(big)
    assert torch.equal(y.nan_to_num(), qx.qgemm_i8_scaled(a, w, sa, sw, bias=bias, dtype=dtype).nan_to_num())
    other = torch.ones(M, dtype=torch.bool, device="cuda")
    other[rows] = False
    if M > 10:
        assert torch.isnan(y[4]).all()
        other[4] = False
    assert torch.equal(y[other], plain[other])
    want, tol = ref.product(ref.quantize(big[rows])[0], w, ref.quantize(big[rows])[1], sw, bias)
    assert float(want.abs().max()) < 3e38 and float((want / sw.cpu()).abs().max()) > 3.5e38     # what this is about
    if dtype != F32:
        tol = tol + ref.half_ulp(dtype) * (want.abs() + tol)
    assert ((y[rows].cpu().double() - want).abs() <= tol).all()


def test_small_rows_and_large_weights():
    # and the other way round, with a sum of nothing: 0 times the product of both scales would be NaN
    a = torch.tensor([[1, -1], [1, 1]], dtype=torch.int8, device="cuda")
    w = torch.tensor([[1, 1], [127, -128]], dtype=torch.int8, device="cuda")
    sa, sw = torch.tensor([1e30, 1e-30], device="cuda"), torch.tensor([1e30, 1e10], device="cuda")
    y = qx.qgemm_i8_scaled(a, w, sa, sw, dtype=F32).cpu()
    assert y[0, 0] == 0 and y[0, 1] == float("inf")
    want, tol = ref.product(a, w, sa, sw)
    assert ((y[1].double() - want[1]).abs() <= tol[1]).all()


# on each side of the rules by which a kernel is chosen
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(17, 1, 64), (24, 100, 8192), (32, 1000, 300), (32, 2047, 1501), (33, 2047, 1501),
                                   (64, 16383, 129), (64, 16400, 129), (512, 16400, 65), (513, 16400, 65)])
def test_layers_on_each_side_of_a_rule(dtype, M, N, K):
    g = gen(M + N)
    x = normal(g, M, K, dtype=dtype)
    w = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int32).to(torch.int8).cuda()
    sw = torch.rand(N, generator=g).cuda() * 1e-2
    y = qx.linear_i8(x, w, sw)
    a, sa = qx.quantize_rows_i8(x)
    assert torch.equal(y, qx.qgemm_i8_scaled(a, w, sa, sw, dtype=dtype))
    rows = [0, M // 2, M - 1]
    want, tol = ref.product(a[rows], w, sa[rows], sw)
    floor = 2.0 ** -25 if dtype == F16 else 0
    tol = tol + (ref.half_ulp(dtype) * (want.abs() + tol) if dtype != F32 else 0) + floor
    assert ((y[rows].cpu().double() - want).abs() <= tol).all()


# ---------------------------------------------------------------------------
# long memories
# ---------------------------------------------------------------------------
# A decay close to one is applied thousands of times, so what its rounding adds
# must not point the same way each time.
#
# With new terms of random size each token, n roundings of a state are a random
# walk of n steps of at most U / sqrt(3) (root mean square): four of its
# deviations bound the norm over a head's state.
def walk(n):
    return 4 * (n / 3) ** 0.5 * ref.U


# A state that only decays loses nearly the same number of last places each
# time, and their fraction is rounded the same way each time: an element may be
# n U off after n decays.  Over many elements that is next to nothing, so the
# projection on the state as it should be, sum(x w) / sum(w^2), tells a wrong
# decay from roundings:
#  - errors uniform within n U |w| and independent deviate by n U / sqrt(3)
#    sqrt(sum(w^4)) / sum(w^2), which is n U / sqrt(N) for normally distributed w
#    (sum(w^4) = 3 N, sum(w^2) = N); four of these;
#  - a decay by exp(l), |l| small, takes P = |l| / 2 U places of w = 1 and 2 P of
#    w = 2.  Rounding them has a mean over that range: 1/8 of a place over P at
#    most from the period that the range cuts, 1/12 over P from the falling
#    density of w within the periods; together below 0.42 U / P < U (U / |l|),
#    and never more than U;
#  - the decay itself is rounded by 2^-23 of its logarithm.
# decays: [(how many, logarithm of each)].
def check_decayed(state, S0, decays):
    total = sum(n * x for n, x in decays)
    x, want = state.detach().cpu().double(), S0.cpu().double() * float(torch.tensor(total, dtype=torch.float64).exp())
    if total < -80:      # below fp32's smallest normal number nothing is promised
        assert float(x.abs().max()) <= 1e-34
        return
    n = sum(n for n, _ in decays)
    own = (2 * abs(total) + 1) * ref.U
    assert ref.norm_error(x, want) <= n * ref.U + own
    along = float((x * want).sum() / (want * want).sum()) - 1
    mean = sum(n * ref.U * min(1, ref.U / abs(x) if x else 0) for n, x in decays)
    assert abs(along) <= 4 * n * ref.U / want.numel() ** 0.5 + mean + own, (along, mean)


LONG = [0.0, -1e-6, -7.3e-6, -1e-5, -(2.0 ** -12), -0.01, -0.68, -0.7, -5.0, float("-inf")]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_thousands_of_tokens_keep_a_long_memory(dtype):
    H, d, n = len(LONG), 64, 4096
    g = gen(31)
    ld = torch.tensor(LONG, device="cuda")
    q, k, v = (normal(g, 1, H, n, d, dtype=dtype) for _ in range(3))
    S0 = normal(g, 1, H, d, d, scale=30)
    state = S0.clone()
    for i in range(n):
        out = qx.lin_attn_step(q[:, :, i], k[:, :, i], v[:, :, i], ld, state, scale=0.1)
    o, S = ref.lin_attn(q, k, v, ld, 0.1, S0)
    o2, end = qx.lin_attn(q, k, v, ld, scale=0.1, state=S0)
    for h in range(H):
        # the state's decay and its new term, two roundings a token
        assert ref.norm_error(state[:, h], S[:, h]) <= walk(2 * n), h
        assert ref.norm_error(end[:, h], S[:, h]) <= walk(2 * n), h
        assert ref.norm_error(out[:, h], o[:, h, -1]) <= walk(2 * n) + 4 * ref.U + (ref.half_ulp(dtype) if dtype != F32 else 0), h


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_state_that_only_decays_token_by_token(dtype):
    H, n = len(LONG), 8192
    ld = torch.tensor(LONG, device="cuda")
    S0 = normal(gen(32), 1, H, 64, 96)
    state, zero = S0.clone(), torch.zeros(1, H, 96, dtype=dtype, device="cuda")
    for i in range(n):
        qx.lin_attn_step(zero[..., :64], zero[..., :64], zero, ld, state)
    for h, x in enumerate(ld.tolist()):
        check_decayed(state[:, h], S0[:, h], [(n, x)])


# whole sequences, segments and their scan, segments that add up those before them
@pytest.mark.parametrize("B,H,L,d", [(64, 8, 32768, 64), (1, 8, 1 << 20, 64), (1, 8, 1200, 64), (1, 8, 1 << 18, 128)])
def test_a_state_that_only_decays_over_a_prompt(B, H, L, d):
    # one row of zeros is every row of q, k and v
    x = torch.zeros(d, dtype=BF16, device="cuda").expand(B, H, L, d)
    logs = [-float(a) / L for a in (0, 1e-3, 3.3e-3, 1e-2, 3.7e-2, 0.13, 0.5, 3.0)]
    ld = torch.tensor(logs, device="cuda")
    S0 = normal(gen(33), B, H, d, d)
    _, end = qx.lin_attn(x, x, x, ld, state=S0)
    back = qx.lin_attn_backward(x, x, x, x, ld, d_state=S0)[3] if L <= 1 << 18 else None
    segments = max(qx.plan_lin_attn("bf16", B, H, L, d, d)["k_splits"], 1)
    of_segment = -(-(L // 32) // segments)          # chunks
    for h in range(H):
        x = float(ld[h].double())
        # the segments before the last one, and its chunks
        decays = [(segments - 1, 32 * of_segment * x), (L / 32 - (segments - 1) * of_segment, 32 * x)]
        check_decayed(end[:, h], S0[:, h], decays)
        if back is not None:
            check_decayed(back[:, h], S0[:, h], decays)


def test_ragged_calls_that_make_their_results_in_a_graph():
    B, H, L, d = 3, 2, 600, 64
    g = gen(41)
    q, k, v, do = (normal(g, B, H, L, d, dtype=BF16) for _ in range(4))
    ld = torch.tensor([-0.1, -0.01], device="cuda")
    lens = torch.tensor([L, 5, 0], dtype=torch.int32, device="cuda")

    def work():
        out, end = qx.lin_attn(q, k, v, ld, lens=lens)
        return (out, end, *qx.lin_attn_backward(q, k, v, do, ld, lens=lens))

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = work()
    for rep in range(4):
        lens.copy_(torch.tensor([[L, 5, 0], [1, L, 300], [0, 0, L], [L - 1, 33, 2]][rep], dtype=torch.int32))
        q.copy_(normal(gen(rep), B, H, L, d, dtype=BF16))
        for t in res:
            t.fill_(3)
        graph.replay()
        for a, b in zip(res, work()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("L,d", [(1000, 64), (1200, 64), (2000, 128)])
def test_a_state_in_place_has_the_bits_of_one_apart(dtype, L, d):
    # few segments add up the states before them, but not where the state is in place
    H = len(LONG)
    g = gen(L)
    q, k, v = (normal(g, 1, H, L, d, dtype=dtype) for _ in range(3))
    ld = torch.tensor(LONG, device="cuda")
    S0 = normal(g, 1, H, d, d, scale=10)
    out, end = qx.lin_attn(q, k, v, ld, state=S0)
    state = S0.clone()
    got, _ = qx.lin_attn(q, k, v, ld, state=state, out_state=state)
    assert torch.equal(got, out) and torch.equal(state, end)
