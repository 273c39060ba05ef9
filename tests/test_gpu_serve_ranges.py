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
