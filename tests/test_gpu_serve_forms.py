"""The plain forms and 64-bit definitions of perf/operators.py quantise as
the operators' definition says, on as many values as it takes to meet those
next to a half; and so do the kernels."""
import pytest

import serve_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _operators():
    from perf import operators
    return operators


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_a_layer_quantise_as_defined(dtype, own):
    # weights that are the identity give the 8-bit values back, times their scale: in float32
    # one rounding, the same for everyone who has the same values and scales
    ops = _operators()
    g = torch.Generator()
    g.manual_seed(17)
    x = torch.randn(16384, 256, generator=g).to(dtype)
    s = dict(op="linear", dt="f32" if dtype == F32 else "bf16", x=x.cuda(),
             w=torch.eye(256).to(torch.int8).cuda(), scale_w=torch.ones(256).cuda(), bias_t=None)
    ops.own = own
    try:
        y = ops.run(s).cpu()
    finally:
        ops.own = False
    q, sa = ref.quantize(x)
    assert torch.equal(y, (q.float() * sa[:, None]).to(dtype))


def test_definition_in_64_bits_quantises_as_defined():
    ops = _operators()
    case = dict(op="linear", dt="f32", M=3000, N=40, K=4096, bias=False)
    y = ops.exact(case, 3).cpu()
    s = ops.prepare(case, 3)
    q, sa = ref.quantize(s["x"])
    want, _ = ref.product(q, s["w"], sa, s["scale_w"])
    # the sums are exact whole numbers, so three roundings of 2^-53 on each side
    assert ((y - want).abs() <= 6 * 2.0 ** -53 * want.abs()).all()
