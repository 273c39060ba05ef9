"""On the host: the largest numbers of heads that linear attention is
documented to take, on both sides; calls with a missing operand; and which of
the 8-bit kernels a size gets."""
import pytest

import test_serve_host as host
from paper_2606_09905_amd import qx
from test_serve_host import double  # noqa: F401  (a fixture)

# (dk, dv): heads that a prompt takes, that its gradients take
HEADS = [((64, 64), 1 << 24, 1 << 24), ((8, 56), 1 << 24, 1 << 24),
         ((64, 72), (1 << 24) - 1, (1 << 24) - 1), ((72, 64), 1 << 24, (1 << 24) - 1), ((128, 128), (1 << 24) - 1, (1 << 24) - 1),
         ((33, 64), (1 << 24) - 1, (1 << 24) - 1), ((64, 136), (1 << 23) - 1, (1 << 23) - 1),
         ((256, 64), 1 << 24, (1 << 23) - 1), ((256, 256), (1 << 23) - 1, (1 << 23) - 1)]


def _both_sides(call, heads, **kw):
    assert call(B=1, H=heads, **kw) == qx.OK, host.last()
    assert call(B=1, H=heads + 1, **kw) == qx.ERR_UNSUPPORTED
    # whatever bounds it, the message names the heads, and nothing that the call does not have
    assert "H" in host.last() and "L" not in host.last(), host.last()


@pytest.mark.parametrize("d,prompt,gradients", HEADS)
@pytest.mark.parametrize("dt", [0, 2])
def test_heads_of_prompts_and_gradients(double, dt, d, prompt, gradients):  # noqa: F811
    _both_sides(lambda **kw: host.attn(double, **kw), prompt, dt=dt, n=32, dk=d[0], dv=d[1])
    _both_sides(lambda **kw: host.back(double, **kw), gradients, dt=dt, n=32, dk=d[0], dv=d[1])


@pytest.mark.parametrize("dv", [1, 32, 33, 128, 250, 256])
def test_heads_of_one_token(double, dv):  # noqa: F811
    _both_sides(lambda **kw: host.step(double, **kw), ((1 << 24) - 1) // -(-dv // 32), dk=64, dv=dv)


@pytest.mark.parametrize("name,args", [("quant", "x q s"), ("product", "a w sa sw y"), ("linear", "x w sw y ws"),
                                       ("attn", "q k v g o"), ("step", "q k v g s o"),
                                       ("back", "q k v do g dq dk_ dv_ ws")])
@pytest.mark.parametrize("n", [40, 600])
def test_nothing_is_enqueued_without_an_operand(double, name, args, n):  # noqa: F811
    kw = dict(n=n) if name in ("attn", "back") else {}
    need = name != "back" or qx.plan_lin_attn_backward("bf16", 2, 3, n, 64, 64)["workspace_bytes"]
    for arg in args.split():
        if arg == "ws" and not need:
            continue
        before = qx.testing_counters()["launches"]
        assert host.CALLS[name](double, **{arg: None}, **kw) == qx.ERR_INVALID_ARG, arg
        assert host.last() and qx.testing_counters()["launches"] == before, arg


@pytest.mark.parametrize("N", [1, 64, 1024, 2047, 2048, 9000])
@pytest.mark.parametrize("K", [64, 1501, 8192, 131071])
def test_few_rows_go_to_the_kernel_whose_waves_share_k(N, K):
    for f in (qx.plan_gemm_i8_scaled, qx.plan_linear_i8):
        assert [f("bf16", M, N, K)["tile_m"] for M in (16, 17, 24, 32)] == [16, 32, 32, 32]
        assert f("bf16", 33, N, K)["tile_m"] >= 64


@pytest.mark.parametrize("M,N,K,copied", [(777, 1000, 1501, True), (33, 16383, 1001, True), (33, 16384, 1001, False),
                                          (512, 40000, 4099, False), (513, 40000, 4099, True), (33, 1000, 1008, False),
                                          (32, 1000, 1501, False)])
def test_weights_are_copied_where_it_pays(M, N, K, copied):
    need = qx.plan_linear_i8("bf16", M, N, K)["workspace_bytes"]
    assert (need >= N * K) == copied and need >= M * K
