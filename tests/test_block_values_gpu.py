"""The operators around the linear backward on the GPU, on values where they can go wrong: infinities and NaN, rows of a wide range,
operands whose products are exact; each on the way of working that is meant."""
import pytest
import torch

import block_oracle as ref
import paper_2503_21261_amd as hot
from test_block_ops_gpu import BF16, F32, FNS, close, rand

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("fn", FNS)
def test_gradient_of_a_group_that_held_an_infinity_or_a_nan(fn, dtype):
    """Such a group of a checkpoint reads as NaN, so its gradients are NaN, finite neighbours of the bad element among them, and so are
    the bias sums of its columns; all others are as ever."""
    rows, cols = 300, 100
    x, g = rand((rows, cols), 1, dtype, 2.0), rand((rows, cols), 2, dtype)
    x[3, 5], x[7, 40], x[299, 99] = INF, NAN, -INF          # the last one in a row's short last group
    lost = torch.zeros((rows, cols), dtype=torch.bool)
    lost[3, :32], lost[7, 32:64], lost[299, 96:] = True, True, True
    kept, y = hot.alloc_checkpoint(rows, cols), torch.empty((rows, cols), dtype=dtype, device="cuda")
    gx, gb = torch.empty_like(y), torch.empty(cols, device="cuda")
    hot.hot_activation_forward(hot.ACT_FNS[fn], x.cuda(), y, ckpt=kept)
    hot.hot_activation_backward(hot.ACT_FNS[fn], g.cuda(), gx, ckpt=kept, g_bias=gb, ws=hot.alloc_activation_workspace(rows, cols))
    values = ref.checkpoint(x)[2]
    want, tol, bias, btol = ref.act_grad(fn, ref.f64(g), values, dtype)
    close(gx, want.masked_fill(lost, NAN), tol, "g_x")
    close(gb, bias.masked_fill(lost.any(0), NAN), btol, "g_bias")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_relu_gradient_of_infinities_and_nan(dtype):
    x = torch.tensor([[INF, 1.0, -INF, -1.0, NAN, 0.0, -0.0, 2.0]], dtype=dtype)
    g = torch.full_like(x, 3.0).cuda()
    gx = hot.hot_activation_backward(hot.HOT_ACT_RELU, g, torch.empty_like(g), x=x.cuda())
    want = torch.tensor([[3.0, 3.0, 0.0, 0.0, NAN, 0.0, 0.0, 3.0]], dtype=torch.float64)
    close(gx, want, torch.zeros_like(want), "g_x")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 100, 200, 500, 771, 1500, 4096, 5000, 11008, 16384])
def test_layer_norm_mean_is_the_exact_one_rounded_once(cols, dtype):
    """Rows about zero, with columns that stand out, far from zero, and of the largest numbers.  In 64 bits a lane adds 16 columns and at
    most 25 more additions join the lanes and waves (2^-53 of mean |h| each, and the division), then the mean is rounded: half a step."""
    x = rand((24, cols), cols, dtype)
    x[6:12, ::100] *= 20
    x[12:18] += 300
    x[18:21] *= 1e-30
    x[21:] = x[21:].abs() * 1e37
    y, mean, rstd = torch.empty((24, cols), dtype=dtype, device="cuda"), torch.empty(24, device="cuda"), torch.empty(24, device="cuda")
    hot.hot_layer_norm_forward(x.cuda(), None, None, 1e-6, y, mean, rstd)
    want = ref.f64(x).mean(1)
    close(mean, want, want.abs() * (1 + 2.0 ** -20) * ref.U + 2.0 ** -47 * ref.f64(x).abs().mean(1), "mean")
