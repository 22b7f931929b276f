"""The linear layer and its backward pass where a matrix has more than 2^31 elements: its last rows and
columns against the definition in 64 bits (tolerances: test_gpu_linear.py)."""
import pytest
import torch

from test_gpu_linear import DT, HALF, acc, act64, close, slope64

pytestmark = pytest.mark.gpu

FAR, WIDE = 32768 + 8 + 40, 65536 + 16  # their product is above 2^31
END = 130


def rand(gen, dtype, *shape):
    t = torch.empty(*shape, dtype=DT[dtype], device="cuda")
    return t.normal_(generator=gen)


# many rows of output; wide weights by rows, few tokens and tiles
@pytest.mark.parametrize("dtype,T,k,n", [("bf16", FAR, 72, WIDE), ("f32", FAR, 20, WIDE), ("bf16", 2, WIDE, FAR),
                                         ("bf16", 20, WIDE, FAR), ("bf16", 70, WIDE, FAR), ("f32", 2, WIDE, FAR),
                                         ("f32", 20, WIDE, FAR)])
def test_forward(fpo, dtype, T, k, n):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, W, b = rand(gen, dtype, T, k), rand(gen, dtype, n, k), rand(gen, dtype, n)
    W *= k ** -0.5
    y, z = (torch.empty(T, n, dtype=DT[dtype], device="cuda") for _ in range(2))
    r = rand(gen, dtype, T, n)
    ws = fpo.linear(x, W, y, bias=b, act=fpo.ACT_SILU, residual=r, z_out=z)
    assert fpo.get_device_status(ws) == fpo.OK
    for rows in (slice(0, END), slice(max(0, T - END), T)):
        for cols in (slice(0, END), slice(n - END, n)):
            xs, Ws = x[rows].double(), W[cols].double()
            floor = acc(dtype, k, xs.abs() @ Ws.abs().t())
            want = xs @ Ws.t() + b[cols].double()
            floor = floor + 2.0 ** -22 * (want.abs() + b[cols].double().abs())
            close(z[rows, cols], want, HALF[dtype], floor)
            a = act64("silu", want)
            yw = a + r[rows, cols].double()
            close(y[rows, cols], yw, HALF[dtype], 1.13 * floor + 2.0 ** -17 * a.abs() + 2.0 ** -23 * yw.abs())


# a large signal below the layer, weights and gradients, a large signal of its own
@pytest.mark.parametrize("dtype,T,k,n", [("bf16", FAR, WIDE, 72), ("f32", FAR, WIDE, 20), ("bf16", 20, WIDE, FAR),
                                         ("bf16", 70, WIDE, FAR), ("f32", 20, WIDE, FAR), ("bf16", FAR, 72, WIDE),
                                         ("f32", FAR, 20, WIDE)])
def test_backward(fpo, dtype, T, k, n):
    gen = torch.Generator(device="cuda").manual_seed(2)
    dy, x, W = rand(gen, dtype, T, n), rand(gen, dtype, T, k), rand(gen, dtype, n, k)
    z, z_in = rand(gen, dtype, T, n), rand(gen, dtype, T, k)
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty(n, device="cuda")
    ws = fpo.linear_vjp(dy, x, W, dx, act=fpo.ACT_RELU, z=z, act_in=fpo.ACT_RELU, z_in=z_in, dW=dW, dbias=db)
    assert fpo.get_device_status(ws) == fpo.OK
    del ws
    half = HALF[dtype]

    def signal(rows, cols):  # exact: relu's slope is 0 or 1
        return dy[rows, cols].double() * slope64("relu", z[rows, cols].double())

    for rows in (slice(0, END), slice(max(0, T - END), T)):
        for cols in (slice(0, END), slice(k - min(END, k), k)):
            dz = signal(rows, slice(None))
            Ws = W[:, cols].double()
            s = slope64("relu", z_in[rows, cols].double())
            close(dx[rows, cols], dz @ Ws * s, half, acc(dtype, n, dz.abs() @ Ws.abs()))
    for rows in (slice(0, END), slice(n - min(END, n), n)):
        dz = signal(slice(None), rows)
        for cols in (slice(0, END), slice(k - min(END, k), k)):
            xs = x[:, cols].double()
            close(dW[rows, cols], dz.t() @ xs, half, acc(dtype, T, dz.t().abs() @ xs.abs()))
        close(db[rows], dz.sum(0), 2.0 ** -24, (T / 16 + 640) * 2.0 ** -24 * dz.abs().sum(0))
