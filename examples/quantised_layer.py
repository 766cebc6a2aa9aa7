"""A rotated layer in 4 and 8 bits, end to end: calibrate a rotation on a layer's activations, fold it into the weights,
and run the layer on the microscaled operators.

    residual stream  --dq_rmsnorm_quantize-->  8-bit activations  --dq_mx_matmul-->  hidden        (W1, 4 bits)
    hidden           --dq_rotate_apply, dq_mx_linear (4-bit activations)-->           layer output  (W2, 4 bits)

A rotation commutes with the norm (it keeps every token's length), so the residual stream is kept rotated and W1 takes
gamma and the rotation in; W2 takes in the rotation of the hidden activations.  Prints the relative error of the output
against the fp32 layer, with and without the rotations.

    python examples/quantised_layer.py [--tokens 2048] [--width 1024] [--hidden 2048] [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_04063_b200 as dq  # noqa: E402

EPS = 1e-5


def hadamard(d, seed):
    """Random Hadamard matrix, the latent that calibration starts from."""
    h = torch.ones(1, 1)
    while h.shape[0] < d:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)))
    sign = torch.randint(0, 2, (d,), generator=torch.Generator().manual_seed(seed)) * 2.0 - 1
    return (h / d ** 0.5 * sign).cuda().contiguous()


def calibrate(x, steps, lr=1e-3):
    """The rotation of activations x ([tokens, d] bfloat16) after `steps` calibration steps."""
    z0 = hadamard(x.shape[1], 0)
    handle = dq.dq_calib_init(x, z0, lr=lr, path=dq.DQ_PATH_BF16_TC)
    dq.dq_calib_step(handle, steps)
    rotation = torch.empty_like(z0)
    dq.dq_calib_get_rotation(handle, rotation)
    status = dq.dq_calib_status(handle)
    dq.dq_calib_destroy(handle)
    if status != dq.DQ_OK:
        raise dq.DartQuantError(status, "dq_calib_step")
    return rotation


def quantised_weights(w):
    codes, scales = dq.dq_mx_empty(w.shape[0], w.shape[1], dq.DQ_MXFP4)
    dq.dq_mx_quantize(w.contiguous(), dq.DQ_MXFP4, codes, scales)
    return codes, scales


def layer(x, residual, w1, w2, rotation2):
    """The quantised layer: (output, new residual).  w1, w2: (codes, scales); rotation2: of the hidden activations, or None."""
    tokens, width = x.shape
    hidden, out = w1[0].shape[0], w2[0].shape[0]
    a, a_scales = dq.dq_mx_empty(tokens, width, dq.DQ_MXFP8)
    stream = torch.empty_like(x)
    dq.dq_rmsnorm_quantize(x, None, EPS, dq.DQ_MXFP8, a, a_scales, residual=residual, sum_out=stream)
    h = torch.empty((tokens, hidden), dtype=torch.bfloat16, device="cuda")
    dq.dq_mx_matmul(a, a_scales, dq.DQ_MXFP8, w1[0], w1[1], width, h)
    if rotation2 is not None:
        rotated = torch.empty_like(h)
        dq.dq_rotate_apply(h, rotation2, rotated)
        h = rotated
    y = torch.empty((tokens, out), dtype=torch.bfloat16, device="cuda")
    workspace = torch.empty(dq.dq_mx_linear_workspace(dq.DQ_MXFP4, tokens, hidden), dtype=torch.uint8, device="cuda")
    dq.dq_mx_linear(h, dq.DQ_MXFP4, w2[0], w2[1], y, workspace)
    return y, stream


def main(tokens=2048, width=1024, hidden=2048, steps=20):
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    gamma = 1 + 0.1 * normal(width)
    w1, w2 = normal(hidden, width) / width ** 0.5, normal(width, hidden) / hidden ** 0.5
    outliers = torch.where(torch.rand(width, device="cuda", generator=g) < 0.01, 50.0, 1.0)
    w1 = w1 * (1 + 29 * (torch.rand(hidden, 1, device="cuda", generator=g) < 0.01))   # hidden outlier channels
    x, residual = normal(tokens, width) * outliers, normal(tokens, width)

    def fp32_layer():
        s = x + residual
        n = s * torch.rsqrt(s.square().mean(1, keepdim=True) + EPS) * gamma
        h = n @ w1.t()
        return n, h, h @ w2.t()

    _, h, want = fp32_layer()
    stream = x + residual
    r1 = calibrate((stream * torch.rsqrt(stream.square().mean(1, keepdim=True) + EPS)).bfloat16(), steps)
    r2 = calibrate(h.bfloat16(), steps)

    errors = {}
    for name, q1, q2 in (("plain", None, None), ("rotated", r1, r2)):
        v1, v2 = w1 * gamma, w2
        a, b = x, residual
        if q1 is not None:
            v1, v2, a, b = v1 @ q1, v2 @ q2, x @ q1, residual @ q1
        y, _ = layer(a.bfloat16(), b.bfloat16(), quantised_weights(v1), quantised_weights(v2), q2)
        errors[name] = float((y.float() - want).norm() / want.norm())
    if dq.dq_mx_status() != dq.DQ_OK:
        raise SystemExit("a product gave up waiting")
    return errors


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    for name, value in (("tokens", 2048), ("width", 1024), ("hidden", 2048), ("steps", 20)):
        p.add_argument("--" + name, type=int, default=value)
    result = main(**vars(p.parse_args()))
    print("relative error of the layer's output: %.4f without rotations, %.4f with calibrated rotations"
          % (result["plain"], result["rotated"]))
