"""Calls at the limits of the LoRA linear with dropout and on 4-bit matrices."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2404_15159_amd import binding as B
from test_gpu_q4 import DEV, Q4Linear, check_all, dev, problem

pytestmark = pytest.mark.gpu
SEED, OFFSET = 0x0F1E2D3C4B5A6978, (9 << 33) + 5


@pytest.mark.parametrize("T,d_in,d_out", [(11184817, 8, 64), (5, 11184816, 8)])
def test_rank_term_behind_4_gib(T, d_in, d_out):
    """Rank 64: the rank-r term of dx has an operand of 4 GiB, dy and the matrix have not.  Whole numbers: every product and
    sum is below 2^24 and exact in fp32, so dA and dB are exact and y and dx are rounded once, to the nearest."""
    print(f"case rank term behind 4 GiB T={T} {d_in}->{d_out}", flush=True)
    r, p, s = 64, 0.5, 2.0
    gen = torch.Generator(device=DEV).manual_seed(T)

    def signs(*shape):
        return (torch.randint(0, 2, shape, generator=gen, device=DEV, dtype=torch.int8) * 2 - 1).to(torch.bfloat16)

    x, W, A, Bm = signs(T, d_in), signs(d_out, d_in), signs(r, d_in), signs(d_out, r)
    if d_in > 8:      # (P and the sums over a row of x stay small)
        x[:, 16:] = 0
    dy = torch.zeros((T, d_out), dtype=torch.bfloat16, device=DEV)   # one element a row: V is a row of B
    rows = torch.arange(T, device=DEV)
    dy[rows, rows % d_out] = signs(T)
    f = orc.dropout_factors(T, d_in, p, SEED, OFFSET)
    keep = torch.from_numpy((f > 0).astype(np.uint8)).to(DEV)
    del f
    dims, drop = B.LinearDims(T, d_in, d_out, r, s, B.BF16), B.make_dropout(p, SEED, OFFSET)
    n = B.mixlora_lora_dropout_workspace_bytes(dims, True)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    y, dx = torch.empty((T, d_out), dtype=torch.bfloat16, device=DEV), torch.empty((T, d_in), dtype=torch.bfloat16, device=DEV)
    dA, dB = torch.empty((r, d_in), device=DEV), torch.empty((d_out, r), device=DEV)
    B.mixlora_lora_dropout_forward(dims, W, A, Bm, drop, x, y, ws, n)
    torch.cuda.synchronize()
    print("  forward done", flush=True)
    B.mixlora_lora_dropout_backward(dims, W, None, A, Bm, drop, x, dy, ws, n, dx, dA, dB)
    torch.cuda.synchronize()
    print("  backward done", flush=True)
    del ws
    W, A, Bm = W.float(), A.float(), Bm.float()
    wA, wB = torch.zeros_like(A, dtype=torch.float64), torch.zeros_like(Bm, dtype=torch.float64)
    # (columns in blocks: the library's product into 64 x 11184816 leaves what is behind 2 GiB of its output unwritten)
    for i in range(0, T, 1 << 20):
        j = slice(i, min(i + (1 << 20), T))
        xf, d, k = x[j].float(), dy[j].float(), keep[j].float()
        xd, V = 2.0 * xf * k, d @ Bm
        P = xd @ A.T
        assert torch.equal(y[j], (xf @ W.T + s * (P @ Bm.T)).to(torch.bfloat16)), i
        for c in range(0, d_in, 1 << 20):
            c = slice(c, min(c + (1 << 20), d_in))
            assert torch.equal(dx[j, c], (d @ W[:, c] + 2.0 * s * k[:, c] * (V @ A[:, c])).to(torch.bfloat16)), (i, c)
            wA[:, c] += (s * (V.T @ xd[:, c])).double()
        wB += (s * (d.T @ P)).double()
    assert torch.equal(dA.double(), wA) and torch.equal(dB.double(), wB)


def test_dropout_of_more_elements_than_a_grid_row():
    """fp32: D(x) takes more than one row of its launch (16384 workgroups of 2048 elements)."""
    T, d_in, d_out, r, p = 4100, 8200, 8, 12, 0.3
    print(f"case D(x) in grid rows T={T} {d_in}->{d_out} r={r}", flush=True)
    h, W = problem(T, d_in, d_out, r, 64, "f32", 1)
    m = Q4Linear(h, None, 64, "f32", 2.0, B.make_dropout(p, SEED, OFFSET), W=dev(W, "f32"))
    m.forward()
    m.backward()
    check_all(m.results(), h, W.astype(np.float64), 2.0, orc.dropout_factors(T, d_in, p, SEED, OFFSET), "f32")
