"""Every instance of the kernels behind the LoRA linear on 4-bit matrices, at sizes of which neither rows, columns nor inputs
fill their tiles, against the float64 definition; and the block on matrices that the library has widened."""
import functools

import numpy as np
import pytest
import torch

from oracle import mixlora_oracle as block
from oracle import operators_oracle as orc
from paper_2404_15159_amd import binding as B
from paper_2404_15159_amd import synth
from paper_2404_15159_amd.runner import MixLoraFFN
from test_gpu_q4 import DEV, Q4Linear, check, check_all, packed, problem

import parity_utils as pu

pytestmark = pytest.mark.gpu
SEED, OFFSET = 0x1357246813572468, (1 << 34) + 3


@functools.lru_cache(maxsize=None)
def matrix(d_in, d_out, group):
    return packed(np.random.default_rng(d_out + group).normal(0, 0.02, (d_out, d_in)).astype(np.float32), group)


def forward(T, d_in, d_out, r, group, s=2.0):
    h, _ = problem(T, d_in, 8, r, group, "bf16", T + d_out)
    h["B"] = torch.from_numpy(np.random.default_rng(T).normal(0, 0.08, (d_out, r))).to(torch.bfloat16).float().numpy()
    h["dy"] = np.zeros((T, d_out), np.float32)
    q4, W = matrix(d_in, d_out, group)
    m = Q4Linear(h, q4, group, "bf16", s, back=False)
    m.forward()
    torch.cuda.synchronize()
    m.ws.numpy()
    check("y", m.y.numpy(), orc.linear(h["x"], W, h["A"], h["B"], s)["y"],
          orc.linear_sums(h["x"], W, h["A"], h["B"], s)["y"], 2 * d_in + r, "bf16")


# one launch: one tile per workgroup to 256 row blocks of the matrix, two to 512, three beyond (259, 514 and 515 of them:
# a last workgroup with one tile, and with two); one row, and one, two and four blocks of 16 rows
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 2, 16, 20, 32, 40, 64])
@pytest.mark.parametrize("d_in,d_out,r", [(264, 88, 16), (264, 4136, 8), (264, 4136, 16), (136, 8216, 16), (264, 8232, 8)])
def test_one_launch(d_in, d_out, r, T, group):
    print(f"case one launch T={T} {d_in}->{d_out} r={r} group={group}", flush=True)
    forward(T, d_in, d_out, r, group)


# slices (rank above 16): one, two and four row blocks, eight in two groups of wavefronts; one and more blocks of 128 rows
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 13, 16, 29, 32, 50, 64, 90, 128, 129, 270])
@pytest.mark.parametrize("d_in,d_out,r", [(1304, 88, 24), (264, 4136, 40)])
def test_slices(d_in, d_out, r, T, group):
    print(f"case slices T={T} {d_in}->{d_out} r={r} group={group}", flush=True)
    forward(T, d_in, d_out, r, group)


@pytest.mark.parametrize("T,d_in,d_out,r,p", [(1050, 1864, 2056, 12, 0.1), (1050, 1864, 2056, 64, 0.0)])
def test_four_rows_of_the_masked_term(T, d_in, d_out, r, p):
    """fp32 with 256 workgroups and more of 128 rows x 64 columns in both directions, remainders in both, in place."""
    print(f"case masked term T={T} {d_in}->{d_out} r={r} p={p}", flush=True)
    h, W = problem(T, d_in, d_out, r, 64, "f32", 3)
    q4, Wq = packed(W, 64)
    m = Q4Linear(h, q4, 64, "f32", 2.0, B.make_dropout(p, SEED, OFFSET) if p else None)
    m.forward()
    m.backward()
    check_all(m.results(), h, Wq, 2.0, orc.dropout_factors(T, d_in, p, SEED, OFFSET) if p else None, "f32")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 9, 40, 100, 150, 1030])
def test_largest_inputs_beside_codes(T, group):
    """Up to 2^118 a group's sum of x times level stays finite: 128 x 6 x 2^118 < 2^128.  264 x 6 x 2^98 has seven
    significant bits and is exact in bf16."""
    d_in, d_out = 264, 72
    codes = np.full((d_out, d_in), 7, np.uint8)
    codes[1::2] = 15
    c, s = orc.pack(codes, np.full((d_out, -(-d_in // group)), 2.0 ** -20), group)
    q4 = B.make_q4(torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV).to(torch.bfloat16), group)
    h = dict(x=np.full((T, d_in), 2.0 ** 118, np.float32), A=np.zeros((8, d_in), np.float32), B=np.zeros((d_out, 8), np.float32),
             dy=np.zeros((T, d_out), np.float32))
    m = Q4Linear(h, q4, group, "bf16", 1.0, back=False)
    m.forward()
    torch.cuda.synchronize()
    want = np.tile(np.where(np.arange(d_out) % 2, -1.0, 1.0) * 264 * 6 * 2.0 ** 98, (T, 1))
    assert np.array_equal(m.y.numpy().astype(np.float64), want)


@pytest.mark.parametrize("T", [5, 200])
def test_block_on_widened_matrices(T):
    """The feed-forward block, both directions, with every frozen matrix and its transposed copy widened from codes."""
    cfg = synth.scaled(synth.CONFIGS["llama2_7b"], name="widened", T=T, d=264, d_ff=520, N=8, k=2, r=16)
    print(f"case block on widened matrices T={T}", flush=True)
    host = dict(synth.make_inputs(cfg))
    names, made = ("W_gate", "W_up", "W_down"), {}
    for i, n in enumerate(names):
        rows, cols = host[n].shape
        group = (32, 64, 128)[i]
        W = torch.from_numpy(np.ascontiguousarray(host[n])).to(DEV).to(torch.bfloat16)
        codes = torch.empty(B.mixlora_q4_code_bytes(rows, cols), dtype=torch.uint8, device=DEV)
        scales = torch.empty(B.mixlora_q4_scale_bytes(rows, cols, group) // 2, dtype=torch.bfloat16, device=DEV)
        q4 = B.make_q4(codes, scales, group)
        B.mixlora_q4_quantize(W, B.BF16, rows, cols, q4)
        for name, shape, tr in ((n, (rows, cols), False), (n + "_T", (cols, rows), True)):
            made[name] = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
            B.mixlora_q4_dequantize(q4, rows, cols, tr, made[name], B.BF16)
        host[n] = orc.values(*orc.quantize(W.float().cpu().numpy(), group), group).astype(np.float32)
        assert np.array_equal(made[n].float().cpu().numpy(), host[n])
    m = MixLoraFFN(cfg, host)
    m.t.update(made)
    m.weights = B.make_weights(m.t)
    m.forward()
    m.backward()
    bw = block.backward(host["x"], {n: host[n] for n in synth.WEIGHT_NAMES}, cfg.k, cfg.lora_scale, host["dy"], 1.0,
                        cfg.aux_coeff, "top1")
    pu.compare_all(m.results(), bw["forward"], bw, cfg)
