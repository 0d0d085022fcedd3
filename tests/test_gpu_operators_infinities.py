"""Infinite elements that count, in the LoRA linear on 4-bit matrices and with dropout: results are infinite, with their
sign, or not a number exactly where the 64-bit definition's are."""
import numpy as np
import pytest

from oracle import operators_oracle as orc
from paper_2404_15159_amd import binding as B
from test_gpu_q4 import Q4Linear, dev, packed, problem, rounded


pytestmark = pytest.mark.gpu
SEED, OFFSET = 0x1122334455667788, 21
# T, d_in, d_out, r: the forward on codes in one launch, in slices, in slices with a sliced projection; widened
SHAPES = [(20, 264, 72, 8), (50, 264, 136, 24), (150, 1296, 72, 16), (300, 264, 136, 40), (1030, 264, 72, 64)]


def same_kind(name, got, want):
    for kind in (np.isposinf, np.isneginf, np.isnan):
        assert np.array_equal(kind(got), kind(want)), (name, kind.__name__)


def run(h, W, p, dtype, q4):
    T, d_in = h["x"].shape
    f = orc.dropout_factors(T, d_in, p, SEED, OFFSET) if p else None
    packed_q4, Wq = packed(W, 64)
    m = Q4Linear(h, packed_q4 if q4 else None, 64, dtype, 2.0, B.make_dropout(p, SEED, OFFSET) if p else None,
                 W=None if q4 else dev(W, dtype))
    m.forward()
    m.backward()
    with np.errstate(invalid="ignore"):
        return m.results(), orc.linear(h["x"], Wq if q4 else W, h["A"], h["B"], 2.0, f, h["dy"])


def kept(T, d_in, p):
    return orc.dropout_factors(T, d_in, p, SEED, OFFSET) > 0 if p else np.ones((T, d_in), bool)


@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("p,dtype", [(0.0, "bf16"), (0.5, "bf16"), (0.5, "f32")])
@pytest.mark.parametrize("T,d_in,d_out,r", SHAPES)
def test_sums_of_the_first_factor(T, d_in, d_out, r, p, dtype, q4):
    """dA = s (dy B)^T D(x) with infinite kept elements of x beside factors that bf16 holds exactly (one element of dy a row)
    and beside an infinite one."""
    print(f"case dA T={T} {d_in}->{d_out} r={r} p={p} {dtype} q4={q4}", flush=True)
    h, W = problem(T, d_in, d_out, r, 64, dtype, T + r)
    stay = kept(T, d_in, p)
    h["dy"][:] = 0.0
    h["dy"][np.arange(T), np.arange(T) % d_out] = np.where(np.arange(T) % 3, 1.0, -0.5)
    h["x"][3, np.flatnonzero(stay[3])[5]] = np.inf
    h["x"][T - 1, np.flatnonzero(stay[T - 1])[-9]] = -np.inf
    h["x"][7, np.flatnonzero(stay[7])[20]] = -np.inf
    h["dy"][7, 7 % d_out] = np.inf
    got, want = run(h, W, p, dtype, q4)
    assert np.isposinf(want["dA"]).any() and np.isneginf(want["dA"]).any()
    same_kind("dA", got["dA"], want["dA"])


@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("p,dtype", [(0.0, "bf16"), (0.5, "bf16"), (0.5, "f32")])
@pytest.mark.parametrize("T,d_in,d_out,r", SHAPES)
def test_sums_of_the_second_factor(T, d_in, d_out, r, p, dtype, q4):
    """dB = s dy^T (D(x) A^T) likewise: one kept element of x a row, infinite elements of dy."""
    print(f"case dB T={T} {d_in}->{d_out} r={r} p={p} {dtype} q4={q4}", flush=True)
    h, W = problem(T, d_in, d_out, r, 64, dtype, T + r)
    stay = kept(T, d_in, p)
    h["x"][:] = 0.0
    for t in range(T):
        at = np.flatnonzero(stay[t])
        h["x"][t, at[t % len(at)]] = 1.0 if t % 3 else -0.25
    h["dy"][5, 11], h["dy"][T - 1, 30], h["dy"][9, 8] = np.inf, -np.inf, np.inf
    h["x"][9, np.flatnonzero(stay[9])[9]] = -np.inf      # its only element
    got, want = run(h, W, p, dtype, q4)
    assert np.isposinf(want["dB"]).any() and np.isneginf(want["dB"]).any()
    same_kind("dB", got["dB"], want["dB"])


# ranks that run zero-padded to a multiple of eight, beside ones that do not
@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("p,dtype", [(0.0, "bf16"), (0.5, "bf16"), (0.0, "f32"), (0.5, "f32")])
@pytest.mark.parametrize("T,d_in,d_out,r", [(1, 264, 72, 1), (20, 264, 72, 1), (20, 264, 72, 8), (50, 264, 136, 12),
                                            (100, 264, 136, 20), (150, 1296, 72, 1), (150, 264, 72, 3), (200, 264, 136, 1),
                                            (300, 264, 136, 35), (1030, 264, 72, 1), (1030, 264, 72, 16)])
def test_padded_ranks(T, d_in, d_out, r, p, dtype, q4):
    """An infinite element of x makes x A^T infinite: the rank entries that only fill up a multiple of eight have to stay
    zeros beside it, or zero times infinity reaches every output of the row.  Likewise dy and dy B."""
    print(f"case padded rank T={T} {d_in}->{d_out} r={r} p={p} {dtype} q4={q4}", flush=True)
    h, W = problem(T, d_in, d_out, r, 64, dtype, T + r)
    h["A"], h["B"] = np.abs(h["A"]) + np.float32(0.0625), np.abs(h["B"]) + np.float32(0.0625)   # one sign over all ranks
    stay = kept(T, d_in, p)
    h["x"][T // 2, np.flatnonzero(stay[T // 2])[3]] = np.inf
    h["x"][T - 1, np.flatnonzero(stay[T - 1])[40]] = -np.inf
    h["dy"][T // 3, 17], h["dy"][T - 1, 3] = np.inf, -np.inf
    h = {k: rounded(v, dtype) for k, v in h.items()}
    got, want = run(h, W, p, dtype, q4)
    for n in ("y", "dx"):
        assert np.isposinf(want[n]).any() and np.isneginf(want[n]).any() or T == 1, n
    for n in got:
        same_kind(n, got[n], want[n])
