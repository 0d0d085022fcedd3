"""Dropout on the adapter's input, on an ordinary frozen matrix, against the float64 definition."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2404_15159_amd import binding as B
from test_gpu_q4 import CODE, DEV, Q4Linear, check_all, dev, packed, problem

pytestmark = pytest.mark.gpu
SEED, OFFSET = 0x0123456789ABCDEF, (3 << 40) + 11

CASES = [
    # T, d_in, d_out, r, dtype, p, transposed copy given
    (1, 64, 128, 8, "bf16", 0.5, True),
    (2, 1032, 520, 16, "bf16", 0.1, False),
    (4, 520, 1032, 8, "bf16", 0.0, True),
    (17, 512, 704, 16, "bf16", 0.05, True),
    (60, 264, 264, 64, "bf16", 0.3, False),
    (128, 264, 264, 40, "bf16", 0.05, True),
    (129, 264, 264, 40, "bf16", 0.05, True),
    (200, 1024, 1024, 8, "bf16", 0.1, True),
    (300, 256, 520, 12, "bf16", 0.9, False),
    (513, 192, 320, 24, "bf16", 0.05, True),
    (300, 264, 264, 1, "bf16", 0.0, True),
    (5, 72, 200, 8, "f32", 0.3, True),
    (97, 64, 136, 16, "f32", 0.05, False),
]


@pytest.mark.parametrize("T,d_in,d_out,r,dtype,p,pre", CASES)
def test_linear(T, d_in, d_out, r, dtype, p, pre):
    print(f"case dropout linear T={T} {d_in}->{d_out} r={r} {dtype} p={p} transposed={pre}", flush=True)
    h, W = problem(T, d_in, d_out, r, 64, dtype, T + d_in)
    factors = orc.dropout_factors(T, d_in, p, SEED, OFFSET) if p else None
    Wd = dev(W, dtype)
    m = Q4Linear(h, None, 64, dtype, 2.0, B.make_dropout(p, SEED, OFFSET), W=Wd)
    m.forward()
    m.backward(Wd.T.contiguous() if pre else None)
    check_all(m.results(), h, W.astype(np.float64), 2.0, factors, dtype)


def test_no_dropout_is_p_zero():
    h, W = problem(140, 264, 136, 16, 64, "bf16", 1)
    outs = []
    for drop in (None, B.make_dropout(0.0, 1, 2), B.make_dropout(2.0 ** -18, 1, 2)):   # the last rounds to none
        m = Q4Linear(h, None, 64, "bf16", 2.0, drop, W=dev(W, "bf16"))
        m.forward()
        m.backward()
        outs.append(m.results())
    for o in outs[1:]:
        assert all(np.array_equal(o[n], outs[0][n]) for n in o)


@pytest.mark.parametrize("T", [40, 200])
def test_dropped_infinities_reach_no_gradient(T):
    """dA takes D(x): an infinite or NaN element of x that is dropped adds nothing to it."""
    p = 0.4
    h, W = problem(T, 136, 72, 8, 64, "bf16", 3)
    f = orc.dropout_factors(T, 136, p, SEED, OFFSET)
    gone = np.argwhere(f == 0)[::7]
    h["x"][gone[:, 0], gone[:, 1]] = np.where(np.arange(len(gone)) % 2, np.inf, np.nan)
    m = Q4Linear(h, None, 64, "bf16", 2.0, B.make_dropout(p, SEED, OFFSET), W=dev(W, "bf16"))
    m.forward()
    m.backward()
    got = m.results()
    clean = dict(h, x=np.where(np.isfinite(h["x"]), h["x"], 0.0))
    want = orc.linear(clean["x"], W, h["A"], h["B"], 2.0, f, h["dy"])
    sums = orc.linear_sums(clean["x"], W, h["A"], h["B"], 2.0, f, h["dy"])
    for n in ("dA", "dB"):
        assert np.all(np.abs(got[n] - want[n]) <= 500 * 2.0 ** -23 * sums[n]), n


def test_gradient_against_differences():
    """<y, dy> is linear in x, A and B each: a difference of two forward passes is a product with the gradient."""
    T, p = 33, 0.2
    rng = np.random.default_rng(5)
    h, W = problem(T, 64, 40, 8, 64, "f32", 6)
    drop = B.make_dropout(p, SEED, OFFSET)
    m = Q4Linear(h, None, 64, "f32", 2.0, drop, W=dev(W, "f32"))
    m.forward()
    m.backward()
    g = m.results()
    for n, grad in (("x", "dx"), ("A", "dA"), ("B", "dB")):
        step = rng.normal(size=h[n].shape).astype(np.float32)
        k = Q4Linear(dict(h, **{n: h[n] + step}), None, 64, "f32", 2.0, drop, W=dev(W, "f32"))
        k.forward()
        torch.cuda.synchronize()
        diff = float(((k.y.numpy().astype(np.float64) - g["y"]) * h["dy"]).sum())
        want = float((g[grad].astype(np.float64) * step).sum())
        # fp32 results of sums over at most 64 + 8 terms, then T * 40 of them in 64 bits
        size = float((np.abs(k.y.numpy()).astype(np.float64) * np.abs(h["dy"])).sum())
        assert abs(diff - want) <= 200 * 2.0 ** -24 * size, n


def test_step_on_the_device_moves_the_mask():
    """offset + *step is the stream: the same mask as offset alone with the sum, and a captured graph draws a
    new one whenever the program advances the number, replay for replay equal to eager calls."""
    T, p = 150, 0.5
    h, W = problem(T, 136, 72, 8, 64, "bf16", 7)
    Wd = dev(W, "bf16")
    step = torch.zeros(1, dtype=torch.int64, device=DEV)

    def eager(offset):
        m = Q4Linear(h, None, 64, "bf16", 2.0, B.make_dropout(p, SEED, offset), W=Wd)
        m.forward()
        m.backward(Wd.T.contiguous())
        return m.results()

    W_T = Wd.T.contiguous()
    m = Q4Linear(h, None, 64, "bf16", 2.0, B.make_dropout(p, SEED, OFFSET, step), W=Wd)
    m.forward()
    m.backward(W_T)
    first = m.results()
    want = eager(OFFSET)
    assert all(np.array_equal(first[n], want[n]) for n in first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.forward()
        m.backward(W_T)
    seen = []
    for i in (0, 1, 2, 5, 1):
        step.fill_(i)
        graph.replay()
        got = m.results()
        want = eager(OFFSET + i)
        assert all(np.array_equal(got[n], want[n]) for n in got), i
        seen.append(got["dA"].copy())
    assert not np.array_equal(seen[0], seen[1]) and np.array_equal(seen[1], seen[4])


def test_two_streams_and_workspaces():
    """Two problems on two streams, each with its own workspace, give what they give alone."""
    h, W = problem(200, 264, 136, 16, 64, "bf16", 8)
    q4, _ = packed(W, 64)
    ms = [Q4Linear(h, q4, 64, "bf16", 2.0, B.make_dropout(0.1, SEED, i)) for i in (1, 2)]
    alone = []
    for m in ms:
        m.forward()
        m.backward()
        alone.append(m.results())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ms]
    for _ in range(3):
        for m, s in zip(ms, streams):
            m.forward(s)
            m.backward(stream=s)
    torch.cuda.synchronize()
    for m, a in zip(ms, alone):
        got = m.results()
        assert all(np.array_equal(got[n], a[n]) for n in got)
