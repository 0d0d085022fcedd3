"""Pins of the oracle's 4-bit, dropout and router definitions: published test vectors, closed forms,
autograd, differences."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc


def test_philox_published_vectors():
    """Known answers that the generator's authors distribute for Philox4x32 (7 and 10 rounds)."""
    M = 0xFFFFFFFF
    assert orc.philox((0,) * 4, (0,) * 2, 7) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    assert orc.philox((0,) * 4, (0,) * 2, 10) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert orc.philox((M,) * 4, (M,) * 2, 10) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("p", [0.05, 0.5, 0.9])
def test_dropout_share_and_mean(p):
    f = orc.dropout_factors(64, 1000, p, seed=0x123456789ABCDEF, offset=5 << 33)
    # 64000 draws: five standard deviations
    assert abs((f == 0).mean() - p) < 5 * np.sqrt(p * (1 - p) / f.size)
    assert abs(f.mean() - 1) < 5 * np.sqrt(p / (1 - p) / f.size)
    assert not np.array_equal(f, orc.dropout_factors(64, 1000, p, seed=0x123456789ABCDEF, offset=(5 << 33) + 1))
    assert np.array_equal(f[:, :200], orc.dropout_factors(64, 200, p, seed=0x123456789ABCDEF, offset=5 << 33))


def test_scales_have_six_bits_and_cover():
    rng = np.random.default_rng(0)
    for most in np.concatenate([np.exp(rng.uniform(-60, 80, 500)), 6.0 * 2.0 ** np.arange(-90, 90),
                                6.0 * 33 / 32 * 2.0 ** np.arange(-90, 90)]).astype(np.float32).astype(np.float64):
        s = orc.group_scale(most)
        m = np.frexp(s)[0] * 64
        assert m == round(m) and 6 * s >= most
        assert 6 * s * (1 - 1 / 32) < most * (1 + 1e-12)   # the next smaller one would not do
        # scale x level is exact in bf16
        for lv in orc.LEVELS:
            v = torch.tensor(s * lv, dtype=torch.float64)
            assert v.to(torch.bfloat16).double() == v
    assert orc.group_scale(2.0 ** -101) == 0 and np.isnan(orc.group_scale(np.inf)) and np.isnan(orc.group_scale(2.0 ** 127))


def test_codes_ties_and_signs():
    s = 0.75
    mids = (orc.LEVELS[1:] + orc.LEVELS[:-1]) / 2
    assert [orc.nearest_code(m * s, s) for m in mids] == [0, 2, 2, 4, 4, 6, 6]
    assert [orc.nearest_code(-m * s, s) for m in mids] == [0, 10, 10, 12, 12, 14, 14]
    assert [orc.nearest_code(v * s, s) for v in orc.LEVELS] == list(range(8))
    assert orc.nearest_code(-0.1, s) == 0 and orc.nearest_code(3.0, 0.0) == 0


def test_quantize_is_idempotent_and_near():
    W = np.random.default_rng(1).normal(0, 0.02, (24, 200)).astype(np.float32)
    for group in (32, 64, 128):
        c, s = orc.quantize(W, group)
        V = orc.values(c, s, group)
        # half the widest step (2 levels of 6) of the group's scale
        assert np.all(np.abs(V - W) <= np.repeat(s, group, 1)[:, :200] * 1.0)
        c2, s2 = orc.quantize(V, group)
        assert np.array_equal(orc.values(c2, s2, group), V)


def test_arrays_against_single_elements():
    """The oracle's array forms against its definitions of one code, one byte and one counter."""
    rng = np.random.default_rng(4)
    W = rng.normal(0, 1, (20, 200))
    W[3, :40] = [0.0, -0.0] * 20
    W[5, 150], W[6, 10] = np.nan, np.inf
    W[7, :32] = np.resize(np.array([9.0, .375, 1.125, 1.875, 2.625, 3.75, 5.25, -7.5]), 32)
    for group in (32, 64, 128):
        codes, scales = orc.quantize(W, group)
        data, sc = orc.pack(codes, scales, group)
        kt, per = 2, 128 // group
        for i in range(20):
            for k in range(200):
                g = k // group
                assert codes[i, k] == orc.nearest_code(W[i, k], scales[i, g]), (i, k)
                byte = data[(i // 16 * kt + k // 128) * 1024 + 16 * (16 * (k % 32 // 8) + i % 16) + 4 * (k % 128 // 32) + k % 8 // 2]
                assert (byte >> (4 * (k % 2))) & 15 == codes[i, k]
                got = sc[((i // 16 * kt + g // per) * 16 + i % 16) * per + g % per]
                assert got == scales[i, g] or np.isnan(got) and np.isnan(scales[i, g])
        assert data.size == 4 * 1024 and sc.size == 4 * 16 * per
    f = orc.dropout_factors(3, 20, 0.3, 0x123456789ABCDEF0, (9 << 32) + 4)
    thr = int(np.floor(float(np.float32(0.3)) * 65536 + 0.5))
    for t in range(3):
        for c in range(20):
            w = orc.philox((c // 8, t, 4, 9), (0x9ABCDEF0, 0x12345678))[c % 8 // 2] >> (16 * (c % 2)) & 0xFFFF
            assert f[t, c] == (65536 / (65536 - thr) if w >= thr else 0.0)


def test_linear_against_autograd():
    rng = np.random.default_rng(2)
    x, W, A, B, dy = (rng.normal(size=n) for n in ((9, 16), (24, 16), (3, 16), (24, 3), (9, 24)))
    f = orc.dropout_factors(9, 16, 0.3, 7, 9)
    got = orc.linear(x, W, A, B, 2.0, f, dy)
    t = [torch.tensor(v, requires_grad=True) for v in (x, A, B)]
    y = t[0] @ torch.tensor(W).T + 2.0 * (t[0] * torch.tensor(f)) @ t[1].T @ t[2].T
    y.backward(torch.tensor(dy))
    for n, v in zip(("y", "dx", "dA", "dB"), (y.detach(), t[0].grad, t[1].grad, t[2].grad)):
        assert np.allclose(got[n], v.numpy(), rtol=1e-12, atol=1e-12), n


@pytest.mark.parametrize("mode", ["top1", "topk"])
def test_router_against_autograd_and_differences(mode):
    rng = np.random.default_rng(3)
    z, dw = rng.normal(size=(11, 5)), rng.normal(size=(11, 2))
    mask = rng.random(11) < 0.6
    args = (2, mode, 0.3, 0.2)
    got = orc.router(z, mask, *args, dw, 0.7, 1.3)
    t = torch.tensor(z, requires_grad=True)
    on = torch.tensor(mask)
    p, n = torch.softmax(t, 1), int(mask.sum())
    idx = torch.tensor(got["topk_idx"].astype(np.int64))
    F = torch.zeros(5, dtype=torch.float64)
    for i in np.flatnonzero(mask):
        for j in range(1 if mode == "top1" else 2):
            F[idx[i, j]] += 1.0 / (n * (1 if mode == "top1" else 2))
    bal = 0.3 * 5 * (F * p[on].sum(0) / n).sum()
    zl = 0.2 * torch.logsumexp(t[on], 1).square().mean()
    w = p[on].gather(1, idx[on])
    w = w / w.sum(1, keepdim=True)
    assert np.allclose(got["loss"], [(bal + zl).item(), bal.item(), zl.item()], rtol=1e-12)
    assert np.allclose(got["topk_w"][mask], w.detach().numpy(), rtol=1e-12)
    (0.7 * bal + 1.3 * zl + (w * torch.tensor(dw)[on]).sum()).backward()
    assert np.allclose(got["dlogits"], t.grad.numpy(), rtol=1e-10, atol=1e-14)

    def total(zz):
        o = orc.router(zz, mask, *args)
        # F is held: it carries no gradient
        P = sum((np.exp(zz[i]) / np.exp(zz[i]).sum() for i in np.flatnonzero(mask)), np.zeros(5)) / n
        return 0.7 * 0.3 * 5 * (F.numpy() * P).sum() + 1.3 * o["loss"][2] + (o["topk_w"] * dw)[mask].sum()
    for i, j in ((0, 0), (3, 2), (int(np.flatnonzero(mask)[0]), 4)):
        e = np.zeros_like(z)
        e[i, j] = 1e-6
        assert abs((total(z + e) - total(z - e)) / 2e-6 - got["dlogits"][i, j]) < 1e-8


def test_router_masks():
    z = np.zeros((4, 3))
    z[1] = np.nan
    got = orc.router(z, [1, 0, 1, 1], 2, "top1", 1.0, 1.0)
    assert np.array_equal(got["counts"], [3, 3, 0]) and np.array_equal(got["topk_idx"], [[0, 1], [-1, -1], [0, 1], [0, 1]])
    assert np.allclose(got["loss"], [1 + np.log(3) ** 2, 1, np.log(3) ** 2])   # F = (1, 0, 0), P = 1/3
    none = orc.router(z, [0] * 4, 2, "topk", 1.0, 1.0)
    assert not none["loss"].any() and not none["counts"].any() and not none["dlogits"].any()
