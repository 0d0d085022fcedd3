"""Adapters on a 4-bit frozen base: the operators of a fine-tuning step and of serving it, timed through
the library's entry points (paper_2404_15159_amd.binding) and beside their plain form.

Four operators.
  quantize   a frozen matrix W [d_out, d_in] to 4-bit floating-point codes with one scale per group of
             32, 64 or 128 consecutive inputs of a row, and back to values.
  q4         the LoRA linear  y = x W'^T + s (D(x) A^T) B^T  on such a matrix W', forward and backward.
  dropout    the same linear on an ordinary matrix; D drops elements of the adapter's input by a
             counter-based generator, so that no mask is kept between forward and backward.
  router     softmax routing of logits with Eq. 8-9 and a z-loss over the tokens that a mask keeps,
             per-expert counts, and the gradient with respect to the logits.

With `own` false, run() is elementary torch in 32 bits on the same inputs.
"""
import math

import torch

own = False

DEV = "cuda:0"
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)     # magnitudes of the codes 0-7; bit 3 is the sign
MASK32 = 0xFFFFFFFF


def _linear(kind, T, d_in, d_out, r=16, group=64, p=0.0, dtype="bf16", train=True):
    return dict(kind=kind, T=T, d_in=d_in, d_out=d_out, r=r, group=group, p=p, dtype=dtype, train=train)


def _quantize(d_out, d_in, group, dtype="bf16"):
    return dict(kind="quantize", d_out=d_out, d_in=d_in, group=group, dtype=dtype)


def _router(T, N, k, keep, mode="top1", dtype="f32"):
    return dict(kind="router", T=T, N=N, k=k, keep=keep, mode=mode, dtype=dtype)


def listed():
    cases = {
        # one new token through a gate projection of LLaMA-2 7B: latency and the codes' bytes
        "q4_one_token": _linear("q4", 1, 4096, 11008, train=False),
        # one new token of each of 24 sequences through an attention projection of LLaMA-2 13B
        "q4_decode_24": _linear("q4", 24, 5120, 5120, group=128, train=False),
        # a prompt of ragged length through a key projection with shared heads (LLaMA-3 8B)
        "q4_prompt_517": _linear("q4", 517, 4096, 1024, r=8, group=32, train=False),
        # the usual fine-tuning step: 8 sequences of 512 tokens, dropout of the paper's table
        "q4_train_7b": _linear("q4", 4096, 4096, 4096, p=0.05),
        # the largest: a down projection of LLaMA-2 13B under 8 sequences of 1024 tokens
        "q4_train_13b_down": _linear("q4", 8192, 13824, 5120, group=128),
        # 32-bit storage, every size odd: what numerics are debugged on
        "q4_train_small_f32": _linear("q4", 97, 136, 264, r=12, group=32, p=0.1, dtype="f32"),
        # the usual fine-tuning step on an ordinary base
        "dropout_train_7b": _linear("dropout", 4096, 4096, 4096, p=0.05),
        # a short micro-batch with a large adapter
        "dropout_train_333": _linear("dropout", 333, 5120, 5120, r=64, p=0.1),
        # loading a model: one gate projection
        "quantize_gate_7b": _quantize(11008, 4096, 64),
        # a small matrix in 32 bits whose last group is cut
        "quantize_small_f32": _quantize(264, 1000, 128, dtype="f32"),
        # the router of a 16-expert block under 16 padded sequences of 1024 tokens
        "router_16384": _router(16384, 16, 2, keep=0.7),
        # a short padded micro-batch, logits in 16 bits
        "router_300": _router(300, 8, 2, keep=0.5, mode="topk", dtype="bf16"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["q4_forward", "q4_forward", "q4_forward", "q4_train", "q4_train", "dropout",
                       "dropout", "quantize", "router", "router", "f32"])
    if kind == "router":
        N = rng.choice([4, 7, 8, 16, 33, 64])
        return _router(_log(rng, 1, 16384), N, rng.randint(1, min(N, 6)), rng.choice([0.3, 0.7, 1.0]),
                       rng.choice(["top1", "topk"]), rng.choice(["f32", "f32", "bf16"]))
    shape = rng.choice(["7b", "7b_gate", "7b_down", "13b", "kv", "small", "small"])
    d_in, d_out = {"7b": (4096, 4096), "7b_gate": (4096, 11008), "7b_down": (11008, 4096),
                   "13b": (5120, 5120), "kv": (4096, 1024),
                   "small": (8 * _log(rng, 8, 256), 8 * _log(rng, 8, 256))}[shape]
    group, r = rng.choice([32, 64, 64, 128]), rng.choice([2, 4, 8, 12, 16, 16, 32, 64])
    if kind == "quantize":
        return _quantize(d_out, d_in, group, rng.choice(["bf16", "bf16", "f32"]))
    if kind == "f32":
        return _linear("q4", _log(rng, 1, 300), 8 * _log(rng, 4, 64), 8 * _log(rng, 4, 64), r, group,
                       rng.choice([0.0, 0.1]), "f32", rng.random() < 0.6)
    if kind == "q4_forward":
        return _linear("q4", _log(rng, 1, 2048), d_in, d_out, r, group, train=False)
    p = rng.choice([0.05, 0.1, 0.5])
    if kind == "q4_train":
        return _linear("q4", _log(rng, 64, 8192), d_in, d_out, r, group, rng.choice([0.0, p]))
    return _linear("dropout", _log(rng, 64, 8192), d_in, d_out, r, group, p)


# ---- inputs ---------------------------------------------------------------------------------

SCALE = 2.0                          # alpha / r of every configuration
SEED, STREAM = 0x243F6A8885A308D3, 0x13198A2E03707344 >> 8
BALANCE, ZCOEFF, D_BALANCE, D_Z = 0.01, 0.001, 1.0, 1.0


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _group_scales(W, group):
    """One scale per group of a row: the smallest number of six significant bits that is at least a
    sixth of the group's largest magnitude, so that scale times any code is exact in bf16; 0 where that
    magnitude is below 2^-100, NaN where it is not below 2^127."""
    n, K = W.shape
    G = -(-K // group)
    padded = torch.nn.functional.pad(W.float(), (0, G * group - K)).reshape(n, G, group)
    most = padded.abs().amax(2).double()
    low = (1 << 47) - 1              # of a double's 52 bits of fraction, five stay
    s = (((most / 6).view(torch.int64) + low) & ~low).view(torch.float64)
    s = torch.where(most < 2.0 ** -100, torch.zeros_like(s), s)
    s = torch.where(most < 2.0 ** 127, s, torch.full_like(s, math.nan))
    return padded, s.float()


def _codes(padded, s):
    """Nearest magnitude of LEVELS, ties to the even code; compared with (midpoint * scale), which is
    exact, so no quotient is rounded.  A magnitude of 0 has no sign."""
    a, s = padded.abs(), s.unsqueeze(2)
    c = torch.zeros(padded.shape, dtype=torch.uint8, device=padded.device)
    c += a > 0.25 * s
    c += a >= 0.75 * s
    c += a > 1.25 * s
    c += a >= 1.75 * s
    c += a > 2.5 * s
    c += a >= 3.5 * s
    c += a > 5.0 * s
    c[(s == 0).expand_as(c)] = 0
    return torch.where((padded < 0) & (c > 0), c + 8, c)


def _tiled(codes, s, group):
    """Codes [n, G, group] and scales [n, G] as the library keeps them.  A tile is 16 rows by 128 inputs,
    tiles of a row block are consecutive.  codes: byte 16 (16 h + i) + 4 b + c of a tile holds, of row i,
    inputs 32 b + 8 h + 2 c (low half) and the next one; scales: [tile][row][group of the tile].
    Rows and inputs past the end are zeros."""
    n, G, _ = codes.shape
    nt, kt = -(-n // 16), -(-(G * group) // 128)
    c = torch.zeros((nt * 16, kt * 128), dtype=torch.uint8, device=codes.device)
    c[:n, :G * group] = codes.reshape(n, G * group)
    c = c.reshape(nt, 16, kt, 4, 4, 4, 2).permute(0, 2, 4, 1, 3, 5, 6)     # tile, h, row, b, c, half
    c = (c[..., 0] | (c[..., 1] << 4)).contiguous().reshape(-1)
    per = 128 // group
    t = torch.zeros((nt * 16, kt * per), dtype=torch.bfloat16, device=s.device)
    t[:n, :G] = s.to(torch.bfloat16)
    return c, t.reshape(nt, 16, kt, per).permute(0, 2, 1, 3).contiguous().reshape(-1)


class State:
    """Tensors and handles of one problem, held for its lifetime."""


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    td = _dtype(case)

    def nrm(shape, std):
        return (torch.randn(shape, generator=gen, device=DEV) * std).to(td)

    t = {}
    if case["kind"] == "router":
        T, N = case["T"], case["N"]
        z = torch.randn((T, N), generator=gen, device=DEV) * 1.28      # a unit token on N(0, 0.02^2) weights
        z[:, 0] += 0.8
        t["logits"] = z.to(td)
        # sequences of up to 128 tokens, each padded behind its own length
        L = min(128, T)
        lengths = torch.rand((-(-T // L), 1), generator=gen, device=DEV) * 2 * (1 - case["keep"])
        inside = torch.arange(L, device=DEV)[None, :] < (1 - lengths.clamp(max=1.0)) * L
        t["mask"] = (inside.reshape(-1)[:T] if case["keep"] < 1 else torch.ones(T, dtype=torch.bool, device=DEV)).to(torch.uint8)
        t["d_w"] = torch.randn((T, case["k"]), generator=gen, device=DEV)
        return t
    d_in, d_out = case["d_in"], case["d_out"]
    W = nrm((d_out, d_in), 0.02)
    if case["kind"] == "quantize":
        t["W"] = W
        return t
    if case["kind"] == "q4":
        padded, s = _group_scales(W, case["group"])
        t["codes"], t["scales"] = _tiled(_codes(padded, s), s, case["group"])
    else:
        t["W"] = W
    T, r = case["T"], case["r"]
    t["x"] = nrm((T, d_in), 1.0)
    t["A"] = ((torch.rand((r, d_in), generator=gen, device=DEV) * 2 - 1) / math.sqrt(d_in)).to(td)
    t["B"] = nrm((d_out, r), 0.01)
    if case["train"]:
        t["dy"] = nrm((T, d_out), 1.0)
    return t


def prepare(case, seed):
    s = State()
    s.case, s.seed, s.t = case, SEED + seed, _inputs(case, seed)
    if own:
        s.plan = _plan(s)
    return s


# ---- the library's calls ----------------------------------------------------------------------

def _plan(s):
    """Dims, workspace and output buffers that a program keeps between steps."""
    from paper_2404_15159_amd import binding as B
    case, t, p = s.case, s.t, State()
    p.B, p.code = B, B.BF16 if case["dtype"] == "bf16" else B.F32
    td = _dtype(case)

    def empty(shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEV)

    if case["kind"] == "router":
        T, N, k = case["T"], case["N"], case["k"]
        p.dims = B.RouterDims(T, N, k, BALANCE, ZCOEFF, B.AUX_TOP1 if case["mode"] == "top1" else B.AUX_TOPK, p.code)
        p.ws_bytes = B.mixlora_router_loss_workspace_bytes(p.dims)
        p.ws = empty(p.ws_bytes, torch.uint8)
        p.out = dict(loss=empty(3), counts=empty(N, torch.int32), topk_idx=empty((T, k), torch.int32),
                     topk_w=empty((T, k)), dlogits=empty((T, N), td))
        return p
    d_in, d_out, group = case["d_in"], case["d_out"], case["group"]
    if case["kind"] == "quantize":
        p.codes = empty(B.mixlora_q4_code_bytes(d_out, d_in), torch.uint8)
        scales = empty(B.mixlora_q4_scale_bytes(d_out, d_in, group) // 2, torch.bfloat16)
        p.q4 = B.make_q4(p.codes, scales, group)
        p.out = dict(W=empty((d_out, d_in), td), scales=scales)
        return p
    T, r, train = case["T"], case["r"], case["train"]
    p.dims = B.LinearDims(T, d_in, d_out, r, SCALE, p.code)
    p.drop = B.make_dropout(case["p"], s.seed, STREAM) if case["p"] > 0 else None
    if case["kind"] == "q4":
        p.q4 = B.make_q4(t["codes"], t["scales"], group)
        p.ws_bytes = B.mixlora_q4_linear_workspace_bytes(p.dims, group, train)
    else:
        p.W_T = None
        if train:
            p.W_T = empty((d_in, d_out), td)
            B.mixlora_transpose(t["W"], p.W_T, d_out, d_in, p.code)
        p.ws_bytes = B.mixlora_lora_dropout_workspace_bytes(p.dims, train)
    p.ws = empty(p.ws_bytes, torch.uint8)
    p.out = dict(y=empty((T, d_out), td))
    if train:
        p.out.update(dx=empty((T, d_in), td), dA=empty((r, d_in)), dB=empty((d_out, r)))
    return p


def _run_own(s):
    case, t, p = s.case, s.t, s.plan
    B, o = p.B, p.out
    if case["kind"] == "router":
        B.mixlora_router_loss_forward(p.dims, t["logits"], t["mask"], o["loss"], o["counts"], o["topk_idx"],
                                      o["topk_w"], p.ws, p.ws_bytes)
        B.mixlora_router_loss_backward(p.dims, t["logits"], t["mask"], o["topk_idx"], t["d_w"], D_BALANCE, D_Z,
                                       p.ws, p.ws_bytes, o["dlogits"])
    elif case["kind"] == "quantize":
        B.mixlora_q4_quantize(t["W"], p.code, case["d_out"], case["d_in"], p.q4)
        B.mixlora_q4_dequantize(p.q4, case["d_out"], case["d_in"], False, o["W"], p.code)
    elif case["kind"] == "q4":
        B.mixlora_q4_linear_forward(p.dims, p.q4, t["A"], t["B"], p.drop, t["x"], o["y"], p.ws, p.ws_bytes)
        if case["train"]:
            B.mixlora_q4_linear_backward(p.dims, p.q4, t["A"], t["B"], p.drop, t["x"], t["dy"], p.ws,
                                         p.ws_bytes, o["dx"], o["dA"], o["dB"])
    else:
        B.mixlora_lora_dropout_forward(p.dims, t["W"], t["A"], t["B"], p.drop, t["x"], o["y"], p.ws, p.ws_bytes)
        if case["train"]:
            B.mixlora_lora_dropout_backward(p.dims, t["W"], p.W_T, t["A"], t["B"], p.drop, t["x"], t["dy"],
                                            p.ws, p.ws_bytes, o["dx"], o["dA"], o["dB"])
    return o


# ---- the plain form -----------------------------------------------------------------------------

def _plain_values(codes, scales, d_out, d_in, group):
    """W' in 32 bits from the tiles."""
    nt, kt = -(-d_out // 16), -(-d_in // 128)
    pairs = torch.stack((codes & 15, codes >> 4), 1).reshape(nt, kt, 4, 16, 4, 4, 2)
    c = pairs.permute(0, 3, 1, 4, 2, 5, 6).reshape(nt * 16, kt * 128)[:d_out, :d_in]
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=DEV)
    per = 128 // group
    s = scales.float().reshape(nt, kt, 16, per).permute(0, 2, 1, 3).reshape(nt * 16, kt * per)
    return table[c.long()] * s[:d_out].repeat_interleave(group, 1)[:, :d_in]


def _plain_keep(T, width, p, seed, stream):
    """Which elements stay, and the factor of those.  Counter-based generator of Salmon et al. (2011),
    four 32-bit words, seven rounds: counter (column / 8, row, stream), key seed; column c takes bits
    16 (c % 8) .. + 15 of the 128, and stays where they are at least p 2^16."""
    drop = int(math.floor(p * 65536 + 0.5))
    c0 = torch.arange(-(-width // 8), device=DEV, dtype=torch.int64).expand(T, -1)
    c1 = torch.arange(T, device=DEV, dtype=torch.int64)[:, None].expand_as(c0)
    c2, c3 = torch.full_like(c0, stream & MASK32), torch.full_like(c0, stream >> 32)
    k0, k1 = seed & MASK32, seed >> 32
    for _ in range(7):
        m0, m1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((m1 >> 32) & MASK32) ^ c1 ^ k0, m1 & MASK32, ((m0 >> 32) & MASK32) ^ c3 ^ k1, m0 & MASK32
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    words = torch.stack((c0, c1, c2, c3), 2)
    bits = torch.stack((words & 0xFFFF, words >> 16), 3).reshape(T, -1)[:, :width]
    return bits >= drop, 65536 / (65536 - drop)


def _plain_linear(case, t, seed):
    td = _dtype(case)
    x, A, Bm = t["x"].float(), t["A"].float(), t["B"].float()
    if case["kind"] == "q4":
        W = _plain_values(t["codes"], t["scales"], case["d_out"], case["d_in"], case["group"])
    else:
        W = t["W"].float()
    keep, factor = _plain_keep(case["T"], case["d_in"], case["p"], seed, STREAM) if case["p"] > 0 else (None, 1.0)

    def dropped(v):
        return v if keep is None else torch.where(keep, v * factor, torch.zeros_like(v))

    xd = dropped(x)
    P = xd @ A.T
    out = {"y": (x @ W.T + SCALE * (P @ Bm.T)).to(td)}
    if case["train"]:
        dy = t["dy"].float()
        V = dy @ Bm
        out.update(dx=(dy @ W + dropped(SCALE * (V @ A))).to(td), dA=SCALE * (V.T @ xd), dB=SCALE * (dy.T @ P))
    return out


def _plain_router(case, t):
    T, N, k = case["T"], case["N"], case["k"]
    z, on = t["logits"].float(), t["mask"] != 0
    n = on.sum().clamp(min=1).float()
    top = z.amax(1, keepdim=True)
    lse = top + (z - top).exp().sum(1, keepdim=True).log()
    p = (z - lse).exp()
    idx = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    kept = p.gather(1, idx)
    w = kept / kept.sum(1, keepdim=True)
    chosen = torch.nn.functional.one_hot(idx, N) * on[:, None, None]
    counts = chosen.sum((0, 1))
    F = chosen[:, 0].sum(0).float() / n if case["mode"] == "top1" else counts.float() / (n * k)
    P = torch.where(on[:, None], p, torch.zeros_like(p)).sum(0) / n
    balance = BALANCE * N * (F * P).sum()
    z_loss = ZCOEFF * torch.where(on[:, None], lse * lse, torch.zeros_like(lse)).sum() / n
    dz = D_BALANCE * BALANCE * N / n * p * (F - (F * p).sum(1, keepdim=True)) + D_Z * ZCOEFF * 2 / n * lse * p
    dw = t["d_w"]
    dz = dz + torch.zeros_like(z).scatter(1, idx, w * (dw - (w * dw).sum(1, keepdim=True)))
    none = torch.zeros((), device=DEV)
    return dict(loss=torch.stack((balance + z_loss, balance, z_loss)), counts=counts.to(torch.int32),
                topk_idx=torch.where(on[:, None], idx, -1).to(torch.int32), topk_w=torch.where(on[:, None], w, none),
                dlogits=torch.where(on[:, None], dz, none).to(_dtype(case)))


def _plain_quantize(case, t):
    group = case["group"]
    padded, s = _group_scales(t["W"], group)
    c = _codes(padded, s)
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=DEV)
    W = (table[c.long()] * s.unsqueeze(2)).reshape(case["d_out"], -1)[:, :case["d_in"]]
    return dict(W=W.to(_dtype(case)), scales=_tiled(c, s, group)[1])


def run(s):
    if own:
        return _run_own(s)
    if s.case["kind"] == "router":
        return _plain_router(s.case, s.t)
    if s.case["kind"] == "quantize":
        return _plain_quantize(s.case, s.t)
    return _plain_linear(s.case, s.t, s.seed)


def work(case):
    """Inputs read once, outputs written once; the frozen product and its input gradient, the rank-r
    products, a few operations per element for the rest."""
    E = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "router":
        T, N, k = case["T"], case["N"], case["k"]
        return {"bytes": 2 * E * T * N + T * (1 + 12 * k), "flops": 12.0 * T * N}
    d_in, d_out, group = case["d_in"], case["d_out"], case["group"]
    held = d_in * d_out / 2 + 2 * d_out * -(-d_in // group)
    if case["kind"] == "quantize":
        return {"bytes": 2 * E * d_in * d_out + held, "flops": 10.0 * d_in * d_out}
    T, r = case["T"], case["r"]
    by = (held if case["kind"] == "q4" else E * d_in * d_out) + E * (T * (d_in + d_out) + r * (d_in + d_out))
    fl = 2.0 * T * (d_in * d_out + r * (d_in + d_out))
    if case["train"]:
        by += E * T * (d_in + d_out) + 4 * r * (d_in + d_out)
        fl += 2.0 * T * (d_in * d_out + 2 * r * (d_in + d_out))
    return {"bytes": by, "flops": fl}


# ---- 64-bit reference -----------------------------------------------------------------------

def _exact_values(codes, scales, d_out, d_in, group):
    """W' element by element from the place and the bits of its code."""
    kt, per = -(-d_in // 128), 128 // group
    n = torch.arange(d_out, device=DEV)[:, None]
    k = torch.arange(d_in, device=DEV)[None, :]
    tile = (n // 16) * kt + k // 128
    byte = tile * 1024 + ((k % 32) // 8 * 16 + n % 16) * 16 + (k % 128) // 32 * 4 + (k % 8) // 2
    c = (codes[byte] >> (4 * (k % 2)).to(torch.uint8)).int()
    e, m = (c >> 1) & 3, (c & 1).double()
    v = torch.where(e > 0, (1 + m / 2) * (1 << e) / 2, m / 2)
    v = torch.where((c & 8) > 0, -v, v)
    return v * scales.double()[(tile * 16 + n % 16) * per + (k % 128) // group]


def _exact_keep(T, width, p, seed, stream):
    import numpy as np
    low = np.uint64(MASK32)
    blocks = (width + 7) // 8
    x = [np.tile(np.arange(blocks, dtype=np.uint64), T), np.repeat(np.arange(T, dtype=np.uint64), blocks),
         np.full(T * blocks, stream % 2 ** 32, np.uint64), np.full(T * blocks, stream // 2 ** 32, np.uint64)]
    for i in range(7):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        ka, kb = np.uint64((seed + i * 0x9E3779B9) % 2 ** 32), np.uint64((seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32)
        x = [(b >> np.uint64(32)) ^ x[1] ^ ka, b & low, (a >> np.uint64(32)) ^ x[3] ^ kb, a & low]
    bits = np.stack([(w >> np.uint64(16 * h)) & np.uint64(0xFFFF) for w in x for h in (0, 1)], 1)
    drop = round(p * 65536)
    kept = (bits >= drop).reshape(T, blocks * 8)[:, :width]
    return torch.from_numpy(kept).to(DEV).double() * (65536 / (65536 - drop))


def _exact_router(case, t):
    N, k = case["N"], case["k"]
    rows = t["mask"].nonzero()[:, 0]
    z = t["logits"].double()[rows].requires_grad_()
    n = max(1, len(rows))
    p = torch.softmax(z, 1)
    order = torch.argsort(-z.detach(), dim=1, stable=True)[:, :k]
    w = torch.softmax(z.gather(1, order), 1)
    counts = torch.bincount(order.reshape(-1), minlength=N)
    F = (torch.bincount(order[:, 0], minlength=N) if case["mode"] == "top1" else counts / k).double() / n
    balance = BALANCE * N * (F * p.sum(0) / n).sum()
    z_loss = ZCOEFF * torch.logsumexp(z, 1).square().sum() / n
    (D_BALANCE * balance + D_Z * z_loss + (w * t["d_w"].double()[rows]).sum()).backward()
    T = case["T"]
    idx = torch.full((T, k), -1, dtype=torch.int32, device=DEV)
    wide, dz = torch.zeros((T, k), dtype=torch.float64, device=DEV), torch.zeros((T, N), dtype=torch.float64, device=DEV)
    idx[rows], wide[rows], dz[rows] = order.to(torch.int32), w.detach(), z.grad
    return dict(loss=torch.stack((balance + z_loss, balance, z_loss)).detach(), counts=counts.to(torch.int32),
                topk_idx=idx, topk_w=wide, dlogits=dz)


def exact(case, seed):
    t = _inputs(case, seed)
    if case["kind"] == "router":
        return _exact_router(case, t)
    d_in, d_out, group = case["d_in"], case["d_out"], case["group"]
    if case["kind"] == "quantize":
        # the nearest level of every weight, from its definition: the distance to each of them
        import numpy as np
        W = t["W"].double()
        at = torch.arange(d_in, device=DEV) // group
        most = torch.zeros((d_out, int(at[-1]) + 1), dtype=torch.float64, device=DEV)
        most.scatter_reduce_(1, at.expand_as(W), W.abs(), "amax")
        m, e = np.frexp(most.cpu().numpy() / 6)
        s = torch.from_numpy(np.ldexp(np.ceil(m * 64), e - 6)).to(DEV)[:, at]
        best, off = torch.zeros_like(W), W.abs().clone()
        for i in (2, 4, 6, 1, 3, 5, 7):     # even codes first: a tie stays with them
            d = (W.abs() - LEVELS[i] * s).abs()
            better = d < off
            best, off = torch.where(better, LEVELS[i] * s, best), torch.where(better, d, off)
        return dict(W=torch.where(W < 0, -best, best), scales=None)
    x, A, Bm = (t[n].double().requires_grad_(case["train"]) for n in ("x", "A", "B"))
    W = _exact_values(t["codes"], t["scales"], d_out, d_in, group) if case["kind"] == "q4" else t["W"].double()
    xd = x * _exact_keep(case["T"], d_in, case["p"], SEED + seed, STREAM) if case["p"] > 0 else x
    y = torch.cat((x, SCALE * xd @ A.T), 1) @ torch.cat((W, Bm), 1).T
    out = {"y": y.detach()}
    if case["train"]:
        y.backward(t["dy"].double())
        out.update(dx=x.grad, dA=A.grad, dB=Bm.grad)
    return out
