"""Timed cases of the microscaled operators: the feed-forward block of a language model, trained and served.

A microscaled row is cut into blocks of 32 values with one power of two each: 4-bit floating point (E2M1: 0, 0.5, 1,
1.5, 2, 3, 4, 6) for what enters the product, 8-bit integers (steps of 1/64) for what the backward pass reads again.

Kinds of cases:
  codec   a tensor quantised to codes and scales and the values these stand for
  linear  y = Q4(x) W4^T + b on weights quantised once: serving, from one token to a long prompt
  train   a training step of that layer: forward with x kept in 8 bits, then dx, dw and db
  act     f(gate) * up, forward with both inputs kept in 8 bits, and backward from what was kept
  norm    layer norm, forward with its input kept in 8 bits, and backward from that with both weights' gradients

Where ``own`` is false ``run`` computes the operators in elementary torch operations in 32 bits; where it is true it calls
the library.  ``exact`` is the same from the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 32


def _code_pitch(K, bits):            # bytes of a row of codes: whole units of 128 values
    return -(-K // 128) * 16 * bits


def _scale_pitch(K):                 # bytes of a row of scales: whole units of 16
    return -(-K // 512) * 16


# ------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token's activations on their way into a product
        dict(name="codec_token", kind="codec", bits=4, rows=1, K=4096, type="bf16", pad=0),
        # a checkpoint of an odd batch, taken from columns of a wider tensor
        dict(name="codec_ragged", kind="codec", bits=8, rows=999, K=4609, type="f16", pad=7),
        # a layer's weights, quantised once when the model is loaded
        dict(name="codec_weights", kind="codec", bits=4, rows=16384, K=8192, type="bf16", pad=0),
        # a single token through a layer: the decoding loop
        dict(name="linear_token", kind="linear", M=1, N=4096, K=4096, type="bf16", bias=False),
        # a serving batch on a layer of odd sizes
        dict(name="linear_batch", kind="linear", M=37, N=5001, K=2309, type="f16", bias=True),
        # a long prompt
        dict(name="linear_prompt", kind="linear", M=8192, N=8192, K=4096, type="bf16", bias=False),
        # a training step of a small layer of odd sizes
        dict(name="train_small", kind="train", M=515, N=771, K=577, type="bf16", bias=True),
        # a training step of a large one
        dict(name="train_large", kind="train", M=8192, N=4096, K=4096, type="bf16", bias=True),
        # the gated activation of a short sequence, and of a full batch
        dict(name="act_small", kind="act", f="gelu", rows=77, K=2049, type="f32"),
        dict(name="act_large", kind="act", f="silu", rows=8192, K=8192, type="bf16"),
        # the norm before the block, likewise
        dict(name="norm_small", kind="norm", rows=130, K=1000, type="f16"),
        dict(name="norm_large", kind="norm", rows=16384, K=4096, type="bf16"),
    ]


def _spread(rng, lo, hi):
    """A size between lo and hi, even over its logarithm; half of the larger ones are whole multiples of 64."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 128 and rng.random() < 0.5:
        n = n // 64 * 64
    n = max(lo, min(hi, n))
    return n if n != 3072 else n + 1


def draw(rng):
    kind = rng.choice(["codec", "linear", "train", "act", "norm"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "codec":
        K = _spread(rng, 1, 16384)
        rows = _spread(rng, 1, min(65536, (1 << (26 if t == "f32" else 27)) // K))
        return dict(kind=kind, bits=rng.choice([4, 8]), rows=rows, K=K, type=t, pad=rng.choice([0, 0, 1, 8]))
    if kind == "linear":
        N, K = _spread(rng, 16, 8192), _spread(rng, 32, 8192)
        M = _spread(rng, 1, min(8192, (1 << 38) // (N * K)))
        return dict(kind=kind, M=M, N=N, K=K, type=t, bias=rng.random() < 0.5)
    if kind == "train":
        N, K = _spread(rng, 16, 4096), _spread(rng, 32, 4096)
        M = _spread(rng, 1, min(8192, (1 << (35 if t == "f32" else 36)) // (N * K)))
        return dict(kind=kind, M=M, N=N, K=K, type=t, bias=rng.random() < 0.5)
    K = _spread(rng, 16, 8192 if kind == "norm" else 16384)
    rows = _spread(rng, 1, min(32768, (1 << (25 if t == "f32" else 26)) // K))
    if kind == "act":
        return dict(kind=kind, f=rng.choice(["silu", "gelu"]), rows=rows, K=K, type=t)
    return dict(kind=kind, rows=rows, K=K, type=t)


def work(case):
    e, k = BYTES[case["type"]], case["kind"]
    if k in ("linear", "train"):
        M, N, K = case["M"], case["N"], case["K"]
        w = N * K * 17 / 32
        if k == "linear":
            return {"bytes": e * M * K + w + e * M * N + 4 * N * case["bias"], "flops": 2 * M * N * K}
        # x and dy in, the weights' codes, y, dx, dw and db out; the checkpoint goes out and comes back
        return {"bytes": e * M * (2 * K + 2 * N) + w + 4 * N * K + 4 * N + 2 * M * K * 33 / 32, "flops": 6 * M * N * K}
    n = case["rows"] * case["K"]
    if k == "codec":
        return {"bytes": n * (2 * e + (17 / 32 if case["bits"] == 4 else 33 / 32)), "flops": 4 * n}
    if k == "act":                   # gate, up, dy in; y, dgate, dup out; two checkpoints out and back
        return {"bytes": n * (6 * e + 4 * 33 / 32), "flops": 50 * n}
    return {"bytes": n * (4 * e + 2 * 33 / 32), "flops": 20 * n}


# ------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, k = TYPES[case["type"]], case["kind"]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(scale)

    def activations(rows, K, pad=0):
        """Channels of different spread, a few of them much wider than the rest, some with an offset."""
        spread = torch.exp(0.5 * normal(K + pad))
        spread *= torch.where(torch.rand(K + pad, generator=g, device="cuda") < 0.01, 16.0, 1.0)
        return (normal(rows, K + pad) * spread + 0.2 * normal(K + pad)).to(t)[:, pad:]

    if k == "codec":
        return dict(x=activations(case["rows"], case["K"], case["pad"]))
    if k in ("linear", "train"):
        M, N, K = case["M"], case["N"], case["K"]
        d = dict(x=activations(M, K), w=normal(N, K, scale=K ** -0.5), b=normal(N) if case["bias"] else None)
        if k == "train":
            d["dy"] = normal(M, N, scale=0.01).to(t)
        return d
    rows, K = case["rows"], case["K"]
    d = dict(x=activations(rows, K), dy=normal(rows, K, scale=0.01).to(t))
    if k == "act":
        d["up"] = normal(rows, K).to(t)
    else:
        d["gamma"], d["beta"] = 1.0 + 0.2 * normal(K), 0.2 * normal(K)
    return d


def prepare(case, seed):
    """The inputs; for a layer its weights' codes and scales; and the results' and the library's buffers."""
    s = _inputs(case, seed)
    s["case"], k, t = case, case["kind"], TYPES[case["type"]]
    if k in ("linear", "train"):
        s["w_codes"], s["w_scales"] = _store4(s.pop("w"))
    if not own:
        return s
    import paper_2105_11010_amd as sq

    def empty(*shape, dtype=t):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def coded(rows, K, bits):
        return (empty(rows, sq.sparq_mx_code_bytes(K, bits), dtype=torch.uint8),
                empty(rows, sq.sparq_mx_scale_bytes(K), dtype=torch.uint8))

    if k == "codec":
        s["codes"], s["scales"] = coded(case["rows"], case["K"], case["bits"])
        s["y"] = empty(case["rows"], case["K"])
    elif k == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        s["y"] = empty(M, N)
        s["ws"] = empty(sq.sparq_mx_linear_workspace_bytes(M, N, K), dtype=torch.uint8)
    elif k == "train":
        M, N, K = case["M"], case["N"], case["K"]
        s["x4"], s["x8"] = coded(M, K, 4), coded(M, K, 8)
        s["y"], s["dx"] = empty(M, N), empty(M, K)
        s["dw"], s["db"] = empty(N, K, dtype=torch.float32), empty(N, dtype=torch.float32)
        s["ws"] = empty(max(sq.sparq_mx_gemm_workspace_bytes(M, N, K), sq.sparq_mx_linear_dx_workspace_bytes(M, N, K),
                            sq.sparq_mx_linear_dw_workspace_bytes(M, N, K)), dtype=torch.uint8)
    else:
        rows, K = case["rows"], case["K"]
        s["x8"], s["y"], s["dx"] = coded(rows, K, 8), empty(rows, K), empty(rows, K)
        if k == "act":
            s["up8"], s["dup"] = coded(rows, K, 8), empty(rows, K)
        else:
            s["mean"], s["rstd"] = empty(rows, dtype=torch.float32), empty(rows, dtype=torch.float32)
            s["dgamma"], s["dbeta"] = empty(K, dtype=torch.float32), empty(K, dtype=torch.float32)
            s["ws"] = empty(sq.sparq_mx_norm_grad_workspace_bytes(rows, K), dtype=torch.uint8)
    return s


# ------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------
EPS = 1e-5


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2105_11010_amd as sq
    case, k = s["case"], s["case"]["kind"]
    if k == "codec":
        p = "codes%d" % case["bits"], "scales%d" % case["bits"]
        sq.sparq_mx_quantize(s["x"], **{p[0]: s["codes"], p[1]: s["scales"]})
        sq.sparq_mx_dequantize(s["codes"], s["scales"], case["bits"], s["y"])
        return s["y"]
    if k == "linear":
        sq.sparq_mx_linear(s["x"], s["w_codes"], s["w_scales"], s["y"], bias=s["b"], workspace=s["ws"])
        return s["y"]
    if k == "train":
        x4, x8 = s["x4"], s["x8"]
        sq.sparq_mx_quantize(s["x"], codes4=x4[0], scales4=x4[1], codes8=x8[0], scales8=x8[1])
        sq.sparq_mx_gemm(x4[0], x4[1], s["w_codes"], s["w_scales"], case["K"], s["y"], bias=s["b"], workspace=s["ws"])
        sq.sparq_mx_linear_dx(s["dy"], s["w_codes"], s["w_scales"], s["dx"], workspace=s["ws"])
        sq.sparq_mx_linear_dw(s["dy"], x8[0], x8[1], s["dw"], db=s["db"], workspace=s["ws"])
        return [s["y"], s["dx"], s["dw"], s["db"]]
    if k == "act":
        kept = dict(gate_codes=s["x8"][0], gate_scales=s["x8"][1], up_codes=s["up8"][0], up_scales=s["up8"][1])
        sq.sparq_mx_act(case["f"], s["x"], s["y"], up=s["up"], **kept)
        sq.sparq_mx_act_grad(case["f"], s["dy"], dgate=s["dx"], dup=s["dup"], **kept)
        return [s["y"], s["dx"], s["dup"]]
    c, sc = s["x8"]
    sq.sparq_mx_norm(s["x"], s["gamma"], s["beta"], EPS, s["y"], mean=s["mean"], rstd=s["rstd"], codes=c, scales=sc)
    sq.sparq_mx_norm_grad(s["dy"], c, sc, s["mean"], s["rstd"], s["gamma"], s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"],
                          workspace=s["ws"])
    return [s["y"], s["dx"], s["dgamma"], s["dbeta"]]


def _blocks(x):
    """x in 32 bits as [rows][blocks][32] and each block's floor(log2 max|x|); blocks of zeros get -127."""
    rows, K = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -K % BLOCK)).view(rows, -1, BLOCK)
    top = b.abs().amax(-1, keepdim=True)
    return b, torch.where(top > 0, torch.frexp(top)[1] - 1, -127)


def _pow2(e):
    """2^e, to the bit (e beyond a normal number's exponent: blocks of zeros only)."""
    return (e.clamp(-126, 127).int() + 127 << 23).view(torch.float32)


def _values4(x):
    """The 4-bit values of x in units of the block's scale, and the scale's exponent."""
    b, e = _blocks(x)
    e = (e - 2).clamp(-127, 127)
    a = b * _pow2(-e)
    step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
    return (torch.round(a / step) * step).clamp(-6, 6), e


def _values8(x):
    b, e = _blocks(x)
    e = e.clamp(-127, 127)
    return torch.round(b * _pow2(-e) * 64).clamp(-127, 127) / 64, e


def _whole(v, e, K):
    return (v * _pow2(e)).flatten(1)[:, :K]


def _store4(w):
    """Codes and scales of w as a model file holds them: two values a byte, the lower one first."""
    N, K = w.shape
    v, e = _values4(w)
    a = v.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (v < 0).to(torch.uint8) << 3
    code = code.view(N, -1, 2)
    codes = torch.zeros(N, _code_pitch(K, 4), dtype=torch.uint8, device=w.device)
    codes[:, : code.shape[1]] = code[..., 0] | code[..., 1] << 4
    scales = torch.zeros(N, _scale_pitch(K), dtype=torch.uint8, device=w.device)
    scales[:, : e.shape[1]] = (e[..., 0] + 127).to(torch.uint8)
    return codes, scales


_VALUE4 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _read4(codes, scales, K):
    """The values that codes and scales stand for."""
    table = torch.tensor(_VALUE4, device=codes.device)
    blocks = -(-K // BLOCK)
    c = codes[:, : 16 * blocks].int()
    v = torch.stack((table[c & 15], table[c >> 4]), -1).view(c.shape[0], blocks, BLOCK)
    return _whole(v, scales[:, :blocks, None].int() - 127, K)


def _run_plain(s):
    case, k = s["case"], s["case"]["kind"]
    t, K = TYPES[case["type"]], case["K"]
    if k == "codec":
        return _whole(*(_values4 if case["bits"] == 4 else _values8)(s["x"]), K).to(t)
    if k in ("linear", "train"):
        w = _read4(s["w_codes"], s["w_scales"], K)
        y = _whole(*_values4(s["x"]), K) @ w.t()
        if s["b"] is not None:
            y = y + s["b"]
        if k == "linear":
            return y.to(t)
        kept, dy = _whole(*_values8(s["x"]), K), s["dy"].float()
        return [y.to(t), (dy @ w).to(t), dy.t() @ kept, dy.sum(0)]
    kept, x, dy = _whole(*_values8(s["x"]), K), s["x"].float(), s["dy"].float()
    if k == "act":
        up, kept_up = s["up"].float(), _whole(*_values8(s["up"]), K)
        value, slope = _act(case["f"], kept)
        return [(_act(case["f"], x)[0] * up).to(t), (dy * kept_up * slope).to(t), (dy * value).to(t)]
    mean = x.mean(1, keepdim=True)
    rstd = torch.rsqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    y = (x - mean) * rstd * s["gamma"] + s["beta"]
    xh, d = (kept - mean) * rstd, dy * s["gamma"]
    dx = rstd * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
    return [y.to(t), dx.to(t), (dy * xh).sum(0), dy.sum(0)]


def _act(f, x):
    """f(x) and f'(x)."""
    if f == "silu":
        sig = 1 / (1 + torch.exp(-x))
        return x * sig, sig * (1 + x * (1 - sig))
    cdf = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
    return x * cdf, cdf + x * torch.exp(-0.5 * x * x) * (0.5 / math.pi) ** 0.5


# ------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------------------
def _exact_quantised(x, bits):
    """Each block's values on the grid of its power of two: nearest, ties to the even code, at most the largest code."""
    x = x.double()
    rows, K = x.shape
    blocks = -(-K // BLOCK)
    padded = torch.zeros(rows, blocks * BLOCK, dtype=torch.float64, device=x.device)
    padded[:, :K] = x
    b = padded.reshape(rows * blocks, BLOCK)
    largest = b.abs().max(1).values
    power = torch.pow(2.0, torch.floor(torch.log2(largest.clamp_min(2.0 ** -149))))
    power = torch.where(power > largest, power / 2, power)          # (a logarithm rounded up to a whole number)
    power = torch.where(power * 2 <= largest, power * 2, power)
    if bits == 8:
        unit = power.clamp_min(2.0 ** -127)[:, None] / 64
        q = torch.round(b / unit).clamp(-127, 127) * unit
    else:
        unit = (power / 4).clamp_min(2.0 ** -127)[:, None]
        grid = torch.tensor(_VALUE4[:8], dtype=torch.float64, device=x.device)
        between = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device=x.device)
        a = b.abs() / unit
        up, down = torch.bucketize(a, between, right=True), torch.bucketize(a, between, right=False)
        q = torch.copysign(grid[torch.where(up % 2 == 0, up, down)], b) * unit
    return q.reshape(rows, blocks * BLOCK)[:, :K]


def exact(case, seed):
    d, k = _inputs(case, seed), case["kind"]
    if k == "codec":
        return _exact_quantised(d["x"], case["bits"])
    if k in ("linear", "train"):
        w = _exact_quantised(d["w"], 4)
        y = torch.matmul(_exact_quantised(d["x"], 4), w.T)
        if d["b"] is not None:
            y += d["b"].double()
        if k == "linear":
            return y
        dy = d["dy"].double()
        return [y, torch.matmul(dy, w), torch.matmul(dy.T, _exact_quantised(d["x"], 8)), dy.sum(0)]
    x, dy, kept = d["x"].double(), d["dy"].double(), _exact_quantised(d["x"], 8)
    if k == "act":
        up, kept_up = d["up"].double(), _exact_quantised(d["up"], 8)
        if case["f"] == "silu":
            s0, s1 = torch.special.expit(x), torch.special.expit(kept)
            value, slope = kept * s1, s1 + kept * s1 * torch.special.expit(-kept)
        else:
            s0, s1 = torch.special.ndtr(x), torch.special.ndtr(kept)
            value, slope = kept * s1, s1 + kept * torch.exp(-kept.square() / 2) / math.sqrt(2 * math.pi)
        return [x * s0 * up, dy * kept_up * slope, dy * value]
    mean = x.sum(1) / x.shape[1]
    var = (x - mean[:, None]).square().sum(1) / x.shape[1]
    sigma = torch.sqrt(var + EPS)[:, None]
    gamma, beta = d["gamma"].double(), d["beta"].double()
    xh = (kept - mean[:, None]) / sigma
    d = dy * gamma
    n = x.shape[1]
    dx = (n * d - d.sum(1, keepdim=True) - xh * (d * xh).sum(1, keepdim=True)) / (n * sigma)
    return [(x - mean[:, None]) / sigma * gamma + beta, dx, (dy * xh).sum(0), dy.sum(0)]
