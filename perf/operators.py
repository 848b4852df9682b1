"""4-bit layers and the answers of a classifier: what programs ask of the library, and the same in plain tensor operations.

Three operators.  `quant` rounds activations to microscaled 4-bit floating point (blocks of 32 channels that share a power
of two; e2m1 elements) and reads them back.  `conv` is a pointwise layer on weights held in that form, which rounds its
activations to it too, with sums in fp32.  `logp` turns logits into log probabilities of given classes, entropy and the
most probable classes.  Sizes come from the classifier and the pointwise layers of MobileNet-v1 and of the benchmark's
sweep, or are the generic ones of wide projections and large vocabularies.
"""
import math

import torch

own = False


def listed():
    return [
        # Pooled features of one image on their way into the classifier: the smallest call.
        dict(name="quant-1x1024-f32", op="quant", m=1, k=1024, dtype="float32"),
        # Half-precision feature maps of nine 14 x 14 images with an odd number of channels.
        dict(name="quant-1764x517-f16", op="quant", m=1764, k=517, dtype="float16"),
        # The activations of a long prompt, bfloat16.
        dict(name="quant-16384x8192-bf16", op="quant", m=16384, k=8192, dtype="bfloat16"),
        # The network's classifier on one image.
        dict(name="conv-m1-1024-1000-f32", op="conv", m=1, k=1024, n=1000, dtype="float32", relu=False),
        # One token through a wide projection: weights are read once and that is the time.
        dict(name="conv-m1-4096-16384-bf16", op="conv", m=1, k=4096, n=16384, dtype="bfloat16", relu=False),
        # A small batch of tokens, an odd number, through a square projection.
        dict(name="conv-m13-8192-8192-f16", op="conv", m=13, k=8192, n=8192, dtype="float16", relu=False),
        # A pointwise layer on three 14 x 14 images, fp32 in and out, output channels that fill no tile.
        dict(name="conv-m588-1024-516-f32", op="conv", m=588, k=1024, n=516, dtype="float32", relu=True),
        # A long prompt through a square projection: bound by arithmetic.
        dict(name="conv-m8192-8192-8192-bf16", op="conv", m=8192, k=8192, n=8192, dtype="bfloat16", relu=False),
        # The classes of 64 images, the serving batch of the benchmark.
        dict(name="logp-64x1000-f32-top5", op="logp", rows=64, v=1000, top=5, dtype="float32", masked=False),
        # One token out of a large vocabulary.
        dict(name="logp-1x131072-bf16-top20", op="logp", rows=1, v=131072, top=20, dtype="bfloat16", masked=False),
        # Constrained decoding: an odd vocabulary of which most is masked out.
        dict(name="logp-37x50257-f16-top8-masked", op="logp", rows=37, v=50257, top=8, dtype="float16", masked=True),
        # Scoring a long text.
        dict(name="logp-2048x131072-bf16-top1", op="logp", rows=2048, v=131072, top=1, dtype="bfloat16", masked=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {c["name"]: work(c) for c in listed()}
    cap = {"quant": most["quant-16384x8192-bf16"], "conv": most["conv-m8192-8192-8192-bf16"], "logp": most["logp-2048x131072-bf16-top1"]}
    while True:
        op, dtype = rng.choice(["quant", "conv", "conv", "logp", "logp"]), rng.choice(["float32", "float16", "bfloat16", "bfloat16"])
        if op == "quant":
            case = dict(op=op, m=_log_int(rng, 1, 65536), k=_log_int(rng, 16, 16384), dtype=dtype)
        elif op == "conv":
            # Channels in multiples of 8, as layers have them, or any number.
            step = rng.choice([1, 8, 8])
            case = dict(op=op, m=_log_int(rng, 1, 8192), k=step * _log_int(rng, 64 // step, 16384 // step),
                        n=step * _log_int(rng, 16 // step, 16384 // step), dtype=dtype, relu=rng.choice([False, True]))
        else:
            case = dict(op=op, rows=_log_int(rng, 1, 4096), v=_log_int(rng, 10, 262144), top=0, dtype=dtype,
                        masked=rng.choice([False, False, True]))
            case["top"] = min(case["v"], rng.choice([0, 1, 5, 20, 32]))
        w = work(case)
        if all(w[key] <= cap[op][key] for key in w):
            return case


def work(case):
    size = 4 if case["dtype"] == "float32" else 2
    if case["op"] == "logp":
        # One exponential, two sums and a comparison a class; indexes and log probabilities of four bytes.
        elements = case["rows"] * case["v"]
        return {"bytes": size * elements + case["rows"] * (4 + 4 + 4 + 8 * case["top"]), "flops": 6 * elements}
    m, k = case["m"], case["k"]
    if case["op"] == "quant":
        # The values, the 4-bit elements with their scales, and the values they stand for.
        return {"bytes": m * (2 * size * k + 17 * -(-k // 32)), "flops": 4 * m * k}
    n = case["n"]
    return {"bytes": size * m * (k + n) + 17 * n * -(-k // 32) + 4 * n, "flops": 2 * m * n * k}


# ---- the 4-bit form in tensor operations ------------------------------------------------------------

def _blocks(x):
    """[rows, channels] as [rows, blocks, 32], the last block filled up with zeros."""
    pad = -x.shape[1] % 32
    return torch.nn.functional.pad(x, (0, pad)).view(x.shape[0], -1, 32)


def _exponent(b):
    """The exponent of a block's scale: two below that of its largest magnitude, not below -127."""
    largest = b.abs().amax(dim=2)
    e = torch.frexp(largest).exponent - 3
    return torch.where(largest == 0, -127, e.clamp(min=-127))


def _round_e2m1(v):
    """The nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with v's sign; ties to the one whose code is even; 6 above 6."""
    a = v.abs()
    q = 0.5 * ((a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float())
    q = q + (a > 2.5).float() + (a >= 3.5).float() + 2 * (a > 5).float()
    return torch.copysign(q, v)


def _power(e):
    """2^e as fp32, e from -127: 2^-127 is below the smallest normal number and its bits are 0x00400000."""
    return torch.where(e > -127, (e + 127) << 23, 0x00400000).to(torch.int32).view(torch.float32)


def _read_back(x):
    """fp32 values -> the values that their 4-bit form stands for, [rows, channels]."""
    b = _blocks(x)
    e = _exponent(b)
    # x / 2^e in two exact factors: 2^-e alone may leave the range of fp32
    half = torch.div(-e, 2, rounding_mode="floor")
    v = b * _power(half)[..., None] * _power(-e - half)[..., None]
    return (_round_e2m1(v) * _power(e)[..., None]).flatten(1)[:, :x.shape[1]]


def _encode(x):
    """fp32 [rows, channels] -> (codes uint8 [rows, 16 * blocks], scales uint8 in tiles of 128 rows by 4 blocks)."""
    b = _blocks(x)
    e = _exponent(b)
    q = _round_e2m1(b * _power(-e)[..., None])       # weights are far from the ends of fp32's range
    a = q.abs()
    code = torch.where(a <= 2, 2 * a, torch.where(a < 6, a + 2, 7)).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    code = code.view(x.shape[0], -1, 2)
    rows, blocks = e.shape
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -blocks % 4, 0, -rows % 128))
    s = s.view(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)
    return (code[..., 0] | (code[..., 1] << 4)).contiguous(), s


def _scale_bytes(scales, rows, blocks):
    """The tiles of scales as [rows, blocks]."""
    tiles = scales.view(-(-rows // 128), -(-blocks // 4), 32, 4, 4)
    return tiles.permute(0, 3, 2, 1, 4).reshape(-(-rows // 128) * 128, -1)[:rows, :blocks]


def _decode(codes, scales, k):
    """The fp32 values of a 4-bit matrix, [rows, k]."""
    rows, blocks = codes.shape[0], codes.shape[1] // 16
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = grid[torch.stack((codes & 15, codes >> 4), dim=2).int()].view(rows, blocks, 32)
    e = _scale_bytes(scales, rows, blocks).int() - 127
    return (v * _power(e)[..., None]).view(rows, -1)[:, :k]


# ---- inputs -----------------------------------------------------------------------------------------

def prepare(case, seed):
    gpu = torch.Generator(device="cuda").manual_seed(seed)
    dtype = getattr(torch, case["dtype"])
    op = case["op"]

    def normal(*shape):
        return torch.randn(shape, generator=gpu, device="cuda")

    if op == "logp":
        rows, v, top = case["rows"], case["v"], case["top"]
        # Logits of a trained model: a wide bulk and a few classes far above it, another number of them in each row.
        x = 2.5 * normal(rows, v)
        peaks = torch.randint(v, (rows, min(v, 8)), generator=gpu, device="cuda")
        x.scatter_add_(1, peaks, 6 + 4 * normal(rows, min(v, 8)))
        targets = torch.where(torch.rand((rows,), generator=gpu, device="cuda") < 0.7, peaks[:, 0],
                              torch.randint(v, (rows,), generator=gpu, device="cuda"))
        if case["masked"]:
            # A grammar allows about a fifth of the classes, the given one among them.
            x.masked_fill_(torch.rand((rows, v), generator=gpu, device="cuda") > 0.2, -math.inf)
            x.scatter_(1, targets[:, None], 2.0)
        return dict(op=op, rows=rows, v=v, top=top, x=x.to(dtype), targets=targets.int(),
                    logprob=torch.empty((rows,), device="cuda"), entropy=torch.empty((rows,), device="cuda"),
                    index=torch.empty((rows, top), device="cuda", dtype=torch.int32), alternatives=torch.empty((rows, top), device="cuda"))
    m, k = case["m"], case["k"]
    # Activations of a trained network: every channel has a spread of its own, a few stand out.
    spread = torch.exp(0.5 * normal(k))
    spread = torch.where(torch.rand((k,), generator=gpu, device="cuda") < 0.005, 20 * spread, spread)
    x = (normal(m, k) * spread).to(dtype)
    codes_bytes, scales_bytes = m * 16 * -(-k // 32), 512 * -(-m // 128) * -(-k // 128)
    state = dict(op=op, m=m, k=k, x=x)
    if op == "quant":
        return dict(state, codes=torch.empty((codes_bytes,), device="cuda", dtype=torch.uint8),
                    scales=torch.empty((scales_bytes,), device="cuda", dtype=torch.uint8), y=torch.empty_like(x))
    n = case["n"]
    w_codes, w_scales = _encode(normal(n, k) / math.sqrt(k))
    return dict(state, n=n, relu=case["relu"], w_codes=w_codes, w_scales=w_scales, bias=0.1 * normal(n),
                y=torch.empty((m, n), device="cuda", dtype=dtype),
                workspace=torch.empty((codes_bytes + scales_bytes,), device="cuda", dtype=torch.uint8))


# ---- one pass ---------------------------------------------------------------------------------------

def run(state):
    op, x = state["op"], state["x"]
    if own:
        import paper_2310_19509_b200 as sbnn
        if op == "quant":
            m, k = state["m"], state["k"]
            sbnn.mxfp4_quantize(x, k, state["codes"], state["scales"], m, k)
            sbnn.mxfp4_dequantize(state["codes"], state["scales"], state["y"], k, m, k)
            return state["y"]
        if op == "conv":
            sbnn.conv1x1_mxfp4(state["w_codes"], state["w_scales"], state["bias"], x, state["k"], state["y"], state["n"],
                               state["m"], state["k"], state["n"], sbnn.SBNN_RELU if state["relu"] else 0, state["workspace"])
            return state["y"]
        sbnn.logprobs(x, state["v"], state["rows"], state["v"], state["targets"], 1, state["logprob"], state["entropy"],
                      state["top"], state["index"], state["alternatives"])
        return {key: state[key] for key in (("logprob", "entropy", "index", "alternatives") if state["top"] else ("logprob", "entropy"))}
    if op == "quant":
        return _read_back(x.float()).to(x.dtype)
    if op == "conv":
        y = _read_back(x.float()) @ _decode(state["w_codes"], state["w_scales"], state["k"]).T + state["bias"]
        return (y.clamp(min=0) if state["relu"] else y).to(x.dtype)
    return _plain_logprobs(x.float(), state["targets"], state["top"])


def _plain_logprobs(x, targets, top):
    largest = x.amax(dim=1, keepdim=True)
    e = (x - largest).exp()
    total = e.sum(dim=1, keepdim=True)
    lse = largest + total.log()
    # 0 * -inf is no part of the mean
    mean = (e * x.clamp(min=torch.finfo(torch.float32).min)).sum(dim=1, keepdim=True) / total
    out = {"logprob": (x.gather(1, targets.long()[:, None]) - lse)[:, 0], "entropy": (lse - mean)[:, 0]}
    if top:
        # Value first, then the lower index: the bits of fp32 in the order of its values, above the index's complement.
        bits = (x + 0.0).view(torch.int32).long()
        key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) | (0xFFFFFFFF - torch.arange(x.shape[1], device=x.device))
        index = 0xFFFFFFFF - (key.topk(top, dim=1).values & 0xFFFFFFFF)
        out["index"], out["alternatives"] = index.int(), x.gather(1, index) - lse
    return out


# ---- the definition in 64 bits -------------------------------------------------------------------------

def exact(case, seed):
    def read_back(x):
        """The values of the 4-bit form by distance from every value it has; of two as near the one with the even code."""
        rows, k = x.shape
        out = torch.empty_like(x)
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=x.device, dtype=torch.float64)
        even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device=x.device)
        for r in range(0, rows, 1024):
            b = torch.nn.functional.pad(x[r:r + 1024], (0, -k % 32)).unflatten(1, (-1, 32))
            largest = b.abs().amax(dim=2, keepdim=True)
            exponent = (largest.view(torch.int64) >> 52) - 1023           # floor(log2): all these are normal numbers in 64 bits
            scale = torch.ldexp(torch.ones_like(largest), exponent.clamp(min=-125) - 2)
            a = (b.abs() / scale).clamp(max=6)
            best, nearest = torch.full_like(a, math.inf), torch.zeros_like(a)
            for i in even_first:
                d = (a - grid[i]).abs()
                nearest = torch.where(d < best, grid[i], nearest)
                best = torch.minimum(best, d)
            out[r:r + 1024] = (torch.where(b < 0, -nearest, nearest) * scale).flatten(1)[:, :k]
        return out

    state = prepare(case, seed)
    x = state["x"].double()
    if case["op"] == "quant":
        return read_back(x)
    if case["op"] == "conv":
        rows, blocks, k = case["n"], -(-case["k"] // 32), case["k"]
        low, high = state["w_codes"] % 16, torch.div(state["w_codes"], 16, rounding_mode="floor")
        code = torch.stack((low, high), dim=2).view(rows, -1).long()
        a = code % 8
        # e2m1: one bit of fraction, two of exponent; exponent 0 holds 0 and 0.5
        value = torch.where(a < 2, a * 0.5, (1 + (a % 2) * 0.5) * torch.tensor([0, 1, 2, 4], device="cuda")[a // 2]) * (1 - 2 * (code // 8)).double()
        r, b = torch.arange(rows, device="cuda")[:, None], torch.arange(blocks, device="cuda")[None, :]
        at = (r // 128 * -(-k // 128) + b // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + b % 4
        scale = torch.ldexp(torch.ones((), device="cuda", dtype=torch.float64), state["w_scales"][at].int() - 127)
        w = (value.view(rows, blocks, 32) * scale[..., None]).view(rows, -1)[:, :k]
        y = read_back(x) @ w.T + state["bias"].double()
        return torch.relu(y) if case["relu"] else y
    out = {"logprob": [], "entropy": [], "index": None, "alternatives": []}
    for r in range(0, case["rows"], 256):
        part, targets = x[r:r + 256], state["targets"][r:r + 256].long()
        logp = torch.log_softmax(part, dim=1)
        out["logprob"].append(logp.gather(1, targets[:, None])[:, 0])
        out["entropy"].append(-torch.where(logp > -math.inf, logp.exp() * logp, 0.0).sum(dim=1))
        if case["top"]:
            out["alternatives"].append(logp.gather(1, part.sort(dim=1, descending=True, stable=True).indices[:, :case["top"]]))
    return {key: torch.cat(parts) if parts else None for key, parts in out.items()}
