"""Calls of the layers in 8-bit integers and of the group norm, with inputs for each: linear layers from one token to a
long prefill, norms from one image of few positions to many large ones, and a layer behind its norm.

`own` False: the operators in elementary torch operations.  `own` True: the entry points of paper_2308_07641_amd as a
program would call them: weights packed once and kept, workspace and output buffers too.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
SMALLEST = 2.0 ** -100          # tokens whose largest magnitude is below this are scaled as if it were this


def _linear(name, M, N, B, x_dtype="bf16", y_dtype="f32", x_token_major=False, y_token_major=False, bias=False):
    case = {"op": "linear", "M": M, "N": N, "B": B, "x_dtype": x_dtype, "y_dtype": y_dtype, "x_token_major": x_token_major,
            "y_token_major": y_token_major, "bias": bias}
    return dict(case, name=name) if name else case


def _norm(name, images, P, C, groups, act, x_dtype="bf16", y_dtype="bf16", y_token_major=True):
    case = {"op": "norm", "images": images, "P": P, "C": C, "groups": groups, "act": act, "x_dtype": x_dtype, "y_dtype": y_dtype,
            "y_token_major": y_token_major}
    return dict(case, name=name) if name else case


def _block(name, images, P, C, groups, act, M, x_dtype="bf16"):
    # (bf16 results: a value of the norm that lies within an fp32 rounding of the border between two codes may take either)
    case = {"op": "block", "images": images, "P": P, "C": C, "groups": groups, "act": act, "M": M, "x_dtype": x_dtype}
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest layer, one fp32 vector: what a call costs when there is next to nothing to do
        _linear("int8_tiny", 256, 256, 1, x_dtype="f32"),
        # one decoding step of a single sequence through a feed-forward layer of a large language model
        _linear("int8_decode", 16384, 4096, 1),
        # the same step for a batch of 16 sequences, as a row-per-token program with a bf16 residual stream calls it
        _linear("int8_decode_b16", 16384, 4096, 16, y_dtype="bf16", x_token_major=True, y_token_major=True, bias=True),
        # a prefill chunk of the same layer
        _linear("int8_prefill_b256", 16384, 4096, 256, y_dtype="bf16", x_token_major=True, y_token_major=True, bias=True),
        # the prefill of a very large layer: bound by the matrix cores
        _linear("int8_prefill_b2048", 36864, 9216, 2048, y_dtype="bf16", x_token_major=True, y_token_major=True, bias=True),
        # the pointwise layer of a convolutional network at many positions, feature-major like its convolutions
        _linear("int8_pointwise", 2048, 512, 12544),
        # activations that arrive in fp32, odd sizes everywhere
        _linear("int8_fp32_odd", 1000, 2047, 197, x_dtype="f32", x_token_major=True, y_token_major=True, bias=True),
        # the norm of the innermost stage of an image network, one image: latency
        _norm("norm_8x8", 1, 64, 320, 32, "silu"),
        # the same network's middle stage, a batch of images
        _norm("norm_32x32", 8, 1024, 640, 32, "silu"),
        # its outermost stage at full resolution: bound by memory
        _norm("norm_128x128", 16, 16384, 256, 32, "silu"),
        # odd sizes in fp32, written channel by channel for a convolution behind it
        _norm("norm_7x7_fp32", 5, 49, 1155, 21, "gelu", x_dtype="f32", y_dtype="f32", y_token_major=False),
        # a layer behind its norm row by row (layer norm: one position, one group), 2048 tokens of a language model
        _block("norm_int8_rows", 2048, 1, 4096, 1, "none", 4096),
    ]


def _log(rng, lo, hi):
    """A size spread over the logarithm of lo .. hi; every third one is a multiple of 64 where the range allows."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 128 and rng.random() < 1 / 3:
        v = v // 64 * 64
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.random()
    if kind < 0.5:
        # layers of 16 to 36864 rows and 16 to 16384 features, 1 to 16384 tokens
        while True:
            c = _linear(None, _log(rng, 16, 36864), _log(rng, 16, 16384), _log(rng, 1, 16384), rng.choice(("bf16", "bf16", "f32")),
                        rng.choice(("bf16", "f32")), rng.random() < 0.6, rng.random() < 0.6, rng.random() < 0.5)
            if c["M"] * c["N"] * c["B"] <= 3 << 37 and max(c["M"], c["N"]) * c["B"] <= 1 << 27:
                return c
    # 1 to 64 images (rows: 1 to 4096) of 1 to 16384 positions, 1 to 64 groups of 1 to 128 channels
    while True:
        P = 1 if kind > 0.9 else _log(rng, 2, 16384)
        images = _log(rng, 1, 4096 if P == 1 else 64)
        groups = rng.choice((1, 1, 8, 32)) if P == 1 else rng.choice((1, 4, 21, 32, 32, 32, 64))
        C = groups * _log(rng, 1, 8192 // groups if P == 1 else 128)
        if C >= 8 and images * P * C <= 1 << 26:
            break
    act, x_dtype = rng.choice(("none", "silu", "silu", "gelu", "relu")), rng.choice(("bf16", "bf16", "f32"))
    if kind > 0.8:
        M = _log(rng, 16, 8192)
        if M * C * images * P <= 1 << 38 and M * images * P <= 1 << 27:
            return _block(None, images, P, C, groups, act, M, x_dtype)
    return _norm(None, images, P, C, groups, act, x_dtype, rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.75)


def _torch_type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _weights(g, M, N):
    """Rows of normal weights as a program gets them from a checkpoint in 8 bits: codes and a scale for each row."""
    w = torch.randn((M, N), generator=g, device=DEV)
    top = w.abs().amax(1)
    codes = w.mul_((127 / top)[:, None]).round_().to(torch.int8)
    return codes, top / (127 * math.sqrt(N))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    if case["op"] == "linear":
        M, N, B = case["M"], case["N"], case["B"]
        x = torch.randn((B, N) if case["x_token_major"] else (N, B), generator=g, device=DEV)
        # a few features far larger than the rest, as the activations of language models have them
        far = torch.randint(0, N, (max(1, N // 256),), generator=g, device=DEV)
        if case["x_token_major"]:
            x[:, far] *= 8
        else:
            x[far] *= 8
        s["x"] = x.to(_torch_type(case["x_dtype"]))
        s["bias"] = torch.randn(M, generator=g, device=DEV) if case["bias"] else None
    else:
        images, P, C = case["images"], case["P"], case["C"]
        x = torch.randn((images, P, C), generator=g, device=DEV)
        # channels with means and spreads of their own
        x = x * (0.5 + torch.rand(C, generator=g, device=DEV)) + torch.randn(C, generator=g, device=DEV)
        s["x"] = x.to(_torch_type(case["x_dtype"]))
        s["gamma"] = 1 + 0.2 * torch.randn(C, generator=g, device=DEV)
        s["beta"] = 0.2 * torch.randn(C, generator=g, device=DEV)
    if case["op"] != "norm":
        s["w"], s["t"] = _weights(g, case["M"], case["N"] if case["op"] == "linear" else case["C"])
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    import paper_2308_07641_amd as tsvd
    f32, bf16, fm, tm = tsvd.TSVD_F32, tsvd.TSVD_BF16, tsvd.TSVD_FEATURE_MAJOR, tsvd.TSVD_TOKEN_MAJOR
    s["tsvd"] = tsvd
    if s["op"] != "norm":
        s["handle"] = tsvd.tsvd_int8_pack(s["w"], s["t"])
    if s["op"] == "linear":
        s["x_layout"], s["y_layout"] = tm if s["x_token_major"] else fm, tm if s["y_token_major"] else fm
        s["y_code"] = bf16 if s["y_dtype"] == "bf16" else f32
        x_code = bf16 if s["x_dtype"] == "bf16" else f32
        nbytes = tsvd.tsvd_int8_workspace_bytes(s["handle"], s["B"], x_code, s["x_layout"])
        s["y"] = torch.empty((s["B"], s["M"]) if s["y_token_major"] else (s["M"], s["B"]), dtype=_torch_type(s["y_dtype"]), device=DEV)
    else:
        s["act_code"] = {"none": tsvd.TSVD_ACT_NONE, "relu": tsvd.TSVD_ACT_RELU, "silu": tsvd.TSVD_ACT_SILU, "gelu": tsvd.TSVD_ACT_GELU}[s["act"]]
        nbytes = tsvd.tsvd_group_norm_workspace_bytes(s["images"], s["P"], s["C"], s["groups"])
        rows = s["images"] * s["P"]
        if s["op"] == "norm":
            s["y_code"], s["y_layout"] = bf16 if s["y_dtype"] == "bf16" else f32, tm if s["y_token_major"] else fm
            shape = (s["images"], s["P"], s["C"]) if s["y_token_major"] else (s["C"], s["images"], s["P"])
            s["y"] = torch.empty(shape, dtype=_torch_type(s["y_dtype"]), device=DEV)
        else:
            s["codes"] = torch.empty((rows, tsvd.tsvd_int8_row_bytes(s["C"])), dtype=torch.int8, device=DEV)[:, :s["C"]]
            s["scales"] = torch.empty(rows, dtype=torch.float32, device=DEV)
            s["y"] = torch.empty((rows, s["M"]), dtype=torch.bfloat16, device=DEV)
    s["workspace"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)


def run(s):
    if own:
        tsvd = s["tsvd"]
        if s["op"] == "linear":
            return tsvd.tsvd_int8_forward(s["handle"], s["x"], x_layout=s["x_layout"], bias=s["bias"], y=s["y"], y_dtype=s["y_code"],
                                          y_layout=s["y_layout"], workspace=s["workspace"])
        if s["op"] == "norm":
            return tsvd.tsvd_group_norm(s["x"], s["groups"], s["gamma"], s["beta"], eps=EPS, act=s["act_code"], y=s["y"], y_dtype=s["y_code"],
                                        y_layout=s["y_layout"], workspace=s["workspace"])
        codes, scales = tsvd.tsvd_group_norm_int8(s["x"], s["groups"], s["gamma"], s["beta"], eps=EPS, act=s["act_code"], codes=s["codes"],
                                                  scales=s["scales"], workspace=s["workspace"])
        return tsvd.tsvd_int8_product(s["handle"], codes, scales, y=s["y"], y_dtype=tsvd.TSVD_BF16, y_layout=tsvd.TSVD_TOKEN_MAJOR)
    if s["op"] == "linear":
        y = _plain_layer(s["x"] if s["x_token_major"] else s["x"].t(), s["w"], s["t"], s["bias"])
        return (y if s["y_token_major"] else y.t()).to(_torch_type(s["y_dtype"])).contiguous()
    if s["op"] == "norm":
        y = _plain_norm(s["x"].float(), s)
        return (y if s["y_token_major"] else y.permute(2, 0, 1)).to(_torch_type(s["y_dtype"])).contiguous()
    # (64 bits up to the codes: values next to the border between two of them)
    y = _plain_norm(s["x"].double(), s)
    return _plain_layer(y.reshape(-1, s["C"]).float(), s["w"], s["t"], None).to(torch.bfloat16)


def _plain_layer(x, w, t, bias):
    top = x.float().abs().amax(1).clamp_min(SMALLEST).double()
    scale, inverse = (top / 127).float(), (127 / top).float()
    codes = (x.double() * inverse.double()[:, None]).round().float()      # (in 64 bits: ties and values next to them)
    y = codes @ w.float().t() * scale[:, None] * t
    return y if bias is None else y + bias


def _plain_norm(x, s):
    images, P, C = x.shape
    v = x.reshape(images, P, s["groups"], C // s["groups"])
    v = v - v.mean((1, 3), keepdim=True)
    v = v / (v.square().mean((1, 3), keepdim=True) + EPS).sqrt()
    y = v.reshape(images, P, C) * s["gamma"] + s["beta"]
    if s["act"] == "relu":
        return y.clamp_min(0)
    if s["act"] == "silu":
        return y / (1 + torch.exp(-y))
    if s["act"] == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "linear":
        M, N, B = case["M"], case["N"], case["B"]
        moved = M * N + 4 * M + N * B * size[case["x_dtype"]] + M * B * size[case["y_dtype"]] + (4 * M if case["bias"] else 0)
        return {"bytes": moved, "flops": 2 * M * N * B}
    values, C = case["images"] * case["P"] * case["C"], case["C"]
    if case["op"] == "norm":
        return {"bytes": values * (size[case["x_dtype"]] + size[case["y_dtype"]]) + 8 * C, "flops": 10 * values}
    M, rows = case["M"], case["images"] * case["P"]
    return {"bytes": values * size[case["x_dtype"]] + 8 * C + M * C + 4 * M + 2 * M * rows, "flops": 2 * M * values + 10 * values}


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].to(torch.float64)
    if case["op"] == "linear":
        rows = x if case["x_token_major"] else x.transpose(0, 1)
    else:
        # a row for each group of an image
        G, C = case["groups"], case["C"]
        by_group = x.unflatten(2, (G, C // G)).transpose(1, 2).flatten(2)
        var, mean = torch.var_mean(by_group, dim=2, correction=0, keepdim=True)
        h = ((by_group - mean) * torch.rsqrt(var + EPS)).unflatten(2, (case["P"], C // G)).transpose(1, 2).flatten(2)
        h = torch.addcmul(s["beta"].double(), h, s["gamma"].double())
        if case["act"] == "relu":
            h = torch.where(h > 0, h, torch.zeros_like(h))
        elif case["act"] == "silu":
            h = h * torch.special.expit(h)
        elif case["act"] == "gelu":
            h = h * torch.special.ndtr(h)
        if case["op"] == "norm":
            return h if case["y_token_major"] else h.movedim(2, 0).contiguous()
        rows = h.flatten(0, 1)
    # a code is the whole number next to the value times the stored (32-bit) 127 / largest; the stored scale is 1 / 127 of the largest
    largest = torch.maximum(rows.amax(1), -rows.amin(1)).clamp(min=SMALLEST).to(torch.float32).double()
    q = torch.round(rows * (127 / largest).to(torch.float32).unsqueeze(1))
    y = torch.empty((rows.shape[0], case["M"]), dtype=torch.float64, device=rows.device)
    for m in range(0, case["M"], 4096):
        part = s["w"][m:m + 4096].double()
        y[:, m:m + 4096] = torch.mm(q, part.t().contiguous()) * torch.outer(largest / 127, s["t"][m:m + 4096].double())
    if case.get("bias"):
        y += s["bias"]
    return y if case["op"] == "block" or case["y_token_major"] else y.t().contiguous()
