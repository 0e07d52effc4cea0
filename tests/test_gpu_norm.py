"""Group norm with an activation against a plain implementation in 64 bits.

Tolerance, from the formula's roundings in fp32 (u = 2^-24): a mean is off by at most D u mean|x|, with D = 512 additions that a value passes through at
most; 1 / sqrt(v + eps) by (D + 8) u of itself, and by the mean's square, which is smaller; then one subtraction, two products and a sum; none of the
activations is steeper than 1.13; silu's exponential carries |h| u of its own value and silu at most 4 u more, gelu 4 u |h|.  bf16: half a step more."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U, D = 2.0 ** -24, 512
ACTS = ("none", "relu", "silu", "gelu")


@pytest.fixture(scope="module")
def tsvd():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no fallback")
    import paper_2308_07641_amd as t
    t.load_library()
    return t


def plain_norm(x, groups, gamma, beta, eps, act):
    """x [images, P, C] float64 -> (y, tolerance) in 64 bits."""
    from scipy.special import erf
    images, P, C = x.shape
    v = x.reshape(images, P, groups, C // groups)
    mean = v.mean((1, 3), keepdims=True)
    rstd = 1 / np.sqrt(((v - mean) ** 2).mean((1, 3), keepdims=True) + eps)
    size = np.abs(v).mean((1, 3), keepdims=True)
    shape = np.broadcast_to
    d, rstd, off = (v - mean).reshape(x.shape), shape(rstd, v.shape).reshape(x.shape), shape(D * U * size, v.shape).reshape(x.shape)
    g, b = (np.ones(C) if gamma is None else gamma.astype(np.float64)), (np.zeros(C) if beta is None else beta.astype(np.float64))
    h = d * rstd * g + b
    slope = rstd * np.abs(g)
    tol = 1.13 * (slope * (1 + (D + 8) * U) * (off + 2 * U * np.abs(d)) + np.abs(h - b) * (D + 16) * U + (slope * off) ** 2 + 2 * U * (np.abs(h) + np.abs(b)))
    if act == "relu":
        y = np.maximum(h, 0)
    elif act == "silu":
        y = h / (1 + np.exp(-h))
        tol = tol + np.abs(y) * (2 * np.abs(h) + 4) * U
    elif act == "gelu":
        y = 0.5 * h * (1 + erf(h / np.sqrt(2)))
        tol = tol + 4 * U * np.abs(h)
    else:
        y = h
    return y, tol + 1e-44


def values(rng, images, P, C, kind="plain"):
    x = rng.standard_normal((images, P, C)) * rng.uniform(0.5, 2, size=C) + rng.standard_normal(C)
    if kind == "far":                     # means far from zero beside small deviations; the first value of all far from the rest
        x = 1000 + 0.5 * x
        x[:, 0, 0] = -3000
    if kind == "same":                    # groups without any deviation
        x = np.full_like(x, 0.7)
    return x


def on_gpu(x, dtype, pitch=0, offset=0):
    import torch
    v = torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    images, P, C = v.shape
    buf = torch.full((images * P * (C + pitch) + offset,), float("nan"), dtype=v.dtype, device="cuda:0")
    view = buf[offset:].view(images, P, C + pitch)[:, :, :C]
    view.copy_(v)
    return view, v.double().numpy()


# images, positions, channels, groups
SHAPES = [(1, 1, 1, 1), (1, 1, 8, 8), (2, 1, 96, 1), (3, 1, 100, 4), (1, 64, 320, 32), (2, 49, 55 * 3, 3), (5, 49, 1155, 21), (3, 7, 13, 13), (2, 300, 24, 3), (1, 1000, 10, 5),
          (4, 1, 4096, 1), (3, 1, 2050, 1), (2, 1, 8200, 1), (70, 1, 768, 1), (2, 5, 4100, 2), (1, 2100, 64, 32), (2, 33, 640, 32), (1, 3000, 7, 1), (2, 17, 128, 128), (1, 2, 20000, 1),
          (3, 130, 96, 1), (2, 40, 520, 8), (1, 5000, 40, 8), (1, 4, 2048, 1024), (1, 300, 1000, 1),
          (70, 11, 100, 4), (65, 30, 33, 11), (9, 1, 2832, 8), (3, 1, 9000, 9), (2, 3000, 72, 9), (2, 2000, 200, 2), (3, 900, 65, 5), (1, 5000, 8, 2),
          (700, 3, 40, 8), (1100, 1, 72, 9), (600, 4, 320, 32), (2, 700, 60, 4), (2, 900, 130, 13), (2, 600, 300, 4), (2, 300, 700, 7), (3, 90, 1500, 4), (2, 70, 3001, 1), (1, 30, 6000, 8),
          (5, 1, 5000, 8), (2, 16306, 64, 64), (600, 9, 67, 1), (3, 1, 16001, 1), (100, 40, 330, 33), (8, 500, 64, 8), (4, 777, 294, 21), (1, 714, 292, 4), (2, 300, 45, 5), (1, 1530, 1984, 64), (100, 300, 217, 7), (2, 3000, 217, 7), (9, 700, 198, 22)]


def params(rng, C, which):
    gamma = (1 + 0.3 * rng.standard_normal(C)).astype(np.float32) if which & 1 else None
    beta = (0.5 * rng.standard_normal(C)).astype(np.float32) if which & 2 else None
    return gamma, beta


def gpu_params(gamma, beta):
    import torch
    return tuple(None if a is None else torch.from_numpy(a).to("cuda:0") for a in (gamma, beta))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images,P,C,G", SHAPES)
def test_norm_against_64_bits(tsvd, images, P, C, G, dtype):
    import torch
    rng = np.random.default_rng(images + 3 * P + 7 * C + G)
    for k, (act, kind) in enumerate((("silu", "plain"), ("none", "far"), ("gelu", "plain"), ("relu", "plain"), ("silu", "same"))):
        gamma, beta = params(rng, C, (3, 1, 2, 0, 3)[k])
        pitch, offset = ((0, 0), (3, 1), (8, 8), (0, 0), (1, 0))[k]
        x, ref = on_gpu(values(rng, images, P, C, kind), dtype, pitch, offset)
        eps = (1e-5, 1e-3, 1e-6, 1e-5, 1e-5)[k]
        want, tol = plain_norm(ref, G, gamma, beta, np.float64(np.float32(eps)), act)
        g, b = gpu_params(gamma, beta)
        for y_tm in (True, False):
            for y_bf16 in (False, True):
                print(f"case norm {images} {P} {C} {G} {dtype} {act} {kind} y_tm={y_tm} bf16={y_bf16}", flush=True)
                y = tsvd.tsvd_group_norm(x, G, g, b, eps=eps, act=ACTS.index(act), y_dtype=tsvd.TSVD_BF16 if y_bf16 else tsvd.TSVD_F32,
                                         y_layout=tsvd.TSVD_TOKEN_MAJOR if y_tm else tsvd.TSVD_FEATURE_MAJOR)
                got = y.double().cpu().numpy()
                got = got if y_tm else got.transpose(1, 2, 0)
                assert got.shape == want.shape
                assert np.all(np.abs(got - want) <= tol + (2.0 ** -8 * (np.abs(want) + tol) if y_bf16 else 0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images,P,C,G", SHAPES)
def test_norm_to_codes(tsvd, images, P, C, G, dtype):
    """A code times its scale is within half a step of the value in 64 bits (and its tolerance); the scale within the tolerance of the largest value."""
    import torch
    rng = np.random.default_rng(images + 5 * P + 11 * C + G)
    for act, kind in (("none", "plain"), ("silu", "far"), ("gelu", "plain")):
        print(f"case norm codes {images} {P} {C} {G} {dtype} {act} {kind}", flush=True)
        gamma, beta = params(rng, C, 3)
        x, ref = on_gpu(values(rng, images, P, C, kind), dtype)
        want, tol = plain_norm(ref, G, gamma, beta, np.float64(np.float32(1e-5)), act)
        want, tol = want.reshape(-1, C), tol.reshape(-1, C)
        q, s = tsvd.tsvd_group_norm_int8(x, G, *gpu_params(gamma, beta), act=ACTS.index(act))
        q, s = q.double().cpu().numpy(), s.double().cpu().numpy()
        top, off = np.abs(want).max(1), tol.max(1)
        assert np.all(np.abs(127 * s - top) <= off + 4 * U * top)
        assert np.all(np.abs(q).max(1) == 127)
        assert np.all(np.abs(q * s[:, None] - want) <= 0.5 * s[:, None] * (1 + 1e-5) + tol + off[:, None])


# rows, one launch (lanes of 64, 256, 512), pieces and codes of each
FAR = [(3, 1, 512, 1), (600, 9, 64, 8), (1, 333, 8, 1), (2, 100, 64, 2), (2, 1999, 32, 4), (1, 10007, 8, 2), (2, 5003, 96, 3), (1, 1201, 256, 1), (2, 49, 1280, 4), (3, 7, 5000, 1)]


@pytest.mark.parametrize("images,P,C,G", FAR)
def test_means_far_from_zero(tsvd, images, P, C, G):
    """Means 2^21 and 2^23 times the deviations: channels c - d, c + d in turn, all exact in fp32, and so are a thread's mean c and deviations d whatever it holds (whole vectors).
    What is left: the squares of a thread (8 additions), the joined variance, 1 / sqrt and the product: 16 roundings of 2^-24 and one of 2^-23."""
    import torch
    for c, d in ((2.0 ** 17, 2.0 ** -4), (2.0 ** 20, 2.0 ** -3)):
        print(f"case far {images} {P} {C} {G} {c}", flush=True)
        x = torch.full((images, P, C), c, device="cuda:0")
        x[..., ::2] -= d
        x[..., 1::2] += d
        eps = np.float64(np.float32(1e-9))
        want = d / np.sqrt(d * d + eps)
        y = tsvd.tsvd_group_norm(x, G, eps=1e-9).double()
        assert float((y[..., 1::2] - want).abs().max()) <= 18 * U * want and float((y[..., ::2] + want).abs().max()) <= 18 * U * want
        q, s = tsvd.tsvd_group_norm_int8(x, G, eps=1e-9)
        assert bool((q[:, 1::2] == 127).all()) and bool((q[:, ::2] == -127).all())
        assert float((s.double() * 127 - want).abs().max()) <= 20 * U * want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images,P,C,G", FAR + [(5, 1, 100, 1), (20, 1, 128, 1), (9, 1, 250, 1), (5, 1, 513, 1), (3, 1, 1001, 1), (3, 1, 2048, 1), (3, 1, 4095, 1), (2, 1, 8191, 1), (2, 1, 16384, 1)])
def test_groups_without_deviation(tsvd, images, P, C, G, dtype):
    """All values of a group alike: every deviation is exactly 0, whatever the value, and y is beta to the last bit."""
    import torch
    beta = torch.randn(C, device="cuda:0")
    gamma = torch.randn(C, device="cuda:0")
    for value in (100000.3, -0.7, 3.0e-5, 1.0e30):
        print(f"case alike {images} {P} {C} {G} {dtype} {value}", flush=True)
        x = torch.full((images, P, C), value, device="cuda:0", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
        y = tsvd.tsvd_group_norm(x, G, gamma, beta, y_dtype=tsvd.TSVD_F32)
        assert torch.equal(y, beta.expand(images, P, C))
        q, s = tsvd.tsvd_group_norm_int8(x, G, gamma, beta)
        codes, scale = tsvd.tsvd_int8_quantize(beta[None])
        assert torch.equal(q, codes.expand(images * P, C)) and torch.equal(s, scale.expand(images * P))


@pytest.mark.parametrize("images,P,C,G", [(2, 50, 64, 4), (3, 1, 512, 1), (1, 3000, 96, 32), (2, 600, 16, 2)])
def test_a_value_that_is_no_number_stays_in_its_group(tsvd, images, P, C, G):
    import torch
    x = torch.randn((images, P, C), device="cuda:0")
    clean = tsvd.tsvd_group_norm(x, G)
    for bad in (float("nan"), float("inf")):
        z = x.clone()
        z[images - 1, P // 2, C - 1] = bad
        y = tsvd.tsvd_group_norm(z, G)
        assert torch.isnan(y[images - 1, :, C - C // G:]).all()
        y[images - 1, :, C - C // G:] = clean[images - 1, :, C - C // G:]
        assert torch.equal(y, clean)


def test_rows_and_images_of_two_dimensions(tsvd):
    import torch
    x = torch.randn((3, 20, 6, 5), device="cuda:0").to(memory_format=torch.channels_last)          # [images, C, H, W] in memory as [images, H, W, C]
    v = x.permute(0, 2, 3, 1)
    want = torch.nn.functional.group_norm(x.double(), 4).float()
    y = tsvd.tsvd_group_norm(v, 4)
    assert y.shape == v.shape and torch.allclose(y.permute(0, 3, 1, 2), want, atol=1e-5)
    f = tsvd.tsvd_group_norm(v, 4, y_layout=tsvd.TSVD_FEATURE_MAJOR)
    assert f.shape == (20, 3, 6, 5) and torch.equal(f, y.permute(3, 0, 1, 2))
    rows = torch.randn((7, 48), device="cuda:0")
    assert torch.allclose(tsvd.tsvd_group_norm(rows, 1), torch.nn.functional.layer_norm(rows, (48,)), atol=1e-5)
    assert torch.equal(tsvd.tsvd_group_norm(rows[:, None, :], 1)[:, 0], tsvd.tsvd_group_norm(rows, 1))


@pytest.mark.parametrize("images,P,C,G", [(1, 64, 320, 32), (2, 4000, 64, 8), (30, 1, 1000, 1)])
def test_captured_and_replayed(tsvd, images, P, C, G):
    import torch
    x = torch.randn((images, P, C), device="cuda:0")
    n = tsvd.tsvd_group_norm_workspace_bytes(images, P, C, G)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda:0")
    y, q, s = torch.empty_like(x), torch.empty((images * P, tsvd.tsvd_int8_row_bytes(C)), dtype=torch.int8, device="cuda:0")[:, :C], torch.empty(images * P, device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tsvd.tsvd_group_norm(x, G, y=y, act=tsvd.TSVD_ACT_SILU, workspace=ws)
        tsvd.tsvd_group_norm_int8(x, G, codes=q, scales=s, workspace=ws)
    for r in range(3):
        x.copy_(torch.randn((images, P, C), device="cuda:0"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, tsvd.tsvd_group_norm(x, G, act=tsvd.TSVD_ACT_SILU))
        q2, s2 = tsvd.tsvd_group_norm_int8(x, G)
        assert torch.equal(q, q2) and torch.equal(s, s2)


def test_norm_layer_convolution_together(tsvd):
    """A block as a network has it: norm + silu into codes, a pointwise layer in 8 bits on them, a norm written channel by channel, and a 3 x 3 convolution in ternary form on that.
    Each step against the steps before it, in 64 bits."""
    import torch
    from oracle import conv as oc
    rng = np.random.default_rng(21)
    images, H, W, C, M = 2, 9, 7, 48, 32
    x, ref = on_gpu(values(rng, images, H * W, C), "bf16")
    gamma, beta = params(rng, C, 3)
    q, s = tsvd.tsvd_group_norm_int8(x, 8, *gpu_params(gamma, beta), act=tsvd.TSVD_ACT_SILU)
    w = rng.integers(-127, 128, size=(M, C)).astype(np.int8)
    t = (rng.random(M) * 1e-2).astype(np.float32)
    h8 = tsvd.tsvd_int8_pack(torch.from_numpy(w).to("cuda:0"), torch.from_numpy(t).to("cuda:0"))
    y = tsvd.tsvd_int8_product(h8, q, s, y_dtype=tsvd.TSVD_BF16, y_layout=tsvd.TSVD_TOKEN_MAJOR)
    want, tol = plain_norm(ref, 8, gamma, beta, 1e-5, "silu")
    want, tol = want.reshape(-1, C), tol.reshape(-1, C)
    step = np.abs(want).max(1, keepdims=True) / 127
    lin = want @ (w * t[:, None].astype(np.float64)).T
    bound = (0.5 * step + tol + tol.max(1, keepdims=True)) * 1.001 @ np.ones((C, 1)) * np.abs(w * t[:, None].astype(np.float64)).max(1)[None, :]
    assert np.all(np.abs(y.double().cpu().numpy() - lin) <= bound + 2.0 ** -8 * np.abs(lin) * 1.01 + 2.0 ** -8 * bound)
    z = tsvd.tsvd_group_norm(y.view(images, H, W, M), 4, y_dtype=tsvd.TSVD_BF16, y_layout=tsvd.TSVD_FEATURE_MAJOR)
    want, tol = plain_norm(y.double().cpu().numpy().reshape(images, H * W, M), 4, None, None, 1e-5, "none")
    got = z.double().cpu().numpy().reshape(M, images, H * W).transpose(1, 2, 0)
    assert np.all(np.abs(got - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol))
    K, co = 40, 12
    Um, V = rng.choice([-1, 0, 1], size=(co, K)).astype(np.int8), rng.choice([-1, 0, 1], size=(K, M * 9)).astype(np.int8)
    S = (rng.random(K) * 0.1).astype(np.float32)
    h = tsvd.tsvd_pack(Um, S, V)
    out = tsvd.tsvd_conv2d_forward(h, 0, M, co, 3, 3, z, pad=(1, 1))
    ref = oc.tsvd_conv2d(z.float().cpu().numpy().transpose(1, 0, 2, 3), Um, S, V, 0, co, M, 3, 3, (1, 1), (1, 1), (1, 1))
    assert np.max(np.abs(out.double().cpu().numpy().transpose(1, 0, 2, 3) - ref)) <= 2e-3 * np.max(np.abs(ref))
    tsvd.tsvd_free(h)
    tsvd.tsvd_int8_free(h8)


def test_refusals(tsvd):
    import torch
    x = torch.randn((2, 5, 24), device="cuda:0")
    side = torch.cuda.Stream().cuda_stream
    for args, kw in (((x, 5), {}), ((x, 0), {}), ((x.half(), 4), {}), ((x.cpu(), 4), {}), ((x[0, 0], 4), {}), ((x[:, :0], 4), {}), ((x.transpose(1, 2), 5), {}), ((x[:, ::2], 4), {}),
                     ((x, 4), {"eps": 0.0}), ((x, 4), {"eps": float("nan")}), ((x, 4), {"act": 4}), ((x, 4), {"gamma": torch.ones(23, device="cuda:0")}),
                     ((x, 4), {"beta": torch.ones(24)}), ((x, 4), {"y": torch.empty((2, 5, 23), device="cuda:0")}), ((x, 4), {"y": torch.empty((2, 5, 24))}),
                     ((x, 4), {"workspace": torch.empty(8, dtype=torch.uint8, device="cuda:0")}), ((x, 4), {"stream": side})):
        with pytest.raises((ValueError, TypeError, tsvd.TsvdError)):
            tsvd.tsvd_group_norm(*args, **kw)
    for kw in ({"codes": torch.empty((10, 24), dtype=torch.int8, device="cuda:0")}, {"scales": torch.empty(9, device="cuda:0")}, {"stream": side}):
        with pytest.raises((ValueError, TypeError, tsvd.TsvdError)):
            tsvd.tsvd_group_norm_int8(x, 4, **kw)
    # every third position of a longer tensor has one pitch, and is taken
    long = torch.randn((1, 15, 24), device="cuda:0")
    assert torch.equal(tsvd.tsvd_group_norm(long[:, ::3], 4), tsvd.tsvd_group_norm(long[:, ::3].contiguous(), 4))
