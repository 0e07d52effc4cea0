"""CPU-only tests of the layers in 8-bit integers and of the group norm: exported symbols, sizes, and refusals, which all come before any device work."""
import ctypes
import os
import re

import pytest

import paper_2308_07641_amd as tsvd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_function_is_exported_and_bound():
    lib = tsvd.load_library()
    for header in ("tsvd_int8.h", "tsvd_norm.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names = set(re.findall(r"\b(tsvd_[a-z0-9_]+)\s*\(", text))
        assert names
        for n in names:
            assert hasattr(lib, n) and hasattr(tsvd, n), n


def test_sizes():
    assert [tsvd.tsvd_int8_row_bytes(n) for n in (0, -1, 1, 128, 129, 131071, 131072)] == [0, 0, 128, 128, 256, 131072, 0]
    assert tsvd.tsvd_int8_packed_bytes(1, 1) == 256 + 2048 and tsvd.tsvd_int8_packed_bytes(17, 129) == 256 + 2 * 4 * 1024
    assert tsvd.tsvd_int8_packed_bytes(0, 5) == 0 and tsvd.tsvd_int8_packed_bytes(5, 0) == 0 and tsvd.tsvd_int8_packed_bytes(5, 1 << 17) == 0
    assert tsvd.tsvd_int8_packed_bytes((1 << 24) + 1, 4) == 0
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (1, 1, 6, 4), (1, 1, (1 << 20) + 1, 1), (1 << 16, 1 << 15, 8, 1)):
        assert tsvd.tsvd_group_norm_workspace_bytes(*bad) == 0
    assert tsvd.tsvd_group_norm_workspace_bytes(1, 1, 8, 1) >= 256


EINVAL, EUNSUPPORTED = 1, 5


def test_int8_calls_check_their_arguments_first():
    lib = tsvd.load_library()
    buf = (ctypes.c_char * 4096)()
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    out = ctypes.c_void_p()

    def quantize(x=p, dtype=0, layout=1, B=2, N=32, ldx=32, codes=p, ldq=32, s=p, ws=None, nbytes=0):
        return lib.tsvd_int8_quantize(x, dtype, layout, B, N, ldx, codes, ldq, s, ws, nbytes, None)

    for bad in (dict(x=None), dict(codes=None), dict(s=None), dict(dtype=2), dict(layout=2), dict(B=0), dict(N=0), dict(ldx=31), dict(layout=0, ldx=1), dict(ldq=31), dict(ldq=40),
                dict(codes=p + 8), dict(nbytes=8), dict(ws=p + 8, nbytes=256), dict(layout=0, B=64, N=8192, ldx=64, ldq=8192),
                dict(layout=0, B=64, N=8192, ldx=64, ldq=8192, ws=p, nbytes=16)):
        assert quantize(**bad) == EINVAL, bad
    assert tsvd.tsvd_int8_quantize_workspace_bytes(64, 8192, 1) == 0 and tsvd.tsvd_int8_quantize_workspace_bytes(64, 8192, 0) > 0
    assert quantize(N=1 << 17, ldx=1 << 17, ldq=1 << 17) == EUNSUPPORTED and quantize(B=(1 << 24) + 1) == EUNSUPPORTED

    def pack(w=p, ldw=32, t=p, M=4, N=32, d=None, nbytes=0, o=ctypes.byref(out)):
        return lib.tsvd_int8_pack(w, ldw, t, M, N, d, nbytes, None, o)

    for bad in (dict(w=None), dict(t=None), dict(o=None), dict(M=0), dict(N=0), dict(ldw=31), dict(d=p, nbytes=100), dict(d=p + 64, nbytes=1 << 20), dict(nbytes=5)):
        assert pack(**bad) == EINVAL, bad
    assert pack(N=1 << 17, ldw=1 << 17) == EUNSUPPORTED and pack(M=(1 << 24) + 1) == EUNSUPPORTED
    assert out.value is None
    assert lib.tsvd_int8_info(None, None, None) == EINVAL
    assert lib.tsvd_int8_workspace_bytes(None, 4, 0, 0) == 0
    assert lib.tsvd_int8_product(None, p, 32, p, 1, None, p, 0, 0, 1, None) == EINVAL
    assert lib.tsvd_int8_forward(None, p, 0, 0, 1, 1, None, p, 0, 0, 1, p, 4096, None) == EINVAL
    lib.tsvd_int8_free(None)


def test_norm_calls_check_their_arguments_first():
    lib = tsvd.load_library()
    buf = (ctypes.c_char * 8192)()
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    nan, inf = float("nan"), float("inf")

    def norm(x=p, dtype=0, images=1, P=2, C=32, ldx=32, groups=4, eps=1e-5, act=0, y=p, y_dtype=0, y_layout=1, ldy=32, ws=p, nbytes=4096):
        return lib.tsvd_group_norm(x, dtype, images, P, C, ldx, groups, None, None, eps, act, y, y_dtype, y_layout, ldy, ws, nbytes, None)

    shared = (dict(x=None), dict(y=None), dict(dtype=2), dict(images=0), dict(P=0), dict(C=0), dict(groups=0), dict(groups=5), dict(ldx=31), dict(eps=0.0), dict(eps=-1.0), dict(eps=nan),
              dict(eps=inf), dict(act=-1), dict(act=4), dict(ws=None), dict(ws=p + 8), dict(nbytes=0))
    for bad in shared + (dict(y_dtype=2), dict(y_layout=2), dict(ldy=31), dict(y_layout=0, ldy=1)):
        assert norm(**bad) == EINVAL, bad
    assert norm(C=1 << 21, ldx=1 << 21, ldy=1 << 21) == EUNSUPPORTED and norm(images=1 << 20, P=1 << 12) == EUNSUPPORTED

    def codes(x=p, dtype=0, images=1, P=2, C=32, ldx=32, groups=4, eps=1e-5, act=0, y=p, ldq=32, s=p, ws=p, nbytes=4096):
        return lib.tsvd_group_norm_int8(x, dtype, images, P, C, ldx, groups, None, None, eps, act, y, ldq, s, ws, nbytes, None)

    for bad in shared + (dict(s=None), dict(y=p + 8), dict(ldq=31), dict(ldq=16), dict(ldq=40)):
        assert codes(**bad) == EINVAL, bad


def test_packing_needs_a_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    out = ctypes.c_void_p()
    buf = (ctypes.c_char * 4096)()
    p = ctypes.addressof(buf)
    assert tsvd.load_library().tsvd_int8_pack(p, 32, p, 4, 32, None, 0, None, ctypes.byref(out)) == 4 and out.value is None


@pytest.mark.parametrize("x_dtype", [0, 1])
def test_codes_of_feature_major_activations_take_every_feature(x_dtype):
    """One launch holds all features in registers or reads x twice; else there are two launches, and they need scratch.  On both sides of every border of the rules."""
    tokens = sorted({b + d for b in (8, 16, 64, 512, 1024, 4096, 32704, 32768, 1 << 20, (1 << 24) - 1) for d in (-1, 0, 1)} | {1, 2})
    features = sorted({n + d for n in (64, 512, 1024, 2048, 4096, 8192, 16384, (1 << 17) - 2) for d in (-1, 0, 1)} | {1, 4100, 9216, 14381})
    for B in tokens:
        for N in features:
            holds = tsvd.tsvd_tuning_int8_columns(B, N, x_dtype)
            assert (holds == -1) == (tsvd.tsvd_int8_quantize_workspace_bytes(B, N, tsvd.TSVD_FEATURE_MAJOR) > 0), (B, N)
            assert holds in (-1, 0) or holds >= N, (B, N, holds)
    assert tsvd.tsvd_tuning_int8_columns(0, 5, x_dtype) == tsvd.tsvd_tuning_int8_columns(5, 1 << 17, x_dtype) == -1


def test_norm_refuses_views_whose_positions_have_no_pitch():
    """Positions that share their memory (a broadcast view), overlap or stand at different distances are refused by their strides, before anything asks where they are; every pitch of
    C or more passes on to the next check, which on the CPU is the one for the device."""
    import torch
    row, images = torch.zeros(1, 24), torch.zeros(2, 1, 24)
    wide = torch.zeros(2, 3, 4, 40)[..., :24]
    refused = (row.expand(5, 24), row[None].expand(1, 5, 24), row[None].expand(2, 1, 24), row[None].expand(2, 5, 24), images.expand(2, 5, 24),
               torch.zeros(2, 1, 120)[:, :, :24].expand(2, 5, 24), torch.zeros(5, 1, 24).transpose(0, 1).expand(2, 5, 24), row[None, None].expand(2, 3, 4, 24),
               torch.zeros(2, 1, 1, 24).expand(2, 1, 4, 24), torch.zeros(100).as_strided((4, 24), (20, 1)), torch.zeros(300).as_strided((2, 3, 24), (144, 24, 1)),
               torch.zeros(2, 5, 24).transpose(0, 1), torch.zeros(5, 24, 2)[:, :, 0],
               wide[:, :1])                              # (rows 40 apart, images 480 where four rows take 160)
    for x in refused:
        for call in (tsvd.tsvd_group_norm, tsvd.tsvd_group_norm_int8):
            with pytest.raises(ValueError, match="a pitch of C or more"):
                call(x, 4)
    for x in (row, images, wide, wide[0], wide[:, :, :1, :][:, :1], wide.flatten(0, 2), torch.zeros(1, 15, 24)[:, ::3], torch.zeros(2, 1, 100)[:, :, :24].transpose(0, 1)):
        for call in (tsvd.tsvd_group_norm, tsvd.tsvd_group_norm_int8):
            with pytest.raises(ValueError, match="live on the GPU"):
                call(x, 4)


def test_a_handle_of_the_other_kind_is_a_type_error():
    """Ternary and 8-bit handles of one layer have the same sizes but nothing else in common: every function takes its own kind only, whatever else is wrong with the call."""
    import torch
    ternary, int8 = tsvd.Handle(None, 8, 4, 16), tsvd.Int8Handle(None, 8, 16)
    x, y, codes, scales = torch.zeros(16, 2), torch.zeros(8, 2), torch.zeros((2, 16), dtype=torch.int8), torch.zeros(2)

    class Looks:
        ptr, M, K, N = None, 8, 4, 16

    for h in (int8, Looks(), None, 5):
        for call in (lambda: tsvd.tsvd_forward(h, x), lambda: tsvd.tsvd_forward_ex(h, x), lambda: tsvd.tsvd_forward_io(h, x), lambda: tsvd.tsvd_forward_noalloc(h, x, y),
                     lambda: tsvd.tsvd_conv2d_forward(h, 0, 16, 8, 1, 1, x.view(16, 1, 2, 1)), lambda: tsvd.tsvd_unpack(h), lambda: tsvd.tsvd_info(h),
                     lambda: tsvd.tsvd_workspace_bytes(h, 2, 0), lambda: tsvd.tsvd_workspace_bytes_ex(h, 2, 0, 0), lambda: tsvd.tsvd_tuning_forward_stages(h, x, y, 7),
                     lambda: tsvd.tsvd_tuning_tile_shapes(h, 2), lambda: tsvd.tsvd_tuning_one_launch(h, 2), lambda: tsvd.tsvd_tuning_split_tiles(h, 2, 0),
                     lambda: tsvd.tsvd_tuning_tiles_by_xcd(h, 2, 0), lambda: tsvd.tsvd_tuning_read_clocks(h, 1)):
            with pytest.raises(TypeError, match="Handle"):
                call()
    for h in (ternary, Looks(), None, 5):
        for call in (lambda: tsvd.tsvd_int8_forward(h, x), lambda: tsvd.tsvd_int8_product(h, codes, scales), lambda: tsvd.tsvd_int8_info(h),
                     lambda: tsvd.tsvd_int8_workspace_bytes(h, 2, 0, 0)):
            with pytest.raises(TypeError, match="Int8Handle"):
                call()
    for free, h in ((tsvd.tsvd_free, int8), (tsvd.tsvd_int8_free, ternary), (tsvd.tsvd_free, Looks()), (tsvd.tsvd_int8_free, 5)):
        with pytest.raises(TypeError):
            free(h)
    for free, h in ((tsvd.tsvd_free, None), (tsvd.tsvd_int8_free, None), (tsvd.tsvd_free, ternary), (tsvd.tsvd_int8_free, int8)):
        free(h)
    # one's own kind, released: the library refuses it
    for call in (lambda: tsvd.tsvd_info(ternary), lambda: tsvd.tsvd_int8_info(int8)):
        with pytest.raises(tsvd.TsvdError):
            call()

    class Own(tsvd.Int8Handle):
        pass

    with pytest.raises(tsvd.TsvdError):
        tsvd.tsvd_int8_info(Own(None, 8, 16))
