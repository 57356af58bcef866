"""Arguments of the layer-replay entry points are validated before any device work."""
import numpy as np
import pytest

from paper_2608_11034_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.lib()


def attn(**kw):
    a = np.zeros(1, dtype=binding.ATTN_DTYPE)
    d = dict(dtype=binding.DT_BF16, batch=2, q_len=32, kv_len=48, q_heads=4, kv_heads=2, head_dim=64, causal=1, window=0, scale=0.125,
             q_stride=(8192, 256, 64), k_stride=(6144, 128, 64), v_stride=(6144, 128, 64), o_stride=(8192, 256, 64),
             do_stride=(8192, 256, 64))
    d.update(kw)
    for n, x in d.items():
        a[0][n] = x
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=binding.DT_F32), binding.ERR_UNSUPPORTED), (dict(dtype=99), binding.ERR_INVALID), (dict(batch=0), binding.ERR_INVALID),
    (dict(q_heads=0), binding.ERR_INVALID), (dict(kv_heads=3), binding.ERR_INVALID), (dict(kv_heads=0), binding.ERR_INVALID),
    (dict(head_dim=0), binding.ERR_INVALID), (dict(head_dim=136), binding.ERR_UNSUPPORTED), (dict(head_dim=20), binding.ERR_UNSUPPORTED),
    (dict(causal=2), binding.ERR_INVALID), (dict(causal=0, window=5), binding.ERR_INVALID), (dict(scale=0.0), binding.ERR_INVALID),
    (dict(scale=-1.0), binding.ERR_INVALID), (dict(scale=float("nan")), binding.ERR_INVALID), (dict(scale=float("inf")), binding.ERR_INVALID),
    (dict(q_len=2 ** 31), binding.ERR_UNSUPPORTED), (dict(q_len=2 ** 28), binding.ERR_UNSUPPORTED), (dict(kv_len=2 ** 31), binding.ERR_UNSUPPORTED),
    (dict(k_stride=(6144, 0, 64)), binding.ERR_INVALID), (dict(v_stride=(6144, 132, 64)), binding.ERR_ALIGN),
    (dict(do_stride=(8192, 256, 65)), binding.ERR_ALIGN)])
def test_attention_descriptions_are_checked(kw, code):
    with pytest.raises(binding.ScoutError) as e:
        binding.scout_attn_workspace(attn(**kw).ctypes.data)
    assert e.value.code == code


def test_attention_scratch_and_pointers_are_checked(lib):
    a = attn()
    f, b = binding.scout_attn_workspace(a.ctypes.data)
    assert f % 256 == 0 and b % 256 == 0 and b >= 2 * 4 * 32 * 8
    # strides of axes of one element do not matter
    binding.scout_attn_workspace(attn(batch=1, q_stride=(0, 256, 64), o_stride=(3, 256, 64)).ctypes.data)
    at = a.ctypes.data
    assert lib.scout_attn_workspace(at, None, None) == lib.scout_attn_workspace(None, None, None) == binding.ERR_INVALID
    assert lib.scout_attn_forward(at, 0, 256, 256, 0, 0, 256, 256, 256, f, 0) == binding.ERR_INVALID
    assert lib.scout_attn_forward(at, 8, 256, 256, 0, 0, 256, 256, 256, f, 0) == binding.ERR_ALIGN
    assert lib.scout_attn_backward(at, 256, 256, 256, 256, 256, 256, 0, 0, 256, 256, 256, 256, b - 1, 0) == binding.ERR_INVALID
    assert lib.scout_attn_backward(at, 256, 256, 256, 256, 256, 256, 0, 0, 256, 256, 256, 0, b, 0) == binding.ERR_INVALID
    assert lib.scout_attn_backward(at, 256, 256, 256, 256, 256, 256, 0, 0, 256, 264, 256, 256, b, 0) == binding.ERR_ALIGN


def test_checkpoint_arguments_are_checked(lib):
    p, u, w = lib.scout_ckpt_pack, lib.scout_ckpt_unpack, lib.scout_ckpt_wgrad
    B, F, H = binding.DT_BF16, binding.DT_F32, binding.DT_F16
    assert p(binding.DT_I64, 1, 1, 256, 1, 256, 1, 256, 0) == binding.ERR_UNSUPPORTED
    assert p(77, 1, 1, 256, 1, 256, 1, 256, 0) == binding.ERR_INVALID
    assert p(B, 4, 32, 0, 32, 256, 32, 256, 0) == binding.ERR_INVALID
    assert p(B, 4, 32, 256, 31, 256, 32, 256, 0) == binding.ERR_INVALID
    assert u(B, 4, 32, 256, 31, 256, 256, 32, 0) == binding.ERR_INVALID
    assert u(F, 4, 32, 256, 32, 256, 258, 32, 0) == binding.ERR_ALIGN
    assert p(B, 0, 32, 0, 0, 0, 0, 0, 0) == binding.OK
    assert p(B, 2 ** 41, 1, 256, 1, 256, 1, 256, 0) == binding.ERR_UNSUPPORTED
    with pytest.raises(binding.ScoutError) as e:
        binding.scout_ckpt_wgrad_workspace(F, 8, 8, 8)
    assert e.value.code == binding.ERR_UNSUPPORTED
    n = binding.scout_ckpt_wgrad_workspace(B, 4096, 64, 64)
    assert n > 0                                              # one tile of outputs: its tokens are split
    assert w(B, F, 4096, 64, 64, 256, 64, 256, 64, 256, 256, 64, 0, 256, n - 1, 0) == binding.ERR_INVALID
    assert w(B, H, 8, 8, 8, 256, 8, 256, 8, 256, 256, 8, 0, 256, 0, 0) == binding.ERR_INVALID       # dW neither fp32 nor dy's type
    assert w(B, F, 8, 8, 8, 256, 7, 256, 8, 256, 256, 8, 0, 256, 0, 0) == binding.ERR_INVALID
    assert w(B, F, 8, 8, 8, 256, 8, 256, 8, 256, 258, 8, 0, 256, 0, 0) == binding.ERR_ALIGN
    assert w(B, F, 8, 8, 8, 256, 8, 256, 8, 256, 256, 8, 2, 256, 0, 0) == binding.ERR_INVALID
    assert w(B, F, 8, 0, 8, 0, 0, 0, 8, 0, 0, 8, 0, 0, 0, 0) == binding.OK
