"""What the rotation and the paged cache refuse before anything reaches a GPU."""
import ctypes

import pytest
import torch

from paper_2410_23079_b200 import BuzzPaged, binding, norm_rope
from tests import paged_reference as ref

lib = binding.load_library()
OK_ROPE = dict(q_heads=8, kv_heads=2, head_dim=128, rotary_dim=64, dtype=1, interleaved=0, eps=1e-6, reserved=0,
               q_stride=1024, k_stride=256, q_out_stride=1024, k_out_stride=256)
OK_PAGED = dict(layers=2, pages=8, page_tokens=32, q_heads=8, kv_heads=2, head_dim=128, dtype=1, cache_dtype=2, flags=0)
OK_BUFFERS = dict(k=256, v=512, k_scale=768, v_scale=1024, bounds=None, status=1280)


@pytest.mark.parametrize("over", [dict(q_heads=0), dict(kv_heads=0), dict(head_dim=96), dict(rotary_dim=0), dict(rotary_dim=24),
                                  dict(rotary_dim=144), dict(dtype=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                  dict(reserved=1), dict(q_stride=1023), dict(q_stride=1028), dict(k_stride=128), dict(k_out_stride=252),
                                  dict(q_out_stride=1016)])
def test_norm_rope_shapes(over):
    sh = binding._RopeShape(**{**OK_ROPE, **over})
    assert lib.buzz_norm_rope(ctypes.byref(sh), 256, 256, 256, 256, None, None, 256, 256, 4, None) == -1


def test_norm_rope_pointers():
    sh = binding._RopeShape(**OK_ROPE)
    good = [256, 256, 256, 256, None, None, 256, 256]
    for i, bad in [(0, None), (1, None), (2, None), (3, None), (6, None), (7, None), (0, 8), (1, 8), (2, 2), (3, 2), (4, 8), (5, 8), (6, 8), (7, 8)]:
        args = list(good)
        args[i] = bad
        assert lib.buzz_norm_rope(ctypes.byref(sh), *args, 4, None) == -1, (i, bad)
    assert lib.buzz_norm_rope(ctypes.byref(sh), *good, -1, None) == -1
    assert lib.buzz_norm_rope(None, *good, 4, None) == -1
    for over in (dict(q_out_stride=2048), dict(k_out_stride=512)):                    # in place, but not where the rows were
        assert lib.buzz_norm_rope(ctypes.byref(binding._RopeShape(**{**OK_ROPE, **over})), 256, 512, 256, 256, None, None, 256, 512, 4, None) == -1
    assert lib.buzz_norm_rope(ctypes.byref(sh), *[None] * 8, 0, None) == 0          # no tokens: nothing to do


@pytest.mark.parametrize("over", [dict(layers=0), dict(pages=0), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=256),
                                  dict(q_heads=6), dict(q_heads=7), dict(q_heads=32), dict(kv_heads=0), dict(head_dim=32), dict(dtype=2),
                                  dict(cache_dtype=0), dict(cache_dtype=4), dict(flags=2)])
def test_paged_shapes(over):
    h = ctypes.c_void_p(1)
    sh, buf = binding._PagedShape(**{**OK_PAGED, **over}), binding._PagedBuffers(**OK_BUFFERS)
    assert lib.buzz_paged_create(ctypes.byref(h), ctypes.byref(sh), ctypes.byref(buf)) == -1
    assert h.value is None


@pytest.mark.parametrize("over", [dict(k=None), dict(v=None), dict(status=None), dict(k_scale=None), dict(v_scale=None), dict(k=8),
                                  dict(v=4), dict(k_scale=12), dict(bounds=2), dict(status=4)])
def test_paged_buffers(over):
    h = ctypes.c_void_p()
    sh, buf = binding._PagedShape(**OK_PAGED), binding._PagedBuffers(**{**OK_BUFFERS, **over})
    assert lib.buzz_paged_create(ctypes.byref(h), ctypes.byref(sh), ctypes.byref(buf)) == -1


def test_calls_without_an_object():
    n = ctypes.c_size_t()
    assert lib.buzz_paged_workspace_bytes(None, 1, 1, 0, ctypes.byref(n), ctypes.byref(n)) == -1
    assert lib.buzz_paged_append(None, 0, 256, 256, None, 1, 1, 1, 256, 256, 1, None) == -1
    assert lib.buzz_paged_read(None, 0, 256, 256, None, 1, 1, 1, 256, 256, 1, None) == -1
    assert lib.buzz_paged_decode(None, 0, 256, 256, 256, 1, 1, 1, None, 0, 256, None, 256, 256, None) == -1
    assert lib.buzz_paged_select(None, 0, 256, 256, 256, 1, 1, 1, 0, 1, 1, 256, 256, 256, None) == -1
    assert lib.buzz_paged_status(None, None) == -1
    assert lib.buzz_paged_launch_count(None) == 0
    lib.buzz_paged_destroy(None)


def test_no_cpu_fallback():
    x = torch.zeros(2, 1, 64)
    with pytest.raises(ValueError):
        norm_rope(x, x, torch.zeros(2, dtype=torch.int32), torch.ones(8))
    if not torch.cuda.is_available():
        with pytest.raises(RuntimeError):
            BuzzPaged(layers=1, pages=1, page_tokens=16, q_heads=1, kv_heads=1, head_dim=64, dtype=torch.float32)


def test_reference_quantisation_agrees_with_the_type():
    """The 64-bit codes of the tests against torch's own conversion to the 8-bit type."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(64, 128, generator=g) * torch.exp(3 * torch.randn(64, 1, generator=g))
    x[3] = 0
    codes, scale = ref.quantise(x, torch.float8_e4m3fn)
    y = (x / scale[:, None].float()).clamp(-448, 448).to(torch.float8_e4m3fn)
    assert torch.equal(codes, y.double())
    codes, scale = ref.quantise(x, torch.int8)
    assert torch.equal(codes, (x / scale[:, None].float()).clamp(-127, 127).round().double())


def test_reference_choice_by_hand():
    """Four pages, one head, worked below; ties to the lowest page."""
    q = torch.tensor([[2.0, -1.0]])
    bounds = torch.tensor([[[[-1.0, -2.0], [1.0, 5.0]]], [[[0.0, 0.0], [3.0, 1.0]]], [[[-9.0, -4.0], [1.0, 0.0]]], [[[0.0, 0.0], [0.0, 0.0]]]])
    # page 0: 2*1 + (-1)(-2) = 4; page 1: 2*3 + 0 = 6; page 2: 2*1 + 4 = 6; page 3: 0
    assert ref.choose(q, bounds, 0, 1, 1) == [[1, 3]]
    assert ref.choose(q, bounds, 0, 1, 2) == [[1, 2, 3]]
    assert ref.choose(q, bounds, 1, 1, 1) == [[0, 1, 3]]
    assert ref.choose(q, bounds, 0, 1, 3) == [[0, 1, 2, 3]]
