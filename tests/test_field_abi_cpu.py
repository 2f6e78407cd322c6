"""Host-side checks of the operators over the candidates of a field that need no GPU."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2004_13940_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2004_13940_amd import build
        build.build()
    return binding.load()


def test_candidates_struct_layout_matches_header():
    from paper_2004_13940_amd import binding
    at = {name: getattr(binding.fm_candidates, name).offset for name, _ in binding.fm_candidates._fields_}
    assert ctypes.sizeof(binding.fm_candidates) == 48
    assert at == dict(V=0, w=8, mask=16, v_stride=24, mask_stride=32, v_type=40, scale=44)


@pytest.mark.parametrize("args,code", [
    ((0, 8, 1, 0, 0), -4), ((1 << 31, 8, 1, 0, 0), -4), ((10, 0, 1, 0, 0), -1), ((10, 65, 1, 0, 0), -1), ((10, 260, 1, 0, 0), -1),
    ((10, 8, 0, 0, 0), -4), ((10, 8, 1 << 31, 0, 0), -4), ((10, 8, 1, -1, 0), -4), ((10, 8, 1, 65, 0), -4),
    ((10, 8, 1, 0, -1), -4), ((10, 8, 1, 0, 4097), -4)])
def test_handles_of_bad_sizes_are_refused(lib, args, code):
    h = ctypes.c_void_p(None)
    assert lib.fm_field_create(*args, ctypes.byref(h)) == code
    assert not h.value and lib.fm_field_last_error(None)


def test_null_handles(lib):
    assert lib.fm_field_create(10, 8, 1, 0, 0, None) == -1
    assert lib.fm_field_destroy(None) == 0
    assert lib.fm_field_logprobs(None, None, 1, None, 8, 0, None, None, None, None, 0, None, None, None) == -1
    assert lib.fm_field_distill(None, None, 1, None, 8, 1, None, None, None, None, None, None, None, None) == -1


def test_binding_refuses_to_run_without_a_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    from paper_2004_13940_amd import binding
    with pytest.raises(RuntimeError):
        binding.Field(10, 8, 1)
