"""What the operators between the q/k/v and the o product refuse, before anything touches a GPU."""
from __future__ import annotations

import ctypes as C
import os

import pytest

from paper_2412_17560_amd import binding

NULL, SHAPE, UNSUPPORTED, RANGE, HIP, ALIGN = 1, 2, 3, 4, 6, 8
AT = 1 << 20        # an aligned address that no call gets to use


def rotate(**change):
    a = dict(q=AT, q_row=1024, q_head=128, q_heads=8, k=AT, k_row=256, k_head=128, k_heads=2, rows=3, dim=128, qw=AT, kw=AT, eps=1e-6,
             table=AT, n_positions=10, rotary=128, interleaved=0, positions=AT, qo=AT, qo_row=1024, qo_head=128, ko=AT, ko_row=256, ko_head=128)
    assert not set(change) - set(a)
    return binding._lib().gqsa_qk_norm_rotate(*{**a, **change}.values(), None)


def prompt(**change):
    a = dict(q=AT, q_row=1024, q_head=128, q_heads=8, q_rows=5, k=AT, k_row=256, k_head=128, v=AT, v_row=256, v_head=128, kv_heads=2,
             k_rows=5, dim=128, q_starts=AT, k_starts=AT, n_seqs=2, scale=0.1, out=AT, out_row=1024, out_head=128)
    assert not set(change) - set(a)
    return binding._lib().gqsa_prompt_attend(*{**a, **change}.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(q=None), NULL), (dict(qo=None), NULL), (dict(k=None), NULL), (dict(ko=None), NULL), (dict(table=None), NULL),
    (dict(positions=None), NULL), (dict(q=AT + 8), ALIGN), (dict(qo=AT + 2), ALIGN), (dict(q_row=1028), ALIGN), (dict(k_head=12), ALIGN),
    (dict(qw=AT + 8), ALIGN), (dict(kw=AT + 4), ALIGN), (dict(table=AT + 8), ALIGN), (dict(positions=AT + 2), ALIGN),
    (dict(q_row=-8), SHAPE), (dict(q_head=1 << 41), SHAPE), (dict(q_heads=0), SHAPE), (dict(k_heads=-1), SHAPE), (dict(rows=-1), SHAPE),
    (dict(rows=(1 << 25) + 1), SHAPE), (dict(n_positions=-1), SHAPE), (dict(q_heads=1025), UNSUPPORTED), (dict(dim=120), UNSUPPORTED),
    (dict(dim=0), UNSUPPORTED), (dict(dim=272), UNSUPPORTED), (dict(rotary=24), UNSUPPORTED), (dict(rotary=144), UNSUPPORTED),
    (dict(rotary=-16), UNSUPPORTED), (dict(eps=-1.0), RANGE), (dict(eps=float("nan")), RANGE), (dict(eps=float("inf")), RANGE)])
def test_norm_rotate_refuses(change, status):
    assert rotate(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(out=None), NULL), (dict(q_starts=None), NULL), (dict(k_starts=None), NULL),
    (dict(q=AT + 8), ALIGN), (dict(v_row=260), ALIGN), (dict(out_head=4), ALIGN), (dict(q_starts=AT + 1), ALIGN), (dict(k_row=-256), SHAPE),
    (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(q_heads=7), SHAPE), (dict(q_rows=-1), SHAPE), (dict(k_rows=-1), SHAPE),
    (dict(n_seqs=0), SHAPE), (dict(q_rows=(1 << 25) + 1), SHAPE), (dict(q_heads=2048), UNSUPPORTED), (dict(n_seqs=65537), UNSUPPORTED),
    (dict(dim=96), UNSUPPORTED), (dict(k_row=(1 << 23) + 8), UNSUPPORTED), (dict(scale=float("nan")), RANGE), (dict(scale=float("-inf")), RANGE)])
def test_prompt_attend_refuses(change, status):
    assert prompt(**change) == status


def test_no_rows_is_no_work():
    assert rotate(rows=0, q=None) == 0 and prompt(q_rows=0, q=None) == 0


@pytest.mark.parametrize("args, status", [
    ((0, 32, 1, 64), SHAPE), ((1, 0, 1, 64), SHAPE), ((1, 32, 0, 64), SHAPE), ((1, 16, 1, 64), UNSUPPORTED), ((1, 48, 1, 64), UNSUPPORTED),
    ((1, 8192, 1, 64), UNSUPPORTED), ((1, 32, 1025, 64), UNSUPPORTED), ((1, 32, 1, 80), UNSUPPORTED), (((1 << 30) + 1, 32, 1, 64), UNSUPPORTED)])
def test_cache_create_refuses(args, status):
    out = C.c_void_p(123)
    assert binding._lib().gqsa_cache_create(*args, C.byref(out)) == status
    assert out.value is None
    assert binding._lib().gqsa_cache_create(*args, None) == NULL


def test_calls_without_a_cache():
    lib = binding._lib()
    info = binding._CacheInfo()
    assert lib.gqsa_cache_info(None, C.byref(info)) == NULL
    for copy in (lib.gqsa_cache_append, lib.gqsa_cache_read):
        assert copy(None, AT, 64, 64, AT, 64, 64, 1, AT, 1, AT, None, 1, None) == NULL
    assert lib.gqsa_cache_attend(None, AT, 64, 64, 1, 1, AT, 1, AT, None, 1, 1.0, AT, 64, 64, None) == NULL
    lib.gqsa_cache_free(None)


def test_under_address_and_undefined_behaviour_sanitizers():
    from paper_2412_17560_amd import build as lib_build
    from test_sanitizers import _run_under
    if lib_build.HOST_ONLY:
        pytest.skip("this is that run")
    lib = lib_build.build_sanitized()
    runtime = lib_build.sanitizer_runtime()
    if not os.path.exists(runtime):
        pytest.skip(f"no AddressSanitizer runtime at {runtime}")
    _run_under(runtime, {"GQSA_LIBRARY": lib}, ["tests/test_attention_abi.py"])
