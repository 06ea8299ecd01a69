"""What the calls of a decoding step of several drafted tokens refuse, before anything touches a GPU: with no handle, and with one that lies in host memory only (a call
that refuses nothing ends at the device it was made for)."""
from __future__ import annotations

import ctypes as C
import os

import pytest

from paper_2412_17560_amd import binding

NULL, SHAPE, UNSUPPORTED, RANGE, HIP, BUFSIZE, ALIGN = 1, 2, 3, 4, 6, 7, 8
AT = 1 << 20        # an aligned address that no call gets to use


class _Cache(C.Structure):      # (gqsa_attention.hpp)
    _fields_ = [("n_pages", C.c_int64), ("page_tokens", C.c_int), ("kv_heads", C.c_int), ("head_dim", C.c_int), ("device", C.c_int),
                ("d_pages", C.c_void_p), ("d_partials", C.c_void_p), ("d_arrivals", C.c_void_p)]


class _Verifier(C.Structure):   # (gqsa_verify.hpp)
    _fields_ = [("max_seqs", C.c_int), ("max_vocab", C.c_int), ("device", C.c_int), ("d_sums", C.c_void_p), ("d_arrivals", C.c_void_p)]


CACHE = _Cache(10, 32, 2, 64, -1, None, None, None)
VERIFIER = _Verifier(3, 100, -1, None, None)


def tree(**change):
    a = dict(c=C.addressof(CACHE), q=AT, q_row=256, q_head=64, q_heads=4, rows=2, pages=AT, max_pages=2, lengths=AT, starts=AT, n_seqs=1, masks=AT, words=1, scale=0.1,
             out=AT, o_row=256, o_head=64)
    assert not set(change) - set(a)
    return binding._lib().gqsa_cache_attend_tree(*{**a, **change}.values(), None)


def append(**change):
    a = dict(c=C.addressof(CACHE), q=AT, q_row=256, q_head=64, q_heads=4, k=AT, k_row=128, k_head=64, v=AT, v_row=128, v_head=64, rows=2, qw=AT, kw=AT, eps=1e-6, table=AT,
             n_positions=9, rotary=64, interleaved=0, positions=AT, qo=AT, qo_row=256, qo_head=64, ko=AT, ko_row=128, ko_head=64, pages=AT, max_pages=2, lengths=AT,
             starts=AT, n_seqs=1)
    assert not set(change) - set(a)
    return binding._lib().gqsa_cache_append_rotated(*{**a, **change}.values(), None)


def keep(**change):
    a = dict(c=C.addressof(CACHE), rows=2, pages=AT, max_pages=2, lengths=AT, starts=AT, n_seqs=1, path=AT, accepted=AT)
    assert not set(change) - set(a)
    return binding._lib().gqsa_cache_keep(*{**a, **change}.values(), None)


def verify(**change):
    a = dict(v=C.addressof(VERIFIER), target=AT, target_row=100, draft=None, draft_row=0, vocab=100, rows=6, tokens=AT, parents=AT, uniforms=AT, finals=AT, starts=AT,
             n_seqs=3, path=AT, out=AT, accepted=AT)
    assert not set(change) - set(a)
    return binding._lib().gqsa_verify(*{**a, **change}.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(), HIP), (dict(c=None), NULL), (dict(q=None), NULL), (dict(out=None), NULL), (dict(masks=None), NULL), (dict(pages=None), NULL), (dict(lengths=None), NULL),
    (dict(words=0), SHAPE), (dict(words=-1), SHAPE), (dict(words=(1 << 15) + 1), UNSUPPORTED), (dict(words=1 << 15), HIP), (dict(masks=AT + 2), ALIGN), (dict(q_heads=3), SHAPE),
    (dict(starts=None), SHAPE), (dict(starts=None, n_seqs=2), HIP), (dict(rows=-1), SHAPE), (dict(rows=(1 << 25) + 1), SHAPE), (dict(scale=float("inf")), RANGE),
    (dict(scale=float("nan")), RANGE), (dict(q=AT + 8), ALIGN), (dict(o_head=60), ALIGN), (dict(q_row=-8), SHAPE), (dict(n_seqs=65537), UNSUPPORTED), (dict(q_heads=2048), UNSUPPORTED)])
def test_attend_tree_refuses(change, status):
    assert tree(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(), HIP), (dict(c=None), NULL), (dict(q=None), NULL), (dict(qo=None), NULL), (dict(q=None, qo=None, q_heads=0), HIP), (dict(k=None), NULL), (dict(v=None), NULL),
    (dict(ko=None), HIP), (dict(table=None), NULL), (dict(table=None, rotary=0, positions=None), HIP), (dict(positions=None), HIP), (dict(qw=None, kw=None), HIP),
    (dict(pages=None), NULL), (dict(q_heads=-1), SHAPE), (dict(q_heads=1025), UNSUPPORTED), (dict(q_heads=7), HIP), (dict(rotary=24), UNSUPPORTED), (dict(rotary=80), UNSUPPORTED),
    (dict(rotary=-16), UNSUPPORTED), (dict(n_positions=-1), SHAPE), (dict(eps=float("nan")), RANGE), (dict(eps=-1.0), RANGE), (dict(ko=AT + 2), ALIGN), (dict(qw=AT + 8), ALIGN),
    (dict(kw=AT + 8), ALIGN), (dict(table=AT + 4), ALIGN), (dict(positions=AT + 1), ALIGN), (dict(ko_row=12), ALIGN), (dict(v_head=-64), SHAPE), (dict(starts=None), SHAPE),
    (dict(rows=-1), SHAPE), (dict(max_pages=0), SHAPE), (dict(max_pages=(1 << 20) + 1), UNSUPPORTED)])
def test_append_rotated_refuses(change, status):
    assert append(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(), HIP), (dict(c=None), NULL), (dict(path=None), NULL), (dict(accepted=None), NULL), (dict(pages=None), NULL), (dict(path=AT + 2), ALIGN), (dict(accepted=AT + 1), ALIGN),
    (dict(starts=None), SHAPE), (dict(n_seqs=0), SHAPE), (dict(rows=-1), SHAPE), (dict(lengths=AT + 2), ALIGN)])
def test_keep_refuses(change, status):
    assert keep(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(), HIP), (dict(v=None), NULL), (dict(target=None), NULL), (dict(tokens=None), NULL), (dict(uniforms=None), NULL), (dict(finals=None), NULL), (dict(path=None), NULL),
    (dict(out=None), NULL), (dict(accepted=None), NULL), (dict(parents=None), HIP), (dict(draft=AT), UNSUPPORTED), (dict(draft=AT, parents=None), HIP), (dict(vocab=101), BUFSIZE),
    (dict(n_seqs=4), BUFSIZE), (dict(vocab=0), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=(1 << 25) + 1), SHAPE), (dict(n_seqs=0), SHAPE), (dict(starts=None), SHAPE),
    (dict(starts=None, rows=3), HIP), (dict(target=AT + 2), ALIGN), (dict(tokens=AT + 1), ALIGN), (dict(draft=AT + 2, parents=None), ALIGN), (dict(accepted=AT + 2), ALIGN),
    (dict(target_row=-1), SHAPE), (dict(draft_row=-4), SHAPE), (dict(target_row=(1 << 31) + 1), SHAPE)])
def test_verify_refuses(change, status):
    assert verify(**change) == status


def test_no_rows_is_no_work():
    assert tree(rows=0, q=None) == 0 and append(rows=0, k=None) == 0 and keep(rows=0, path=None) == 0


@pytest.mark.parametrize("args, status", [((0, 10), SHAPE), ((1, 0), SHAPE), ((65537, 10), UNSUPPORTED), ((1, (1 << 22) + 1), UNSUPPORTED), ((65536, 1 << 19), SHAPE)])
def test_verify_create_refuses(args, status):
    out = C.c_void_p(123)
    assert binding._lib().gqsa_verify_create(*args, C.byref(out)) == status
    assert out.value is None
    assert binding._lib().gqsa_verify_create(*args, None) == NULL
    binding._lib().gqsa_verify_free(None)


def test_under_address_and_undefined_behaviour_sanitizers():
    from paper_2412_17560_amd import build as lib_build
    from test_sanitizers import _run_under
    if lib_build.HOST_ONLY:
        pytest.skip("this is that run")
    lib = lib_build.build_sanitized()
    runtime = lib_build.sanitizer_runtime()
    if not os.path.exists(runtime):
        pytest.skip(f"no AddressSanitizer runtime at {runtime}")
    _run_under(runtime, {"GQSA_LIBRARY": lib}, ["tests/test_drafts_abi.py"])
