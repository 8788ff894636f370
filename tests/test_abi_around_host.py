"""Refusals of the calls around the attention, without a GPU: every one of these returns before a launch.  The
plan is a block of host memory that begins with the problem, which is all that the checks read."""
import ctypes

import pytest

from paper_2602_24082_b200 import binding as B
from paper_2602_24082_b200 import build as build_mod
from paper_2602_24082_b200 import workloads as W


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.lib()


@pytest.fixture(scope="module")
def plan():
    w = W.Workload("e", [[(5, (2, 4))]], 4, 2, 64, seed=0)
    p, keep = B.make_problem(w.descriptors(), 4, 2, 64, w.total_tokens)
    buf = ctypes.create_string_buffer(4096)
    ctypes.memmove(buf, ctypes.byref(p), ctypes.sizeof(p))
    buf.keep = (p, keep)
    return buf


class Policy(ctypes.Structure):
    _fields_ = [("advantage_mode", ctypes.c_int32), ("reduction", ctypes.c_int32)] + [
        (n, ctypes.c_double) for n in ("clip_low", "clip_high", "kl_coef", "scale", "eps")]


A = 4096     # an aligned address that nothing reads


def test_token_logp(lib, plan):
    fwd = [plan, A, 0, 100, 100, A, 0, 1.0, A, A, None]
    bwd = [plan, A, 0, 100, 100, A, 0, 1.0, A, A, A, 2 * A, 100, None]
    for call, good in ((lib.pp_token_logp, fwd), (lib.pp_token_logp_bwd, bwd)):
        for i, bad, code in ((0, None, -1), (1, None, -1), (5, None, -1), (8, None, -1), (9, None, -1), (3, 99, -1), (4, 0, -1),
                             (4, -5, -1), (2, 3, -2), (2, -1, -2), (7, 0.0, -1), (7, -1.0, -1), (7, float("nan"), -1),
                             (7, float("inf"), -1), (1, A + 1, -4), (9, A + 4, -4)):
            args = list(good)
            args[i] = bad
            assert call(*args) == code, (call, i, bad)
    for i, bad, code in ((10, None, -1), (11, None, -1), (12, 99, -1), (11, A + 1, -4)):
        args = list(bwd)
        args[i] = bad
        assert lib.pp_token_logp_bwd(*args) == code
    same = list(bwd)
    same[11], same[12] = A, 101               # the logits' memory under another stride
    assert lib.pp_token_logp_bwd(*same) == -1


def test_policy_loss(lib, plan):
    nan = float("nan")
    good = dict(advantage_mode=2, reduction=0, clip_low=0.2, clip_high=0.2, kl_coef=0.0, scale=1.0, eps=1e-6)
    call = lambda o, *a: lib.pp_policy_loss(plan, None if o is None else ctypes.byref(Policy(**o)), *a)
    args = (A, None, None, A, None, None, A, A, A, None, None)
    for name, bad in (("advantage_mode", 4), ("advantage_mode", -1), ("reduction", 2), ("clip_low", -0.1), ("clip_low", 1.1),
                      ("clip_low", nan), ("clip_high", -0.1), ("clip_high", nan), ("clip_high", 1e31), ("kl_coef", -1.0), ("kl_coef", nan),
                      ("scale", nan), ("scale", 1e31), ("eps", 0.0), ("eps", nan)):
        assert call(dict(good, **{name: bad}), *args) == -1, name
    assert call(None, *args) == -1
    for i in (0, 3, 6, 7, 8):
        assert call(good, *[None if j == i else x for j, x in enumerate(args)]) == -1
    assert lib.pp_policy_loss(None, ctypes.byref(Policy(**good)), *args) == -1


def test_axes(lib, plan):
    assert lib.pp_position_ids_axes(None, 0, None, None, A, A, None) == -1
    for args in ((-1, A, A, A, A), (1, None, A, A, A), (1, A, None, A, A), (0, None, None, None, A), (0, None, None, A, None)):
        assert lib.pp_position_ids_axes(plan, *args, None) == -1
    axis = ctypes.create_string_buffer(bytes([0, 1, 2] * 10 + [0, 0]), 32)
    good = [plan, A, 256, 2 * A, 128, 3 * A, 256, 4 * A, 128, A, 3, axis, 10000.0, 0, None]
    for i, bad, code in ((0, None, -1), (1, None, -1), (3, None, -1), (5, None, -1), (7, None, -1), (9, None, -1), (11, None, -1),
                         (2, 248, -1), (4, 120, -1), (6, 248, -1), (8, 120, -1), (10, 0, -1), (10, 5, -1), (10, 2, -1),
                         (12, 1.0, -1), (12, float("nan"), -1), (12, 1e13, -1), (1, A + 8, -4), (7, A + 8, -4), (2, 260, -4),
                         (8, 132, -4)):
        args = list(good)
        args[i] = bad
        assert lib.pp_rope_qk_axes(*args) == code, (i, bad)
    for i, j in ((5, 6), (7, 8)):             # in place under another stride
        args = list(good)
        args[i], args[j] = args[i - 4], args[j] + 8
        assert lib.pp_rope_qk_axes(*args) == -1
    for i, other in ((5, 7), (7, 5), (5, 3), (7, 1)):     # one tensor's output on the other tensor
        args = list(good)
        args[i] = args[other]
        assert lib.pp_rope_qk_axes(*args) == -1, (i, other)


def test_sizes_beyond_32_bit_indices(lib, plan):
    w = W.Workload("e", [[(5, (2, 4))]], 4, 2, 64, seed=0)
    p, keep = B.make_problem(w.descriptors(), 4, 2, 64, 2 ** 31 - 1000)
    long = ctypes.create_string_buffer(4096)
    ctypes.memmove(long, ctypes.byref(p), ctypes.sizeof(p))
    axis = ctypes.create_string_buffer(bytes(32), 32)
    policy = ctypes.byref(Policy(2, 0, 0.2, 0.2, 0.0, 1.0, 1e-6))
    assert lib.pp_token_logp(long, A, 0, 100, 100, A, 0, 1.0, A, A, None) == -2
    assert lib.pp_token_logp(plan, A, 0, 2 ** 31, 2 ** 30 + 1, A, 0, 1.0, A, A, None) == -2
    assert lib.pp_token_logp_bwd(long, A, 0, 100, 100, A, 0, 1.0, A, A, A, 2 * A, 100, None) == -2
    assert lib.pp_policy_loss(long, policy, A, None, None, A, None, None, A, A, A, None, None) == -2
    assert lib.pp_rope_qk_axes(long, A, 256, 2 * A, 128, 3 * A, 256, 4 * A, 128, A, 3, axis, 10000.0, 0, None) == -2
    assert lib.pp_position_ids_axes(long, 0, None, None, A, A, None) == -2
    assert lib.pp_position_ids_axes(plan, 12, A, A, A, A, None) == -1      # more spans than tokens


def test_more_spans_than_32_bit_indices_of_their_sides(lib):
    """Three int32 sides a span: entries from 2^31 on begin with span 715827883."""
    w = W.Workload("e", [[(5, (2, 4))]], 4, 2, 64, seed=0)
    p, keep = B.make_problem(w.descriptors(), 4, 2, 64, 2 ** 31 - 70000)
    long = ctypes.create_string_buffer(4096)
    ctypes.memmove(long, ctypes.byref(p), ctypes.sizeof(p))
    for n in (2 ** 24 + 1, 715827883, 2 ** 30, 2 ** 31 - 70000):
        assert lib.pp_position_ids_axes(long, n, None, None, A, A, None) == -2
    assert lib.pp_position_ids_axes(long, 2 ** 24, None, None, A, A, None) == -1       # (no arrays)


def test_outputs_that_overlap_their_inputs(lib, plan):
    """11 tokens.  Rows that share bytes are refused.  Rows side by side in one buffer are not: those calls go on to the
    check of alignment, which a shift of all by 8 bytes ends."""
    bwd = lambda x, d, V, stride: lib.pp_token_logp_bwd(plan, x, 0, stride, V, A, 0, 1.0, A, A, A, d, stride, None)
    x = 1 << 20
    for shift in (2, 100, 198, 400 - 198, 398, 400 + 20, 4000, 4000 + 198, -2, -198, -398, -4000, -4000 - 198):
        assert bwd(x, x + shift, 100, 200) == -1, shift
    axis = ctypes.create_string_buffer(bytes([0, 1, 2] * 10 + [0, 0]), 32)
    rope = lambda q, k, qo, ko, s: lib.pp_rope_qk_axes(plan, q, s, k, s, qo, s, ko, s, A, 3, axis, 10000.0, 0, None)
    s, h, far = 640, 128, 1 << 22           # a token of the fused buffer: 10 heads of 64, 128 bytes each; q 4 of them, k 2
    for args in ((x, x + 4 * h, x + h, far), (x, x + 4 * h, x + 3 * h, far), (x + h, x + 5 * h, x, far), (x, x + 4 * h, far, x + 5 * h),
                 (x, x + 4 * h, far, x + 3 * h), (x, x + 4 * h, x + 5 * h, far), (x, far, x + 7 * h, far), (far, x, 2 * far, x + 2 * s + h),
                 (x, x + 4 * h, far, far + 3 * h), (x, x + 4 * h, far + 2 * s * 9 + h, far), (x, far, x + 10 * 2 * s + 3 * h, 3 * far)):
        assert rope(*args, s) == -1, args
    # side by side, one after the other, in place: nothing but the alignment is wrong
    for args in ((x, x + 4 * h, x + 6 * h, far), (x, x + 4 * h, far, x + 6 * h), (x, x + 4 * h, x, x + 4 * h), (x, x + 4 * h, far, far + 4 * h),
                 (x, far, x + 10 * 2 * s + 4 * h, 3 * far), (far, x, 2 * far, x - 10 * 2 * s - 2 * h)):
        assert rope(*[a + 8 for a in args], s) == -4, args
