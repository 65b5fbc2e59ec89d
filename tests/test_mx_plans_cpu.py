"""The 4-bit product's choice of kernels (dn::gemm_mx4_plan, a host function of the library) and the
sizes that no launch of it can hold: a launch has less than 2^32 threads."""

import ctypes as C

import pytest

from paper_2511_06724_amd import dn
from tests.plans import CUS

P = 4096  # a 16-byte aligned address that is never followed
THREADS = {(32, 32): 512, (32, 64): 512, (128, 256): 256, (64, 128): 256, (64, 160): 320}


class Plan(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("bm", "bn", "small")]


def plan(M, N, K, geglu=False):
    """(bm, bn, small): N counts the accumulator's columns."""
    f = getattr(dn.lib, "_ZN2dn13gemm_mx4_planEiiibi")
    f.argtypes, f.restype = [C.c_int] * 3 + [C.c_bool, C.c_int], Plan
    g = f(M, N, K, geglu, CUS)
    return g.bm, g.bn, g.small


def groups(M, N, bm, bn, small=0):
    mt, nt = -(-M // bm), -(-N // bn)
    return mt * (nt - small) + -(-M // 64) * small if bm == 128 else mt * nt


@pytest.mark.parametrize("M,N,K,want,us,other", [
    (200, 1280, 5120, (32, 32), 9.4, "64 x 128 tiles 11.0"), (128, 5120, 2560, (64, 128), 6.2, "few rows 8.4"),
    (4096, 4096, 4096, (128, 256), 39.8, "64 x 128 58"), (2048, 1280, 5120, (64, 160), 15.0, "64 x 128 19.8"),
    (700, 1280, 2560, (64, 128), 8.4, "64 x 160 9.2")])
def test_plans_are_the_measured_best(M, N, K, want, us, other):
    assert plan(M, N, K)[:2] == want, f"{us} us wanted, {other}"


@pytest.mark.parametrize("M,N,K,want,us,other", [
    (77, 10240, 1280, (32, 64, 0), 5.8, "tiles 8.6"), (300, 5120, 640, (128, 256, 20), 5.6, "128 rows 7.2"),
    (8192, 5120, 640, (128, 256, 0), 29.0, "64 rows 33.7"), (2048, 10240, 1280, (128, 256, 8), 22.4, "128 rows 24.8")])
def test_geglu_plans_are_the_measured_best(M, N, K, want, us, other):
    assert plan(M, N, K, geglu=True) == want, f"{us} us wanted, {other}"


@pytest.mark.parametrize("geglu", [False, True])
def test_plans_fit_a_launch(geglu):
    """Whatever passes the checks of the call is given tiles that one launch holds."""
    for M in (1, 33, 1000, 10 ** 6, 2 ** 24, 2 ** 28 + 1, 2 ** 30, 2 ** 30 + 1, 2 ** 31 - 128):
        for N in (64, 128, 192, 256, 320, 640, 5120, 2 ** 18, 2 ** 22):
            if -(-M // 128) * -(-N // 256) * 256 >= 2 ** 32:
                continue
            bm, bn, small = plan(M, N, 128, geglu)
            assert groups(M, N, bm, bn, small) * THREADS[bm, bn] < 2 ** 32, (M, N, bm, bn, small)


@pytest.mark.parametrize("M,N,K,geglu", [(2 ** 31 - 1, 32, 128, 0), (2 ** 31 - 127, 32, 128, 1), (2 ** 30, 288, 128, 0), (2 ** 24, 2 ** 18, 128, 0)])
def test_more_tiles_than_a_launch_holds_refused(M, N, K, geglu):
    assert dn.lib.dn_op_linear(dn.DN_MXFP4, P, P, None, None, 0, P, 0, M, N, K, geglu, None) == dn.DN_EINVAL
    assert b"one launch" in dn.lib.dn_last_error()


def test_a_product_that_only_the_largest_tiles_hold_is_planned_with_them():
    """2^24 tiles of 64 rows are one more than a launch holds: 73 GB of x, 69 GB of bf16 y."""
    assert plan(2 ** 30, 32, 128)[:2] == (128, 256)


def test_geglu_tiles_are_not_all_small_for_a_short_last_round():
    for M in (65664, 10 ** 6 + 100, 2 ** 30 + 1):
        for N in (64, 256):
            assert plan(M, N, 640, geglu=True) == (128, 256, 0), (M, N)
    assert plan(33024, 512, 640, geglu=True) == (128, 256, 1)
