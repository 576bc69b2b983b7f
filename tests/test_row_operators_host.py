"""Refusals of dropout, the root-mean-square norm and the rows of 8 bits, which need no GPU; and the generator that their GPU tests compare
with, against published answers."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import binding
from tests.philox import kept, philox

P = 1 << 20          # an aligned address that is never used
A = 1 << 24          # apart from it
EINVAL, ECAPACITY = -1, -2


def call(name, good, **change):
    """The call with `good` arguments (a dict in order), some of them changed: its code.  Only for calls that are refused."""
    args = dict(good)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(binding._calls(), name)(*args.values())


def test_generator_gives_the_published_words():
    """Known answers of Philox-4x32 with ten rounds, as its authors publish them."""
    def words(counter, seed):
        return [int(w[0]) for w in philox([np.array([c], dtype=np.uint64) for c in counter], seed)]

    assert words([0] * 4, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert words([ones] * 4, ones << 32 | ones) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], 0x299F31D0 << 32 | 0xA4093822) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_generator_is_fair():
    """16 bits a value: 2^18 values at p = 0.3 keep 0.7 of them to five deviations, and each column of eight does."""
    k = kept(2048, 128, 0.3, 5, 7)
    assert abs(k.mean() - 0.7) < 5 * (0.21 / k.size) ** 0.5
    assert np.all(abs(k.reshape(-1, 8).mean(0) - 0.7) < 5 * (0.21 / (k.size / 8)) ** 0.5)
    assert not np.array_equal(k, kept(2048, 128, 0.3, 5, 8)) and not np.array_equal(k, kept(2048, 128, 0.3, 6, 7))
    assert np.array_equal(k[100:300, :50], kept(200, 50, 0.3, 5, 7, row0=100))


DROP = dict(dtype=0, X=P, ldx=24, R=None, ldr=0, m=100, C=24, drop=6554, seed=1, offset=2, d_offset=None, row0=0, Y=A, ldy=24, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": 2}, {"dtype": -1}, {"m": -1}, {"m": 1 << 31}, {"C": 0}, {"C": 16385, "ldx": 16385, "ldy": 16385}, {"ldx": 23}, {"ldy": 23}, {"R": 2 * A, "ldr": 23},
    {"drop": -1}, {"drop": 65537}, {"row0": -1}, {"row0": (1 << 32) - 99}, {"d_offset": P + 4}, {"X": None}, {"Y": None}, {"X": P + 2}, {"Y": A + 1},
    {"R": A + 2, "ldr": 24}, {"Y": P + 16}, {"Y": P, "ldy": 28}, {"R": A + 4, "ldr": 24}, {"dtype": 1, "Y": A + 1},
])
def test_dropout_add_refuses(change):
    assert call("dropout_add", DROP, **change) == EINVAL


def test_dropout_of_no_rows_is_done():
    assert call("dropout_add", DROP, m=0, X=None, Y=None, row0=1 << 32) == 0


NORM = dict(dtype=0, X=P, ldx=24, R=None, ldr=0, m=100, C=24, gamma=P, eps=1e-6, drop=0, seed=0, offset=0, d_offset=None, row0=0, out_type=0, Y=A, ldy=24,
            scale=None, S=2 * A, lds=24, rstd=3 * A, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": 2, "out_type": 2}, {"out_type": 1}, {"out_type": 3}, {"out_type": -1}, {"dtype": 1}, {"m": -1}, {"C": 0}, {"C": 16385, "ldx": 16385, "ldy": 16385, "lds": 16385},
    {"ldx": 23}, {"ldy": 23}, {"lds": 23}, {"R": 4 * A, "ldr": 20}, {"eps": -1e-9}, {"eps": float("nan")}, {"eps": float("inf")}, {"drop": 65537}, {"row0": -5},
    {"X": None}, {"Y": None}, {"out_type": 2}, {"X": P + 2}, {"S": 2 * A + 2}, {"Y": A + 3}, {"gamma": P + 2}, {"rstd": 3 * A + 1}, {"out_type": 2, "scale": A + 2},
    {"S": A}, {"S": P + 4}, {"Y": P + 96}, {"R": A + 4, "ldr": 24}, {"out_type": 2, "scale": 5 * A, "Y": P}, {"out_type": 2, "scale": 5 * A, "Y": 2 * A + 9599},
])
def test_rms_norm_fwd_refuses(change):
    assert call("rms_norm_fwd", NORM, **change) == EINVAL


BWD = dict(dtype=0, S=P, lds=24, G=A, ldg=24, D=None, ldd=0, m=100_000, C=24, gamma=P, rstd=P, drop=6554, seed=0, offset=0, d_offset=None, row0=0, dX=3 * A, lddx=24,
           dR=5 * A, lddr=24, dgamma=P, ws=7 * A, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": 2}, {"m": -1}, {"C": 0}, {"lds": 23}, {"ldg": 23}, {"lddx": 23}, {"lddr": 23}, {"D": 9 * A, "ldd": 1}, {"drop": -3}, {"row0": 1 << 32}, {"S": None}, {"G": None},
    {"rstd": None}, {"S": P + 2}, {"dX": 3 * A + 2}, {"dR": 5 * A + 1}, {"dgamma": P + 2}, {"ws": 7 * A + 2}, {"ws": None}, {"dX": 5 * A}, {"dX": A + 8}, {"dR": P + 96, "lddr": 24},
    {"dX": 5 * A + 96 * 7},
])
def test_rms_norm_bwd_refuses(change):
    assert call("rms_norm_bwd", BWD, **change) == EINVAL


def test_rms_norm_bwd_needs_its_workspace():
    b = ctypes.c_size_t(0)
    query = sagnn.lib().rms_norm_bwd_workspace_bytes
    assert query(100_000, 24, ctypes.byref(b)) == 0 and b.value > 0
    assert call("rms_norm_bwd", BWD, ws_bytes=b.value - 1) == ECAPACITY
    assert query(1, 24, ctypes.byref(b)) == 0 and b.value == 0
    assert query(-1, 24, ctypes.byref(b)) == EINVAL and query(5, 16385, ctypes.byref(b)) == EINVAL and query(5, 24, None) == EINVAL


PACK = dict(Q=P, ldq=24, scale=P, n=100, C=24, rows=P, N=50, out_type=0, out=A, ldo=24, stream=None)


@pytest.mark.parametrize("change", [
    {"out_type": 2}, {"ldq": 23}, {"ldo": 23}, {"C": 0}, {"n": -1}, {"N": -1}, {"n": 1 << 31}, {"rows": None, "N": 101}, {"Q": None}, {"scale": None}, {"out": None},
    {"out": A + 2}, {"rows": P + 2}, {"scale": P + 1}, {"out": P}, {"out": P + 2396}, {"out_type": 1, "out": A + 1},
])
def test_spmm_pack_rows_e4m3_refuses(change):
    assert call("spmm_pack_rows_e4m3", PACK, **change) == EINVAL


def test_pack_of_no_rows_is_done():
    assert call("spmm_pack_rows_e4m3", PACK, N=0, out=None, rows=None) == 0


def test_binding_refuses():
    x = torch.zeros(4, 8)
    for f in (lambda: sagnn.dropout_add(x, 0.1, 0), lambda: sagnn.rms_norm(x), lambda: sagnn.rms_norm_e4m3(x), lambda: sagnn.rms_norm_bwd(x, x, x[:, 0]),
              lambda: sagnn.spmm_pack_rows_e4m3(x.to(torch.float8_e4m3fn), x[:, 0])):
        with pytest.raises(ValueError, match="no CPU path"):
            f()
    for bad in (-0.1, 1.1, float("nan")):
        with pytest.raises(ValueError, match="probability"):
            binding._drop_args(bad, 0, 0, 0)
    for seed, offset in ((-1, 0), (1 << 64, 0), (0, -1)):
        with pytest.raises(ValueError, match="64 bits"):
            binding._drop_args(0.5, seed, offset, 0)
    assert binding._drop_args(0.5, 3, 4, 5) == (32768, 3, 4, None, 5) and binding._drop_args(1.0, 0, 0, 0)[0] == 65536
