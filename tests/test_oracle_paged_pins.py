"""Pins of the paged cache's oracle by facts that do not retype it: the dense
oracle's rows, torch's float8 conversion, and the error bounds of the formats."""

import numpy as np
import pytest
import torch

import oracle
from oracle import paged


def rnd(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def test_chunk_rows_are_the_causal_reads_rows():
    q, k, v = rnd(1, 2, 23, 8), rnd(2, 2, 23, 8), rnd(3, 2, 23, 5)
    beta = np.exp(rnd(4, 2, 5))
    want = oracle.fem_softmax(q[None], k[None], v[None], beta)[0]  # [H, T, dv]
    for n in (1, 7, 23):
        new = q[:, 23 - n:].transpose(1, 0, 2)
        got = oracle.fem_paged(new, [k], [v], beta, [0, n])
        np.testing.assert_allclose(got.transpose(1, 0, 2), want[:, 23 - n:], rtol=0, atol=1e-12)


def test_ragged_batch_groups_and_encoder():
    beta = np.exp(rnd(5, 2, 4))
    ks = [rnd(10 + b, 2, n, 6) for b, n in enumerate((9, 4, 1))]
    vs = [rnd(20 + b, 2, n, 4) for b, n in enumerate((9, 4, 1))]
    q = rnd(30, 8, 6, 6)  # three query heads a cached head; the last two tokens are nobody's
    starts = [0, 5, 5, 6]
    got = oracle.fem_paged(q, ks, vs, beta, starts, causal=False)
    assert np.isnan(got[6:]).all()
    for t, b in ((0, 0), (4, 0), (5, 2)):
        for h in range(6):
            want = oracle.fem_softmax_decode(q[t, h][None, None], ks[b][None, [h // 3]],
                                             vs[b][None, [h // 3]], [ks[b].shape[1]], beta[[h // 3]])
            np.testing.assert_allclose(got[t, h], want[0, 0], rtol=0, atol=1e-12)
    assert np.isnan(oracle.fem_paged(q[:1], [ks[0][:, :0]], [vs[0][:, :0]], beta, [0, 1],
                                     causal=False)).all()


@pytest.mark.parametrize("kind,half", [("e4m3", 2.0 ** -4), ("int8", None)])
def test_storing(kind, half):
    x = torch.from_numpy(rnd(6, 50, 64) * 2.0 ** np.random.default_rng(7).integers(-30, 30, (50, 1)))
    x = x.bfloat16().double().numpy()
    codes, byte = oracle.codes_of(x, kind)
    got = oracle.values_of(codes, byte, kind)
    step = 2.0 ** (byte.astype(float) - 127).repeat(32, -1)
    # the scale is the smallest that reaches the block's largest value
    top = np.abs(x).reshape(50, 2, 32).max(-1)
    s = step.reshape(50, 2, 32)[..., 0]
    assert (top <= paged.LARGEST[kind] * s).all() and (top > paged.LARGEST[kind] * s / 2).all()
    if half is None:  # integers: half a step of the scale
        assert (np.abs(got - x) <= step / 2).all()
    else:             # half a step relative, or half the smallest step
        assert (np.abs(got - x) <= np.maximum(half * np.abs(x), step * 2.0 ** -10)).all()
        y = torch.from_numpy(x / step).float().to(torch.float8_e4m3fn)
        assert (y.view(torch.uint8).numpy() == codes).all()
    # every value is a bf16 number, and storing it again changes nothing
    assert (torch.from_numpy(got).bfloat16().double().numpy() == got).all()
    assert (oracle.stored(got, kind) == got).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_storing_borders(kind):
    x = np.zeros((6, 32))
    x[1, 3] = 2.0 ** -126             # below the least scale's smallest code: zero
    x[2, 0], x[2, 1] = -np.inf, 1.0   # the block is NaN
    x[3, 5] = np.nan
    x[4, 0] = paged.LARGEST[kind]     # reaches the largest code exactly
    x[4, 1:4] = 0.5, 1.5, -2.5        # ties of the integers
    x[5, 0] = 3.3895313892515355e38   # the largest bf16
    codes, byte = oracle.codes_of(x, kind)
    assert (byte[:2, 0] == 27).all() and (codes[:2] == 0).all()
    assert (byte[2:4, 0] == 255).all() and np.isnan(oracle.values_of(codes, byte, kind)[2:4]).all()
    assert byte[4, 0] == 127
    if kind == "int8":
        assert list(codes[4, 1:4].view(np.int8)) == [0, 2, -2]
    v = oracle.values_of(codes, byte, kind)
    assert v[4, 0] == paged.LARGEST[kind] and np.isfinite(v[5]).all()
