"""The models of a generating step against other definitions of the same, on the CPU."""
import math

import numpy as np
import pytest
import torch

import step_model as model


def test_weights_are_probabilities():
    rng = np.random.default_rng(1)
    for scale in (1.0, 0.3, 2.7):
        x = np.concatenate([rng.standard_normal(3000) * 4, [11.0, 11.0, -np.inf, -3.4e38, 20.0]]).astype(np.float32)
        w, _ = model.weights(x, scale)
        want = np.exp2((x.astype(np.float64) - x.max()) * scale * np.log2(np.e)) * 2.0**40
        # P is within 2^-21, t within three roundings of up to 41; below 1 the weight is cut to whole numbers
        assert (np.abs(w - want) <= want * (2.0**-21 + 41 * math.log(2) * 3 * 2.0**-24) + 1).all()
        assert w[x == x.max()].tolist() == [2**40] and not w[np.isneginf(x)].any()


def test_drawn_tokens_follow_their_probabilities():
    rng = np.random.default_rng(2)
    x = rng.standard_normal(23) * 2
    x[5] = x[6] = x.max() + 0.5
    for kw in (dict(top_k=0, top_p=1.0, min_p=0.0), dict(top_k=7, top_p=1.0, min_p=0.0), dict(top_k=0, top_p=0.8, min_p=0.0),
               dict(top_k=12, top_p=0.9, min_p=0.1)):
        n = 4096
        drawn = [model.sample(x, (i + 0.5) / n, scale=1.0, **kw) for i in range(n)]
        p = np.exp(x.astype(np.float32).astype(np.float64))
        order = np.argsort(-p, kind="stable")
        keep = order[:kw["top_k"] or len(x)]
        share = np.cumsum(p[keep]) / p[keep].sum()
        keep = keep[:int(np.searchsorted(share, kw["top_p"])) + 1] if kw["top_p"] < 1 else keep
        keep = keep[p[keep] >= kw["min_p"] * p.max()]
        want = np.zeros(len(x))
        want[keep] = p[keep] / p[keep].sum()
        got = np.bincount([i for i, _, _ in drawn], minlength=len(x)) / n
        assert np.abs(got - want).max() <= 1.5 / n and {k for _, _, k in drawn} == {len(keep)}
        for i, lp, _ in drawn[::97]:
            assert abs(lp - math.log(want[i])) <= 2.0**-20


def test_stored_values_are_the_nearest_that_8_bits_hold():
    """Against the type of torch, and every code against its value."""
    codes = np.arange(256)
    as_torch = torch.from_numpy(codes.astype(np.uint8)).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(model.held(codes, np.int64(127)), as_torch, equal_nan=True)
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((500, 48)) * 10.0 ** rng.uniform(-38, 30, (500, 1))).astype(np.float32)
    x[3] = 0
    x[4, 1] = np.inf
    x[5, 2] = np.nan
    x[6] = 0
    x[6, 0] = 448.0 * 2.0**-130
    x[7, 0] = 448.0
    x[8, 0] = 449.0
    x = torch.from_numpy(x).bfloat16()
    values, code, power = model.stored(x.double().numpy())
    fine = np.isfinite(x.double().numpy())
    scaled = (x.double() * torch.exp2(127.0 - torch.from_numpy(power).double())[:, None]).float()
    want = scaled.to(torch.float8_e4m3fn)
    assert np.array_equal(want.view(torch.uint8).numpy()[fine], code[fine]) and not np.isfinite(values[~fine]).any()
    assert np.array_equal(model.held(np.where(fine, code, 127), power)[fine], values[fine])
    most = np.where(fine, np.abs(x.double().numpy()), 0).max(1)
    at = most / 2.0**(power - 127.0)
    assert (((at > 224) | (power == 1)) & (at <= 448)).all()
    assert (np.abs(values - x.double().numpy())[fine] <= np.maximum(2.0**-4 * np.abs(x.double().numpy()),
                                                                    2.0**-10 * 2.0**(power - 127.0)[:, None])[fine]).all()


@pytest.mark.parametrize("eps", [1e-6, 1e-2])
def test_norms_by_hand(eps):
    x, y = np.array([[3.0, 4.0]]), np.array([[1.0, -2.0]])
    s, h = model.norm(x, np.array([2.0, 1.0]), y, np.array([1.0, 0.5]), np.array([0.5, 2.0]), -1.0, eps)
    r = math.sqrt(2.5 + eps)
    assert np.allclose(s, [[3.0 - 0.5 / r, 4.0 + 2.0 / r]], rtol=1e-15)
    assert np.allclose(h, s / math.sqrt((s * s).mean() + eps) * [2.0, 1.0], rtol=1e-15)
