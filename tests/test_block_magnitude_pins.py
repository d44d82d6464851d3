"""Pin of the error bound that ``oracle.block`` gives with ``magnitude=True``: the sums of
the absolute values of every term, also inside the slope of the gate."""
from __future__ import annotations

import numpy as np

import oracle.block as ob


def test_the_gates_slope_near_its_zero_is_a_sum_of_two_terms():
    # One channel, one step, C = 0: dz = dy h0 u p (1 + z (1 - p)), whose bracket vanishes at
    # z = -1.2784645.  In float32 the bracket alone is off by up to 2^-24 (1 + |z| (1 - p))
    # times its three roundings and that of p.
    z = (-1.2784645 + np.linspace(-1e-5, 1e-5, 401)).astype(np.float32)
    T = len(z)
    one = np.ones((1, T, 1))
    args = dict(dy=one, A=np.array([[-1.0]]), dt=one, Bm=one[..., None], Cm=0 * one[..., None], u=one, h0=np.ones(1),
                z=z.reshape(1, T, 1))
    ref = ob.selective_grad(**args)["dz"].ravel()
    mag = ob.selective_grad(**args, magnitude=True)["dz"].ravel()
    p = (np.float32(1) / (np.float32(1) + np.exp(-z))).astype(np.float32)
    got = p * (np.float32(1) + z * (np.float32(1) - p))
    assert np.abs(ref).max() < 1e-5
    assert (np.abs(got.astype(np.float64) - ref) <= 16 * 2.0 ** -24 * mag).all()
    assert (mag < 1).all()
