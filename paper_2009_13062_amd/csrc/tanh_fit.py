#!/usr/bin/env python3
"""Fits of the tanh polynomials in logprob_kernels.h (kTanhNearFit, kTanhWideFit).

tanh(u) / u is a smooth function of w = u^2.  The polynomial of a degree that is nearest to it on [0, r^2] in the relative error has degree + 2 points of the same largest error with
signs in turn; the exchange below (Remez) looks for them: it solves for the polynomial and that error on a set of points, takes the extrema of the error for the next set, and ends when they
stay.  Coefficients are then rounded to float32.  Needs numpy only.

    python tanh_fit.py            prints the coefficients (constant term first), the error of the fit and that of its evaluation in float32
"""
import numpy as np

NEAR = (0.35, 3)                                   # largest |u|, degree in u^2
WIDE = (0.8, 5)


def quotient(w):
    """tanh(u) / u of w = u^2"""
    u = np.sqrt(np.maximum(w, 1e-300))
    return np.where(w > 0, np.tanh(u) / u, 1.0)


def fit(reach, degree, rounds=30):
    n = degree + 2
    at = (1 - np.cos(np.pi * np.arange(n) / (n - 1))) / 2 * reach * reach
    grid = np.linspace(0, reach * reach, 200001)
    for _ in range(rounds):
        A = np.hstack([np.vander(at, degree + 1, increasing=True), ((-1.0) ** np.arange(n) * quotient(at))[:, None]])
        c = np.linalg.solve(A, quotient(at))[:-1]
        error = np.polyval(c[::-1], grid) / quotient(grid) - 1
        ends = [0] + list(np.nonzero(np.diff(np.sign(error)))[0] + 1) + [len(grid)]
        extrema = [a + int(np.argmax(np.abs(error[a:b]))) for a, b in zip(ends[:-1], ends[1:])]
        if len(extrema) != n:
            break
        at = grid[extrema]
    return [float(x) for x in c.astype(np.float32)]


def tanh_f32(u, c):
    """u P(u^2) in float32, each multiply-add rounded once"""
    u = np.asarray(u, np.float32)
    w = (u * u).astype(np.float32)
    p = np.full_like(u, np.float32(c[-1]))
    for x in c[-2::-1]:
        p = (p.astype(np.float64) * w + np.float32(x)).astype(np.float32)
    return (u * p).astype(np.float32)


def max_relative_error(c, reach, n=400001):
    u = np.linspace(1e-6, reach, n).astype(np.float32)
    return float(np.abs(tanh_f32(u, c) / np.tanh(u.astype(np.float64)) - 1).max())


if __name__ == "__main__":
    for reach, degree in (NEAR, WIDE):
        c = fit(reach, degree)
        print("up to %g: %s, in float32 within 2^%.2f" % (reach, c, np.log2(max_relative_error(c, reach))))
