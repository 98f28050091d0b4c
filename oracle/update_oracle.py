"""Newton-Schulz products in binary64, from their formulas (numpy; test infrastructure only)."""
import numpy as np


def orthogonalize(x, coefficients, eps, scale, roundings=None):
    """One matrix.  roundings: (result, a bound of its error in the Frobenius norm) where every stored number is within `stored` of itself or within `floor`,
    and a sum of k products within `summed(k)` of the sum of their magnitudes: roundings = (stored, floor, summed)."""
    x = x.astype(np.float64)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    x = x / (np.linalg.norm(x) + eps)
    n, m = x.shape
    stored, floor, summed = roundings or (0.0, 0.0, lambda k: 0.0)
    size = np.linalg.norm
    error = stored * size(x) + floor * (n * m) ** 0.5
    for a, b, c in coefficients:
        g = x @ x.T
        p = a * np.eye(n) + b * g + c * (g @ g)
        s = np.linalg.svd(x, compute_uv=False)
        top_g = s[0] ** 2
        # what the step makes of the error that it finds: the largest slope between any two values of s p(s^2) on -top .. top
        t = np.linspace(0, 1.01 * s[0], 20001)
        slope = max(np.max(np.abs(a + 3 * b * t ** 2 + 5 * c * t ** 4)), np.max(np.abs(a + b * t ** 2 + c * t ** 4)))
        dg = (summed(m) + stored) * size(x) ** 2 + floor * n
        dp = (abs(b) + 2 * abs(c) * top_g) * dg + abs(c) * summed(n) * size(g) ** 2 + 4 * stored * (abs(a) * n ** 0.5 + abs(b) * size(g) + abs(c) * size(g @ g)) + 2 * floor * n
        new = p @ x
        error = 1.01 * slope * error + dp * s[0] + summed(n) * size(p) * size(x) + stored * size(new) + floor * (n * m) ** 0.5
        x = new
    x = (x.T if tall else x) * scale
    return (x, error * abs(scale)) if roundings else x


def kept(v, bits):
    """v with so many significant bits."""
    m, e = np.frexp(v)
    return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)


def in_bits(x, coefficients, eps, bits, result=24):
    """One matrix with no more rows than columns, as products of operands of so many significant bits make it: bits has those of the operands of X X^T, of G G and
    of P X (P's, X's).  Sums in binary64, everything that they give rounded to `result` bits."""
    x = kept(x.astype(np.float64) / (np.linalg.norm(x.astype(np.float64)) + eps), result)
    for a, b, c in coefficients:
        y = kept(x, bits["gram"])
        g = kept(y @ y.T, result)
        h = kept(g, bits["square"])
        p = kept(a * np.eye(len(g)) + b * g + c * (h @ h), result)
        x = kept(kept(p, bits["poly"]) @ kept(x, bits["apply"]), result)
    return x


def step_in(x, coefficients, eps, dtype=np.float32):
    """The same in numpy's products of a type."""
    x = (x.astype(np.float64) / (np.linalg.norm(x.astype(np.float64)) + eps)).astype(dtype)
    for a, b, c in np.asarray(coefficients, dtype):
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x


def as_binary32(got, want, plain):
    """Whether a result is as near to binary64's (want) as binary32's own (plain) is, within a factor of four; where little is summed binary32 rounds a X once, and
    pairs of 22 bits show three of their roundings, 3 2^-22."""
    size = np.linalg.norm
    return bool(size(got - want) <= 4 * size(plain - want) + 3 * 2.0 ** -22 * size(want))
