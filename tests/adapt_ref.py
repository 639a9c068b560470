"""Plain float64 definitions of the adapter and orthogonalisation operators (numpy), and error bounds."""
import numpy as np

U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # unit roundoff: 24, 8 and 11 significant bits
U32 = 2.0 ** -24


def pairs_of_rows(T, offsets, adapter, S):
    """The pair of each row, -1 for none."""
    out = np.full(T, -1, dtype=np.int64)
    for i, a in enumerate(adapter):
        lo, hi = max(0, int(offsets[i])), min(T, int(offsets[i + 1]))
        if 0 <= a < S:
            out[lo:hi] = a
    return out


def forward(x, W, bias, A, B, scale, pair):
    """y, v and the sums of absolute values behind each entry of y and v."""
    y = x @ W.T
    ay = np.abs(x) @ np.abs(W).T
    if bias is not None:
        y = y + bias
        ay = ay + np.abs(bias)
    v = np.zeros((x.shape[0], A.shape[1]))
    av = np.zeros_like(v)
    for a in range(A.shape[0]):
        t = np.flatnonzero(pair == a)
        if t.size:
            v[t] = x[t] @ A[a].T
            av[t] = np.abs(x[t]) @ np.abs(A[a]).T
            y[t] += scale[a] * (v[t] @ B[a].T)
            ay[t] += abs(scale[a]) * (av[t] @ np.abs(B[a]).T)
    return y, v, ay, av


def backward(dy, x, W, A, B, scale, pair, v):
    dx, adx = dy @ W, np.abs(dy) @ np.abs(W)
    dA, dB = np.zeros(A.shape), np.zeros(B.shape)
    aA, aB = np.zeros(A.shape), np.zeros(B.shape)
    for a in range(A.shape[0]):
        t = np.flatnonzero(pair == a)
        if t.size:
            u, au = dy[t] @ B[a], np.abs(dy[t]) @ np.abs(B[a])
            s = scale[a]
            dx[t] += s * (u @ A[a])
            adx[t] += abs(s) * (au @ np.abs(A[a]))
            dA[a], aA[a] = s * (u.T @ x[t]), abs(s) * (au.T @ np.abs(x[t]))
            dB[a], aB[a] = s * (dy[t].T @ v[t]), abs(s) * (np.abs(dy[t]).T @ np.abs(v[t]))
    return dx, dA, dB, adx, aA, aB


def bound(ref, absolute, terms, dtype, out=None):
    """Elementwise error bound of a result that is rounded once to ``out``.

    Sums of ``terms`` products in float32 in any order: (terms + 16) u32 of the
    sum of absolute values.  The 16 covers what each factor may lose when it
    goes to the matrix cores as a sum of two 16-bit numbers: float32 as two
    float16 (2^-22 each and the dropped product, 12 u32).  Factors that were
    computed before (v, u) go as two bfloat16 (relative 2^-16) where the type
    is bfloat16: 256 u32.  The absolute floor covers float16 sub-normals of rows
    scaled to their largest value.
    """
    extra = 16.0 if dtype != "bf16" else 256.0
    return (U[out or dtype] * np.abs(ref) + (terms + extra) * U32 * absolute * 1.01
            + 2.0 ** -36 * np.max(absolute, initial=0.0) + (6e-8 if (out or dtype) == "f16" else 1e-38))


def newton_schulz(G, steps, coefficients, eps):
    """[b, m, n] float64."""
    X = G / (np.sqrt(np.sum(G * G, axis=(1, 2), keepdims=True)) + eps)
    tall = X.shape[1] > X.shape[2]
    X = X.transpose(0, 2, 1) if tall else X
    for k in range(steps):
        a, b, c = coefficients[k]
        P = X @ X.transpose(0, 2, 1)
        X = a * X + (b * P + c * (P @ P)) @ X
    return X.transpose(0, 2, 1) if tall else X


# Relative error (2-norm over the stack) allowed to the orthogonalised result.
# float32: the first steps multiply small singular values by a = 3.4 each, 485 in
# five steps, and with them rounding errors of 2^-24 relative to ||X_0||_F = 1;
# spread over the matrix that is at most 2^-24 * 485 = 2.9e-5 of the result's
# norm, which is at least 0.7 of its root rank.  float16: its own rounding, at
# most 2^-11, besides.  bfloat16: its own, at most 2^-8 and in the 2-norm under 2^-9 (a
# third of 2^-16 in the mean square, over the values 1 to 2), and products of
# operands of 11 bits: p'(s)-weighted rounding of X, P and the polynomial, each at
# most 2^-12 times (a + 2|b| + 4c) / 0.7 = 30 in one direction, root-mean-square
# a fifth of that: 1.5e-3 a step, added in quadrature over the last three.
NS_TOL = {"f32": 3e-5, "f16": 2.0 ** -11 + 3e-5, "bf16": 2.0 ** -9 + 2.6e-3}
