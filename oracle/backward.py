"""Oracle: gradients of the layer's forward pass (test infrastructure, CPU only), fp64, from the formulas.

The paper trains nothing; these are the derivatives of the forward definitions in combine.py, routing.py and
ffn.py.  The duplication plan only says where a row is computed and has no gradient.
"""
import numpy as np


def combine_backward(dout, y_perm, row_of_assign, topk_w, topk_idx, E):
    """(dy_perm [A, d], dtopk_w [T, k], dlogits [T, E]) of out[t] = sum_j w[t, j] y_perm[row(t, j)] with
    w[t] = softmax of the selected logits."""
    dout, y = np.asarray(dout, np.float64), np.asarray(y_perm, np.float64)
    w = np.asarray(topk_w, np.float64)
    T, k = w.shape
    rows = np.asarray(row_of_assign, np.int64).reshape(T, k)
    dy = np.zeros(y.shape)
    dw = np.zeros((T, k))
    dlogits = np.zeros((T, E))
    for t in range(T):
        for j in range(k):
            dy[rows[t, j]] = w[t, j] * dout[t]
            dw[t, j] = np.sum(dout[t] * y[rows[t, j]])
        for j in range(k):
            dlogits[t, topk_idx[t, j]] = w[t, j] * (dw[t, j] - np.sum(w[t] * dw[t]))
    return dy, dw, dlogits


def ffn_rows_backward(x, dy, W1, W3, W2):
    """(dx, dW1, dW3, dW2) of the rows of one expert, y = (silu(x W1) * (x W3)) W2; W3 None: y = max(x W1, 0) W2."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    W1, W2 = np.asarray(W1, np.float64), np.asarray(W2, np.float64)
    a = x @ W1
    dh = dy @ W2.T
    if W3 is None:
        da = np.where(a > 0, dh, 0.0)
        return da @ W1.T, x.T @ da, None, np.maximum(a, 0.0).T @ dy
    W3 = np.asarray(W3, np.float64)
    b = x @ W3
    s = 1.0 / (1.0 + np.exp(-a))
    da = dh * b * (s + a * s * (1.0 - s))
    db = dh * a * s
    return da @ W1.T + db @ W3.T, x.T @ da, x.T @ db, (a * s * b).T @ dy


def grouped_ffn_backward(x_perm, dy_perm, seg_offsets, slot_expert, W1, W3, W2):
    """(dx_perm, dW1, dW3, dW2): replicas of an expert share its gradient; an expert without rows has a gradient of
    zeros.  Rows of slots that hold no expert stay at zero."""
    x_perm, dy_perm = np.asarray(x_perm, np.float64), np.asarray(dy_perm, np.float64)
    dx = np.zeros(x_perm.shape)
    grads = [None if W is None else np.zeros(W.shape) for W in (W1, W3, W2)]
    for s, e in enumerate(slot_expert):
        lo, hi = int(seg_offsets[s]), int(seg_offsets[s + 1])
        if hi == lo or e < 0:
            continue
        out = ffn_rows_backward(x_perm[lo:hi], dy_perm[lo:hi], W1[e], None if W3 is None else W3[e], W2[e])
        dx[lo:hi] = out[0]
        for g, o in zip(grads, out[1:]):
            if g is not None:
                g[e] += o
    return (dx, *grads)
