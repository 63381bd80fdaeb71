"""Group norm with an activation over channels-last images in fp64, and its gradient (test infrastructure)."""
import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def _act(z, act):
    """Value and slope."""
    if act == "silu":
        s = np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))
        return z * s, s + z * s * (1 - s)
    if act == "gelu":
        cdf = 0.5 * (1 + _erf(z / math.sqrt(2)))
        return z * cdf, cdf + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, np.ones_like(z)


def _grouped(x, groups):
    B, Hh, Ww, C = x.shape
    return x.reshape(B, Hh * Ww, groups, C // groups)


def group_norm(x, weight, bias, groups, eps, act):
    """out, mean [B, groups], 1 / sqrt(var + eps) [B, groups]."""
    g = _grouped(x, groups)
    mean = g.mean((1, 3))
    rstd = 1 / np.sqrt(g.var((1, 3)) + eps)
    xhat = ((g - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)
    z = xhat * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)
    return _act(z, act)[0], mean, rstd


def group_norm_bwd(x, weight, bias, groups, eps, act, d_out):
    """dx, dweight, dbias."""
    _, mean, rstd = group_norm(x, weight, bias, groups, eps, act)
    w = np.ones(x.shape[3]) if weight is None else weight
    xhat = ((_grouped(x, groups) - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)
    g = d_out * _act(xhat * w + (0.0 if bias is None else bias), act)[1]
    dxhat, h = _grouped(g * w, groups), _grouped(xhat, groups)
    m = dxhat.shape[1] * dxhat.shape[3]
    s1, s2 = dxhat.sum((1, 3), keepdims=True), (dxhat * h).sum((1, 3), keepdims=True)
    dx = rstd[:, None, :, None] * (dxhat - s1 / m - h * s2 / m)
    return dx.reshape(x.shape), (g * xhat).sum((0, 1, 2)), g.sum((0, 1, 2))
