"""LayerNorm over rows and its gradients in float64 -- TEST INFRASTRUCTURE, NOT PRODUCT CODE.

    y = u gamma + beta,  u = (x - mean) / sqrt(var + eps)
    dx = rstd (a - mean(a) - u mean(a u)),  a = gamma dy;   dgamma = sum dy u;   dbeta = sum dy

Pins (tests/test_operators_cpu.py): the library LayerNorm in float64, gradients against differences.
"""
import numpy as np


def layernorm_rows_numpy(x, gamma, beta, eps):
    """(y, mean_rstd [M][2])"""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * np.asarray(gamma, np.float64) + np.asarray(beta, np.float64), np.stack([mean, rstd], 1)


def layernorm_rows_gradients_numpy(x, mean_rstd, gamma, dy):
    """(dx, dgamma, dbeta)"""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    mean, rstd = np.asarray(mean_rstd, np.float64).T[:, :, None]
    u = (x - mean) * rstd
    a = dy * np.asarray(gamma, np.float64)
    return rstd * (a - a.mean(1, keepdims=True) - u * (a * u).mean(1, keepdims=True)), (dy * u).sum(0), dy.sum(0)
