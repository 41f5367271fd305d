"""Plain numpy fp64 forms of the operators for parameters outside the low-rank path, written from their definitions in include/lordo.h."""
import numpy as np
import torch

from oracle import lordo_oracle as lo

BLOCK = 256


def f32(x: float) -> float:
    return float(np.float32(x))


def to64(t: torch.Tensor) -> np.ndarray:
    return t.detach().double().cpu().numpy()


def table_grad(tokens: np.ndarray, dY: np.ndarray, V: int, scale: float) -> np.ndarray:
    """[K][V][d] from tokens [K][T] and dY [K][T][d]."""
    K, T, d = dY.shape
    out = np.zeros((K, V, d))
    for k in range(K):
        inside = (tokens[k] >= 0) & (tokens[k] < V)
        np.add.at(out[k], tokens[k][inside], dY[k][inside])
    return out * scale


def lookup(W: np.ndarray, tokens: np.ndarray, scale: float) -> np.ndarray:
    K, V, d = W.shape
    out = np.zeros(tokens.shape + (d,))
    for k in range(K):
        inside = (tokens[k] >= 0) & (tokens[k] < V)
        out[k][inside] = W[k][tokens[k][inside]] * scale
    return out


def random16(seed: int, purpose: int, index: int, number: int, n: int) -> np.ndarray:
    """The 16 bits of elements 0 .. n-1: four consecutive ones share a word of the generator, low bits first."""
    key = lo.mix64_int((lo.stream_key(seed, purpose, 0, index, 0) + lo._GOLDEN * (number + 1)) & lo._MASK)
    w = lo.random_words(key, (n + 3) // 4)
    return np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for s in (0, 16, 32, 48)], axis=1).reshape(-1)[:n].astype(np.int64)


def second16(u: np.ndarray) -> np.ndarray:
    return (u * 40503) % 65536


def scale_exponents(a: np.ndarray) -> np.ndarray:
    """Exponent of the scale of each block of 256 magnitudes: the largest lies in [128, 256) times it; at least -126."""
    pad = np.zeros(-(-a.size // BLOCK) * BLOCK)
    pad[:a.size] = a
    top = pad.reshape(-1, BLOCK).max(axis=1)
    return np.maximum(np.frexp(top)[1] - 8, -126) * (top > 0) + -126 * (top == 0)


def grid(t: np.ndarray) -> np.ndarray:
    """Distance of E4M3 codes at magnitude t."""
    return np.exp2(np.maximum(np.frexp(t)[1] - 1, -6) - 3)


def round8(x: np.ndarray, u: np.ndarray, positive: bool):
    """(values of the codes without scale, exponents of the scales, distance of the rounding's argument to the nearest border in steps)."""
    e = scale_exponents(np.abs(x))
    t = np.abs(x) * np.exp2(-e.repeat(BLOCK)[:x.size].astype(float))
    step = grid(t)
    y = t / step + (u + 0.5) / 65536
    q = np.floor(y) * step
    if positive:
        q = np.where(x > 0, np.maximum(q, 2.0 ** -9), q)
    return np.copysign(q, x), e, np.abs(y - np.rint(y))


def adamw(W, m, v, g, lr, beta1, beta2, omega, eps, wd, s, least=0.0):
    """One step in 64 bits: (W, m, v, size of the update before lr). least: below this v counts as 0."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    v = np.where(v < least, 0.0, v)
    up = (omega * m / (1 - beta1 ** s) + (1 - omega) * g) / (np.sqrt(v / (1 - beta2 ** s)) + eps)
    return W - lr * (up + wd * W), m, v, up


def clip(grads, rho, scope=0):
    """[n_tensors][K] coefficients of gradients [K][n]."""
    if not rho > 0:
        return np.ones((len(grads), grads[0].shape[0]))
    sq = np.stack([(g.reshape(g.shape[0], -1) ** 2).sum(axis=1) for g in grads])
    if scope == 0:
        sq = np.repeat(sq.sum(axis=0, keepdims=True), len(grads), axis=0)
    return np.minimum(1.0, rho / (np.sqrt(sq) + 1e-6))
