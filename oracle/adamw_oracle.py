"""Oracle of the list operators (test infrastructure, never the product path): AdamW with decoupled weight decay, the
global gradient norm with its clip factor, and the scaling by that factor, in fp64 numpy from their formulas.  Imports
nothing from the HIP package.  The 8-bit number format has its own oracle (``q8_oracle``)."""
import numpy as np


def adamw(w, g, m, v, beta1, beta2, eps, lr, weight_decay, k):
    """One step k >= 1 on fp64 arrays; returns (w, m, v, n), n the normalised update."""
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    n = (m / (1.0 - beta1 ** k)) / (np.sqrt(v / (1.0 - beta2 ** k)) + eps)
    return (1.0 - lr * weight_decay) * w - lr * n, m, v, n


def grad_stats(grads, grad_scale, max_norm):
    """(norm, factor, finite) of a list of fp64 arrays taken together."""
    finite = all(bool(np.all(np.isfinite(g))) for g in grads)
    if not finite:
        return float("nan"), 0.0, 0.0
    norm = abs(grad_scale) * float(np.sqrt(sum(float(np.sum(g * g)) for g in grads)))
    return norm, grad_scale * min(1.0, max_norm / (norm + 1e-6)), 1.0
