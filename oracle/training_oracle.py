"""Plain numpy oracle, in 64 bits, of what surrounds the stack calls of a training step: the LM head's log-probabilities and
their gradient, the preference and the policy loss, and the 8-bit checkpoints.  Loops where loops are the definition."""
import numpy as np

GROUP = 32


# ---- LM head --------------------------------------------------------------------------------------
def head_fwd(U, W, labels, scale=1.0):
    """logp [b] (0 where the label is not in the vocabulary) and lse [b]."""
    z = scale * (np.asarray(U, np.float64) @ np.asarray(W, np.float64).T)
    top = z.max(axis=1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    logp = np.zeros(len(z))
    for i, y in enumerate(labels):
        if 0 <= y < z.shape[1]:
            logp[i] = z[i, y] - lse[i]
    return logp, lse


def head_dz(U, W, labels, dlogp, scale=1.0):
    U, W = np.asarray(U, np.float64), np.asarray(W, np.float64)
    z = scale * (U @ W.T)
    _, lse = head_fwd(U, W, labels, scale)
    dz = np.zeros_like(z)
    for i, y in enumerate(labels):
        if 0 <= y < z.shape[1]:
            dz[i] = -np.exp(z[i] - lse[i])
            dz[i, y] += 1.0
            dz[i] *= scale * dlogp[i]
    return dz


def head_bwd(U, W, labels, dlogp, scale=1.0):
    dz = head_dz(U, W, labels, dlogp, scale)
    return dz @ np.asarray(W, np.float64), dz.T @ np.asarray(U, np.float64)


# ---- losses ---------------------------------------------------------------------------------------
def _log_sigmoid(h):
    return -np.log1p(np.exp(-h)) if h >= 0 else h - np.log1p(np.exp(h))


def _counted(offsets, mask, k):
    return [t for t in range(int(offsets[k]), int(offsets[k + 1])) if mask is None or mask[t]]


def preference(logp, ref, mask, offsets, beta, smooth=0.0, margin=0.0, mean=False, grad_scale=1.0):
    logp = np.asarray(logp, np.float64)
    n = (len(offsets) - 1) // 2
    d = np.zeros(len(logp))
    rewards, margins, total = np.zeros(2 * n), np.zeros(n), 0.0
    for i in range(n):
        tok = [_counted(offsets, mask, 2 * i + j) for j in (0, 1)]
        per = [beta / max(1, len(t)) if mean else beta for t in tok]
        r = [p * sum(logp[t] - (0.0 if ref is None else float(ref[t])) for t in ts) for p, ts in zip(per, tok)]
        h = r[0] - r[1] - margin
        total += -(1 - smooth) * _log_sigmoid(h) - smooth * _log_sigmoid(-h)
        slope = -(1 - smooth) * np.exp(_log_sigmoid(-h)) + smooth * np.exp(_log_sigmoid(h))
        for sign, p, ts in ((1, per[0], tok[0]), (-1, per[1], tok[1])):
            d[ts] = grad_scale * sign * slope * p / n
        rewards[2 * i:2 * i + 2] = r
        margins[i] = h
    return dict(loss=total / n if n else 0.0, margins=margins, rewards=rewards, dlogp=d)


def policy(logp, old, ref, adv, mask, offsets, low, high, kl_coef=0.0, by_sequence=False, per_token=False, grad_scale=1.0):
    logp = np.asarray(logp, np.float64)
    n = len(offsets) - 1
    tok = [_counted(offsets, mask, k) for k in range(n)]
    live, every = sum(len(t) > 0 for t in tok), sum(len(t) for t in tok)
    d = np.zeros(len(logp))
    size = np.zeros(len(logp))      # of the terms that a token's gradient and loss are made of
    loss = kl = clipped = 0.0
    for k, ts in enumerate(tok):
        for t in ts:
            w = 1.0 / (len(ts) * live) if by_sequence else 1.0 / every
            A = float(adv[t if per_token else k])
            rho = np.exp(logp[t] - float(old[t]))
            bound = min(max(rho, 1 - low), 1 + high)
            over = bound * A < rho * A
            q = 0.0 if ref is None else float(ref[t]) - logp[t]
            excess = np.expm1(q) - q if abs(q) > 1e-2 else q * q * (0.5 + q * (1 / 6 + q * (1 / 24 + q * (1 / 120 + q / 720))))
            loss += w * (kl_coef * excess - min(rho * A, bound * A))
            kl += w * excess
            clipped += w * over
            d[t] = grad_scale * w * ((0.0 if over else -rho * A) - kl_coef * np.expm1(q))
            size[t] = abs(grad_scale) * w * ((0.0 if over else rho * abs(A)) * (1 + abs(logp[t] - float(old[t]))) + abs(kl_coef) * abs(np.expm1(q)))
    return dict(loss=loss, kl=kl, clipped=clipped, dlogp=d, size=size)


# ---- 8-bit checkpoints ----------------------------------------------------------------------------
def ckpt_pack(X):
    """q int8 [rows x 32 groups] and e uint8 [rows x groups] of a float32 matrix."""
    X = np.asarray(X, np.float32)
    rows, cols = X.shape
    groups = -(-cols // GROUP)
    q = np.zeros((rows, groups * GROUP), np.int8)
    e = np.zeros((rows, groups), np.uint8)
    for i in range(rows):
        for g in range(groups):
            x = X[i, g * GROUP:(g + 1) * GROUP].astype(np.float64)
            if not np.isfinite(x).all():
                e[i, g] = 255
                continue
            most = np.abs(x).max()
            power = max(int(np.frexp(most)[1]) - 1 if most > 0 else -10 ** 6, -120) - 6
            e[i, g] = power + 127
            q[i, g * GROUP:g * GROUP + len(x)] = np.clip(np.rint(x * 2.0 ** -power), -127, 127)
    return q, e


def ckpt_unpack(q, e, cols):
    power = np.where(e == 255, np.nan, 2.0 ** (e.astype(np.float64) - 127))
    return (q.astype(np.float64).reshape(len(q), -1, GROUP) * power[:, :, None]).reshape(len(q), -1)[:, :cols].astype(np.float32)
