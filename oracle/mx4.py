"""Microscaled 4-bit rows in plain numpy, 64 bits (the oracle of the 4-bit calls).

From the definition (OCP Microscaling Formats v1.0: E2M1 elements, E8M0 scales,
blocks of 32) and the row layout that include/scone.h states.
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_bytes(cols: int) -> int:
    g = -(-cols // 128)
    return -(-68 * g // 16) * 16


def quantize(x: np.ndarray) -> np.ndarray:
    """Packed rows of x [n, cols] (any float type)."""
    x = np.asarray(x)
    n, cols = x.shape
    g = -(-cols // 128)
    out = np.zeros((n, row_bytes(cols)), np.uint8)
    for r in range(n):
        for b in range(-(-cols // 32)):
            v = x[r, 32 * b:32 * b + 32].astype(np.float64)
            if not np.isfinite(v).all():
                out[r, 64 * g + b] = 255
                continue
            top = np.abs(v).max()
            e = -127 if top == 0 else max(int(np.floor(np.log2(top))) - 2, -127)
            if top > 0 and not 2.0 ** np.floor(np.log2(top)) <= top:  # log2 rounded up
                e = max(e - 1, -127)
            out[r, 64 * g + b] = e + 127
            a = np.abs(v) * 2.0 ** -e
            for i, (m, s) in enumerate(zip(a, np.signbit(v))):
                d = np.abs(GRID - m)
                near = np.flatnonzero(d == d.min())
                code = near[0] if near.size == 1 or near[0] % 2 == 0 else near[1]
                k = 32 * b + i
                out[r, k // 2] |= (int(code) | (8 if s else 0)) << (4 * (k % 2))
    return out


def values(rows: np.ndarray, cols: int) -> np.ndarray:
    """The values [n, cols] of packed rows, in 64 bits."""
    g = -(-cols // 128)
    codes = np.empty((rows.shape[0], 128 * g), np.uint8)
    codes[:, 0::2] = rows[:, :64 * g] & 15
    codes[:, 1::2] = rows[:, :64 * g] >> 4
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    s = rows[:, 64 * g:68 * g].astype(np.float64)
    scale = np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return (v * np.repeat(scale, 32, axis=1))[:, :cols]


def rounded(x: np.ndarray) -> np.ndarray:
    """values(quantize(x)) for finite x [..., cols], cols a multiple of 32, at once."""
    v = np.asarray(x, np.float64).reshape(-1, 32)
    _, e = np.frexp(np.abs(v).max(axis=1, keepdims=True))       # top in [2^(e-1), 2^e)
    scale = np.exp2(np.maximum(e - 3.0, -127.0))
    a = np.abs(v) / scale
    # the grid's steps: 1/2 below 2, 1 below 4, then 2; rint takes ties to even
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    return np.copysign(np.minimum(np.rint(a / step) * step, 6.0) * scale, v).reshape(np.shape(x))


def linear(x: np.ndarray, w: np.ndarray, bias=None, gelu=False, residual=None):
    """act(x w^T + bias) + residual, and sum |x| |w| (what sums round relative to)."""
    y = x @ w.T
    size = np.abs(x) @ np.abs(w).T
    if bias is not None:
        y = y + bias
        size = size + np.abs(bias)
    if gelu:
        from scipy.special import erfc
        y = 0.5 * y * erfc(-y * np.sqrt(0.5))
    if residual is not None:
        y = y + residual
    return y, size


def fgram_forward(fgrams, lengths, tok_emb, params, n_layers, n_heads):
    """F's rows by a model whose linear weights and their inputs are held in 4 bits, the
    inputs rounded to bf16 before (and q, k, v); 64 bits in between.  The model is that
    of oracle/fgram_model.py."""
    from . import fgram_model as m
    d = tok_emb.shape[1]
    W = {k: rounded(v) for k, v in params.items() if k.split(".")[-1].startswith("w_")}
    out = np.zeros((len(lengths), d))
    for n in np.unique(lengths):
        sel = np.flatnonzero(lengths == n)
        G = len(sel)
        h = tok_emb[np.asarray(fgrams)[sel, :n]] + params["pos"][:n]
        for l in range(n_layers):
            p = {k.split(".")[1]: v for k, v in params.items() if k.startswith(f"l{l}.")}
            w = {k.split(".")[1]: v for k, v in W.items() if k.startswith(f"l{l}.")}
            a = m.round_bf16(m.layer_norm(h, p["ln1_g"], p["ln1_b"]))
            qkv = m.round_bf16(rounded(a) @ w["w_qkv"].T + p["b_qkv"])
            q, k, v = (qkv[..., i * d:(i + 1) * d].reshape(G, n, n_heads, d // n_heads)
                       .transpose(0, 2, 1, 3) for i in range(3))
            o = m.causal_attention(q, k, v).transpose(0, 2, 1, 3).reshape(G, n, d)
            h = h + rounded(m.round_bf16(o)) @ w["w_o"].T + p["b_o"]
            a = m.round_bf16(m.layer_norm(h, p["ln2_g"], p["ln2_b"]))
            f = m.round_bf16(m.gelu(rounded(a) @ w["w_fc1"].T + p["b_fc1"]))
            h = h + rounded(f) @ w["w_fc2"].T + p["b_fc2"]
        out[sel] = m.layer_norm(h[:, n - 1], params["lnf_g"], params["lnf_b"])
    return out
