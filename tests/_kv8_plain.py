"""Plain statements of the 8-bit cache and of attention over it, for the GPU tests: numpy in 32 bits where codes are
decided, torch in 64 bits elsewhere."""
import numpy as np
import torch

BLOCK = 64
U = 2.0 ** -8            # half a step of bf16, relative


def blocks(segments):
    """(first token, tokens) of every block."""
    out, first = [], 0
    for n in segments:
        out += [(first + t, min(BLOCK, n - t)) for t in range(0, n, BLOCK)]
        first += n
    return out


def quantise(x, segments, lens=None):
    """x [B, H, L, 64] (float32 array) -> (codes int8, scales float32, rows that count [B, L], blocks that hold any)."""
    B, H, L, _ = x.shape
    codes = np.zeros(x.shape, np.int8)
    bl = blocks(segments)
    scales = np.zeros((B, H, len(bl)), np.float32)
    counts = np.ones((B, L), bool) if lens is None else np.arange(L)[None] < np.asarray(lens)[:, None]
    for b in range(B):
        for i, (t, n) in enumerate(bl):
            n = int(counts[b, t:t + n].sum())
            if n == 0:
                continue
            rows = x[b, :, t:t + n]
            s = np.abs(rows).reshape(H, -1).max(1).astype(np.float32) / np.float32(127)
            scales[b, :, i] = s
            with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
                q = rows / s[:, None, None]
            q = np.where(s[:, None, None] > 0, np.clip(np.rint(q), -127, 127), 0)
            codes[b, :, t:t + n] = q.astype(np.int8)
    return codes, scales, counts


def dequantise(codes, scales, segments):
    """float64 [B, H, L, 64] tensor of s * code."""
    row_block = torch.cat([torch.full((n,), i) for i, (_, n) in enumerate(blocks(segments))] or [torch.zeros(0)]).long()
    return codes.double() * scales.double()[:, :, row_block.to(codes.device)][..., None]


def attention(q, k, v, keep, sm):
    """64-bit attention: (out, sum of weights x |v|, largest sum of |q_d k_d| x sm of a row's kept pairs).  keep
    broadcasts over [B, H, n, L]; heads of k, v are repeated as query heads need them; an empty row is zero."""
    G = q.shape[1] // k.shape[1]
    q, k, v = q.double(), k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    if k.shape[2] == 0:
        return torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q[..., :1])
    kt = k.transpose(-1, -2).contiguous()
    s = torch.matmul(q, kt) * sm
    keep = keep.expand(s.shape)
    s = s.masked_fill(~keep, -torch.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -torch.inf, m, torch.zeros_like(m)))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    size = (torch.matmul(q.abs(), kt.abs()) * sm).masked_fill(~keep, 0.0).amax(-1, keepdim=True)
    return torch.matmul(p, v), torch.matmul(p, v.abs()), size


def assert_close(got, want, tol):
    err = (got.double() - want).abs()
    worst = (err - tol).max().item() if err.numel() else 0.0
    assert torch.isfinite(got).all() and worst <= 0, f"off by {err.max().item():.3e}, {worst:.3e} above its tolerance"
