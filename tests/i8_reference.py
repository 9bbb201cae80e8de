"""Plain 64-bit forms of the 8-bit levels and the experts' products in 8-bit integers (tests only)."""
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}              # half the smallest step
U = 2.0 ** -24


def levels(x):
    """Levels (int64) and scales of rows [..., K]; torch.round takes halves to even."""
    v = x.double()
    top = v.abs().amax(-1, keepdim=True)
    return torch.round(127 * v / torch.where(top > 0, top, torch.ones_like(top))).long(), (top / 127).squeeze(-1)


def tiles(level):
    """[H][N][K] levels as tacg_i8_pack lays them out, one by one."""
    H, N, K = level.shape
    q = torch.zeros((H, -(-N // 16), -(-K // 64), 4, 16, 16), dtype=torch.int8)
    n, c = torch.meshgrid(torch.arange(N), torch.arange(K), indexing="ij")
    for h in range(H):
        q[h, n // 16, c // 64, c % 64 // 16, n % 16, c % 16] = level[h].to(torch.int8)
    return q


def products(qx, sx, ids, qw, sw, mode, slot=None, gate=None):
    """(values, what 32-bit arithmetic may be off before the last rounding).  qx [T][K] or [T][k][K] levels and sx their scales,
    qw [H][N][K] and sw [H][N]; ids [T][k] (None: slot j takes matrix j).

    Terms are off by the scales (2^-24), their product, the sum as a float and the product of both: 4 U, and U for a gate and for each
    addition.  silu(a) = a / (1 + exp(-a)) changes by at most 1 + |a| times a relative change of a; its exp is off by |a| U for the
    argument and 4 U in itself, and 5 U more for sum, quotient and product: 16 (1 + |a|) U in all."""
    T = qx.shape[0]
    H, N, K = qw.shape
    k = H if ids is None else ids.shape[1]
    y = torch.zeros((T, k, N), dtype=torch.float64)
    served = torch.zeros((T, k), dtype=torch.bool)
    for t in range(T):
        for j in range(k):
            h = j if ids is None else int(ids[t, j])
            if ids is not None and h >= 0 and slot is not None:
                h = int(slot[h])
            if h < 0:
                continue
            served[t, j] = True
            x, s = (qx[t, j], sx[t, j]) if qx.dim() == 3 else (qx[t], sx[t])
            y[t, j] = (qw[h].double() @ x[:K].double()) * (sw[h].double() * s.double())
    if mode == "each":
        return y, 4 * U * y.abs()
    if mode == "glu":
        a, b = y[..., :N // 2], y[..., N // 2:]
        v = a * torch.sigmoid(a) * b
        return v, 16 * U * (1 + a.abs()) * v.abs() + 1e-37 * b.abs()
    g = torch.where(served, torch.ones(()) if gate is None else gate, torch.zeros(())).double()[:, :, None]
    return (g * y).sum(1), (5 + k) * U * (g * y).abs().sum(1)


def within(got, want, off, dtype):
    """Whether a result is what one rounding of a value within `off` can be."""
    d = (got.double().cpu() - want).abs()
    tol = off * (1 + HALF[dtype]) + HALF[dtype] * want.abs() * (1 + 1e-6) + TINY[dtype]
    return bool((d <= tol).all())
