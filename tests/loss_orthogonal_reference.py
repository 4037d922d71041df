"""Plain forms in 64 bits of the loss over a large vocabulary and of orthogonalised updates, with bounds on what the library's arithmetic may be off."""
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}      # of a rounding, relative
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}    # half of the smallest number
MUON = (3.4445, -4.7750, 2.0315)


def loss_and_gradients(h, w, y, g, ignore=-100):
    """losses, dh, dw of sum_t g_t losses_t, and bounds of what each may be off, all in float64.

    Logits: products are exact; a sum over 256 of k is made in 16 steps, each of which may cut off 2^-23 of the sum of magnitudes so far (and as much
    again inside the step), the parts are added with 2^-24 each: (32 + D / 256) 2^-23 S for S = sum |h_d w_d|, largest over the vocabulary.
    Losses: two logits' errors, exponentials (2 ulp), sums of V of them (parts of 32 and then some) and a logarithm: 2^-19 (1 + |loss|) beside.
    The gradients' logits are summed without parts: D / 16 steps.  dz: that as a relative error of exp, one rounding to 16 bits; dz is held
    against p + [v = y], so that a difference close to 0 is not.  Products of dz: K / 16 steps of 2 * 2^-23; one rounding of the result."""
    T, D = h.shape
    V = w.shape[0]
    hd, wd = h.double(), w.double()
    valid = y != ignore
    hd = torch.where(valid[:, None], hd, torch.zeros((), dtype=torch.float64, device=h.device))
    at = torch.where(valid, y, torch.zeros_like(y))[:, None]
    z = hd @ wd.t()
    S = (hd.abs() @ wd.abs().t()).amax(1)
    lse = torch.logsumexp(z, 1)
    losses = torch.where(valid, lse - z.gather(1, at)[:, 0], torch.zeros((), dtype=torch.float64, device=h.device))
    loss_tol = torch.where(valid, 2 * (32 + D / 256) * 2.0 ** -23 * S + 2.0 ** -19 * (1 + losses.abs() + lse.abs()), torch.zeros_like(S))
    gv = torch.where(valid, g.double(), torch.zeros((), dtype=torch.float64, device=h.device))[:, None]
    p = (z - lse[:, None]).exp()
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    dz = gv * (p - one)
    half = HALF_STEP[h.dtype]
    z_tol = (2 * (2 * D / 16 + 2) * 2.0 ** -23 * S + 2.0 ** -19 * (1 + lse.abs()))[:, None]
    dz_tol = gv.abs() * (p * z_tol + 2.0 ** -23) + half * dz.abs() * (1 + z_tol) + gv.abs().max() * 2.0 ** -38
    def products(a, tol, b, k):
        return tol @ b.abs() + a.abs() @ b.abs() * (2 * k / 16 + 2) * 2.0 ** -23
    dh, dw = dz @ wd, dz.t() @ hd
    dh_tol = products(dz, dz_tol, wd, V) * valid[:, None] + half * dh.abs() * 1.01 + SMALLEST[h.dtype]
    dw_tol = products(dz.t(), (dz_tol * valid[:, None]).t(), hd, T) + half * dw.abs() * 1.01 + SMALLEST[h.dtype]
    return (losses, dh, dw), (loss_tol, dh_tol, dw_tol)


def orthogonal(u, steps=5, f=MUON, double=True):
    """Through the smaller Gram matrix, in float64 or, for what products in fp32 lose, in float32."""
    a, b, c = f
    x = u.double() if double else u.float()
    tall = x.shape[-2] > x.shape[-1]
    x = x.transpose(-1, -2) if tall else x
    norm = x.double().square().sum((-1, -2), keepdim=True).sqrt()
    x = torch.where(norm > 0, x.double() / norm, torch.zeros_like(x.double())).to(x.dtype)
    for _ in range(steps):
        m = x @ x.transpose(-1, -2)
        x = a * x + (b * m + c * (m @ m)) @ x
    return x.transpose(-1, -2) if tall else x


def off(a, b, lost=0.0):
    """|a - b| / |b| of each matrix, the largest of a batch; 0 for 0.  lost: what each element may be off besides."""
    a, b = a.double().flatten(-2), b.double().flatten(-2)
    n = b.norm(dim=-1)
    d = ((a - b).norm(dim=-1) - lost * a.shape[-1] ** 0.5).clamp(min=0)
    return float((d / torch.where(n > 0, n, torch.ones_like(n))).max())


# X is kept times 2^13 in two fp16 parts, whose smallest step is 2^-24: an element is off by up to 2^-38 whatever its size.  That is nothing beside
# singular values near 1, but coefficients with a = 0 take them to their third power each step, and out of every type's range (0.2 to the
# 81st behind four steps).
KEPT_TO = 2.0 ** -38
