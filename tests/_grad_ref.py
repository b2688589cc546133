"""Attention with an optional skip mask or additive bias, and its gradients, in 64 bits, with
elementwise bounds of what a kernel with bf16 operands and 32-bit sums may be off by.

Half a step of a rounding is U16 = 2^-8 (bf16) or U32 = 2^-24 of the value.  The kernels round
P and dS to bf16 for the products, and the results to bf16.  They sum delta in 32 bits; only dq
begins with the rounded output's delta' and corrects for it afterwards (see dq below).  Per logit the
32-bit arithmetic is off by at most ETA (128 products and their sum, the product with the scale, the
difference to the LSE and the LSE's own rounding), and exp2 and log2 by a few units in the last
place.

dq = scale (sum D k - r sum Pr k) with D = bf16(P (dP - delta')), r = sum D and Pr = bf16(P).  With
e = delta - delta' and D = dS + e P + eps, sum dS = 0 and sum P = 1 give r = e + sum eps (and the
rounding of that sum), so that dq is off by
    scale (sum eps k - (sum eps) sum Pr k + e sum (P - Pr) k),
|eps| <= what dk's dS is off by + (half a step) |e| P.  An eps therefore counts with its own key and
with the row's mean one; most of it cancels (eps is largest where P is), which a bound by absolute
values does not see.
"""

import math

import torch

U16, U32 = 2.0 ** -8, 2.0 ** -24


class Ref:
    """o, lse, dq, dk, dv, ds (float64) and bounds b_o, b_lse, b_dq, b_dk, b_dv of one problem
    q [B, H, n_q, d], k, v [B, H, n_k, d], do like q (or None).  bias [H or 1, n_q, n_k] in
    natural units (-inf: closed); skip [B, H, n_q, n_k] bool.  library_forward: the kernel gets o
    and the LSE from a forward call, which is off by their own bounds, not rounded from here."""

    def __init__(self, q, k, v, do=None, scale=None, bias=None, skip=None, library_forward=False):
        q, k, v = (x.detach().double() for x in (q, k, v))
        scale = 1.0 / math.sqrt(q.shape[-1]) if scale is None else scale
        t = lambda x: x.transpose(-1, -2).contiguous()
        s = scale * (q @ t(k))
        size = scale * (q.abs() @ t(k.abs()))
        if bias is not None:
            bias = bias.double()
            s = s + bias
            size = size + bias.masked_fill(torch.isinf(bias), 0.0).abs()
        if skip is not None:
            s = s.masked_fill(skip, -math.inf)
        lse = torch.logsumexp(s, -1)
        none = torch.isinf(lse)
        self.p = torch.exp(s - lse.masked_fill(none, 0.0)[..., None])
        self.lse = lse
        self.o = self.p @ v
        finite = s.masked_fill(torch.isinf(s), 0.0).abs()
        eta = U32 * (130 * size + 6 * finite + 4 * lse.masked_fill(none, 0.0).abs()[..., None] + 16)
        # P: the logit's error twice (its own and, in the mean, the LSE's)
        worst = (eta * self.p).sum(-1, keepdim=True)
        rel = eta + worst
        a = self.p @ v.abs()
        self.b_lse = worst[..., 0] + 4 * U32 * (1 + lse.masked_fill(none, 0.0).abs())
        self.b_o = U16 * self.o.abs() + (U16 + U32 * s.shape[-1]) * a + (rel * self.p) @ v.abs()
        if do is None:
            return
        do = do.detach().double()
        dp = do @ t(v)
        delta = (do * self.o).sum(-1, keepdim=True)
        self.ds = self.p * (dp - delta)
        self.dv = t(self.p) @ do
        self.dq = scale * (self.ds @ k)
        self.dk = scale * (t(self.ds) @ q)
        if library_forward:
            rel = rel + 2 * self.b_lse[..., None]
        d_o = self.b_o if library_forward else U16 * self.o.abs()
        d_dp = 130 * U32 * (do.abs() @ t(v.abs()))
        n = U32 * max(s.shape[-1], s.shape[-2])
        # delta as the sum of P dP, and what delta' is off by
        d_delta = (self.p * (d_dp + (rel + n) * dp.abs())).sum(-1, keepdim=True)
        d_prime = ((d_o + 130 * U32 * self.o.abs()) * do.abs()).sum(-1, keepdim=True)
        self.b_ds = 1.01 * (rel * self.ds.abs() + self.p * (d_dp + d_delta + 2 * U32 * (dp.abs() + delta.abs())))
        b_k = self.b_ds + (U16 + n) * self.ds.abs()
        # dq: eps and e (P - Pr)
        b_q = b_k + 2 * (U16 + n + rel) * self.p * (d_prime + d_delta)
        self.b_dv = U16 * self.dv.abs() + t((U16 + n + rel) * self.p) @ do.abs()
        mean_k = self.p @ k.abs()
        self.b_dq = U16 * self.dq.abs() + scale * (b_q @ k.abs() + 1.01 * b_q.sum(-1, keepdim=True) * mean_k)
        self.b_dk = U16 * self.dk.abs() + scale * (t(b_k) @ q.abs())

    def add_table(self, bucket, n_buckets):
        """dtable [n_buckets, H] and b_dtable; bucket [n_q, n_k] of every pair, -1: closed."""
        at = bucket.flatten().clamp(min=0).long()
        closed = (bucket < 0).flatten()
        for name, x in (("dtable", self.ds),
                        ("b_dtable", self.b_ds + U32 * bucket.numel() ** 0.5 * self.ds.abs())):
            x = x.sum(0).flatten(1).masked_fill(closed, 0.0)
            out = torch.zeros(x.shape[0], n_buckets, dtype=torch.float64, device=x.device)
            setattr(self, name, out.index_add_(1, at, x).t().contiguous())
        self.b_dtable = self.b_dtable + 2 * U32 * self.dtable.abs()

    def check(self, **got):
        """Every named result within its bound, elementwise; returns the largest share used."""
        worst = {}
        for name, x in got.items():
            ref, bound = getattr(self, name), getattr(self, "b_" + name)
            x = x.double().reshape(ref.shape)
            same = torch.isinf(ref)
            assert torch.equal(same, torch.isinf(x)) and not torch.isnan(x).any(), name
            if same.all():
                continue
            off = (x - ref)[~same].abs()
            # what underflows bf16 or fp32 on the way is far below 1e-30
            use = (off / (1.02 * bound[~same] + 1e-30)).max().item()
            worst[name] = use
            assert use <= 1.0, f"{name}: {use:.2f} of its bound"
        return worst


def distance_matrix(x, n_q, n_k):
    """[..., n_q, n_k] of x [..., n_q + n_k - 1] over key - query, from -(n_q - 1) up."""
    i = torch.arange(n_q, device=x.device)[:, None]
    return x[..., torch.arange(n_k, device=x.device)[None, :] - i + n_q - 1]


def skip_pairs(mask, N, tile_q, tile_k):
    """[B, H, N, N] bool of a skip mask [B, H, units, decisions]."""
    dev = mask.device
    u = torch.arange(N, device=dev) // tile_q
    d = torch.arange(N, device=dev) // tile_k
    return mask.bool()[:, :, u][:, :, :, d]


def random_qkv(B, H, n_q, n_k, seed, std=1.3, with_do=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda n, s: (torch.randn(B, H, n, 128, generator=g) * s).to(torch.bfloat16).cuda()
    q, k, v = r(n_q, std), r(n_k, std), r(n_k, 1.0)
    return (q, k, v, r(n_q, 1.0)) if with_do else (q, k, v)
