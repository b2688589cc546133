"""Inputs whose table gradient is sharp: dout is zero but for one query row a head, another in each,
so that every bucket sums over one row's keys, and dout . v has one sign throughout a block of 32
keys, so that none of a block's sum cancels."""

import math

import torch


class TableCase:
    """q [1, H, n_q, 128], k, v [1, H, n_k, 128], do, o, lse, table, bucket, and in `ref` the 64-bit
    gradient of the rows that count (with dtable and its bound).  A head for every 32 queries."""

    def __init__(self, kind, n_q, n_k, device):
        import paper_2606_16317_amd as dsa
        from _grad_ref import Ref

        g = torch.Generator().manual_seed(n_q + n_k)
        self.H = H = -(-n_q // 32)
        h = torch.arange(H)
        self.rows = rows = torch.clamp(32 * h + (11 * h + 13) % 32, max=n_q - 1)
        if kind == "random":                 # runs of any length, some closed
            n = n_q + n_k - 1
            m = torch.randint(-1, 7, (n,), generator=g).repeat_interleave(
                torch.randint(1, 90, (n,), generator=g))[:n].to(torch.int32)
            self.nb = 7
        else:
            m = torch.from_numpy(dsa.dsattn_relative_buckets(
                n_q, n_k, 32, 128, q_first=max(0, n_k - n_q), causal=kind == "causal"))
            self.nb = 32
        self.table = 0.7 * torch.randn(self.nb, H, generator=g)
        bf16 = lambda x: x.to(torch.bfloat16)
        q_row = bf16(0.4 * torch.randn(H, 128, generator=g))
        k = bf16(torch.randn(n_k, 128, generator=g))
        side = torch.sign(torch.randn(128, generator=g))
        sign = torch.sign(torch.randn(-(-n_k // 32), generator=g)).repeat_interleave(32)[:n_k]
        v = bf16(0.25 * sign[:, None] * side + 0.25 * torch.randn(n_k, 128, generator=g))
        do_row = bf16(side.expand(H, 128) * 1.0)

        self.at = m[torch.arange(n_k)[None] - rows[:, None] + n_q - 1].long()   # [H, n_k]
        bias = torch.where(self.at < 0, -math.inf,
                           self.table.t().gather(1, self.at.clamp(min=0)).double())
        one = lambda x: x[None, :, None].contiguous()
        heads = lambda x: x[None, None].expand(1, H, -1, -1)
        on = lambda x: x.to(device)
        self.ref = ref = Ref(on(one(q_row)), on(heads(k)), on(heads(v)), on(one(do_row)),
                             bias=on(bias)[:, None])
        # add_table by head: each has its own row, so its own distances
        closed = on(self.at < 0)
        index = on(self.at.clamp(min=0))
        from _grad_ref import U32
        for name, x in (("dtable", ref.ds),
                        ("b_dtable", ref.b_ds + U32 * n_k ** 0.5 * ref.ds.abs())):
            x = x[0, :, 0].masked_fill(closed, 0.0)
            out = torch.zeros(H, self.nb, dtype=torch.float64, device=x.device)
            setattr(ref, name, out.scatter_add_(1, index, x).t().contiguous())
        ref.b_dtable = ref.b_dtable + 2 * U32 * ref.dtable.abs()

        def place(row):
            x = torch.zeros(1, H, n_q, 128, dtype=torch.bfloat16)
            x[0, h, rows] = row
            return on(x)

        self.q, self.do, self.o = place(q_row), place(do_row), place(bf16(ref.o[0, :, 0].cpu()))
        self.lse = torch.full((1, H, n_q), 20.0)     # of the rows that do not count: any number
        self.lse[0, h, rows] = ref.lse[0, :, 0].float().cpu()
        self.lse, self.table, self.bucket = on(self.lse), on(self.table), on(m)
        self.k, self.v = on(heads(k)).contiguous(), on(heads(v)).contiguous()
