"""GPU tests of what only large backward passes and calls of many heads reach: long visit lists of
masks up to the longest, units by XCD under a bias, and every block's share of the table's gradient
of long rows."""

import math

import pytest

from test_gpu_attn_bwd import announce, backward, gpu, random_mask  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("tile_q,tile_k", [(32, 32), (32, 64), (128, 128)])
@pytest.mark.parametrize("kept", [0.02, 0.3])
def test_masks_of_more_tiles_than_a_wave_or_a_pass_of_the_list(tile_q, tile_k, kept):
    """140 tiles: three rounds of 64 when the gaps are closed, two passes of 128 before."""
    from _grad_ref import Ref, random_qkv, skip_pairs

    N = 8930
    announce(f"masked backward N={N} kept={kept} tile {tile_q} x {tile_k}")
    q, k, v, do = random_qkv(1, 2, N, N, tile_q + tile_k)
    mask = random_mask(1, 2, N, tile_q, tile_k, kept, N)
    ref = Ref(q, k, v, do, skip=skip_pairs(mask, N, tile_q, tile_k))
    got = backward(q, k, v, ref, do, mask_in=mask, tile_q=tile_q, tile_k=tile_k)
    print(ref.check(**got), flush=True)


def test_the_longest_masks():
    """262144 rows, 4096 tiles: units that keep four of them, the last one always, and one that
    keeps all, so that lists of both kernels reach their full length; the last tiles' numbers are
    the largest that a list holds."""
    import paper_2606_16317_amd as dsa
    from _grad_ref import U16, U32, Ref, random_qkv

    N, unit, tile, full = 262144, 128, 64, 5
    n_u, n_t = N // unit, N // tile
    announce(f"masked backward N={N}")
    q, k, v, do = random_qkv(1, 1, N, N, 3)
    at = torch.arange(n_u)
    last = torch.full_like(at, n_t - 1)
    tiles = torch.stack([2 * at % (n_t - 1), (2 * at + 501) % (n_t - 1),
                         (2 * at + 2222) % (n_t - 1), last], 1).cuda()
    mask = torch.ones(n_u, n_t, dtype=torch.uint8, device="cuda").scatter_(1, tiles, 0)
    mask[full] = 0
    assert int((mask == 0).sum()) == 4 * (n_u - 1) + n_t

    # every unit but the full one as a batch of its own over the keys that it keeps
    some = torch.tensor([u for u in range(n_u) if u != full], device="cuda")
    by_unit = lambda x: x.view(n_u, 1, unit, 128)
    keys = lambda x: x.view(n_t, tile, 128)[tiles[some]].reshape(len(some), 1, 4 * tile, 128)
    parts = [(some, tiles[some], Ref(by_unit(q)[some], keys(k), keys(v), by_unit(do)[some])),
             (torch.tensor([full], device="cuda"), torch.arange(n_t, device="cuda")[None],
              Ref(by_unit(q)[full:full + 1], k, v, by_unit(do)[full:full + 1]))]

    o, lse = torch.zeros_like(q), torch.zeros(1, 1, N, device="cuda")
    whole = Ref.__new__(Ref)
    for name in ("dq", "b_dq"):
        setattr(whole, name, torch.zeros(q.shape, dtype=torch.float64, device="cuda"))
    for name in ("dk", "dv", "b_dk", "b_dv"):
        setattr(whole, name, torch.zeros(n_t, tile, 128, dtype=torch.float64, device="cuda"))
    # rows that a key's sums go over, beyond those of its part, and the sums' sizes
    rows = unit * (mask == 0).sum(0).double()
    size = {n: torch.zeros_like(whole.dk) for n in ("dk", "dv")}
    for units, kept, ref in parts:
        by_unit(o)[units] = ref.o.to(torch.bfloat16)
        lse.view(n_u, 1, unit)[units] = ref.lse.float()
        for name in ("dq", "b_dq"):
            by_unit(getattr(whole, name))[units] = getattr(ref, name)
        add = lambda to, x: to.index_add_(0, kept.flatten(), x.reshape(-1, tile, 128))
        for name in ("dk", "dv", "b_dk", "b_dv"):
            add(getattr(whole, name), getattr(ref, name))
        t = lambda x: x.transpose(-1, -2).contiguous()
        add(size["dv"], t(ref.p) @ by_unit(do)[units].double().abs())
        add(size["dk"], t(ref.ds.abs()) @ by_unit(q)[units].double().abs() / math.sqrt(128))
    for name in ("dk", "dv"):
        bound = getattr(whole, "b_" + name)
        bound += U32 * rows[:, None, None] * size[name]
        for x in (name, "b_" + name):
            setattr(whole, x, getattr(whole, x).view(q.shape))
    del parts, ref
    got = dsa.dsattn_attn_bwd(dsa.RULE_MASK, q, k, v, o, lse, do,
                              mask_in=mask.view(1, 1, n_u, n_t))
    print(whole.check(dq=got[0], dk=got[1], dv=got[2]), flush=True)


def test_masked_call_captured():
    import paper_2606_16317_amd as dsa
    from _grad_ref import Ref, random_qkv, skip_pairs

    announce("masked backward captured")
    N = 700
    q, k, v, do = random_qkv(1, 3, N, N, 22)
    mask = random_mask(1, 3, N, 32, 64, 0.3, 5)
    ref = Ref(q, k, v, do, skip=skip_pairs(mask, N, 32, 64))
    o, lse = ref.o.to(torch.bfloat16), ref.lse.float()
    call = lambda m, *out, **kw: dsa.dsattn_attn_bwd(dsa.RULE_MASK, q, k, v, o, lse, do, *out,
                                                     mask_in=m, tile_q=32, **kw)
    first = call(mask)
    print(ref.check(dq=first[0], dk=first[1], dv=first[2]), flush=True)
    ws = torch.empty(dsa.dsattn_attn_bwd_workspace_bytes(1, 3, N), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for _ in range(3)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(mask, *outs, workspace=ws)
    for _ in range(3):
        for x in outs:
            x.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
        call(torch.zeros_like(mask))


@pytest.mark.parametrize("B,H,n,kind", [(1, 1024, 200, "both"), (1, 1024, 200, "causal"),
                                        (1, 1032, 200, "both"), (2, 208, 520, "causal")])
def test_units_by_xcd(B, H, n, kind):
    """A multiple of 8 heads with 2048 groups and more: whole rounds, some left over, some shared
    between workgroups.  Every head has a table of its own."""
    from test_gpu_bias_attn import backward, forward, make

    announce(f"bias step B={B} H={H} n={n} {kind}")
    q, k, v, do, table, m, ref = make(B, H, n, n, kind, H)
    print(ref.check(**forward(q, k, v, table, m)), flush=True)
    print(ref.check(**backward(q, k, v, table, m, ref, do)), flush=True)


@pytest.mark.parametrize("kind,n_q,n_k", [("both", 3001, 3001), ("causal", 3001, 3001),
                                          ("random", 3001, 1600), ("both", 700, 5000)])
def test_every_block_of_the_table_gradient(kind, n_q, n_k):
    """One query row a head: the sums have few pairs, so a block that is lost or counted for another
    bucket shows (test_grad_host.py shows that it would)."""
    import paper_2606_16317_amd as dsa
    from _table_case import TableCase

    announce(f"table gradient {kind} n_q={n_q} n_k={n_k}")
    c = TableCase(kind, n_q, n_k, "cuda")
    got = dsa.dsattn_bias_attn_bwd(c.q, c.k, c.v, c.table, c.bucket, c.o, c.lse, c.do)
    print(c.ref.check(dtable=got[3]), flush=True)
    empty = torch.ones(c.H, n_q, dtype=torch.bool, device="cuda")
    empty[torch.arange(c.H), c.rows] = False
    assert not got[0][0][empty].any()


def by_distance(x):
    """Sums of x [R, n] over column - row, from -(R - 1) up."""
    R, n = x.shape
    return torch.nn.functional.pad(x.flip(0), (0, R)).flatten()[:R * (n + R - 1)].view(R, -1).sum(0)


@pytest.mark.parametrize("n,heads,causal", [(3001, 4, False), (32760, 1, False), (32760, 1, True)])
def test_table_gradient_of_long_rows_by_norm(n, heads, causal):
    """Errors of a pair's dS are independent but for a row's (its LSE's rounding, its delta), so in
    units of 1e-7 of a dS: the logit (128 products in eight steps of sums of some 2 times the logit,
    and the product with the scale) 7, exp2 1, the LSE's rounding 5, sums of 80 values in 32 bits 3;
    delta's, 0.3 of it for every pair alike, adds up over the keys that share a row (some 1900 of
    32760, 175 of 3001: e^(-s^2) of them for logits of deviation s = 1.7) and counts with the root of
    their number: 3 and 10.  All in one direction: 26e-7.

    The errors e x of independent terms x add up to e times the root of the sum of x^2, whatever the
    terms themselves add up to: where the two far buckets have nearly all of a row, whose dS sum up
    to zero, the gradient is a small difference (7.0 where that root is 43.9, in the third head of
    3001 rows), and an error of 5e-7 of the root is 33e-7 of the gradient.  So the root is what the
    norm of the error is held against."""
    import paper_2606_16317_amd as dsa
    from _grad_ref import random_qkv

    announce(f"table gradient by norm n={n} causal={causal}")
    nb = 32
    q, k, v, do = random_qkv(1, heads, n, n, 6)
    bucket = torch.from_numpy(dsa.dsattn_relative_buckets(n, n, nb, 4096 if causal else 128,
                                                          causal=causal)).cuda()
    table = torch.randn(nb, heads, generator=torch.Generator().manual_seed(9)).cuda()
    o, lse = torch.empty_like(q), torch.empty(1, heads, n, device="cuda")
    want, square = (torch.zeros(nb + 1, heads, dtype=torch.float64, device="cuda") for _ in range(2))
    index = torch.where(bucket < 0, nb, bucket).long()
    j = torch.arange(n, device="cuda")
    for h in range(heads):
        bias = torch.cat([table[:, h].double(), torch.full((1,), -math.inf, device="cuda").double()])
        bias = bias[index]
        kt, vt = (x[0, h].double().t().contiguous() for x in (k, v))
        sums = torch.zeros(2, 2 * n - 1, dtype=torch.float64, device="cuda")
        for lo in range(0, n, 2048):
            hi = min(n, lo + 2048)
            i = torch.arange(lo, hi, device="cuda")
            s = q[0, h, i].double() @ kt / math.sqrt(128) + bias[j[None] - i[:, None] + n - 1]
            row = torch.logsumexp(s, 1)
            p = torch.exp(s - row[:, None])
            oi = p @ v[0, h].double()
            g = do[0, h, i].double()
            ds = p * (g @ vt - (g * oi).sum(1, keepdim=True))
            sums[0, n - hi:2 * n - 1 - lo] += by_distance(ds)
            sums[1, n - hi:2 * n - 1 - lo] += by_distance(ds * ds)
            o[0, h, i], lse[0, h, i] = oi.to(torch.bfloat16), row.float()
        want[:, h].index_add_(0, index, sums[0])
        square[:, h].index_add_(0, index, sums[1])
    got = dsa.dsattn_bias_attn_bwd(q, k, v, table, bucket, o, lse, do)[3].double()
    off, root = (got - want[:nb]).norm(dim=0), square[:nb].sum(0).sqrt()
    print((off / root).tolist(), (off / want[:nb].norm(dim=0)).tolist(), flush=True)
    assert (off / root).max().item() <= 3e-6
