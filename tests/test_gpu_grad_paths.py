"""GPU tests of what only large backward passes and calls of many heads reach: long visit lists of
masks up to the longest, and units by XCD under a bias."""

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
