"""GPU tests of the backward pass (``dsattn_attn_bwd``) against 64 bits, elementwise within
derived bounds; against differences of the forward function; after this library's own forward
calls; captured, on a side stream, and repeated."""

import math
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_16317_amd as dsa

    dsa.lib()


def announce(msg):
    print(f"\n[case] {msg}", flush=True)
    sys.stdout.flush()


def backward(q, k, v, ref, do, **kw):
    import paper_2606_16317_amd as dsa

    rule = dsa.RULE_MASK if "mask_in" in kw else dsa.RULE_DENSE
    out = dsa.dsattn_attn_bwd(rule, q, k, v, ref.o.to(torch.bfloat16), ref.lse.float(), do, **kw)
    torch.cuda.synchronize()
    return dict(zip(("dq", "dk", "dv"), out))


@pytest.mark.parametrize("N", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 777, 1409])
def test_dense(N):
    from _grad_ref import Ref, random_qkv

    B, H = (2, 3) if N < 300 else (1, 2)
    announce(f"dense backward B={B} H={H} N={N}")
    q, k, v, do = random_qkv(B, H, N, N, N)
    ref = Ref(q, k, v, do)
    print(ref.check(**backward(q, k, v, ref, do)), flush=True)


@pytest.mark.parametrize("scale", [0.02, 0.5])
def test_scale(scale):
    from _grad_ref import Ref, random_qkv

    announce(f"dense backward scale={scale}")
    q, k, v, do = random_qkv(1, 2, 300, 300, 5, std=1.0)
    ref = Ref(q, k, v, do, scale=scale)
    print(ref.check(**backward(q, k, v, ref, do, scale=scale)), flush=True)


def test_rows_with_one_key_of_nearly_all_the_weight():
    """dS is then a small difference of P dP and P delta: the output's own rounding must not
    stand in it."""
    from _grad_ref import Ref, random_qkv

    announce("peaked rows")
    q, k, v, do = random_qkv(1, 2, 500, 500, 41, std=2.5)
    ref = Ref(q, k, v, do)
    assert int((ref.p.amax(-1) > 0.9).sum()) > 100
    got = backward(q, k, v, ref, do)
    print(ref.check(**got), flush=True)


def random_mask(B, H, N, tile_q, tile_k, kept, seed):
    g = torch.Generator().manual_seed(seed)
    n_u, n_d = -(-N // tile_q), -(-N // tile_k)
    mask = (torch.rand(B, H, n_u, n_d, generator=g) >= kept).to(torch.uint8)
    mask[0, 0, n_u // 2] = 1                 # rows that keep nothing
    mask[-1, -1, :, n_d // 2] = 1            # keys that no row keeps
    mask[mask != 0] = 3                      # any nonzero byte skips
    return mask.cuda()


@pytest.mark.parametrize("tile_q", [32, 128])
@pytest.mark.parametrize("tile_k", [32, 64, 128])
@pytest.mark.parametrize("N,kept", [(1, 0.5), (33, 0.5), (64, 0.5), (129, 0.6), (500, 0.3),
                                    (1111, 0.1), (1500, 0.9)])
def test_masks(N, kept, tile_q, tile_k):
    from _grad_ref import Ref, random_qkv, skip_pairs

    B, H = (2, 2) if N < 600 else (1, 2)
    announce(f"masked backward N={N} kept={kept} tile {tile_q} x {tile_k}")
    q, k, v, do = random_qkv(B, H, N, N, N + tile_q + tile_k)
    mask = random_mask(B, H, N, tile_q, tile_k, kept, N)
    ref = Ref(q, k, v, do, skip=skip_pairs(mask, N, tile_q, tile_k))
    got = backward(q, k, v, ref, do, mask_in=mask, tile_q=tile_q, tile_k=tile_k)
    print(ref.check(**got), flush=True)
    empty = torch.isinf(ref.lse)
    assert empty.any() and not got["dq"][empty].any()


def test_mask_that_keeps_nothing_and_mask_that_keeps_all():
    import paper_2606_16317_amd as dsa
    from _grad_ref import Ref, random_qkv, skip_pairs

    announce("empty and full masks")
    N = 321
    q, k, v, do = random_qkv(1, 2, N, N, 9)
    mask = torch.ones(1, 2, 11, 6, dtype=torch.uint8, device="cuda")
    ref = Ref(q, k, v, do, skip=skip_pairs(mask, N, 32, 64))
    got = backward(q, k, v, ref, do, mask_in=mask, tile_q=32)
    assert not any(x.any() for x in got.values())
    full = Ref(q, k, v, do)
    a = backward(q, k, v, full, do)
    b = backward(q, k, v, full, do, mask_in=torch.zeros_like(mask), tile_q=32)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("H,N", [(128, 500), (130, 500), (515, 100), (700, 70)])
def test_whole_rounds_of_workgroups_and_a_remainder(H, N):
    """512 row groups at a time go without a split, the rest may be shared: none, few or most."""
    from _grad_ref import Ref, random_qkv, skip_pairs

    announce(f"backward H={H} N={N}")
    q, k, v, do = random_qkv(1, H, N, N, H)
    ref = Ref(q, k, v, do)
    print(ref.check(**backward(q, k, v, ref, do)), flush=True)
    mask = random_mask(1, H, N, 32, 32, 0.5, 6)
    ref = Ref(q, k, v, do, skip=skip_pairs(mask, N, 32, 32))
    got = backward(q, k, v, ref, do, mask_in=mask, tile_q=32, tile_k=32)
    print(ref.check(**got), flush=True)


def test_masked_places_may_hold_anything():
    """NaN and infinities in rows that kept nothing, and in keys that no row kept, go nowhere."""
    import paper_2606_16317_amd as dsa
    from _grad_ref import Ref, random_qkv, skip_pairs

    announce("NaN in masked places")
    N, tile = 400, 32
    q, k, v, do = random_qkv(1, 2, N, N, 14)
    mask = random_mask(1, 2, N, tile, tile, 0.5, 4)
    mask[:, :, 3] = mask[:, :, 12] = 1           # rows, the ragged last ones among them
    mask[..., 5] = mask[..., 12] = 1             # keys
    ref = Ref(q, k, v, do, skip=skip_pairs(mask, N, tile, tile))
    o = ref.o.to(torch.bfloat16)
    for lo, hi in ((96, 128), (384, 400)):
        for x, bad in ((q, math.nan), (do, math.inf), (o, math.nan)):
            x[:, :, lo:hi] = bad
    for lo, hi in ((160, 192), (384, 400)):
        k[:, :, lo:hi], v[:, :, lo:hi] = math.nan, -math.inf
    got = dsa.dsattn_attn_bwd(dsa.RULE_MASK, q, k, v, o, ref.lse.float(), do, mask_in=mask,
                              tile_q=tile, tile_k=tile)
    print(ref.check(dq=got[0], dk=got[1], dv=got[2]), flush=True)


@pytest.mark.parametrize("rule,param,tile_q,tile_k", [
    ("RULE_DENSE", 0.0, 128, 64), ("RULE_DYNSPARSE_LAMBDA", -3.0, 128, 64),
    ("RULE_DYNSPARSE_LAMBDA", -3.0, 32, 32), ("RULE_DYNSPARSE_LAMBDA", -3.0, 32, 128),
    ("RULE_BLASST", 3e-2, 32, 64)])
def test_after_the_library_forward(rule, param, tile_q, tile_k):
    """A whole step: a rule's forward call, then the backward pass of its output."""
    import paper_2606_16317_amd as dsa
    from synth import make_video_qkv
    from _grad_ref import Ref, skip_pairs
    from _parity import to_device

    announce(f"forward {rule} {param} tile {tile_q} x {tile_k}, then backward")
    qn, kn, vn, _ = make_video_qkv(1, 2, (2, 13, 33), 6.0, 6.0, True, 7)
    q, k, v = (to_device(x) for x in (qn, kn, vn))
    N = q.shape[2]
    do = torch.randn(q.shape, generator=torch.Generator("cuda").manual_seed(1),
                     device="cuda").to(torch.bfloat16)
    lse = torch.empty(q.shape[:3], device="cuda")
    mask = torch.empty(1, 2, -(-N // tile_q), -(-N // tile_k), dtype=torch.uint8, device="cuda")
    o = dsa.dsattn_attn_fwd_ex(getattr(dsa, rule), param, q, k, v, tile_q=tile_q, tile_k=tile_k,
                               lse_out=lse, mask_out=mask)
    kw = dict(tile_q=tile_q, tile_k=tile_k)
    if rule == "RULE_DENSE":
        got = dsa.dsattn_attn_bwd(dsa.RULE_DENSE, q, k, v, o, lse, do, **kw)
    else:
        assert 0.05 < mask.float().mean() < 0.95
        got = dsa.dsattn_attn_bwd(dsa.RULE_MASK, q, k, v, o, lse, do, mask_in=mask, **kw)
    ref = Ref(q, k, v, do, skip=skip_pairs(mask, N, tile_q, tile_k), library_forward=True)
    print(ref.check(dq=got[0], dk=got[1], dv=got[2]), flush=True)


def test_against_differences():
    """<gradient, direction> is the slope of the loss <o, do> along it."""
    from _grad_ref import Ref, random_qkv, skip_pairs

    announce("differences")
    N, h = 150, 1e-4
    q, k, v, do = random_qkv(1, 2, N, N, 77, std=1.0)
    mask = random_mask(1, 2, N, 32, 32, 0.6, 3)
    skip = skip_pairs(mask, N, 32, 32)
    ref = Ref(q, k, v, do, skip=skip)
    got = backward(q, k, v, ref, do, mask_in=mask, tile_q=32, tile_k=32)
    g = torch.Generator().manual_seed(8)
    for i, name in enumerate(("dq", "dk", "dv")):
        d = torch.randn(q.shape, generator=g).double().cuda()
        at = [x.double() for x in (q, k, v)]
        loss = []
        for sign in (1.0, -1.0):
            x = list(at)
            x[i] = x[i] + sign * h * d
            loss.append((Ref(*x, skip=skip).o * do.double()).sum().item())
        slope = (loss[0] - loss[1]) / (2 * h)
        mine = (got[name].double() * d).sum().item()
        room = (getattr(ref, "b_" + name) * d.abs()).sum().item()
        # the difference itself is off by h^2 / 6 of the third derivative: far below `room`
        assert abs(mine - slope) <= room, (name, mine, slope, room)


def test_repeated_captured_and_side_stream():
    import paper_2606_16317_amd as dsa
    from _grad_ref import Ref, random_qkv

    announce("repeated, captured and side-stream calls")
    N = 400
    q, k, v, do = random_qkv(1, 3, N, N, 21)
    ref = Ref(q, k, v, do)
    o, lse = ref.o.to(torch.bfloat16), ref.lse.float()
    first = [x.clone() for x in dsa.dsattn_attn_bwd(dsa.RULE_DENSE, q, k, v, o, lse, do)]
    again = dsa.dsattn_attn_bwd(dsa.RULE_DENSE, q, k, v, o, lse, do)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = dsa.dsattn_attn_bwd(dsa.RULE_DENSE, q, k, v, o, lse, do, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))
    # a graph with its own workspace and outputs, replayed with other work between
    ws = torch.empty(dsa.dsattn_attn_bwd_workspace_bytes(1, 3, N), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for _ in range(3)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dsa.dsattn_attn_bwd(dsa.RULE_DENSE, q, k, v, o, lse, do, *outs, workspace=ws)
    for _ in range(3):
        for x in outs:
            x.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
        dsa.dsattn_attn_bwd(dsa.RULE_DENSE, v, q, k, o, lse, do)


def test_refusals():
    import paper_2606_16317_amd as dsa
    from _grad_ref import random_qkv

    announce("refusals")
    N = 70
    q, k, v, do = random_qkv(1, 1, N, N, 2)
    o, lse = q.clone(), torch.zeros(1, 1, N, device="cuda")
    call = lambda rule=dsa.RULE_DENSE, **kw: dsa.dsattn_attn_bwd(
        rule, *(kw.pop(n, x) for n, x in (("q", q), ("k", k), ("v", v), ("o", o), ("lse", lse),
                                          ("do", do))), **kw)
    with pytest.raises(RuntimeError, match="mask_in must be non-null"):
        call(dsa.RULE_MASK)
    with pytest.raises(RuntimeError, match="dense rule or a skip mask"):
        call(dsa.RULE_DYNSPARSE_LAMBDA)
    with pytest.raises(RuntimeError, match="unknown rule"):
        call(9)
    with pytest.raises(RuntimeError, match="dq must not overlap q"):
        call(dq=q)
    with pytest.raises(RuntimeError, match="dv must not overlap dk"):
        x = torch.empty_like(q)
        call(dk=x, dv=x)
    with pytest.raises(RuntimeError, match="workspace too small"):
        call(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(RuntimeError, match="256-byte aligned"):
        call(workspace=torch.empty(9000, dtype=torch.uint8, device="cuda")[64:])
    with pytest.raises(RuntimeError, match="scale must be finite"):
        call(scale=math.inf)
    with pytest.raises(RuntimeError, match="tile shape"):
        call(tile_k=48)
    with pytest.raises(TypeError):
        call(do=do.float())
    with pytest.raises(ValueError):
        call(do=do[:, :, :-1])
    with pytest.raises(ValueError):
        call(lse=lse[..., :-1])
    with pytest.raises(TypeError):
        call(lse=lse.double())
    with pytest.raises(ValueError):
        call(dsa.RULE_MASK, mask_in=torch.zeros(1, dtype=torch.uint8, device="cuda"), tile_q=32)
    empty = torch.empty(1, 0, N, 128, dtype=torch.bfloat16, device="cuda")
    out = dsa.dsattn_attn_bwd(dsa.RULE_DENSE, empty, empty, empty, empty, lse[:, :0].contiguous(),
                              empty)
    assert all(x.shape == empty.shape for x in out)
    torch.cuda.synchronize()


@pytest.mark.parametrize("masked", [False, True])
def test_a_row_with_a_nan_lse_stays_visible(masked):
    """A diverged row's LSE makes its dq, and dk and dv of the keys that it kept, NaN."""
    import paper_2606_16317_amd as dsa
    from _grad_ref import Ref, random_qkv

    announce(f"NaN LSE masked={masked}")
    N = 200
    q, k, v, do = random_qkv(1, 2, N, N, 33)
    mask = torch.zeros(1, 2, 7, 4, dtype=torch.uint8, device="cuda")
    mask[0, 1, 2, 3] = 1                        # rows 64 .. 95 do not keep keys 192 .. 199
    ref = Ref(q, k, v, do)
    o, lse = ref.o.to(torch.bfloat16), ref.lse.float()
    kw = dict(tile_q=32, mask_in=mask) if masked else {}
    rule = dsa.RULE_MASK if masked else dsa.RULE_DENSE
    first = dsa.dsattn_attn_bwd(rule, q, k, v, o, lse, do, **kw)
    lse[0, 1, 70] = math.nan
    dq, dk, dv = dsa.dsattn_attn_bwd(rule, q, k, v, o, lse, do, **kw)
    assert dq[0, 1, 70].isnan().all()
    same = torch.ones(1, 2, N, dtype=torch.bool, device="cuda")
    same[0, 1, 70] = False
    assert torch.equal(dq[same], first[0][same])
    kept = 192 if masked else N
    for x, y in ((dk, first[1]), (dv, first[2])):
        assert x[0, 1, :kept].isnan().all()
        assert torch.equal(x[0, 1, kept:], y[0, 1, kept:]) and torch.equal(x[0, 0], y[0, 0])
    torch.cuda.synchronize()
