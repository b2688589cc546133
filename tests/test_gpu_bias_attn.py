"""GPU tests of attention with a learned position bias by buckets, forward and backward
(``dsattn_bias_attn_fwd``, ``dsattn_bias_attn_bwd``), against 64 bits, elementwise within derived
bounds; a whole training step; single tokens over a growing cache; captured and side-stream
calls; refusals."""

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


def bucket_map(kind, n_q, n_k, seed):
    """(int32 map of every distance, number of buckets)."""
    import paper_2606_16317_amd as dsa

    n = n_q + n_k - 1
    g = torch.Generator().manual_seed(seed)
    if kind == "both":
        m, nb = dsa.dsattn_relative_buckets(n_q, n_k, 32, 128, q_first=max(0, n_k - n_q)), 32
    elif kind == "causal":
        m, nb = dsa.dsattn_relative_buckets(n_q, n_k, 16, 300, q_first=max(0, n_k - n_q),
                                            causal=True), 16
    elif kind == "single":               # every distance its own, as far as they go
        m, nb = torch.arange(n) % 512, 512
    elif kind == "one":                  # all pairs one bucket
        m, nb = torch.zeros(n), 1
    elif kind == "random":               # runs of any length, some closed, some out of range
        m = torch.randint(-1, 8, (n,), generator=g).repeat_interleave(
            torch.randint(1, 90, (n,), generator=g))[:n]
        m[m == 7] = 1 << 30
        nb = 7
    elif kind == "window":               # distances beyond 70 closed: rows far from the keys see none
        d = torch.arange(n) - (n_q - 1)
        m, nb = torch.where(d.abs() <= 70, d.abs() // 9, torch.tensor(-5)), 8
    elif kind == "late":                 # only keys at least 40 later are open
        d = torch.arange(n) - (n_q - 1)
        m, nb = torch.where(d >= 40, 0, -1), 1
    elif kind == "shut":
        m, nb = torch.full((n,), -1), 4
    return torch.as_tensor(m).to(torch.int32).cuda(), nb


KINDS = ["both", "causal", "single", "one", "random", "window", "late", "shut"]
SHAPES = [(1, 1), (1, 37), (1, 2000), (5, 3), (33, 64), (64, 33), (127, 200), (128, 128), (129, 65),
          (300, 300), (31, 1409), (700, 333)]


def make(B, H, n_q, n_k, kind, seed, room=0):
    """q, k, v, do, table, map and the reference."""
    from _grad_ref import Ref, distance_matrix, random_qkv

    q, k, v, do = random_qkv(B, H, n_q, n_k + room, seed)
    m, nb = bucket_map(kind, n_q, n_k, seed)
    g = torch.Generator().manual_seed(seed + 1)
    table = torch.randn(nb, H, generator=g).cuda()
    at = distance_matrix(m, n_q, n_k).long()
    at = torch.where((at >= 0) & (at < nb), at, -1)
    bias = table.t()[:, at.clamp(min=0)].double().masked_fill(at < 0, -math.inf)
    ref = Ref(q, k[:, :, :n_k], v[:, :, :n_k], do, bias=bias)
    ref.add_table(at, nb)
    return q, k, v, do, table, m, ref


def forward(q, k, v, table, m, **kw):
    import paper_2606_16317_amd as dsa

    lse = torch.full(q.shape[:3], float("nan"), device="cuda")
    o = torch.full_like(q, float("nan"))
    dsa.dsattn_bias_attn_fwd(q, k, v, table, m, o=o, lse_out=lse, **kw)
    torch.cuda.synchronize()
    return {"o": o, "lse": lse}


def backward(q, k, v, table, m, ref, do):
    import paper_2606_16317_amd as dsa

    out = dsa.dsattn_bias_attn_bwd(q, k, v, table, m, ref.o.to(torch.bfloat16), ref.lse.float(), do)
    torch.cuda.synchronize()
    return dict(zip(("dq", "dk", "dv", "dtable"), out))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n_k", SHAPES)
def test_forward(n_q, n_k, kind):
    announce(f"bias forward n_q={n_q} n_k={n_k} {kind}")
    q, k, v, _, table, m, ref = make(2, 3, n_q, n_k, kind, n_q + n_k, room=5)
    k[:, :, n_k:] = float("nan")             # rows beyond the keys are not read
    v[:, :, n_k:] = float("nan")
    print(ref.check(**forward(q, k, v, table, m, n_k=n_k)), flush=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n_k", SHAPES)
def test_backward(n_q, n_k, kind):
    announce(f"bias backward n_q={n_q} n_k={n_k} {kind}")
    q, k, v, do, table, m, ref = make(2, 3, n_q, n_k, kind, n_q + n_k)
    got = backward(q, k, v, table, m, ref, do)
    print(ref.check(**got), flush=True)
    empty = torch.isinf(ref.lse)
    assert not got["dq"][empty].any()


def test_longer_rows_and_more_workgroups():
    announce("bias step n=3001, 8 heads")
    q, k, v, do, table, m, ref = make(1, 8, 3001, 3001, "both", 4)
    print(ref.check(**forward(q, k, v, table, m)), flush=True)
    print(ref.check(**backward(q, k, v, table, m, ref, do)), flush=True)


def test_closed_by_the_table():
    """A bias of -inf, or below -30000, closes a bucket for its head alone; a row may keep none."""
    from _grad_ref import Ref, distance_matrix, random_qkv

    announce("closed by the table")
    n, H = 260, 2
    q, k, v, do = random_qkv(1, H, n, n, 12)
    m, nb = bucket_map("both", n, n, 0)
    table = torch.randn(nb, H, generator=torch.Generator().manual_seed(1)).cuda()
    table[:10, 0] = -math.inf
    table[16:, 1] = torch.finfo(torch.float32).min
    table[3:, 1] = -math.inf                 # head 1 keeps distances 0, -1, -2 ...
    table[0, 1] = -3e38                      # ... and of those not 0: the first row has nothing
    bias = table.double().t()[:, distance_matrix(m, n, n).long()]
    bias = bias.masked_fill(bias < -1e30, -math.inf)
    ref = Ref(q, k, v, do, bias=bias)
    ref.add_table(distance_matrix(m, n, n), nb)
    assert torch.isinf(ref.lse).sum() == 1
    print(ref.check(**forward(q, k, v, table, m)), flush=True)
    print(ref.check(**backward(q, k, v, table, m, ref, do)), flush=True)


@pytest.mark.parametrize("low", [-math.inf, -3.4e38, -1e9, -65504.0, -3.1e4, -2.9e4, -1e4])
def test_masking_numbers(low):
    """Masking numbers close their pairs, and leave rows with nothing else without a key; down to
    -30000 they are biases, which rows with nothing else share."""
    from _grad_ref import Ref, distance_matrix, random_qkv

    announce(f"masking number {low}")
    n = 200
    q, k, v, do = random_qkv(1, 2, n, n, 3)
    d = torch.arange(-(n - 1), n)
    m = torch.where(d > 40, 0, 1).to(torch.int32).cuda()      # later keys far enough have a value
    table = torch.tensor([[0.25, -0.5], [low, low]]).cuda()
    at = distance_matrix(m, n, n)
    bias = table.double().t()[:, at.long()]
    if low < -3e4:
        bias = bias.masked_fill(bias < -3e4, -math.inf)
    ref = Ref(q, k, v, do, bias=bias)
    ref.add_table(at, 2)
    assert torch.isinf(ref.lse).any() == (low < -3e4)
    print(ref.check(**forward(q, k, v, table, m)), flush=True)
    print(ref.check(**backward(q, k, v, table, m, ref, do)), flush=True)


@pytest.mark.parametrize("H,n_q,n_k", [(512, 70, 100), (171, 257, 120), (515, 100, 200),
                                       (700, 1, 300)])
@pytest.mark.parametrize("kind", ["both", "random"])
def test_whole_rounds_of_workgroups_and_a_remainder(H, n_q, n_k, kind):
    """512 row groups at a time go without a split, the rest may be shared: none, few or most."""
    announce(f"bias step H={H} n_q={n_q} n_k={n_k} {kind}")
    q, k, v, do, table, m, ref = make(1, H, n_q, n_k, kind, H)
    print(ref.check(**forward(q, k, v, table, m)), flush=True)
    print(ref.check(**backward(q, k, v, table, m, ref, do)), flush=True)


def test_cache_beyond_32_bit_offsets():
    """A token over 40 heads of 450000 rows each, 2.3e9 numbers, of which 700 are keys."""
    import paper_2606_16317_amd as dsa

    announce("cache of 2.3e9 numbers")
    H, rows, n = 40, 450000, 700
    q, k, v, _, table, m, ref = make(1, H, 1, n, "causal", 77)
    cache = [torch.empty(1, H, rows, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for c, x in zip(cache, (k, v)):
        c[:, :, :n] = x
    lse = torch.empty(1, H, 1, device="cuda")
    o = dsa.dsattn_bias_attn_fwd(q, *cache, table, m, n_k=n, lse_out=lse)
    print(ref.check(o=o, lse=lse), flush=True)


def test_gradients_beyond_32_bit_offsets():
    """65 heads of 262144 keys, 2.2e9 numbers; the last head against 64 bits."""
    import paper_2606_16317_amd as dsa
    from _grad_ref import Ref, distance_matrix, random_qkv

    announce("gradients of 2.2e9 numbers")
    H, n_q, n_k = 65, 33, 262144
    m, nb = bucket_map("both", n_q, n_k, 0)
    table = torch.randn(nb, H, generator=torch.Generator().manual_seed(2)).cuda()
    q, k, v, do = random_qkv(1, 1, n_q, n_k, 8)
    at = distance_matrix(m, n_q, n_k)
    ref = Ref(q, k, v, do, bias=table[:, -1:].double().t()[:, at.long()])
    ref.add_table(at, nb)
    full = lambda x: torch.cat([x.new_zeros(1, H - 1, *x.shape[2:]), x], 1)
    lse = ref.lse.float()
    got = dsa.dsattn_bias_attn_bwd(*(full(x) for x in (q, k, v)), table, m,
                                   full(ref.o.to(torch.bfloat16)), full(lse), full(do))
    got = dict(zip(("dq", "dk", "dv"), (x[:, -1:] for x in got[:3])), dtable=got[3][:, -1:])
    print(ref.check(**got), flush=True)


@pytest.mark.parametrize("n_q,n_k", [(3, 0), (0, 3), (0, 0)])
def test_no_keys_or_no_queries(n_q, n_k):
    import paper_2606_16317_amd as dsa

    announce(f"n_q={n_q} n_k={n_k}")
    q = torch.ones(1, 2, n_q, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.ones(1, 2, n_k, 128, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(4, 2, device="cuda")
    m = torch.zeros(8, dtype=torch.int32, device="cuda")
    got = forward(q, k, k, table, m)
    assert not got["o"].any() and (got["lse"] == -math.inf).all()
    out = dsa.dsattn_bias_attn_bwd(q, k, k, table, m, q, got["lse"], q,
                                   dtable=torch.full_like(table, float("nan")))
    assert not any(x.any() for x in out)


@pytest.mark.parametrize("B", [0, 2])
def test_empty_batch(B):
    import paper_2606_16317_amd as dsa

    announce(f"B={B}, n_q = 0")
    q = torch.ones(B, 2, 0 if B else 4, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.ones(B, 2, 4, 128, dtype=torch.bfloat16, device="cuda")
    table, m = torch.zeros(4, 2, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    out = dsa.dsattn_bias_attn_bwd(q, k, k, table, m, q, torch.zeros(q.shape[:3], device="cuda"), q,
                                   dtable=torch.full_like(table, float("nan")))
    assert not any(x.any() for x in out)


def test_tokens_over_a_growing_cache():
    """A rollout: a prompt, then single tokens, against one causal call over all of them; the
    maps of the steps are slices of the longest one."""
    import paper_2606_16317_amd as dsa

    announce("growing cache")
    n, prompt, B, H = 200, 150, 2, 4
    q, k, v, _, table, _, ref = make(B, H, n, n, "causal", 31)
    longest = torch.from_numpy(dsa.dsattn_relative_buckets(1, n, 16, 300, q_first=n - 1,
                                                           causal=True)).cuda()
    cache_k, cache_v = torch.full_like(k, float("nan")), torch.full_like(v, float("nan"))
    for i in [prompt, *range(prompt + 1, n + 1)]:
        lo = 0 if i == prompt else i - 1
        cache_k[:, :, lo:i], cache_v[:, :, lo:i] = k[:, :, lo:i], v[:, :, lo:i]
        step = q[:, :, lo:i].contiguous()
        if lo:
            m = longest[n - i:]
        else:
            m = torch.from_numpy(dsa.dsattn_relative_buckets(i, i, 16, 300, causal=True)).cuda()
        got = forward(step, cache_k, cache_v, table, m, n_k=i)
        rows = type("Rows", (), {})()
        for name in ("o", "lse"):
            for p in ("", "b_"):
                setattr(rows, p + name, getattr(ref, p + name)[:, :, lo:i])
        type(ref).check(rows, **got)


def test_a_training_step():
    """Forward, a loss and its gradients through an autograd function a user would write."""
    import paper_2606_16317_amd as dsa

    from _grad_ref import Ref, distance_matrix

    announce("training step")

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, table, bucket):
            lse = torch.empty(q.shape[:3], device=q.device)
            o = dsa.dsattn_bias_attn_fwd(q, k, v, table, bucket, lse_out=lse)
            ctx.save_for_backward(q, k, v, table, bucket, o, lse)
            return o

        @staticmethod
        def backward(ctx, do):
            return (*dsa.dsattn_bias_attn_bwd(*ctx.saved_tensors, do.contiguous()), None)

    q, k, v, do, table, m, ref = make(2, 3, 190, 190, "both", 91)
    leaves = [x.clone().requires_grad_() for x in (q, k, v, table)]
    o = Attention.apply(*leaves, m)
    (o * do).sum().backward()
    ref.check(o=o.detach())
    at = distance_matrix(m, 190, 190).long()
    ref = Ref(q, k, v, do, bias=table.t()[:, at], library_forward=True)
    ref.add_table(at, 32)
    print(ref.check(**dict(zip(("dq", "dk", "dv", "dtable"), (x.grad for x in leaves)))), flush=True)


def test_against_differences():
    """<gradient, direction> is the slope of the loss <o, do> along it, the table's too."""
    from _grad_ref import Ref, distance_matrix

    announce("differences")
    n, h = 140, 1e-4
    q, k, v, do, table, m, ref = make(1, 2, n, n, "both", 55)
    got = backward(q, k, v, table, m, ref, do)
    at = distance_matrix(m, n, n).long()
    g = torch.Generator().manual_seed(8)
    for i, name in enumerate(("dq", "dk", "dv", "dtable")):
        leaves = [x.double() for x in (q, k, v, table)]
        d = torch.randn(leaves[i].shape, generator=g).double().cuda()
        loss = []
        for sign in (1.0, -1.0):
            x = list(leaves)
            x[i] = x[i] + sign * h * d
            loss.append((Ref(*x[:3], bias=x[3].t()[:, at]).o * do.double()).sum().item())
        slope = (loss[0] - loss[1]) / (2 * h)
        mine = (got[name].double() * d).sum().item()
        # the difference is off by h^2 / 6 of the third derivative, far below the bound
        room = (getattr(ref, "b_" + name) * d.abs()).sum().item() + 1e-6 * abs(slope)
        assert abs(mine - slope) <= room, (name, mine, slope, room)


@pytest.mark.parametrize("kind", ["both", "one", "random", "single"])
def test_repeated_calls_give_the_same_bits(kind):
    announce(f"repeated {kind}")
    q, k, v, do, table, m, ref = make(2, 3, 500, 700, kind, 2)
    first = {**forward(q, k, v, table, m), **backward(q, k, v, table, m, ref, do)}
    for _ in range(4):
        again = {**forward(q, k, v, table, m), **backward(q, k, v, table, m, ref, do)}
        for name, x in first.items():
            assert torch.equal(x, again[name]), name


def test_captured_and_side_stream():
    import paper_2606_16317_amd as dsa

    announce("captured and side-stream calls")
    # one query: the split and joined form
    for n_q, n_k in ((1, 900), (200, 200)):
        q, k, v, do, table, m, ref = make(1, 2, n_q, n_k, "both", 6)
        o, lse0 = ref.o.to(torch.bfloat16), ref.lse.float()
        first = {**forward(q, k, v, table, m), **backward(q, k, v, table, m, ref, do)}
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        lse = torch.empty_like(lse0)
        out = dsa.dsattn_bias_attn_fwd(q, k, v, table, m, lse_out=lse, stream=side)
        grads = dsa.dsattn_bias_attn_bwd(q, k, v, table, m, o, lse0, do, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first.values(), (out, lse, *grads)))
        ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in
              (dsa.dsattn_bias_attn_workspace_bytes(1, 2, n_q, n_k),
               dsa.dsattn_bias_attn_bwd_workspace_bytes(1, 2, n_q, n_k, 32))]
        outs = [torch.empty_like(x) for x in first.values()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dsa.dsattn_bias_attn_fwd(q, k, v, table, m, o=outs[0], lse_out=outs[1],
                                     workspace=ws[0])
            dsa.dsattn_bias_attn_bwd(q, k, v, table, m, o, lse0, do, *outs[2:], workspace=ws[1])
        for _ in range(3):
            for x in outs:
                x.fill_(float("nan"))
            for x in ws:
                x.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first.values(), outs))
            dsa.dsattn_bias_attn_fwd(q, v, k, table, m)


def test_refusals():
    import paper_2606_16317_amd as dsa

    announce("refusals")
    n = 40
    q, k, v, do, table, m, ref = make(1, 2, n, n, "both", 3)
    lse = ref.lse.float()
    o = ref.o.to(torch.bfloat16)
    fwd = lambda **kw: dsa.dsattn_bias_attn_fwd(
        *[kw.pop(x, y) for x, y in (("q", q), ("k", k), ("v", v), ("table", table), ("m", m))], **kw)
    bwd = lambda **kw: dsa.dsattn_bias_attn_bwd(
        *[kw.pop(x, y) for x, y in (("q", q), ("k", k), ("v", v), ("table", table), ("m", m),
                                    ("o", o), ("lse", lse), ("do", do))], **kw)
    for call in (fwd, bwd):
        with pytest.raises(TypeError):
            call(q=q.half())
        with pytest.raises(TypeError):
            call(table=table.bfloat16())
        with pytest.raises(TypeError):
            call(m=m.long())
        with pytest.raises(ValueError):
            call(m=m[1:])
        with pytest.raises(ValueError):
            call(table=table[:, :1].contiguous())
        with pytest.raises(ValueError):
            call(k=k[:, :1].contiguous(), v=v[:, :1].contiguous())
        with pytest.raises(ValueError):
            call(v=v[:, :, 1:].contiguous())
        with pytest.raises(ValueError):
            call(q=q.transpose(1, 2))
        with pytest.raises(RuntimeError, match="scale must be finite"):
            call(scale=-1.0)
        with pytest.raises(RuntimeError, match="n_buckets must lie"):
            call(table=torch.zeros(513, 2, device="cuda"))
        with pytest.raises(RuntimeError, match="workspace too small"):
            call(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        fwd(n_k=n + 1)
    with pytest.raises(RuntimeError, match="must not overlap"):
        fwd(o=q)
    both = torch.empty(q.numel(), dtype=torch.float32, device="cuda")
    with pytest.raises(RuntimeError, match="lse_out must not overlap o"):
        fwd(o=both.view(torch.bfloat16)[:q.numel()].view(q.shape), lse_out=both[:2 * n])
    with pytest.raises(RuntimeError, match="dk must not overlap k"):
        bwd(dk=k)
    with pytest.raises(RuntimeError, match="dtable must not overlap table"):
        bwd(dtable=table)
    with pytest.raises(ValueError):
        bwd(dtable=table[:-1])
    torch.cuda.synchronize()


@pytest.mark.parametrize("H,n_q,n_k", [(2, 1, 900), (2, 200, 300), (512, 70, 100)])
@pytest.mark.parametrize("bad", ["query", "key"])
def test_a_row_of_nan_logits_stays_visible(H, n_q, n_k, bad):
    """A NaN query, or an infinite key, makes its rows and their LSE NaN whether their keys are split
    over workgroups or not, as the softmax does, and from that LSE the gradients; other heads keep
    their bits."""
    import paper_2606_16317_amd as dsa

    announce(f"NaN logits by a {bad}, H={H} n_q={n_q} n_k={n_k}")
    q, k, v, do, table, m, ref = make(1, H, n_q, n_k, "one", 5)
    first = forward(q, k, v, table, m)
    grads = dsa.dsattn_bias_attn_bwd(q, k, v, table, m, first["o"], first["lse"], do)
    row = n_q // 2
    if bad == "query":
        q[0, 1, row] = math.nan
    else:
        k[0, 1, n_k - 1] = math.inf            # q . k: a sum of infinities of both signs
    got = forward(q, k, v, table, m)
    hit = torch.zeros(1, H, n_q, dtype=torch.bool, device="cuda")
    hit[0, 1, slice(row, row + 1) if bad == "query" else slice(None)] = True
    assert torch.equal(got["lse"].isnan(), hit)
    assert torch.equal(got["o"].isnan(), hit[..., None].expand_as(got["o"]))
    for name, x in got.items():
        assert torch.equal(x[~hit], first[name][~hit]), name
    out = dsa.dsattn_bias_attn_bwd(q, k, v, table, m, got["o"], got["lse"], do)
    assert torch.equal(out[0].isnan(), hit[..., None].expand_as(out[0]))
    assert all(x[:, 1].isnan().all() for x in out[1:3]) and out[3][0, 1].isnan()
    others = [h for h in range(H) if h != 1]
    for x, y in zip(out, grads):
        assert torch.equal(x[:, others], y[:, others])
    torch.cuda.synchronize()


def test_side_stream_calls_keep_their_outputs():
    """Outputs that a call on a side stream makes: memory that the current stream allocates and
    fills right after the call, with the side stream still busy ahead of its kernels, is neither
    theirs nor, once they are dropped, overwritten by them."""
    import paper_2606_16317_amd as dsa

    announce("outputs of a side stream")
    q, k, v, do, table, m, ref = make(1, 2, 300, 300, "both", 6)
    o, lse = ref.o.to(torch.bfloat16), ref.lse.float()
    steps = [lambda **kw: (dsa.dsattn_bias_attn_fwd(q, k, v, table, m, **kw),),
             lambda **kw: dsa.dsattn_bias_attn_bwd(q, k, v, table, m, o, lse, do, **kw),
             lambda **kw: dsa.dsattn_attn_bwd(dsa.RULE_DENSE, q, k, v, o, lse, do, **kw)]
    want = [step() for step in steps]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for step, first in zip(steps, want):
        for drop in (False, True):
            with torch.cuda.stream(side):
                torch.cuda._sleep(20_000_000)              # some milliseconds
            out = step(stream=side)
            if drop:
                del out
            grabbed = [torch.empty_like(x).fill_(7.0) for x in first for _ in range(4)]
            side.synchronize()
            torch.cuda.synchronize()
            assert all((x == 7.0).all() for x in grabbed)
            if not drop:
                torch.cuda.current_stream().wait_stream(side)
                assert all(torch.equal(a, b) for a, b in zip(first, out))
            del grabbed
