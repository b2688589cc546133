"""The training and position-bias operators as measured cases.

Three families stand around the library's forward pass:

* ``bwd``: dq, dk and dv of one attention layer, dense or under a skip mask that an earlier
  call wrote (fine-tuning with the sparse pattern held fixed);
* ``bias``: attention whose logits carry a learned relative position bias, one number per
  head and bucket of the distance key - query, with its log-sum-exp; the queries may be the
  last few positions of a longer cache, down to a single token;
* ``bias_bwd``: the gradients of that layer, the table's among them.

``own`` selects what ``run`` calls: the plain form below (32-bit torch operations) or the
library's entry points.
"""

import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
LARGEST = 10.0 * D * 10 * 32760.0 ** 2      # FLOP of the largest listed case
CHUNK = 2.0 ** 28                           # logits that the plain forms hold at a time


def _case(name, family, heads, n, **more):
    """B batches of `heads` heads of n tokens; `conc_*` is the range of the heads' logit
    spread.  bwd: `masked`, with the decision unit and the share of pairs kept.  bias: n_q
    queries at positions n - n_q .. n - 1 of n keys, in a cache of `room` more rows per
    head; `causal` closes the keys after a query."""
    c = {"family": family, "B": 1, "H": heads, "n": n, "n_q": n, "room": 0, "conc_lo": 0.5,
         "conc_hi": 2.0, "masked": False, "tile_q": 128, "tile_k": 64, "kept": 1.0,
         "buckets": 32, "max_distance": 128, "causal": False}
    if name is not None:
        c["name"] = name
    c.update(more)
    return c


def listed():
    return [
        # One head of a 2 x 32 x 32 test grid: three launches and their latency.
        _case("bwd_tiny", "bwd", 1, 2048),
        # Fine-tuning on a short clip, five 480p latent frames (5 x 30 x 52, ragged).
        _case("bwd_clip", "bwd", 8, 7800),
        # One GPU's 10 of the 40 heads of a 480p layer: the largest call.
        _case("bwd_480p", "bwd", 10, 32760),
        # The same layer under the mask of its forward pass, decided for 32 rows at a time.
        _case("bwd_reuse_480p", "bwd", 10, 32760, masked=True, tile_q=32, kept=0.25),
        # A ragged grid (3 x 17 x 27) under a mask of 32-key decisions, two clips.
        _case("bwd_reuse_small", "bwd", 3, 1377, B=2, masked=True, tile_k=32, kept=0.4),
        # One new token after 32759 others, all 40 heads: the keys and values are read once.
        _case("bias_token", "bias", 40, 32760, n_q=1, room=1560, causal=True),
        # A small ragged layer with an odd number of buckets, distances told apart up to 60.
        _case("bias_small", "bias", 3, 1377, B=2, buckets=121, max_distance=60),
        # The next latent frame (30 x 52 tokens) of a rollout over four earlier ones.
        _case("bias_frame", "bias", 40, 7800, n_q=1560, room=7800, causal=True,
              max_distance=1560),
        # A layer of 24 heads and 27280 tokens, both directions.
        _case("bias_layer", "bias", 24, 27280, max_distance=1024),
        # Training steps: the small layer, the short clip, and one GPU's share of a causal
        # 480p layer.
        _case("bias_bwd_small", "bias_bwd", 3, 1377, B=2, buckets=121, max_distance=60),
        _case("bias_bwd_clip", "bias_bwd", 8, 7800, max_distance=1024),
        _case("bias_bwd_480p", "bias_bwd", 5, 32760, causal=True, max_distance=4096),
    ]


def _spread(rng, lo, hi):
    """A whole number spread over the logarithm of lo..hi."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    family = rng.choice(["bwd", "bwd", "bias", "bias", "bias_bwd"])
    n = _spread(rng, 1, 32760)
    c = _case(None, family, 1, n)
    if family == "bias":
        # a whole layer, or the last tokens of a cache
        c["n_q"] = n if rng.random() < 0.4 else _spread(rng, 1, min(n, 1560))
        c["room"] = rng.choice([0, 0, rng.randint(1, 2000)])
    cost = (4.0 if family == "bias" else 10.0) * D * c["n_q"] * n
    most = max(1, min(40, int(0.5 * LARGEST / cost)))
    c["H"] = _spread(rng, 1, most)
    if c["H"] * n < 60000 and rng.random() < 0.3:
        c["B"] = 2
    c["conc_lo"] = rng.choice([0.25, 0.5, 1.0])
    c["conc_hi"] = rng.choice([1.0, 2.0, 3.0])
    if family == "bwd":
        c["masked"] = rng.random() < 0.5
        if c["masked"]:
            c.update(tile_q=rng.choice([32, 128]), tile_k=rng.choice([32, 64, 64, 128]),
                     kept=round(rng.uniform(0.1, 0.7), 2))
    else:
        c["causal"] = rng.random() < 0.5
        c["buckets"] = rng.choice([8, 16, 32, 32, 64, 2 * rng.randint(2, 128)])
        c["max_distance"] = _spread(rng, c["buckets"], 40000)
    return c


# ---- inputs --------------------------------------------------------------------------


def _noise(c, seed, salt):
    return torch.Generator(device="cuda").manual_seed(7919 * seed + salt)


def _qkv(c, seed):
    """bf16 q [B, H, n_q, D] and k, v [B, H, n + room, D]: half of a head's spread sits in
    a few shared directions, as trained queries and keys have it."""
    B, H, n, n_q = c["B"], c["H"], c["n"], c["n_q"]
    rows = n + c["room"]
    g = _noise(c, seed, 1)
    q = torch.empty(B, H, n_q, D, device="cuda", dtype=torch.bfloat16)
    k = torch.empty(B, H, rows, D, device="cuda", dtype=torch.bfloat16)
    v = torch.empty_like(k)
    conc = torch.rand(H, generator=g, device="cuda") * (c["conc_hi"] - c["conc_lo"]) + c["conc_lo"]
    conc = conc.sqrt().tolist()
    for b in range(B):
        for h in range(H):
            shared = torch.randn(8, D, generator=g, device="cuda")
            for t, m in ((q, n_q), (k, rows)):
                x = torch.randn(m, 8, generator=g, device="cuda") @ shared * 0.25
                x += torch.randn(m, D, generator=g, device="cuda") * 0.7
                t[b, h] = (conc[h] * x).to(torch.bfloat16)
            v[b, h] = torch.randn(rows, D, generator=g, device="cuda").to(torch.bfloat16)
    return q, k, v


def _mask(c, seed):
    """A skip mask [B, H, units, decisions] (1 = skipped) that keeps about the share `kept`:
    whole runs of tiles as a rule leaves them, every unit's own tile, and, in one unit of a
    larger mask, nothing at all."""
    n_u, n_d = -(-c["n"] // c["tile_q"]), -(-c["n"] // c["tile_k"])
    g = _noise(c, seed, 2)
    coarse = torch.rand(c["B"], c["H"], -(-n_u // 4), -(-n_d // 4), generator=g, device="cuda")
    fine = torch.rand(c["B"], c["H"], n_u, n_d, generator=g, device="cuda")
    x = coarse.repeat_interleave(4, 2)[:, :, :n_u].repeat_interleave(4, 3)[..., :n_d]
    mask = 0.7 * x + 0.3 * fine
    # the quantile of the sum that leaves `kept`, from a sample of it
    sample = mask.flatten()[:: max(1, mask.numel() // 100000)].sort().values
    limit = sample[min(sample.numel() - 1, int(c["kept"] * sample.numel()))]
    mask = (mask >= limit).to(torch.uint8)
    unit = torch.arange(n_u, device="cuda")
    mask[:, :, unit, unit * c["tile_q"] // c["tile_k"]] = 0
    if n_u > 4:
        mask[:, :, n_u // 2] = 1
    return mask


def _bucket_map(c):
    """int32 bucket of every distance key - query, from -(n - 1) up to n_q - 1 (-1: closed).
    Half of the buckets (all of them when causal) serve each direction: a distance below
    half of those has its own, the others share by the logarithm up to max_distance."""
    rel = torch.arange(-(c["n"] - 1), c["n_q"], dtype=torch.int64)
    per = c["buckets"] if c["causal"] else c["buckets"] // 2
    alone = max(1, per // 2)
    away = rel.abs().double()
    far = torch.log(away.clamp(min=alone) / alone) / math.log(max(c["max_distance"], alone + 1)
                                                             / alone)
    far = alone + (far * (per - alone) + 1e-9).floor().long()
    b = torch.where(away < alone, rel.abs(), far.clamp(max=per - 1))
    b = torch.where(rel > 0, torch.full_like(b, -1) if c["causal"] else b + per, b)
    return b.to(torch.int32).cuda()


def _table(c, seed):
    """Learned biases [buckets, H]: falling off with the bucket, with noise."""
    g = _noise(c, seed, 3)
    fall = torch.linspace(0.5, -1.5, c["buckets"], device="cuda")[:, None]
    return (fall + 0.7 * torch.randn(c["buckets"], c["H"], generator=g, device="cuda")).contiguous()


def prepare(case, seed):
    c = case
    st = {"case": c}
    st["q"], st["k"], st["v"] = _qkv(c, seed)
    if c["masked"]:
        st["mask"] = _mask(c, seed)
    if c["family"] != "bwd":
        st["table"], st["bucket"] = _table(c, seed), _bucket_map(c)
    if c["family"] != "bias":
        st["do"] = torch.randn(st["q"].shape, generator=_noise(c, seed, 4),
                               device="cuda").to(torch.bfloat16)
        # what the forward pass left behind
        st["o"], st["lse"] = _plain_forward(st)
    return st


# ---- plain forms ---------------------------------------------------------------------


def _blocks(c):
    """(batch, head, first row, row after the last) of row blocks that fit the chunk."""
    rows = max(1, min(c["n_q"], int(CHUNK // max(1, c["n"]))))
    return [(b, h, r0, min(c["n_q"], r0 + rows)) for b in range(c["B"]) for h in range(c["H"])
            for r0 in range(0, c["n_q"], rows)]


def _distances(c, x, r0, r1):
    """Rows r0..r1 of the matrix x[key - query] from a vector over all distances."""
    first = c["n_q"] - 1 - torch.arange(r0, r1, device="cuda")
    return x.unfold(0, c["n"], 1)[first]


def _bias_vector(st, h):
    b = st["bucket"].long()
    x = st["table"][:, h][b.clamp(min=0)]
    return torch.where(b < 0, torch.full_like(x, -math.inf), x)


def _logits(st, q, k, b, h, r0, r1):
    c = st["case"]
    s = (q @ k.t()) * SCALE
    if "table" in st:
        s += _distances(c, _bias_vector(st, h), r0, r1)
    if "mask" in st:
        unit = torch.arange(r0, r1, device="cuda") // c["tile_q"]
        key = torch.arange(c["n"], device="cuda") // c["tile_k"]
        s.masked_fill_(st["mask"][b, h].bool()[unit][:, key], -math.inf)
    return s


def _softmax(s):
    """(probabilities, log-sum-exp); a row with nothing open gets zeros and -inf."""
    m = s.amax(1, keepdim=True)
    top = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = (s - top).exp()
    total = p.sum(1, keepdim=True)
    p /= torch.where(total > 0, total, torch.ones_like(total))
    return p, (top + total.log())[:, 0]


def _plain_forward(st):
    c = st["case"]
    o = torch.empty_like(st["q"])
    lse = torch.empty(o.shape[:3], device="cuda", dtype=torch.float32)
    for b, h, r0, r1 in _blocks(c):
        k, v = (st[n][b, h, :c["n"]].float() for n in ("k", "v"))
        p, lse[b, h, r0:r1] = _softmax(_logits(st, st["q"][b, h, r0:r1].float(), k, b, h, r0, r1))
        o[b, h, r0:r1] = (p @ v).to(torch.bfloat16)
    return o, lse


def _diagonal_sums(x):
    """Sum of x [R, n] over each key - row distance, [n + R - 1] from -(R - 1) up."""
    R, n = x.shape
    skewed = torch.nn.functional.pad(x.flip(0), (0, R)).flatten()[: R * (n + R - 1)]
    return skewed.view(R, n + R - 1).sum(0, dtype=torch.float64)


def _plain_backward(st):
    c = st["case"]
    n = c["n"]
    grads = {x: torch.zeros(st[x].shape, device="cuda", dtype=torch.float32) for x in "qkv"}
    by_distance = torch.zeros(c["H"], n + c["n_q"] - 1, device="cuda", dtype=torch.float64)
    for b, h, r0, r1 in _blocks(c):
        q, do = (st[x][b, h, r0:r1].float() for x in ("q", "do"))
        k, v = (st[x][b, h].float() for x in "kv")
        p, _ = _softmax(_logits(st, q, k, b, h, r0, r1))
        grads["v"][b, h] += p.t() @ do
        dp = do @ v.t()
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        if "table" in st:
            first = c["n_q"] - r1
            by_distance[h, first: first + n + (r1 - r0) - 1] += _diagonal_sums(ds)
        grads["q"][b, h, r0:r1] = (ds @ k) * SCALE
        grads["k"][b, h] += (ds.t() @ q) * SCALE
    out = [grads[x].to(torch.bfloat16) for x in "qkv"]
    if "table" in st:
        bucket = st["bucket"].long()
        by_distance[:, bucket < 0] = 0.0
        dt = torch.zeros(c["buckets"], c["H"], device="cuda", dtype=torch.float64)
        out.append(dt.index_add_(0, bucket.clamp(min=0), by_distance.t().contiguous()).float())
    return tuple(out)


# ---- one pass --------------------------------------------------------------------------


def run(state):
    st, c = state, state["case"]
    if not own:
        return _plain_forward(st) if c["family"] == "bias" else _plain_backward(st)
    import paper_2606_16317_amd as dsa

    if c["family"] == "bias":
        lse = torch.empty(st["q"].shape[:3], device="cuda", dtype=torch.float32)
        o = dsa.dsattn_bias_attn_fwd(st["q"], st["k"], st["v"], st["table"], st["bucket"],
                                     n_k=c["n"], lse_out=lse)
        return o, lse
    if c["family"] == "bias_bwd":
        return dsa.dsattn_bias_attn_bwd(st["q"], st["k"], st["v"], st["table"], st["bucket"],
                                        st["o"], st["lse"], st["do"])
    if c["masked"]:
        return dsa.dsattn_attn_bwd(dsa.RULE_MASK, st["q"], st["k"], st["v"], st["o"], st["lse"],
                                   st["do"], tile_q=c["tile_q"], tile_k=c["tile_k"],
                                   mask_in=st["mask"])
    return dsa.dsattn_attn_bwd(dsa.RULE_DENSE, st["q"], st["k"], st["v"], st["o"], st["lse"],
                               st["do"])


def work(case):
    """Open pairs times the products each needs (two forward, five backward), and every
    input and output once."""
    c = case
    n, n_q = c["n"], c["n_q"]
    heads = c["B"] * c["H"]
    pairs = float(n) * n_q * c["kept"]
    if c["causal"]:
        pairs = float(n_q) * (n - n_q) + 0.5 * n_q * (n_q + 1.0)
    if c["family"] == "bias":
        return {"bytes": heads * (2 * n_q + 2 * n) * D * 2 + heads * n_q * 4 +
                4 * (n + n_q - 1 + c["buckets"] * c["H"]), "flops": 4.0 * D * heads * pairs}
    moved = heads * n * (8 * D * 2 + 4)
    if c["masked"]:
        moved += heads * -(-n // c["tile_q"]) * -(-n // c["tile_k"])
    if c["family"] == "bias_bwd":
        moved += 4 * (2 * n - 1 + 2 * c["buckets"] * c["H"])
    return {"bytes": moved, "flops": 10.0 * D * heads * pairs}


# ---- 64-bit results --------------------------------------------------------------------


def _open64(c, seed, b, h, i, n):
    """(additive bias, open) of queries i (a vector) against all n keys, in float64."""
    j = torch.arange(n, device="cuda")
    if c["family"] == "bwd":
        if not c["masked"]:
            return 0.0, None
        skip = _mask(c, seed)[b, h]
        return 0.0, skip[(i // c["tile_q"])[:, None], (j // c["tile_k"])[None, :]] == 0
    bucket = _bucket_map(c).long()[(j[None, :] - i[:, None]) + c["n_q"] - 1]
    bias = _table(c, seed).double()[:, h]
    return bias[bucket.clamp(min=0)], bucket >= 0


def exact(case, seed):
    c = case
    n, n_q = c["n"], c["n_q"]
    q, k, v = _qkv(c, seed)
    forward = c["family"] == "bias"
    if forward:
        o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    else:
        do = torch.randn(q.shape, generator=_noise(c, seed, 4), device="cuda").to(torch.bfloat16)
        dq, dk, dv = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(3))
        dist = torch.zeros(c["H"], n + n_q - 1, dtype=torch.float64, device="cuda")
    step = max(1, min(n_q, int(1.2e8 // n)))
    for b in range(c["B"]):
        for h in range(c["H"]):
            kh, vh = k[b, h, :n].double(), v[b, h, :n].double()
            kt, vt = kh.t().contiguous(), vh.t().contiguous()
            for lo in range(0, n_q, step):
                i = torch.arange(lo, min(n_q, lo + step), device="cuda")
                qi = q[b, h, i].double()
                s = torch.mm(qi, kt).mul_(SCALE)
                bias, free = _open64(c, seed, b, h, i, n)
                s += bias
                if free is not None:
                    s = torch.where(free, s, torch.full_like(s, -math.inf))
                row = torch.logsumexp(s, 1)
                p = torch.exp(s - torch.where(torch.isinf(row), torch.zeros_like(row),
                                              row)[:, None])
                del s
                if forward:
                    o[b, h, i], lse[b, h, i] = torch.mm(p, vh), row
                    continue
                doi = do[b, h, i].double()
                mean = (doi * torch.mm(p, vh)).sum(1)
                dv[b, h] += torch.mm(p.t(), doi)
                ds = torch.mm(doi, vt).sub_(mean[:, None]).mul_(p)
                del p
                dq[b, h, i] = torch.mm(ds, kh) * SCALE
                dk[b, h] += torch.mm(ds.t(), qi) * SCALE
                if c["family"] == "bias_bwd":
                    at = torch.arange(n, device="cuda")[None, :] - i[:, None] + n_q - 1
                    dist[h].index_add_(0, at.flatten(), ds.flatten())
                del ds
    if forward:
        return o, lse
    if c["family"] == "bwd":
        return dq, dk, dv
    bucket = _bucket_map(c).long()
    dt = torch.stack([dist[:, bucket == x].sum(1) for x in range(c["buckets"])])
    return dq, dk, dv, dt
