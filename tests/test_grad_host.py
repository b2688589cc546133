"""Backward pass: the host side of the C ABI without a GPU -- struct layout, workspace sizes and
the refusals that need no device pointer -- and the 64-bit reference of the GPU tests against
autograd and differences."""

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "dsattn.h")


def _lib():
    import paper_2606_16317_amd as pkg

    if not os.path.exists(pkg.LIB_PATH):
        pytest.skip("libdsattn.so not built")
    return pkg


def header_fields(struct):
    text = open(HEADER).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), text, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = []
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        names += [p.replace("*", " ").split()[-1] for p in decl.split(",")]
    return names


@pytest.mark.parametrize("struct,mirror", [("dsattn_bwd_args", "DsAttnBwdArgs"),
                                           ("dsattn_bias_args", "DsAttnBiasArgs"),
                                           ("dsattn_bias_bwd_args", "DsAttnBiasBwdArgs")])
def test_struct_mirrors(struct, mirror):
    pkg = _lib()
    assert header_fields(struct) == [f[0] for f in getattr(pkg, mirror)._fields_]


def bwd_args(pkg, **kw):
    a = pkg.DsAttnBwdArgs(rule=pkg.RULE_DENSE, B=1, H=1, N=64, d=128, scale=0.1, tile_q=128,
                          tile_k=64)
    for name, x in kw.items():
        setattr(a, name, x)
    return a


@pytest.mark.parametrize("kw,rc,message", [
    (dict(rule=7), -1, "unknown rule"),
    (dict(rule=1), -2, "dense rule or a skip mask"),
    (dict(rule=2), -2, "dense rule or a skip mask"),
    (dict(rule=3), -2, "dense rule or a skip mask"),
    (dict(N=-1), -1, ">= 0"),
    (dict(d=64), -2, "head dimension"),
    (dict(scale=0.0), -1, "scale"),
    (dict(scale=float("nan")), -1, "scale"),
    (dict(tile_q=64), -2, "tile shape"),
    (dict(tile_k=16), -2, "tile shape"),
    (dict(B=300, H=300), -1, "65535"),
    (dict(N=8388608), -1, "N must be"),
    (dict(rule=4, N=262145), -2, "262144"),
    (dict(), -1, "workspace must be non-null"),
])
def test_refusals(kw, rc, message):
    pkg = _lib()
    a = bwd_args(pkg, **kw)
    assert pkg.lib().dsattn_attn_bwd(ctypes.byref(a), None, 0) == rc
    assert message in pkg.last_error()


def test_small_and_host_workspaces_are_refused():
    pkg = _lib()
    a = bwd_args(pkg)
    need = pkg.dsattn_attn_bwd_workspace_bytes(1, 1, 64)
    host = ctypes.create_string_buffer(2 * need + 256)
    at = ctypes.addressof(host)
    assert pkg.lib().dsattn_attn_bwd(ctypes.byref(a), at, need - 1) == -1
    assert "workspace too small" in pkg.last_error()
    assert pkg.lib().dsattn_attn_bwd(ctypes.byref(a), at, need) == -1
    assert "q must be non-null" in pkg.last_error()
    assert pkg.lib().dsattn_attn_bwd(None, None, 0) == -1


@pytest.mark.parametrize("kw", [dict(B=0), dict(H=0), dict(N=0), dict(N=0, rule=4)])
def test_empty_problems_do_nothing(kw):
    pkg = _lib()
    a = bwd_args(pkg, **kw)
    assert pkg.lib().dsattn_attn_bwd(ctypes.byref(a), None, 0) == 0
    assert pkg.last_error() == ""


def test_workspace_sizes():
    pkg = _lib()
    size = pkg.dsattn_attn_bwd_workspace_bytes
    assert size(0, 1, 64) == size(1, 0, 64) == size(1, 1, 0) == size(-1, 1, 1) == 0
    assert size(1, 1, 1) == 2 * 256 and size(1, 1, 65) == 2 * 512
    assert size(2, 40, 32760) == 2 * 80 * 32768 * 4
    assert size(70000, 1, 1) == 0 and size(1, 1, 1 << 24) == 0


def bias_call(pkg, backward, **kw):
    x = dict(B=1, H=2, n_q=64, n_k=64, d=128, n_buckets=8, scale=0.1)
    if not backward:
        x["k_rows"] = kw.get("n_k", 64)
    x.update(kw)
    L = pkg.lib()
    if backward:
        return L.dsattn_bias_attn_bwd(ctypes.byref(pkg.DsAttnBiasBwdArgs(**x)), None, 0)
    return L.dsattn_bias_attn_fwd(ctypes.byref(pkg.DsAttnBiasArgs(**x)), None, 0)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,rc,message", [
    (dict(B=-1), -1, ">= 0"),
    (dict(n_q=-1), -1, ">= 0"),
    (dict(n_k=-1), -1, ">= 0"),
    (dict(scale=float("inf")), -1, "scale"),
    (dict(scale=1e-38), -1, "1e-30"),
    (dict(d=256), -2, "head dimension"),
    (dict(n_buckets=0), -2, "n_buckets"),
    (dict(n_buckets=513), -2, "n_buckets"),
    (dict(B=65536), -1, "65535"),
    (dict(n_q=8388608), -1, "8388607"),
    (dict(n_k=8388608), -1, "8388607"),
    (dict(B=1000, H=60, n_q=8388607), -1, "too large"),
    (dict(), -1, "workspace must be non-null"),
])
def test_bias_refusals(backward, kw, rc, message):
    pkg = _lib()
    assert bias_call(pkg, backward, **kw) == rc
    assert message in pkg.last_error()


def test_no_batch_lays_nothing_out():
    """Without a batch no pair exists: neither table nor bucket is needed, and nothing of their
    layout by distance is planned -- the number of distances decides both."""
    pkg = _lib()
    size = pkg.lib().dsattn_bias_attn_bwd_workspace_bytes
    none = size(0, 2, 0, 0, 8)
    assert size(0, 2, 5000, 7000, 8) == size(0, 2, 5000, 0, 8) == none
    assert size(1, 2, 5000, 7000, 8) > none + 2 * 12000 * 4


@pytest.mark.parametrize("B", [0, 1])
def test_bias_gradient_heads(B):
    """Heads are a dimension of its launches whatever the batch."""
    pkg = _lib()
    assert bias_call(pkg, True, B=B, H=70000) == -1
    assert "65535" in pkg.last_error()
    assert pkg.lib().dsattn_bias_attn_bwd_workspace_bytes(B, 70000, 64, 64, 8) == 0
    assert pkg.lib().dsattn_bias_attn_bwd_workspace_bytes(B, 65535, 64, 64, 8) > 0


def test_bias_cache_and_empty_problems():
    pkg = _lib()
    assert bias_call(pkg, False, n_k=64, k_rows=63) == -1
    assert "k_rows must be >= n_k" in pkg.last_error()
    for kw in (dict(B=0), dict(H=0), dict(n_q=0)):
        assert bias_call(pkg, False, **kw) == 0
    assert bias_call(pkg, True, H=0) == 0
    assert pkg.lib().dsattn_bias_attn_fwd(None, None, 0) == -1
    assert pkg.lib().dsattn_bias_attn_bwd(None, None, 0) == -1


def test_bias_workspace_sizes():
    pkg = _lib()
    fwd, bwd = pkg.dsattn_bias_attn_workspace_bytes, pkg.dsattn_bias_attn_bwd_workspace_bytes
    assert fwd(0, 2, 5, 5) == fwd(1, 0, 5, 5) == fwd(1, 2, 0, 5) == fwd(-1, 2, 5, 5) == 0
    assert bwd(1, 0, 5, 5, 8) == bwd(1, 2, 5, 5, 0) == bwd(1, 2, 5, 5, 513) == 0
    assert fwd(1, 2, 5, 0) > 0 and bwd(0, 2, 5, 5, 8) > 0
    # few queries: the splits' parts come on top of the layout by distance
    one = fwd(1, 40, 1, 32760)
    assert one > 40 * 32760 * 4 and one < 40 * 32760 * 4 + (64 << 20)
    for shape in ((1, 40, 1, 32760), (2, 3, 100, 5000), (1, 1, 1, 1), (1, 2, 8000000, 3)):
        assert fwd(*shape) % 256 == 0 and bwd(*shape, 32) % 256 == 0


def buckets_by_definition(n_q, n_k, q_first, n_buckets, max_distance, causal):
    """In whole numbers: far distance a has bucket E + k where (a / E)^(P - E) lies between the
    k-th and the next power of max_distance / E."""
    P = n_buckets if causal else n_buckets // 2
    E = max(1, P // 2)

    def f(a):
        if a < E:
            return a
        k = 0
        while k < P - E and a ** (P - E) * E ** (k + 1) >= max_distance ** (k + 1) * E ** (P - E):
            k += 1
        return min(P - 1, E + k)

    out = []
    for e in range(n_q + n_k - 1):
        d = e - (n_q - 1) - q_first
        out.append(f(-d) if d <= 0 else -1 if causal else P + f(d))
    return out


@pytest.mark.parametrize("n_q,n_k,q_first,n_buckets,max_distance,causal", [
    (1, 1, 0, 2, 8, False), (5, 7, 0, 32, 128, False), (400, 300, 0, 32, 128, False),
    (400, 300, 17, 32, 128, True), (1, 700, 699, 16, 512, True), (3, 40, 500, 9, 60, False),
    (300, 300, 0, 121, 60, False), (300, 300, 0, 3, 5, True), (130, 130, 0, 64, 1024, False)])
def test_relative_buckets(n_q, n_k, q_first, n_buckets, max_distance, causal):
    pkg = _lib()
    got = pkg.dsattn_relative_buckets(n_q, n_k, n_buckets, max_distance, q_first=q_first,
                                      causal=causal)
    assert got.tolist() == buckets_by_definition(n_q, n_k, q_first, n_buckets, max_distance, causal)


@pytest.mark.parametrize("args", [(0, 1, 32, 128), (1, 0, 32, 128), (8388608, 1, 32, 128),
                                  (1, 1, 1, 128), (1, 1, 32, 8), (1, 1, 32, -5)])
def test_relative_buckets_refusals(args):
    pkg = _lib()
    with pytest.raises(RuntimeError):
        pkg.dsattn_relative_buckets(*args)
    with pytest.raises(RuntimeError):
        pkg.dsattn_relative_buckets(4, 4, 32, 128, q_first=-1)
    assert pkg.lib().dsattn_relative_buckets(4, 4, 0, 32, 128, 0, None) == -1


@pytest.mark.parametrize("bias,skip", [(False, False), (True, False), (False, True), (True, True)])
def test_reference_against_autograd(bias, skip):
    torch = pytest.importorskip("torch")
    from _grad_ref import Ref

    g = torch.Generator().manual_seed(3)
    B, H, n_q, n_k = 2, 2, 9, 13
    q, k, v, do = (torch.randn(B, H, n, 128, generator=g, dtype=torch.float64)
                   for n in (n_q, n_k, n_k, n_q))
    b = torch.randn(H, n_q, n_k, generator=g, dtype=torch.float64) if bias else None
    s = None
    if skip:
        s = torch.rand(B, H, n_q, n_k, generator=g) < 0.4
        s[..., 0] = False
    leaves = [x.clone().requires_grad_() for x in (q, k, v)] + ([b.clone().requires_grad_()]
                                                                if bias else [])
    z = 128 ** -0.5 * leaves[0] @ leaves[1].transpose(-1, -2)
    if bias:
        z = z + leaves[3]
    if skip:
        z = z.masked_fill(s, float("-inf"))
    o = torch.softmax(z, -1) @ leaves[2]
    o.backward(do)
    ref = Ref(q, k, v, do, bias=b, skip=s)
    assert torch.allclose(ref.o, o, atol=1e-12)
    assert torch.allclose(ref.lse, torch.logsumexp(z, -1), atol=1e-12)
    for x, name in zip(leaves, ("dq", "dk", "dv")):
        assert torch.allclose(getattr(ref, name), x.grad, atol=1e-11)
    if bias:
        assert torch.allclose(ref.ds.sum(0), leaves[3].grad, atol=1e-11)


def test_reference_of_rows_with_nothing():
    torch = pytest.importorskip("torch")
    from _grad_ref import Ref

    g = torch.Generator().manual_seed(4)
    q, k, v, do = (torch.randn(1, 1, 5, 128, generator=g, dtype=torch.float64) for _ in range(4))
    skip = torch.zeros(1, 1, 5, 5, dtype=torch.bool)
    skip[..., 2, :] = True
    ref = Ref(q, k, v, do, skip=skip)
    assert ref.lse[0, 0, 2] == -float("inf") and not ref.o[0, 0, 2].any()
    assert not ref.dq[0, 0, 2].any() and not ref.ds[0, 0, 2].any()
    assert all(torch.isfinite(x).all() for x in (ref.dq, ref.dk, ref.dv))


def test_division_of_work(tmp_path):
    """Every visit of every unit by one workgroup, in every order (a host program)."""
    import shutil
    import subprocess

    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("no g++ or HIP headers")
    exe = str(tmp_path / "split_check")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__",
                    "-isystem", "/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "paper_2606_16317_amd", "csrc"),
                    os.path.join(ROOT, "tests", "c_client", "split_check.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.stdout == "ok\n" and res.returncode == 0, res.stdout


@pytest.mark.parametrize("kind,n_q,n_k", [("both", 3001, 3001), ("causal", 3001, 3001),
                                          ("random", 3001, 1600), ("both", 700, 5000)])
def test_the_table_check_misses_no_block(kind, n_q, n_k):
    """In the GPU test of these cases any one block of 32 keys that is left out of the table's
    gradient, or counted twice, exceeds the bound of a bucket; and so does every part of one that goes
    to the next bucket."""
    torch = pytest.importorskip("torch")
    _lib()
    from _table_case import TableCase

    c = TableCase(kind, n_q, n_k, "cpu")
    closed = c.at < 0
    ds = c.ref.ds[0, :, 0].masked_fill(closed, 0.0)                     # [H, n_k]
    n_b = -(-n_k // 32)
    block = torch.arange(n_k) // 32
    part = torch.zeros(c.H, n_b * c.nb, dtype=torch.float64).scatter_add_(
        1, block[None] * c.nb + c.at.clamp(min=0), ds).view(c.H, n_b, c.nb)
    bound = 1.02 * c.ref.b_dtable.t()[:, None]                          # [H, 1, nb]
    open_ = torch.zeros(c.H, n_b).scatter_add_(1, block.expand(c.H, -1), (~closed).float()) > 0
    seen = (part.abs() > bound).any(-1)
    assert open_.any() and seen[open_].all()
    there = part != 0
    moved = (part.abs() > bound) | (part.abs() > bound.roll(-1, -1))
    assert moved[there].all()
