"""Host-only checks of the sequence operators' C ABI (exports, refusals before anything touches a
GPU) and of the 64-bit references that the GPU tests use (against differences and closed cases)."""
import ctypes as C
import math
import os
import re

import pytest
import torch

import dnnseq_ref as ref
from paper_2110_10802_amd import dnnseq as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096  # an aligned, never dereferenced address


def test_exports_and_constants():
    hdr = open(os.path.join(ROOT, "include", "dnnseq.h")).read()
    declared = set(re.findall(r"\b(dnnseq_[a-z_]+)\s*\(", hdr))
    assert declared == set(S.EXPORTS), declared ^ set(S.EXPORTS)
    lib = S.load()
    for name in declared:
        assert hasattr(lib, name), name
    assert int(re.search(r"#define DNNSEQ_MAX_HEAD_DIM (\d+)", hdr).group(1)) == S.MAX_HEAD_DIM
    assert int(re.search(r"#define DNNSEQ_MAX_NORM_COLS (\d+)", hdr).group(1)) == S.MAX_NORM_COLS
    for name, code in S.ACTIVATIONS.items():
        assert int(re.search(rf"DNNSEQ_ACT_{name.upper()} = (\d+)", hdr).group(1)) == code


def _t(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype)


def _attention(**changes):
    q, k = _t(2, 4, 10, 64), _t(2, 2, 30, 64)
    d = S.attention_desc(q, k, k, q)
    for name, value in changes.items():
        target, names = d, name.split("__")
        for n in names[:-1]:
            target = getattr(target, n)
        setattr(target, names[-1], value)
    return d


@pytest.mark.parametrize("changes,status", [
    (dict(dtype=2), -1), (dict(dtype=-1), -1), (dict(batch=-1), -1), (dict(q_heads=0), -1), (dict(kv_heads=0), -1),
    (dict(q_len=-1), -1), (dict(kv_len=-5), -1), (dict(head_dim=0), -1), (dict(causal=2), -1), (dict(scale=0.0), -1),
    (dict(scale=-1.0), -1), (dict(scale=math.inf), -1), (dict(scale=math.nan), -1), (dict(kv_heads=3), -1),
    (dict(q__token=65), -1), (dict(k__head=-64), -1), (dict(o__token=32), -1), (dict(o__head=0), -1),
    (dict(dk__batch=0), -1), (dict(dv__token=0), -1), (dict(dq__token=56), -1), (dict(dq__batch=64), -1),
    (dict(head_dim=60), -2), (dict(head_dim=136, o__token=136, o__head=1360, o__batch=5440, dq__token=136,
                                   dq__head=1360, dq__batch=5440, dk__token=136, dk__head=4080, dk__batch=8160,
                                   dv__token=136, dv__head=4080, dv__batch=8160), -2),
    (dict(k__token=1 << 22), -2), (dict(v__batch=(1 << 40) + 8), -2),
])
def test_attention_refuses_descriptors(changes, status):
    d = _attention(**changes)
    assert S.attention_backward_scratch_bytes(d) == 0
    with pytest.raises(S.DnnSeqError) as e:
        S.attention_backward(d, P, P, P, P, P, P, P, P, P, P)
    assert e.value.status == status
    if not any(n.startswith("d") and "__" in n for n in changes):
        assert S.attention_forward_scratch_bytes(d) == 0
        with pytest.raises(S.DnnSeqError) as e:
            S.attention_forward(d, P, P, P, P)
        assert e.value.status == status


def test_attention_refuses_pointers():
    d = _attention()
    assert S.attention_forward_scratch_bytes(d) == 0 and S.attention_backward_scratch_bytes(d) > 0
    fwd = dict(q=P, k=P, v=P, o=P)
    for name in fwd:
        for value, status in ((None, -1), (P + 8, -4)):
            with pytest.raises(S.DnnSeqError) as e:
                S.attention_forward(d, **dict(fwd, **{name: value}))
            assert e.value.status == status
    for name in ("lse", "q_lens", "kv_lens", "scratch"):
        with pytest.raises(S.DnnSeqError) as e:
            S.attention_forward(d, **fwd, **{name: P + 4})
        assert e.value.status == -4
    bwd = dict(fwd, dout=P, lse=P, dq=P, dk=P, dv=P, scratch=P)
    for name in bwd:
        for value, status in ((None, -3 if name == "scratch" else -1), (P + 8, -4)):
            with pytest.raises(S.DnnSeqError) as e:
                S.attention_backward(d, **dict(bwd, **{name: value}))
            assert e.value.status == status
    long = S.attention_desc(_t(1, 1, 1, 64), _t(1, 1, 100000, 64), _t(1, 1, 100000, 64), _t(1, 1, 1, 64))
    assert S.attention_forward_scratch_bytes(long) > 0
    with pytest.raises(S.DnnSeqError) as e:
        S.attention_forward(long, P, P, P, P)
    assert e.value.status == -3
    assert S.load().dnnseq_attention_forward(None, P, P, P, None, None, P, None, None, None) == -1


def test_attention_desc_reads_views_and_refuses_shapes():
    qkv = _t(2, 10, 3, 4, 64)
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    d = S.attention_desc(q, k, v, _t(2, 4, 10, 64))
    assert (d.q.batch, d.q.head, d.q.token) == (7680, 64, 768) and (d.o.batch, d.o.head, d.o.token) == (2560, 640, 64)
    assert (d.dk.batch, d.dk.token) == (7680, 768) and abs(d.scale - 0.125) < 1e-9
    for bad in (_t(2, 4, 10, 32), _t(2, 4, 10, 64, dtype=torch.float16), _t(2, 4, 10, 64, dtype=torch.float32),
                _t(2, 4, 64, 10).transpose(2, 3)):
        with pytest.raises(ValueError):
            S.attention_desc(q, bad, v, q)
    # nothing to do: accepted without pointers
    empty = S.attention_desc(_t(0, 4, 10, 64), _t(0, 4, 10, 64), _t(0, 4, 10, 64), _t(0, 4, 10, 64))
    S.attention_forward(empty, None, None, None, None)
    S.attention_backward(empty, None, None, None, None, None, None, None, None, None, None)


def test_linear_refusals():
    def call(d, backward=False, **changes):
        if backward:
            a = dict(dict(x=P, w=P, dy=P, z=P, dx=P, dx_add=None, dw=P, db=P, scratch=P), **changes)
            S.linear_backward(d, **a)
        else:
            a = dict(dict(x=P, w=P, y=P, bias=P, residual=P, z=2 * P, scratch=P), **changes)
            S.linear_forward(d, **a)

    def status(d, **kw):
        with pytest.raises(S.DnnSeqError) as e:
            call(d, **kw)
        return e.value.status

    def desc(**changes):
        d = S.linear_desc(_t(5, 64), _t(32, 64), "gelu")
        for n, v in changes.items():
            setattr(d, n, v)
        return d

    for changes, code in ((dict(dtype=3), -1), (dict(activation=9), -1), (dict(activation=-1), -1), (dict(m=-1), -1),
                          (dict(n=0), -1), (dict(k=0), -1), (dict(ldx=56), -1), (dict(ldw=65), -1), (dict(n=36, ldy=40, ldz=40, ldresidual=40, lddy=40), -2),
                          (dict(k=60), -2), (dict(ldw=1 << 22), -2), (dict(dw_fp32=2), -1)):
        assert status(desc(**changes)) == code, changes
        assert status(desc(**changes), backward=True) == code, changes
        assert S.linear_forward_scratch_bytes(desc(**changes)) == 0
        assert S.linear_backward_scratch_bytes(desc(**changes)) == 0
    for name in ("ldy", "ldresidual", "ldz"):
        assert status(desc(**{name: 24})) == -1 and status(desc(**{name: 36})) == -1
        assert status(desc(**{name: 1 << 23})) == -2
    for name, n in (("lddy", 32), ("ldz", 32), ("lddx", 64), ("lddw", 64)):
        assert status(desc(**{name: n - 8}), backward=True) == -1
    assert status(desc(lddx_add=8), backward=True, dx_add=2 * P) == -1
    assert status(desc(lddx_add=72), backward=True, dx_add=P) == -1      # in place with another pitch
    assert status(desc(ldresidual=40)) == -1
    assert status(desc(), z=P) == -1                                      # z over y
    for name in ("x", "w", "y"):
        assert status(desc(), **{name: None}) == -1
    for name in ("x", "w", "y", "bias", "residual", "z", "scratch"):
        assert status(desc(), **{name: P + 8}) == -4, name
    for name in ("x", "w", "dy", "z"):
        assert status(desc(), backward=True, **{name: None}) == -1
    for name in ("x", "w", "dy", "z", "dx", "dx_add", "dw", "db", "scratch"):
        assert status(desc(), backward=True, **{name: P + 8}) == -4, name
    assert status(desc(), backward=True, scratch=None) == -3
    call(desc(), backward=True, dx=None, dw=None, db=None)               # nothing asked for
    call(desc(m=0), x=None, y=None, z=None)                              # nothing to do
    with pytest.raises(ValueError):
        S.linear_desc(_t(5, 64), _t(32, 64), y=_t(5, 64))
    with pytest.raises(ValueError):
        S.linear_desc(_t(5, 64), _t(32, 64, dtype=torch.float16))
    with pytest.raises(KeyError):
        S.linear_desc(_t(5, 64), _t(32, 64), "tanh")


def test_layernorm_refusals():
    def desc(**changes):
        d = S.layernorm_desc(_t(5, 64))
        for n, v in changes.items():
            setattr(d, n, v)
        return d

    def forward(d, **ch):
        S.layernorm_forward(d, **dict(dict(x=P, gamma=P, beta=P, y=2 * P, mean=P, rstd=P), **ch))

    def backward(d, **ch):
        S.layernorm_backward(d, **dict(dict(x=P, dy=P, gamma=P, mean=P, rstd=P, dx=P, dgamma=P, dbeta=P, scratch=P), **ch))

    def status(f, d, **ch):
        with pytest.raises(S.DnnSeqError) as e:
            f(d, **ch)
        return e.value.status

    for f in (forward, backward):
        for changes, code in ((dict(dtype=5), -1), (dict(rows=-1), -1), (dict(cols=0), -1), (dict(eps=-1.0), -1),
                              (dict(eps=math.nan), -1), (dict(ldx=63), -1),
                              (dict(cols=S.MAX_NORM_COLS + 1, **{n: 1 << 20 for n in ("ldx", "ldy", "lddy", "lddx")}), -2)):
            assert status(f, desc(**changes)) == code, changes
    assert status(forward, desc(ldy=60)) == -1 and status(forward, desc(ldx=72), y=P) == -1
    assert status(backward, desc(lddy=60)) == -1 and status(backward, desc(lddx=60)) == -1
    assert status(backward, desc(lddx_add=60), dx_add=2 * P) == -1 and status(backward, desc(lddx_add=72), dx_add=P) == -1
    for name in ("x", "gamma", "beta", "y", "mean", "rstd"):
        assert status(forward, desc(), **{name: None}) == -1 and status(forward, desc(), **{name: P + 2}) == -4
    for name in ("x", "dy", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta"):
        assert status(backward, desc(), **{name: None}) == -1 and status(backward, desc(), **{name: P + 2}) == -4
    assert status(backward, desc(), scratch=None) == -3
    forward(desc(rows=0), x=None, gamma=None, y=None)
    assert S.layernorm_backward_scratch_bytes(desc(rows=0)) == 0 and S.layernorm_backward_scratch_bytes(desc()) > 0


# ---- the references ----------------------------------------------------------------------------

def _differences(f, t, h=1e-5):
    g = torch.zeros_like(t)
    flat, out = t.view(-1), g.view(-1)
    for i in range(flat.numel()):
        keep = float(flat[i])
        flat[i] = keep + h
        up = f()
        flat[i] = keep - h
        out[i] = (up - f()) / (2 * h)
        flat[i] = keep
    return g


@pytest.mark.parametrize("causal,q_lens,kv_lens", [(False, None, None), (True, None, None), (True, [4, 3], [5, 2])])
def test_attention_reference_gradient_against_differences(causal, q_lens, kv_lens):
    gen = torch.Generator().manual_seed(3)
    q, k, v, do = (torch.randn(s, generator=gen, dtype=torch.float64) for s in
                   ((2, 4, 4, 3), (2, 2, 5, 3), (2, 2, 5, 3), (2, 4, 4, 3)))

    def run():
        return ref.attention(q, k, v, 0.6, causal, q_lens, kv_lens, do, dtype=torch.bfloat16)[0]

    want = run()
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        diff = _differences(lambda: float((run()["o"] * do).sum()), t)
        assert torch.allclose(want[name], diff, atol=1e-8), name
    empty = (want["lse"] == -math.inf)
    assert (want["o"][empty] == 0).all() and (want["dq"][empty] == 0).all()
    if q_lens:
        assert empty.any()


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu", "mish"])
def test_linear_and_layernorm_references_against_differences(act):
    gen = torch.Generator().manual_seed(5)
    ref.U[torch.float64], ref.TINY[torch.float64] = 2.0 ** -8, 0.0
    x, w, dy = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((3, 4), (5, 4), (3, 5)))
    z = ref.linear(x, w, activation=act)[0]["z"]
    want = ref.linear_backward(x, w, dy, z, None, act)[0]
    f = lambda: float((ref.linear(x, w, activation=act)[0]["y"] * dy).sum())  # noqa: E731
    assert torch.allclose(want["dx"], _differences(f, x), atol=1e-8)
    assert torch.allclose(want["dw"], _differences(f, w), atol=1e-8)
    gamma, beta, dx = torch.randn(4, generator=gen, dtype=torch.float64), torch.zeros(4, dtype=torch.float64), dy[:, :4].clone()
    want = ref.layernorm_backward(x, dx, gamma, 1e-3)[0]
    f = lambda: float((ref.layernorm(x, gamma, beta, 1e-3)[0]["y"] * dx).sum())  # noqa: E731
    for name, t in (("dx", x), ("dgamma", gamma), ("dbeta", beta)):
        assert torch.allclose(want[name], _differences(f, t), atol=1e-8), name
    del ref.U[torch.float64], ref.TINY[torch.float64]


def test_tolerances_catch_mistakes():
    """A mistake planted in the reference's result is outside the tolerance: one key too many in a
    causal mask, a head read for its neighbour, a bias left out."""
    gen = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn(1, 2, 40, 64, generator=gen).to(torch.float16) for _ in range(3))
    want, tol = ref.attention(q, k, v, 0.125, True)
    wrong, _ = ref.attention(q[:, :, :-1], k[:, :, :], v, 0.125, True)  # bottom-right aligned: one key more each
    assert ((wrong["o"] - want["o"][:, :, :-1]).abs() > tol["o"][:, :, :-1]).float().mean() > 0.5
    assert ((want["o"][:, 0] - want["o"][:, 1]).abs() > tol["o"][:, 1]).float().mean() > 0.9
    x, w = torch.randn(9, 64, generator=gen).half(), torch.randn(16, 64, generator=gen).half()
    a, tol = ref.linear(x, w, torch.full((16,), 0.25))
    assert ((a["y"] - ref.linear(x, w)[0]["y"]).abs() > tol["y"]).all()


@pytest.mark.parametrize("m,n,k", [(0, 64, 64), (0, 4096, 8), (1, 8, 8), (1, 16384, 8), (7, 8, 16384), (1 << 24, 8, 8),
                                   (65, 2056, 4104), (1 << 20, 4096, 64)])
def test_linear_scratch_of_any_size(m, n, k):
    """Sizes only: a number of bytes that is at least the rounded gradient's, and of its order."""
    d = S.linear_desc(_t(1, k), _t(n, k), "gelu")
    d.m = m
    assert S.linear_forward_scratch_bytes(d) < 1 << 40
    assert 2 * m * n <= S.linear_backward_scratch_bytes(d) < (64 << 20) + 80 * (m * n + m * k + n * k)


def _many(batch, q_heads, kv_heads, q_len, kv_len):
    d = S.attention_desc(_t(1, q_heads, 1, 8), _t(1, kv_heads, 1, 8), _t(1, kv_heads, 1, 8), _t(1, q_heads, 1, 8))
    d.batch, d.q_len, d.kv_len = batch, q_len, kv_len
    for t, heads, length in (("q", q_heads, q_len), ("o", q_heads, q_len), ("dout", q_heads, q_len), ("dq", q_heads, q_len),
                             ("k", kv_heads, kv_len), ("v", kv_heads, kv_len), ("dk", kv_heads, kv_len),
                             ("dv", kv_heads, kv_len)):
        s = getattr(d, t)
        s.token, s.head, s.batch = 8, 8 * max(length, 1), 8 * max(length, 1) * heads
    return d


@pytest.mark.parametrize("sizes,taken", [
    ((1 << 15, 32, 8, 1, 4096), False), ((1 << 15, 32, 1, 1, 4096), True), ((1 << 15, 33, 1, 1, 64), False),
    ((3000, 32, 8, 1, 16384), True), ((1, 1, 1, 1 << 28, 1 << 28), True), ((1, 1, 1, (1 << 28) + 8, 8), False),
    ((1, 2, 1, 1 << 28, 8), False), ((1, 2, 1, 1 << 27, 8), True), ((1 << 10, 1 << 10, 1, 64 * 8, 8), False)])
def test_attention_sizes_fit_a_launch(sizes, taken):
    """Descriptors at both sides of the limits: taken ones ask for scratch or a pointer, others are refused."""
    d = _many(*sizes)
    with pytest.raises(S.DnnSeqError) as e:
        S.attention_backward(d, None, None, None, None, None, None, None, None, None, None)
    assert e.value.status == (-1 if taken else -2)
    assert (S.attention_backward_scratch_bytes(d) > 0) == taken
