"""Products with 8-bit weights (onmt_f8_*) against the definition in 64 bits: for every row and block of 128 columns the smallest
power of two that brings the largest entry to 448 or less, entries rounded to the nearest e4m3 value, the product of
what both operands then stand for.

Tolerances, before any run: fp32 results accumulate exact products in fp32, so a sum of K is off by at most K half-steps (2^-24) of the
sum of its products' sizes, and the bias adds half a step of the result. 16-bit results come from an instruction that adds the 128
products of a block at 17 bits or more of the largest: at most 128 x 2^-16 of a block's largest product per block, the
accumulation as above, and half a step of the result's type.
"""

import numpy as np
import pytest
import torch

from paper_1805_11462_amd import ops

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# with p significant bits (24, 8, 11) neighbours in [1, 2) are 2^(1 - p) apart: half a step is up to 2^-p of a value
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
BIG = 1.875 * 2.0 ** 127                   # larger entries, infinities among them, count as this


def round8(x):
    """The values (fp64) that the rows of x stand for, NaN kept."""
    x = np.clip(x.astype(np.float64), -BIG, BIG)
    out = np.zeros_like(x)
    for k in range(0, x.shape[1], 128):
        b = x[:, k:k + 128]
        a = np.max(np.where(np.isnan(b), 0.0, np.abs(b)), axis=1)
        m, ex = np.frexp(a)
        e = np.where(a > 0, np.maximum(ex - 9 + (m > 0.875), -127), 0)[:, None]
        v = np.ldexp(b, -e)
        _, vx = np.frexp(np.maximum(np.abs(v), 2.0 ** -6))
        step = np.ldexp(1.0, vx - 4)
        out[:, k:k + 128] = np.ldexp(np.rint(v / step) * step, e)
    return out


def host(t):
    return t.float().cpu().numpy()


def check(x, w8, bias, out, kind):
    """out against the definition, within the tolerance above."""
    xq, wq = round8(host(x)), round8_cache(w8)
    y = xq @ wq.T
    mag = np.abs(xq) @ np.abs(wq).T
    if bias is not None:
        y = y + host(bias).astype(np.float64)
    K = x.shape[1]
    tol = (K + 1) * 2.0 ** -24 * mag + HALF_STEP[kind] * np.abs(y) + 2.0 ** -24 * np.abs(y)
    if kind != "f32":
        for k in range(0, K, 128):
            top = np.abs(xq[:, k:k + 128]).max(1)[:, None] * np.abs(wq[:, k:k + 128]).max(1)[None, :]
            tol = tol + 128 * 2.0 ** -16 * top
    if kind == "f16":
        tol = tol + 2.0 ** -25
    got = out.double().cpu().numpy()
    bad = np.abs(got - y) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.abs(got - y).max()))


def round8_cache(w8):
    if not hasattr(w8, "ref"):
        w8.ref = round8(w8.source)
    return w8.ref


def weights(w):
    w8 = ops.F8Weights(w)
    w8.source = host(w)
    return w8


def make(M, N, K, kind="f32", seed=0, wkind="f32"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(M, K, generator=g, device="cuda", dtype=torch.float32).to(TYPES[kind])
    w = (torch.randn(N, K, generator=g, device="cuda", dtype=torch.float32) * 0.1).to(TYPES[wkind])
    return x, w, torch.randn(N, generator=g, device="cuda", dtype=torch.float32)


SIZES = [(1, 1, 1), (1, 17, 127), (3, 1000, 64), (5, 300, 128), (16, 64, 129), (17, 333, 500), (33, 4097, 260),
         (64, 50, 65), (65, 129, 1000), (96, 256, 512), (130, 4100, 384), (200, 777, 96), (257, 515, 2050), (300, 64, 4100)]


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_sizes(M, N, K, out):
    print(f"[case] {M} x {K} by {N}, {out}", flush=True)
    x, w, b = make(M, N, K, seed=M + N)
    w8 = weights(w)
    check(x, w8, b, w8.linear(x, b, out_dtype=TYPES[out]), out)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("wkind", ["f32", "bf16", "f16"])
def test_types(kind, wkind):
    for M, N, K in ((7, 130, 200), (150, 300, 513)):
        x, w, b = make(M, N, K, kind, seed=5, wkind=wkind)
        w8 = weights(w)
        for out in TYPES:
            check(x, w8, None, w8.linear(x, out_dtype=TYPES[out]), out)


def test_values_are_the_definitions():
    g = np.random.default_rng(3)
    w = g.standard_normal((37, 700)).astype(np.float32)
    w *= np.exp2(g.integers(-60, 60, w.shape)).astype(np.float32)            # entries far below a block's largest too
    w[0] = 0.0
    w[1, :] = 448.0                              # f = 1.75 exactly
    w[2, :] = np.nextafter(np.float32(448.0), np.float32(1e9))
    w[3, 5] = 3.0e38
    w[4, 600:] = 1e-38
    w[5, :] = 2.0 ** -149
    w[6, ::2] = -0.0
    w[7, 3], w[7, 300] = np.inf, -np.inf
    got = ops.F8Weights(torch.from_numpy(w).cuda()).values().cpu().numpy().astype(np.float64)
    assert np.array_equal(got, round8(w))
    # packing what the values stand for again changes nothing
    again = ops.F8Weights(torch.from_numpy(got.astype(np.float32)).cuda()).values().cpu().numpy()
    assert np.array_equal(again.astype(np.float64), got)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M", [4, 100])
def test_extreme_values(M, out):
    # powers far apart between blocks and rows, zero rows, infinities (the largest finite value), NaN in one row
    x, w, _ = make(M, 200, 400, seed=9)
    x = x * torch.exp2(torch.linspace(-40, 40, M, device="cuda", dtype=torch.float32))[:, None]
    x[:, 128:256] *= 2.0 ** -20
    x[1] = 0
    w[3] = 0
    w8 = weights(w)
    check(x, w8, None, w8.linear(x, out_dtype=TYPES[out]), out)
    x[2, 7] = float("nan")
    y = w8.linear(x, out_dtype=TYPES[out])
    assert y[2, :3].isnan().all() and y[2, 4:].isnan().all()
    assert not y[:2].isnan().any() and not y[3:].isnan().any()
    z = torch.zeros(M, 400, device="cuda", dtype=torch.float32)
    z[0, 0] = float("inf")
    w[:, 0] = 2.0 ** -100
    w8 = weights(w)
    y = w8.linear(z, out_dtype=TYPES[out])
    ref = round8(host(z)) @ round8_cache(w8).T
    assert np.allclose(y.double().cpu().numpy(), ref, rtol=2.0 ** -8, atol=0)


def test_strides_and_odd_addresses():
    for M, N, K in ((6, 77, 131), (150, 301, 259)):
        for kind in ("f32", "bf16"):
            base = torch.randn(M, K + 9, device="cuda", dtype=torch.float32).to(TYPES[kind])
            wbase = torch.randn(N, K + 5, device="cuda", dtype=torch.float32).to(TYPES[kind])
            x, w = base[:, 3:3 + K], wbase[:, 1:1 + K]
            w8 = weights(w)
            for out in ("f32", "bf16"):
                big = torch.full((M, N + 7), 7.0, device="cuda", dtype=TYPES[out])
                y = w8.linear(x, out=big[:, 3:3 + N])
                check(x, w8, None, y, out)
                assert (big[:, :3] == 7).all() and (big[:, 3 + N:] == 7).all()


def test_offsets_past_32_bits():
    M, N, K = 66000, 33000, 40               # 2.2e9 results
    x, w, b = make(M, N, K, "bf16", seed=2)
    w8 = weights(w)
    y = w8.linear(x, b, out_dtype=torch.bfloat16)
    for r in (0, 1, 30000, 65071, 65073, M - 1):
        check(x[r:r + 1], w8, b, y[r:r + 1], "bf16")


def test_other_streams_and_two_calls_at_once():
    x, w, b = make(90, 2000, 500, seed=4)
    w8 = ops.F8Weights(w)
    x2 = x[:7].clone()
    want, want2 = w8.linear(x, b), w8.linear(x2, b)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for st, xx in zip(streams, (x, x2)):
            with torch.cuda.stream(st):
                got.append(w8.linear(xx, b))
        torch.cuda.synchronize()
        assert torch.equal(got[0], want) and torch.equal(got[1], want2)


@pytest.mark.parametrize("M", [3, 200])
def test_captured_and_replayed(M):
    x, w, b = make(M, 1500, 300, seed=6)
    w8 = ops.F8Weights(w)
    w8.linear(x, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = w8.linear(x, b)
    for seed in range(4):
        x.copy_(make(M, 1500, 300, seed=20 + seed)[0])
        graph.replay()
        assert torch.equal(y, w8.linear(x, b))
        torch.cuda.synchronize()


def test_refused_tensors():
    x, w, b = make(4, 100, 64)
    w8 = ops.F8Weights(w)
    for bad in (x.cpu(), x[0], x[:, :63], x.t(), x.double(), x[:, ::2], x.expand(4, 64)[:0], x[:1].expand(4, 64)):
        with pytest.raises(ValueError):
            w8.linear(bad)
    for bad in (b.cpu(), b[:99], b.double(), b.half()):
        with pytest.raises(ValueError):
            w8.linear(x, bad)
    with pytest.raises(ValueError):
        w8.linear(x, out_dtype=torch.float64)
    with pytest.raises(ValueError):
        w8.linear(x, out=torch.empty(4, 99, device="cuda", dtype=torch.float32))
    with pytest.raises(ValueError):
        ops.F8Weights(w.double())
