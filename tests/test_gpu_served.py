"""The served layer on any number of rows and its form for experts (kronq_online_linear,
kronq_online_grouped) through the C ABI against the float64 oracle.

Tolerances (relative Frobenius). A bf16 result is rounded once, at most 2^-8 of each value; its
activations and weights are rounded to fp16 (2^-11 of each factor), and the errors of the terms of
a sum are independent, so that they stay at 2^-11 of the result each, taken twice for sums that
cancel: 2^-8 + 2 * 2 * 2^-11. A fp32 result has activations of 22 bits (2^-22 of each term) and
fp32 sums of at most a few hundred roundings of 2^-24 that add up as their square root, below
16 * 2^-24 = 4 * 2^-22: 8 * 2^-22 with the same factor for cancellation. Up to four rows of one
layer have 30-bit activations and the same sums.
"""
import numpy as np
import pytest
import torch

import oracle as O
import synth
from gpu_util import DEV, note, rel_frob, to_np
from paper_2607_07964_amd import kronq as K

pytestmark = pytest.mark.gpu
TOL = {torch.bfloat16: 2.0 ** -8 + 4 * 2.0 ** -11, torch.float32: 8 * 2.0 ** -22}
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    K.load()
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


class Layer:
    """Seeded codes, scales, zeros and factors of ``experts`` layers, and the oracle's result."""

    def __init__(self, d_out, d_in, bits, group, flags, experts=1, seed=0, bias=True):
        r = np.random.default_rng(seed + d_out + 3 * d_in + bits)
        self.d_out, self.d_in, self.bits, self.group, self.flags = d_out, d_in, bits, group, flags
        ng = d_in // group
        self.codes = r.integers(0, 2 ** bits, size=(experts, d_out, d_in)).astype(np.uint8)
        self.scales = (np.exp(0.3 * r.standard_normal((experts, d_out, ng))) * 0.01).astype(np.float32)
        self.zeros = r.integers(0, 2 ** bits, size=(experts, d_out, ng)).astype(np.float32)
        sign = lambda d: np.where(r.random((experts, d)) < 0.5, -1.0, 1.0)  # noqa: E731
        self.mul_in = (np.exp(0.2 * r.standard_normal((experts, d_in))) * sign(d_in)).astype(np.float32)
        self.mul_out = (np.exp(0.2 * r.standard_normal((experts, d_out))) * sign(d_out)).astype(np.float32)
        self.bias = r.standard_normal((experts, d_out)).astype(np.float32) if bias else None
        self.q28 = {}
        for side, d, bit in (("in", d_in, K.ROT_IN), ("out", d_out, K.ROT_OUT)):
            turn = flags & bit and d % 28 == 0
            self.q28[side] = np.stack([np.linalg.qr(r.standard_normal((28, 28)))[0]
                                       for _ in range(experts)]).astype(np.float32) if turn else None
        self.device()

    def device(self):
        dev = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
        self.packed = K.kronq_pack_codes(dev(self.codes.reshape(-1, self.d_in)), self.bits)
        self.args = [self.packed, dev(self.scales.reshape(-1, self.scales.shape[-1])),
                     dev(self.zeros.reshape(-1, self.zeros.shape[-1])), self.bits, self.group,
                     self.d_in]
        self.factors = [dev(self.mul_in), dev(self.mul_out), dev(self.q28["in"]),
                        dev(self.q28["out"])]
        self.bias_d = dev(self.bias)

    def one(self):
        """Arguments of a single layer's call."""
        return self.args + [None if t is None else t[0] for t in self.factors]

    def dense(self, side, e):
        d = self.d_in if side == "in" else self.d_out
        if not self.flags & (K.ROT_IN if side == "in" else K.ROT_OUT):
            return np.eye(d)
        q = self.q28[side]
        if q is None:
            return O.hadamard(d) / np.sqrt(d)
        q = q[e].astype(np.float64)
        m = d // 28
        return np.kron(q if side == "in" else q.T, O.hadamard(m) / np.sqrt(m))

    def ref(self, x, act="none", residual=None, e=0):
        w = O.dequantize(self.codes[e], self.scales[e].astype(np.float64),
                         self.zeros[e].astype(np.float64), self.group)
        return O.served_linear(w, self.mul_in[e].astype(np.float64),
                               self.mul_out[e].astype(np.float64), self.dense("in", e),
                               self.dense("out", e), x,
                               None if self.bias is None else self.bias[e].astype(np.float64), act,
                               residual)


def rows_of(n, d, dtype, seed=1):
    return torch.randn(n, d, generator=torch.Generator().manual_seed(seed)).to(dtype)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


BOTH, IN, OUT = K.ROT_IN | K.ROT_OUT, K.ROT_IN, K.ROT_OUT


@pytest.mark.parametrize("rows", [1, 2, 4, 5, 31, 32, 33, 64, 65, 100, 129, 257, 1030])
@pytest.mark.parametrize("bits", [2, 3, 4, 8])
def test_linear_rows_and_widths(rows, bits):
    la = Layer(160 if bits == 3 else 256, 512, bits, 128, BOTH if bits != 3 else IN)
    x = rows_of(rows, 512, BF16)
    note(f"linear rows={rows} bits={bits}")
    y = K.kronq_online_linear(*la.one(), x.to(DEV), bias=la.bias_d[0], flags=la.flags)
    y32 = K.kronq_online_linear(*la.one(), x.to(DEV), bias=la.bias_d[0], flags=la.flags,
                                out_dtype=FP32)
    torch.cuda.synchronize()
    ref = la.ref(f64(x))
    assert y.dtype == BF16 and rel_frob(f64(y), ref) < TOL[BF16]
    assert y32.dtype == FP32 and rel_frob(f64(y32), ref) < TOL[FP32]


@pytest.mark.parametrize("d_out,d_in,bits,group,flags,rows,xdt,ydt,act", [
    (448, 896, 4, 128, BOTH, 40, BF16, BF16, "silu"),      # 28 * 16 and 28 * 32
    (896, 3584, 2, 3584, BOTH, 70, FP32, FP32, "gelu"),
    (1792, 128, 8, 128, OUT, 300, BF16, FP32, "relu"),
    (2, 256, 4, 256, BOTH, 9, FP32, BF16, "none"),
    (1, 128, 3, 128, 0, 7, BF16, BF16, "none"),
    (257, 640, 2, 128, 0, 130, FP32, BF16, "gelu"),        # odd sizes, no transform
    (257, 640, 3, 640, 0, 33, BF16, FP32, "silu"),
    (1001, 2176, 8, 128, 0, 90, BF16, BF16, "relu"),
    (64, 16384, 4, 128, BOTH, 6, BF16, FP32, "none"),
    (64, 28672, 2, 128, BOTH, 3, BF16, BF16, "none"),
    (128, 14336, 3, 128, IN, 66, BF16, BF16, "none"),
    (16384, 128, 4, 128, BOTH, 35, BF16, BF16, "none"),
    (28672, 128, 4, 128, OUT, 5, BF16, BF16, "silu"),
    (4096, 4096, 4, 128, BOTH, 70, BF16, BF16, "none"),
])
def test_linear_shapes(d_out, d_in, bits, group, flags, rows, xdt, ydt, act):
    la = Layer(d_out, d_in, bits, group, flags)
    x = rows_of(rows, d_in, xdt)
    res = rows_of(rows, d_out, ydt, seed=2)
    note(f"linear {d_out}x{d_in} bits={bits} group={group} flags={flags} rows={rows} {ydt} {act}")
    y = K.kronq_online_linear(*la.one(), x.to(DEV), bias=la.bias_d[0], act=act,
                              residual=res.to(DEV), flags=flags, out_dtype=ydt)
    torch.cuda.synchronize()
    assert rel_frob(f64(y), la.ref(f64(x), act, f64(res))) < TOL[ydt]


@pytest.mark.parametrize("rows", [3, 50, 200])
@pytest.mark.parametrize("ydt", [BF16, FP32])
def test_linear_strides_in_place_and_canaries(rows, ydt):
    """x and y inside wider buffers of odd strides, the residual being y itself; nothing else of
    the buffers changes."""
    la = Layer(200, 256, 4, 128, IN)
    xw = rows_of(rows, 256 + 24, BF16)
    yw = rows_of(rows + 2, 231, ydt, seed=3).to(DEV)
    before = yw.clone()
    y = yw[1:rows + 1, 7:207]
    note(f"linear strides rows={rows} {ydt}")
    K.kronq_online_linear(*la.one(), xw.to(DEV)[:, 8:264], y=y, residual=y, bias=la.bias_d[0],
                          act="silu", flags=IN)
    torch.cuda.synchronize()
    ref = la.ref(f64(xw[:, 8:264]), "silu", f64(before[1:rows + 1, 7:207]))
    assert rel_frob(f64(y), ref) < TOL[ydt]
    yw[1:rows + 1, 7:207] = before[1:rows + 1, 7:207]
    assert torch.equal(yw, before)


def test_linear_repeats_bit_for_bit_and_rows_are_independent():
    """No atomics: two calls agree; a row with NaN, infinity or zeros leaves the others alone."""
    la = Layer(256, 512, 4, 128, BOTH)
    x = rows_of(150, 512, BF16).to(DEV)
    note("linear repeats, odd rows")
    a = K.kronq_online_linear(*la.one(), x, flags=BOTH)
    b = K.kronq_online_linear(*la.one(), x, flags=BOTH)
    bad = x.clone()
    bad[3, 5], bad[40, 0], bad[77] = float("nan"), float("inf"), 0.0
    c = K.kronq_online_linear(*la.one(), bad, flags=BOTH)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    keep = torch.ones(150, dtype=torch.bool)
    keep[[3, 40, 77]] = False
    assert torch.equal(a[keep.to(DEV)], c[keep.to(DEV)])
    assert not torch.isfinite(c[3].float()).any() and not torch.isfinite(c[40].float()).any()
    assert torch.equal(c[77].float(), torch.zeros(256, device=DEV))


@pytest.mark.parametrize("size", [1e-24, 1e-6, 1e20])
@pytest.mark.parametrize("rows", [2, 20, 100])
def test_linear_ranges_of_activations_and_scales(size, rows):
    """Activations and scales far from 1 (fp16 has neither range), rows of W and x of different
    sizes side by side."""
    la = Layer(256, 256, 4, 128, 0, bias=False)
    la.scales *= np.exp2(np.arange(256) % 40 - 20.0)[None, :, None].astype(np.float32)
    la.device()
    x = rows_of(rows, 256, FP32) * size
    x *= torch.exp2(torch.arange(rows) % 16 - 8.0)[:, None]
    note(f"linear ranges size={size} rows={rows}")
    y = K.kronq_online_linear(*la.one(), x.to(DEV), flags=0, out_dtype=BF16)
    y32 = K.kronq_online_linear(*la.one(), x.to(DEV), flags=0)
    torch.cuda.synchronize()
    ref = la.ref(f64(x))
    unit = np.abs(la.scales[0]).max(1)[None, :] * np.abs(f64(x)).max(1)[:, None]
    assert rel_frob(f64(y) / unit, ref / unit) < TOL[BF16]
    assert rel_frob(f64(y32) / unit, ref / unit) < TOL[FP32]


def test_linear_zeros_outside_the_codes():
    la = Layer(96, 256, 4, 128, 0)
    la.zeros = (la.zeros * 100 - 1000).astype(np.float32)  # -1000 .. 500
    la.device()
    for rows in (3, 40, 200):
        x = rows_of(rows, 256, BF16) + 0.5
        note(f"linear zeros far outside rows={rows}")
        y = K.kronq_online_linear(*la.one(), x.to(DEV), bias=la.bias_d[0], flags=0)
        torch.cuda.synchronize()
        assert rel_frob(f64(y), la.ref(f64(x))) < TOL[BF16]


def test_linear_without_multipliers_and_empty():
    la = Layer(128, 256, 4, 128, BOTH, bias=False)
    la.mul_in[:], la.mul_out[:] = 1, 1
    x = rows_of(9, 256, BF16)
    note("linear without multipliers")
    y = K.kronq_online_linear(*la.args, None, None, None, None, x.to(DEV), flags=BOTH)
    none = K.kronq_online_linear(*la.args, None, None, None, None, x[:0].to(DEV), flags=BOTH)
    torch.cuda.synchronize()
    assert rel_frob(f64(y), la.ref(f64(x))) < TOL[BF16]
    assert none.shape == (0, 128)


def test_linear_agrees_with_the_matvec():
    """One to four rows are kronq_online_matvec's product, and its fp32 result is reproduced."""
    la = Layer(448, 512, 3, 128, BOTH, bias=False)
    for rows in (1, 4):
        x = rows_of(rows, 512, BF16).to(DEV)
        note(f"linear against the matvec rows={rows}")
        a = K.kronq_online_matvec(*la.one(), x, flags=BOTH)
        b = K.kronq_online_linear(*la.one(), x, flags=BOTH, out_dtype=FP32)
        torch.cuda.synchronize()
        assert rel_frob(to_np(b), to_np(a)) < 8 * 2.0 ** -24  # the output transform's sums alone


# ---------------------------------------------------------------------------------------- experts
def grouped_ref(la, x, offsets, y0, act, residual):
    ref = y0.copy()
    for e in range(len(offsets) - 1):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            ref[a:b] = la.ref(x[a:b], act, None if residual is None else residual[a:b], e)
    return ref


@pytest.mark.parametrize("counts,first,pad", [
    ([1], 0, 0), ([0, 1, 0], 0, 0), ([3, 0, 5, 1, 0, 7], 0, 0), ([0, 0, 40], 2, 3),
    ([32, 32, 32], 0, 0), ([31, 1, 33, 64, 127], 0, 5), ([1] * 70, 0, 1), ([300, 0, 2, 150], 1, 0),
    ([0, 0, 0], 0, 4), ([200, 200, 200], 0, 0), ([0] * 299 + [6], 0, 0),
])
@pytest.mark.parametrize("ydt", [BF16, FP32])
def test_grouped_counts(counts, first, pad, ydt):
    """Ragged, empty, misaligned groups; rows of no expert keep their contents."""
    la = Layer(96, 256, 4, 128, IN, experts=len(counts))
    offsets = first + np.cumsum([0] + counts)
    n = int(offsets[-1]) + pad
    x, y0 = rows_of(n, 256, BF16), rows_of(n, 96, ydt, seed=4)
    res = rows_of(n, 96, ydt, seed=5)
    note(f"grouped counts={counts[:8]} first={first} pad={pad} {ydt}")
    y = y0.to(DEV)
    K.kronq_online_grouped(*la.args, *la.factors, x.to(DEV),
                           torch.tensor(offsets, dtype=torch.int32, device=DEV), y,
                           bias=la.bias_d, act="silu", residual=res.to(DEV), flags=IN)
    torch.cuda.synchronize()
    outside = np.ones(n, dtype=bool)
    outside[first:offsets[-1]] = False
    assert np.array_equal(f64(y)[outside], f64(y0)[outside])
    ref = grouped_ref(la, f64(x), offsets, f64(y0), "silu", f64(res))
    assert rel_frob(f64(y), ref) < TOL[ydt]


@pytest.mark.parametrize("d_out,d_in,bits,group,flags,xdt,ydt", [
    (448, 896, 2, 128, BOTH, BF16, BF16), (256, 512, 3, 512, BOTH, FP32, FP32),
    (101, 384, 8, 128, 0, BF16, BF16), (1792, 256, 4, 256, OUT, FP32, BF16),
])
def test_grouped_shapes(d_out, d_in, bits, group, flags, xdt, ydt):
    counts = [5, 0, 90, 33, 2, 70]
    la = Layer(d_out, d_in, bits, group, flags, experts=6)
    offsets = np.cumsum([0] + counts)
    x = rows_of(200, d_in, xdt)
    note(f"grouped {d_out}x{d_in} bits={bits} flags={flags} {ydt}")
    y = K.kronq_online_grouped(*la.args, *la.factors, x.to(DEV),
                               torch.tensor(offsets, dtype=torch.int32, device=DEV),
                               bias=la.bias_d, flags=flags, out_dtype=ydt)
    torch.cuda.synchronize()
    ref = grouped_ref(la, f64(x), offsets, np.zeros((200, d_out)), "none", None)
    assert rel_frob(f64(y), ref) < TOL[ydt]


@pytest.mark.parametrize("offsets", [[0, 50, 20, 60], [-5, 10, 2 ** 30, 60], [70, 70, 0, 0],
                                     [60, 0, 60, 0], [-9, -8, -7, -6]])
def test_grouped_offsets_that_are_not_ascending(offsets):
    """Such offsets reach no memory outside the rows."""
    la = Layer(96, 256, 4, 128, IN, experts=3)
    yw = rows_of(62, 96, BF16, seed=6).to(DEV)
    before = yw.clone()
    x = rows_of(60, 256, BF16).to(DEV)
    note(f"grouped offsets {offsets}")
    K.kronq_online_grouped(*la.args, *la.factors, x,
                           torch.tensor(offsets, dtype=torch.int32, device=DEV), yw[1:61],
                           bias=la.bias_d, flags=IN)
    torch.cuda.synchronize()
    assert torch.equal(yw[0], before[0]) and torch.equal(yw[61], before[61])


# ------------------------------------------------------------------------------- streams and graphs
def test_linear_and_grouped_on_another_stream():
    la = Layer(256, 512, 4, 128, BOTH, experts=2)
    offsets = torch.tensor([0, 30, 90], dtype=torch.int32, device=DEV)
    x = rows_of(90, 512, BF16).to(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    note("served layers on another stream")
    with torch.cuda.stream(s):
        y = K.kronq_online_grouped(*la.args, *la.factors, x, offsets, flags=BOTH)
    torch.cuda.current_stream().wait_stream(s)
    want = K.kronq_online_grouped(*la.args, *la.factors, x, offsets, flags=BOTH)
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_captured_calls_follow_their_inputs():
    """A linear and a grouped call captured into one graph; replays with new activations and new
    offsets, eager work in between, equal the eager results."""
    la = Layer(256, 512, 4, 128, BOTH, experts=4)
    x = rows_of(130, 512, BF16).to(DEV)
    offsets = torch.tensor([0, 10, 60, 60, 130], dtype=torch.int32, device=DEV)
    y1 = torch.zeros(130, 256, dtype=BF16, device=DEV)
    y2 = torch.zeros(130, 256, dtype=BF16, device=DEV)
    one = Layer(256, 512, 4, 128, BOTH)
    ws1 = torch.empty(K.kronq_workspace_bytes(K.OP_LINEAR, 256, 512, 130), dtype=torch.uint8,
                      device=DEV)
    ws2 = torch.empty(K.load().kronq_grouped_workspace_bytes(256, 512, 130, 4), dtype=torch.uint8,
                      device=DEV)

    def calls(a, b):
        K.kronq_online_linear(*one.one(), x, y=a, flags=BOTH, ws=ws1)
        K.kronq_online_grouped(*la.args, *la.factors, x, offsets, b, flags=BOTH, ws=ws2)

    note("captured served layers")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls(y1, y2)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls(y1, y2)
    for i, off in enumerate(([0, 10, 60, 60, 130], [0, 0, 1, 129, 129], [5, 40, 80, 120, 130])):
        x.copy_(rows_of(130, 512, BF16, seed=20 + i))
        offsets.copy_(torch.tensor(off, dtype=torch.int32))
        y1.zero_(), y2.zero_()
        g.replay()
        torch.cuda.synchronize()
        r1, r2 = y1.clone(), y2.clone()
        y1.zero_(), y2.zero_()
        calls(y1, y2)
        torch.cuda.synchronize()
        assert torch.equal(r1, y1) and torch.equal(r2, y2)
