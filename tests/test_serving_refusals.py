"""Arguments that the serving entry points refuse, before anything is enqueued (CPU: no call here
reaches the device), and the pins of their oracle functions."""
import ctypes

import numpy as np
import pytest
import torch

import oracle as O
from paper_2607_07964_amd import kronq as K

NUL = ctypes.c_void_p(0)
FAKE = ctypes.c_void_p(1 << 20)  # never dereferenced: checks fail first
ODD = ctypes.c_void_p((1 << 20) + 2)
BIG = 1 << 40

LINEAR = dict(packed=FAKE, ldp=32, scales=FAKE, zeros=FAKE, ldsz=2, bits=4, group=128, d_out=64,
              d_in=256, mul_in=FAKE, mul_out=FAKE, q28_in=NUL, q28_out=NUL, flags=0, x=FAKE,
              x_dtype=1, ldx=256, n_rows=9, bias=NUL, act=0, residual=NUL, ldr=0, y=FAKE,
              y_dtype=1, ldy=64, ws=FAKE, ws_bytes=BIG, stream=NUL)


def linear(grouped=None, **change):
    a = {**LINEAR, **change}
    args = list(a.values())
    lib = K.load()
    if grouped is None:
        rc = lib.kronq_online_linear(*args)
    else:
        at = list(a).index("bias")
        rc = lib.kronq_online_grouped(*args[:at], *grouped, *args[at:])
    return rc, lib.kronq_last_error().decode()


@pytest.mark.parametrize("change,code,word", [
    (dict(flags=1024), -1, "flag"), (dict(bits=5), -6, "bits"), (dict(act=9), -1, "activation"),
    (dict(d_in=0), -1, "sizes"), (dict(n_rows=-1), -1, "sizes"), (dict(group=64), -2, "group"),
    (dict(group=384), -2, "group"), (dict(d_in=65536, ldp=8192, ldsz=512, ldx=65536), -6, "LDS"),
    (dict(packed=NUL), -1, "packed"), (dict(ldp=28), -1, "packed"), (dict(ldp=34), -1, "packed"),
    (dict(scales=NUL), -1, "scales"), (dict(ldsz=1), -1, "scales"), (dict(mul_in=ODD), -1, "mul_in"),
    (dict(x_dtype=7), -1, "KRONQ_BF16"), (dict(y_dtype=0), -1, "KRONQ_BF16"),
    (dict(flags=8, d_out=96, ldy=96), -6, "96"), (dict(flags=8, d_out=112, ldy=112), -1, "28"),
    (dict(x=NUL), -1, "x must"), (dict(x=ODD), -1, "x must"), (dict(ldx=252), -1, "x must"),
    (dict(ldx=260), -1, "x must"), (dict(y=NUL), -1, "y is"), (dict(ldy=63), -1, "y is"),
    (dict(y_dtype=2, y=ODD), -1, "y is"), (dict(residual=FAKE, ldr=10), -1, "residual"),
    (dict(ws_bytes=16), -5, "workspace"), (dict(ws=NUL), -1, "workspace"),
])
def test_linear_refuses(change, code, word):
    for grouped in (None, (FAKE, 1)):
        rc, msg = linear(grouped, **change)
        assert rc == code and word in msg, (rc, msg)


def test_grouped_refuses():
    assert linear((NUL, 2))[0] == -1
    assert linear((ODD, 2), ws_bytes=BIG)[0] == -1  # offsets misaligned
    assert linear((FAKE, 0))[0] == -6 and linear((FAKE, 5000))[0] == -6
    assert linear((FAKE, 2), ws_bytes=16)[0] == -5


def test_no_rows_do_nothing():
    assert linear(n_rows=0, x=NUL, y=NUL, ws=NUL, ws_bytes=0)[0] == 0
    assert linear((FAKE, 3), n_rows=0, x=NUL, y=NUL, ws=NUL, ws_bytes=0)[0] == 0


def test_workspace_sizes():
    w = K.kronq_workspace_bytes
    assert w(K.OP_LINEAR, 64, 256, 9) >= 2 * 32 * 256 * 2 + 9 * 64 * 4
    assert w(K.OP_LINEAR, 64, 256, 0) == 0 and w(K.OP_LINEAR, -1, 256, 5) == 0
    assert w(K.OP_ATTENTION, 8, 128, 3) >= 8 * 3 * 130 * 4 and w(K.OP_ATTENTION, 8, 128, 0) == 0
    g = K.load().kronq_grouped_workspace_bytes
    assert g(64, 256, 9, 4) >= w(K.OP_LINEAR, 64, 256, 9) // 2 and g(64, 256, 9, 0) == 0


APPEND = dict(k=FAKE, v=FAKE, dtype=1, ldk=256, ldv=256, n_tokens=3, n_kv=2, dim=128, slots=FAKE,
              codes=FAKE, params=FAKE, n_pages=4, page=16, rotate=1, k_hat=NUL, v_hat=NUL,
              stream=NUL)


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=5), -1, "dtype"), (dict(n_tokens=-1), -1, "n_tokens"), (dict(dim=96), -6, "dim"),
    (dict(page=8), -6, "page"), (dict(page=48), -6, "page"), (dict(n_kv=0), -1, "n_kv"),
    (dict(n_pages=0), -1, "n_pages"), (dict(codes=NUL), -1, "codes"), (dict(params=ODD), -1, "codes"),
    (dict(k=NUL), -1, "k and v"), (dict(v=ODD), -1, "k and v"), (dict(ldk=257), -1, "k and v"),
    (dict(ldv=128), -1, "ldk and ldv"), (dict(slots=NUL), -1, "slots"), (dict(slots=ODD), -1, "slots"),
    (dict(k_hat=ODD), -1, "k_hat"),
])
def test_append_refuses(change, code, word):
    lib = K.load()
    rc = lib.kronq_cache_append(*{**APPEND, **change}.values())
    msg = lib.kronq_last_error().decode()
    assert rc == code and word in msg, (rc, msg)


ATTEND = dict(q=FAKE, ldq=1024, n_tokens=4, n_heads=8, n_kv=2, dim=128, codes=FAKE, params=FAKE,
              n_pages=4, page=16, table=FAKE, ldt=3, table_pages=3, lengths=FAKE, n_seqs=4,
              starts=NUL, max_new=1, scale=0.1, rotate=1, out=FAKE, ldo=1024, ws=FAKE, ws_bytes=BIG,
              stream=NUL)


@pytest.mark.parametrize("change,code,word", [
    (dict(dim=100), -6, "dim"), (dict(page=20), -6, "page"), (dict(n_heads=7), -2, "n_heads"),
    (dict(n_heads=0), -2, "n_heads"), (dict(n_tokens=-1), -1, "n_tokens"),
    (dict(n_seqs=70000), -6, "n_seqs"), (dict(q=NUL), -1, "q must"), (dict(q=ODD), -1, "q must"),
    (dict(ldq=1020), -1, "q must"), (dict(ldq=512), -1, "q must"), (dict(out=NUL), -1, "out"),
    (dict(ldo=1000), -1, "out"), (dict(table=NUL), -1, "table"), (dict(table_pages=0), -1, "table"),
    (dict(ldt=2), -1, "table"), (dict(lengths=NUL), -1, "lengths"), (dict(starts=ODD), -1, "lengths"),
    (dict(n_seqs=3), -2, "starts"), (dict(max_new=0), -1, "max_new"), (dict(max_new=5), -1, "max_new"),
    (dict(ws_bytes=64), -5, "workspace"),
])
def test_attention_refuses(change, code, word):
    lib = K.load()
    rc = lib.kronq_cache_attention(*{**ATTEND, **change}.values())
    msg = lib.kronq_last_error().decode()
    assert rc == code and word in msg, (rc, msg)


def test_binding_refuses_host_tensors():
    t = torch.zeros(4, 32, dtype=torch.int32)
    f = torch.zeros(4, 2)
    with pytest.raises(ValueError, match="device"):
        K.kronq_online_linear(t, f, f, 4, 128, 256, None, None, None, None, torch.zeros(2, 256))
    with pytest.raises(ValueError, match="device"):
        K.kronq_cache_append(torch.zeros(1, 1, 64), torch.zeros(1, 1, 64),
                             torch.zeros(1, dtype=torch.int64), *K.kronq_cache_empty(1, 1, 64, 16, "cpu"))
    with pytest.raises(ValueError, match="int32"):
        K.kronq_online_grouped(t, f, f, 4, 128, 256, None, None, None, None, torch.zeros(2, 256),
                               torch.zeros(3, dtype=torch.int64))


# ------------------------------------------------------------------------------------ oracle's pins
def test_served_linear_is_the_online_matvec():
    r = np.random.default_rng(1)
    W, sx, sg = r.standard_normal((16, 32)), np.exp(r.standard_normal(32)), np.exp(r.standard_normal(16))
    si, so = np.where(r.random(32) < 0.5, -1.0, 1.0), np.where(r.random(16) < 0.5, -1.0, 1.0)
    V, U = O.rht_matrix(32, si), O.rht_matrix(16, so)
    x = r.standard_normal((5, 32))
    H = lambda d: O.hadamard(d) / np.sqrt(d)  # noqa: E731
    a = O.served_linear(W, si / sx, so / sg, H(32), H(16), x)
    np.testing.assert_allclose(a, O.online_matvec(W, sx, sg, V, U, x.T).T, rtol=1e-12)
    b = O.served_linear(W, si / sx, so / sg, H(32), H(16), x, bias=np.ones(16), act="silu",
                        residual=x[:, :16])
    z = a + 1
    np.testing.assert_allclose(b, z / (1 + np.exp(-z)) + x[:, :16], rtol=1e-12)


def test_gelu_by_its_integral():
    z = np.array([[-3.0, -0.5, 0.0, 0.7, 2.0]])
    one = np.eye(5)
    got = O.served_linear(one, np.ones(5), np.ones(5), one, one, z, act="gelu")[0]
    for v, g in zip(z[0], got):
        t = np.linspace(-12, v, 200001)
        pdf = np.exp(-t * t / 2) / np.sqrt(2 * np.pi)
        assert abs(g - v * np.sum((pdf[1:] + pdf[:-1]) / 2 * np.diff(t))) < 1e-8


def test_round_up_bf16_is_the_next_pattern():
    r = np.random.default_rng(2)
    v = np.exp2(r.uniform(-90, 90, 200))
    up = O.round_up_bf16(v)
    bits = up.astype(np.float32).view(np.uint32)
    assert np.all(bits & 0xFFFF == 0) and np.all(up >= v)
    below = (bits - 0x10000).view(np.float32).astype(np.float64)
    assert np.all(below < v)
    assert np.all(O.round_up_bf16(up) == up)


def test_cache_grid_is_the_nearest_point():
    r = np.random.default_rng(3)
    v = r.standard_normal((6, 64))
    codes, scale, zero, held = O.cache_grid(v, False)
    assert codes.min() >= 0 and codes.max() <= 15
    for i in range(6):
        points = scale[i] * (np.arange(16) - zero[i])
        best = np.abs(v[i][:, None] - points).min(1)
        np.testing.assert_allclose(np.abs(v[i] - held[i]), best, atol=1e-12)
    # a turned row is the row's coordinates in the Hadamard basis, and keeps its length
    h = O.hadamard(64) / 8
    assert np.array_equal(O.cache_grid(v @ h, False)[0], O.cache_grid(v, True)[0])
    # by hand: 0 .. 15 has scale 1 and zero 0; -15 .. 0 has zero 15; halves go to even
    c, s, z, _ = O.cache_grid(np.arange(16.0)[None], False)
    assert s[0] == 1 and z[0] == 0 and np.array_equal(c[0], np.arange(16))
    c, s, z, _ = O.cache_grid(-np.arange(16.0)[None], False)
    assert s[0] == 1 and z[0] == 15 and np.array_equal(c[0], 15 - np.arange(16))
    assert list(O.cache_grid(np.array([[0.0, 15.0, 0.5, 1.5, 2.5]]), False)[0][0]) == [0, 15, 0, 2, 2]


@pytest.mark.parametrize("part", [0, 1])
def test_cache_words_layout(part):
    r = np.random.default_rng(4)
    codes = r.integers(0, 16, (8, 64))
    w = O.cache_words(codes, part)
    for t in range(8):
        for d in range(64):
            at = t * 8 + d // 8 if part == 0 else (t // 4 * 8 + d // 8) * 4 + t % 4
            assert (int(w[at]) >> (4 * (d % 8))) & 15 == codes[t, d]


def test_causal_attention_by_hand():
    k = np.array([[[1.0, 0.0]], [[0.0, 1.0]], [[1.0, 1.0]]])
    v = np.array([[[1.0, 2.0]], [[3.0, 4.0]], [[5.0, 6.0]]])
    q = np.array([[[0.0, 0.0]], [[np.log(2.0), 0.0]]])
    o = O.causal_attention(q, k, v, 1.0)
    np.testing.assert_allclose(o[0, 0], [2.0, 3.0])  # the mean of the first two
    np.testing.assert_allclose(o[1, 0], (2 * v[0, 0] + v[1, 0] + 2 * v[2, 0]) / 5)
    # more queries than tokens: the first see nothing
    assert np.all(O.causal_attention(np.ones((4, 1, 2)), k, v, 1.0)[0] == 0)
    # shared heads
    o2 = O.causal_attention(np.repeat(q, 2, 1), k, v, 1.0)
    np.testing.assert_allclose(o2[:, 0], o2[:, 1])


@pytest.mark.parametrize("change", [dict(ldp=(1 << 20) + 4), dict(ldsz=(1 << 20) + 1)])
def test_linear_refuses_rows_of_weights_too_far_apart(change):
    """(256 rows of W are addressed with 32-bit offsets)"""
    rc, msg = linear(**change)
    assert rc == -6 and "2^20" in msg, (rc, msg)


def test_attention_refuses_unknown_flags():
    lib = K.load()
    rc = lib.kronq_cache_attention(*{**ATTEND, "rotate": 4}.values())
    assert rc == -1 and "flag" in lib.kronq_last_error().decode()
