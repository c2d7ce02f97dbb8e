"""Operators over packed batches, without a GPU: their oracle against other definitions, and what the
calls refuse before anything is launched."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import packed_oracle as P  # noqa: E402
from oracle import stack_oracle as O  # noqa: E402
from paper_2410_08791_amd import binding as sp  # noqa: E402

BAD = sp.SP_ERR_INVALID_ARG


def test_oracle_e4m3_against_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(P.E4M3), np.isnan(want)) and np.array_equal(np.nan_to_num(P.E4M3), np.nan_to_num(want))
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 6, 4000),
                        P.E4M3[:127], (P.E4M3[:126] + P.E4M3[1:127]) / 2, [0.0, -0.0]]).astype(np.float32)
    assert np.array_equal(P.to_e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert list(P.to_e4m3([np.inf, -np.inf, np.nan])) == [127, 255, 127]


def test_oracle_attention_is_the_stacks_per_request():
    rng = np.random.default_rng(2)
    hq, hkv, hd, cu = 4, 2, 64, [0, 5, 5, 18, 19]
    x = rng.standard_normal((21, (hq + 2 * hkv) * hd))
    for causal in (True, False):
        o, _, _ = P.attention_packed(x, cu, hq, hkv, hd, causal)
        shape = O.StackShape("decoder", 1, hq * hd, hq, hkv, hd, 64, causal, 1e-5)
        for a, b in zip(cu[:-1], cu[1:]):
            if b > a:
                q, k, v = np.split(x[a:b], [hq * hd, (hq + hkv) * hd], axis=1)
                assert np.allclose(o[a:b].reshape(b - a, -1), O.attention(q, k, v, 1, b - a, shape).reshape(b - a, -1), atol=1e-12)
        assert not o[19:].any()


@pytest.mark.parametrize("causal", [True, False])
def test_oracle_gradient_against_differences(causal):
    rng = np.random.default_rng(3)
    hq, hkv, hd, cu = 4, 2, 64, [0, 7, 7, 8, 20]
    x, w = rng.standard_normal((20, (hq + 2 * hkv) * hd)), rng.standard_normal((20, hq, hd))
    o, lse, _ = P.attention_packed(x, cu, hq, hkv, hd, causal)
    dx, _, _ = P.attention_packed_bwd(x, cu, o, w, lse, hq, hkv, hd, causal)
    for _ in range(4):
        u = rng.standard_normal(x.shape)
        h = 1e-5
        loss = [(P.attention_packed(x + s * h * u, cu, hq, hkv, hd, causal)[0] * w).sum() for s in (1, -1)]
        assert abs((loss[0] - loss[1]) / (2 * h) - (dx.reshape(x.shape) * u).sum()) <= 1e-7 * np.abs(dx).sum()


def test_plan_refusals():
    p = 4096         # an aligned address that is never followed: every call below ends in the argument checks
    good = dict(lens=p, cached=p + 64, free=p + 128, n_free=4, table=p + 192, max_blocks=4, cu=p + 256, kv_len=p + 320, slots=p + 384,
                max_tokens=8, info=p + 448, n=3, bs=16)

    def call(**kw):
        a = dict(good, **kw)
        return sp.spk_batch_plan(None, a["lens"], a["cached"], a["free"], a["n_free"], a["table"], a["max_blocks"], a["cu"], a["kv_len"],
                                 a["slots"], a["max_tokens"], a["info"], a["n"], a["bs"])
    for kw in (dict(lens=None), dict(table=None), dict(cu=None), dict(kv_len=None), dict(slots=None), dict(info=None), dict(free=None),
               dict(n=0), dict(n=4097), dict(n_free=-1), dict(max_tokens=0), dict(max_tokens=(1 << 30) + 1), dict(bs=8), dict(bs=48),
               dict(bs=128), dict(max_blocks=0), dict(max_blocks=(1 << 26) + 1), dict(lens=p + 2), dict(slots=p + 1),
               dict(kv_len=p), dict(kv_len=p + 64), dict(cached=p + 260), dict(cu=p - 12), dict(table=p + 140), dict(slots=p + 100),
               dict(slots=p + 324), dict(info=p + 412), dict(info=p + 264), dict(max_tokens=17)):
        assert call(**kw) == BAD, kw


def test_attention_refusals():
    p = 4096
    good = dict(qkv=p, cu=p, o=p, lse=p, n=2, T=64, hq=4, hkv=2, hd=64)
    bwd = dict(good, dO=p, scratch=p, dqkv=p)

    def call(**kw):
        a = dict(good, **kw)
        return sp.spk_attention_packed(None, a["qkv"], a["cu"], a["o"], a["lse"], a["n"], a["T"], a["hq"], a["hkv"], a["hd"], 1)

    def call_bwd(**kw):
        a = dict(bwd, **kw)
        return sp.spk_attention_packed_bwd(None, a["qkv"], a["cu"], a["o"], a["dO"], a["lse"], a["scratch"], a["dqkv"], a["n"], a["T"],
                                           a["hq"], a["hkv"], a["hd"], 1)
    wrong = [dict(qkv=None), dict(cu=None), dict(o=None), dict(n=0), dict(n=4097), dict(T=0), dict(T=(1 << 30) + 1), dict(hq=3),
             dict(hq=0), dict(hkv=0), dict(hq=16386), dict(hd=96), dict(hd=256), dict(qkv=p + 2), dict(o=p + 8), dict(cu=p + 2), dict(T=1 << 29, hq=64)]
    for kw in wrong:
        assert call(**kw) == BAD and call_bwd(**kw) == BAD, kw
    for kw in (dict(dO=None), dict(lse=None), dict(scratch=None), dict(dqkv=None), dict(dqkv=p + 4), dict(scratch=p + 4)):
        assert call_bwd(**kw) == BAD, kw
    assert sp.spk_attention_packed_bwd_scratch_bytes(100, 3) == 1280
    assert sp.spk_attention_packed_bwd_scratch_bytes(0, 3) == 0


def test_cache_refusals():
    p = 4096
    a0 = dict(qkv=p, slots=p, k8=p, v8=p, scales=p, T=8, blocks=4, bs=16, hq=4, hkv=2, hd=64)

    def append(**kw):
        a = dict(a0, **kw)
        return sp.spk_kv8_append(None, a["qkv"], a["slots"], a["k8"], a["v8"], a["scales"], a["T"], a["blocks"], a["bs"], a["hq"],
                                 a["hkv"], a["hd"])
    b0 = dict(qkv=p, k8=p, v8=p, scales=p, table=p, kv_len=p, o=p, scratch=p, B=2, blocks=4, bs=16, mb=4, hq=4, hkv=2, hd=64)

    def attend(**kw):
        a = dict(b0, **kw)
        return sp.spk_kv8_attention(None, a["qkv"], a["k8"], a["v8"], a["scales"], a["table"], a["kv_len"], a["o"], a["scratch"], a["B"],
                                    a["blocks"], a["bs"], a["mb"], a["hq"], a["hkv"], a["hd"])
    both = [dict(qkv=None), dict(k8=None), dict(v8=None), dict(scales=None), dict(blocks=0), dict(blocks=1 << 27), dict(bs=8), dict(bs=128),
            dict(hq=3), dict(hkv=0), dict(hd=80), dict(hd=32), dict(qkv=p + 2), dict(k8=p + 8), dict(v8=p + 1), dict(scales=p + 4)]
    for kw in both:
        assert append(**kw) == BAD and attend(**kw) == BAD, kw
    for kw in (dict(slots=None), dict(T=0), dict(T=(1 << 30) + 1), dict(slots=p + 2)):
        assert append(**kw) == BAD, kw
    for kw in (dict(table=None), dict(kv_len=None), dict(o=None), dict(B=0), dict(B=65536), dict(mb=0), dict(mb=(1 << 26) + 1),
               dict(table=p + 2), dict(o=p + 8), dict(mb=1 << 20, scratch=None)):
        assert attend(**kw) == BAD, kw
    assert sp.spk_kv8_attention_scratch_bytes(2, 4, 16, 4, 2, 80) == 0
    assert sp.spk_kv8_plan(2, 4, 16, 4, 3, (C.c_int * 2)()) == BAD and sp.spk_kv8_plan(2, 4, 16, 4, 2, None) == BAD


def spread(names):
    """An address per array, far from one another and never followed: every call with them below ends in the argument checks."""
    return {name: (i + 1) << 20 for i, name in enumerate(names)}


def test_attention_refuses_overlaps():
    """Outputs over inputs, over one another, by a whole array or by its last bytes."""
    shape = dict(n=2, T=64, hq=4, hkv=2, hd=64)
    wide, rows, row_values = 64 * 8 * 64 * 2, 64 * 4 * 64 * 2, 64 * 4 * 4         # bytes of qkv, of o, of lse
    a = dict(spread(["qkv", "cu", "o", "lse", "dO", "scratch", "dqkv"]), **shape)

    def call(**kw):
        x = dict(a, **kw)
        return sp.spk_attention_packed(None, x["qkv"], x["cu"], x["o"], x["lse"], x["n"], x["T"], x["hq"], x["hkv"], x["hd"], 1)

    def call_bwd(**kw):
        x = dict(a, **kw)
        return sp.spk_attention_packed_bwd(None, x["qkv"], x["cu"], x["o"], x["dO"], x["lse"], x["scratch"], x["dqkv"], x["n"], x["T"],
                                           x["hq"], x["hkv"], x["hd"], 1)
    for kw in (dict(o=a["qkv"]), dict(o=a["qkv"] + wide - 16), dict(o=a["qkv"] - rows + 16), dict(o=a["cu"]), dict(o=a["cu"] - rows + 16),
               dict(lse=a["qkv"]), dict(lse=a["o"] + rows - 4), dict(lse=a["o"] - row_values + 4), dict(lse=a["cu"] + 8)):
        assert call(**kw) == BAD, kw
    for name, size in (("qkv", wide), ("o", rows), ("dO", rows), ("lse", row_values), ("cu", 16)):
        for kw in (dict(dqkv=a[name]), dict(dqkv=a[name] + size - 16), dict(dqkv=a[name] - wide + 16), dict(scratch=a[name]),
                   dict(scratch=a[name] + size - 16), dict(scratch=a[name] - row_values + 16)):
            assert call_bwd(**kw) == BAD, kw
    for kw in (dict(scratch=a["dqkv"]), dict(scratch=a["dqkv"] + wide - 16), dict(scratch=a["dqkv"] - row_values + 16)):
        assert call_bwd(**kw) == BAD, kw
    # what was refused before, by arrays that lie apart
    for kw in (dict(qkv=None), dict(cu=None), dict(o=None), dict(n=0), dict(n=4097), dict(T=0), dict(T=(1 << 30) + 1), dict(hq=3), dict(hq=0),
               dict(hkv=0), dict(hq=16386), dict(hd=96), dict(hd=256), dict(qkv=a["qkv"] + 2), dict(o=a["o"] + 8), dict(cu=a["cu"] + 2)):
        assert call(**kw) == BAD and call_bwd(**kw) == BAD, kw
    for kw in (dict(dO=None), dict(lse=None), dict(scratch=None), dict(dqkv=None), dict(dqkv=a["dqkv"] + 4), dict(scratch=a["scratch"] + 4)):
        assert call_bwd(**kw) == BAD, kw


def test_cache_refuses_overlaps():
    shape = dict(T=8, B=8, blocks=4, bs=16, mb=40, hq=4, hkv=2, hd=64)
    sizes = dict(qkv=8 * 8 * 64 * 2, k8=4 * 16 * 2 * 64, v8=4 * 16 * 2 * 64, scales=4 * 2 * 8, slots=32, table=8 * 40 * 4, kv_len=32, o=8 * 4 * 64 * 2)
    sizes["scratch"] = sp.spk_kv8_attention_scratch_bytes(8, 40, 16, 4, 2, 64)
    assert sizes["scratch"] > 0
    a = dict(spread(sizes), **shape)

    def append(x):
        return sp.spk_kv8_append(None, x["qkv"], x["slots"], x["k8"], x["v8"], x["scales"], x["T"], x["blocks"], x["bs"], x["hq"],
                                 x["hkv"], x["hd"])

    def attend(x):
        return sp.spk_kv8_attention(None, x["qkv"], x["k8"], x["v8"], x["scales"], x["table"], x["kv_len"], x["o"], x["scratch"], x["B"],
                                    x["blocks"], x["bs"], x["mb"], x["hq"], x["hkv"], x["hd"])
    for call, written, others in ((append, ("k8", "v8", "scales"), ("qkv", "slots", "k8", "v8", "scales")),
                                  (attend, ("o", "scratch"), ("qkv", "k8", "v8", "scales", "table", "kv_len", "o", "scratch"))):
        for w in written:
            for other in others:
                if w != other:
                    for at in (a[other], a[other] + sizes[other] - 16, a[other] - sizes[w] + 16):
                        assert call(dict(a, **{w: at})) == BAD, (w, other, at - a[other])
    for kw in (dict(qkv=None), dict(k8=None), dict(v8=None), dict(scales=None), dict(blocks=0), dict(blocks=1 << 27), dict(bs=8), dict(bs=128),
               dict(hq=3), dict(hkv=0), dict(hd=80), dict(hd=32), dict(qkv=a["qkv"] + 2), dict(k8=a["k8"] + 8), dict(v8=a["v8"] + 1),
               dict(scales=a["scales"] + 4)):
        assert append(dict(a, **kw)) == BAD and attend(dict(a, **kw)) == BAD, kw
    for kw in (dict(slots=None), dict(T=0), dict(T=(1 << 30) + 1), dict(slots=a["slots"] + 2)):
        assert append(dict(a, **kw)) == BAD, kw
    for kw in (dict(table=None), dict(kv_len=None), dict(o=None), dict(B=0), dict(B=65536), dict(mb=0), dict(mb=(1 << 26) + 1),
               dict(table=a["table"] + 2), dict(o=a["o"] + 8), dict(scratch=None)):
        assert attend(dict(a, **kw)) == BAD, kw


def test_kv8_plan_covers_the_table():
    out = (C.c_int * 2)()
    rng = np.random.default_rng(5)
    for _ in range(400):
        B, hkv, g = int(rng.integers(1, 400)), int(rng.integers(1, 40)), int(rng.integers(1, 40))
        bs = int(rng.choice([16, 32, 64]))
        mb = int(2.0 ** rng.uniform(0, 26 - np.log2(bs / 16)))
        assert sp.spk_kv8_plan(B, mb, bs, hkv * g, hkv, out) == sp.SP_OK
        splits, per = out
        assert 1 <= splits <= 65535 and per % 64 == 0 and splits * per >= mb * bs and (splits - 1) * per < mb * bs
        need = sp.spk_kv8_attention_scratch_bytes(B, mb, bs, hkv * g, hkv, 128)
        assert need == (0 if splits == 1 else B * hkv * g * splits * 130 * 4)
        # a row of partial results for every 256 positions is room enough
        assert need <= 4 * B * hkv * g * 130 * -(-mb * bs // 256)
