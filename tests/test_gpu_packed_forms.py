"""The forms of the packed operators that batches with many heads or requests take, where the small
batches of test_gpu_packed do not lead: moving maxima, rows that are not finite beside rows that are,
starts that do not ascend, no place for the log-sum-exp, several streams, a captured step.

Which form a call takes follows from T, the number of requests and the heads; the sizes here lie well
on the sides that the comments name."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import packed_oracle as P  # noqa: E402
from paper_2410_08791_amd import binding as sp  # noqa: E402
from paper_2410_08791_amd import synth  # noqa: E402
from tests import test_gpu_packed as B  # noqa: E402
from tests.gpu_util import DEV, bf16_vals, dev_f32, dev_u16, host_u16, ptr, rand_bf16, stream_ptr  # noqa: E402

STEP = 2.0 ** -8          # half a step of bf16, relative
ULP = 2.0 ** -24          # of fp32


def later_moves(scores, causal):
    """How often a row's reference moves behind its first 32 keys (first half of a tile of 64, second half): it
    follows the maximum of 32 keys where that is more than 2^8 above it."""
    L = scores.shape[0]
    ref = np.full(L, -3.4e38)
    moves = [0, 0]
    for at in range(0, L, 32):
        s = scores[:, at:at + 32]
        if causal:
            s = np.where(np.arange(at, at + s.shape[1])[None] <= np.arange(L)[:, None], s, -np.inf)
        top = s.max(-1)
        move = (top - ref) * np.log2(np.e) > 8
        ref = np.where(move, top, ref)
        if at:
            moves[at // 32 & 1] += int(move.sum())
    return moves


@pytest.mark.parametrize("hq,hkv,hd", [(24, 6, 64), (16, 16, 80), (24, 3, 128), (4, 2, 64), (3, 3, 80), (4, 2, 128)])
@pytest.mark.parametrize("causal", [1, 0])
def test_the_running_maximum_moves(hq, hkv, hd, causal):
    """Keys whose magnitude grows along a request, so that sums and outputs are rescaled in both halves of several tiles: blocks of
    128 queries (the first three) and shared-out keys.

    Bounds.  With Q = max_j sum |q k| / sqrt(hd) a row's scores have an error of at most hd ULP Q from their sums and of 8 ULP |s| <= hd ULP
    Q / 8 from the arithmetic of the exponent; the reference passes through at most the range 2 Q of the scores, by
    differences that are rounded three times: 6 ULP Q.  Together under 2 hd ULP Q = d, by which a probability and the sum of them
    may be off, relative; sums of L terms add L ULP each, the hardware's exponential 4 ULP."""
    lens = [700, 190, 33]
    T, cu = sum(lens), B.sums(lens)
    rng = np.random.default_rng(hq + hd + causal)
    x = rng.standard_normal((T, hq + 2 * hkv, hd)) * 2
    place = np.concatenate([np.arange(v) / v for v in lens])
    x[:, hq:hq + hkv] *= (0.25 + 2 * place)[:, None, None]
    bits = synth.f32_to_bf16_bits(x.astype(np.float32)).reshape(T, -1)
    vals = bf16_vals(bits)
    x = vals.reshape(T, -1, hd)
    ob, lse = B.run_forward(bits, cu, T, hq, hkv, hd, causal)
    want, want_lse, weight = P.attention_packed(vals, cu, hq, hkv, hd, causal)
    got, moves = bf16_vals(ob[:T]).reshape(T, hq, hd), np.zeros(2, int)
    for a, b in zip(cu[:-1], cu[1:]):
        for h in range(hq):
            q, k = x[a:b, h], x[a:b, hq + h // (hq // hkv)]
            moves += later_moves(q @ k.T / np.sqrt(hd), causal)
            d = 2 * hd * ULP * (np.abs(q) @ np.abs(k).T).max(-1) / np.sqrt(hd)
            off = 2 * d + 2 * (b - a + 4) * ULP
            o, w = want[a:b, h], weight[a:b, h]
            assert np.all(np.abs(got[a:b, h] - o) <= STEP * (w + np.abs(o)) + off[:, None] * w * (1 + 2 * STEP))
            assert np.all(np.abs(lse[:hq * T].reshape(hq, T)[h, a:b] - want_lse[h, a:b]) <= off)
    print("later moves, first and second half of a tile:", moves, flush=True)
    assert moves.min() >= 50 * hq


@pytest.mark.parametrize("hq,hkv,hd", [(2, 1, 64), (40, 40, 64), (170, 170, 64), (2, 2, 80), (40, 20, 80), (20, 20, 80), (2, 2, 128), (80, 80, 128)])
@pytest.mark.parametrize("causal", [1, 0])
def test_rows_that_are_not_finite_stay_with_their_request(hq, hkv, hd, causal):
    """Infinite and NaN rows, outputs and gradients of one request leave the bits of its neighbours alone, forward and backward:
    few and many heads, 32, 64 and 128 keys per work-group of the backward; requests end inside tiles."""
    rng = np.random.default_rng(hq + hd)
    lens, T, bad = [70, 40, 130], 240, slice(70, 110)
    cu, n = B.sums(lens), 3
    bits, _ = rand_bf16(rng, (T, (hq + 2 * hkv) * hd))
    db, _ = rand_bf16(rng, (T, hq * hd), 0.5)
    outs = []
    for dirty in (False, True):
        q, d = bits.copy(), db.copy()
        if dirty:
            q[bad, ::3], q[bad, 1::3], d[bad, ::2], d[bad, 1::2] = B.NAN16, 0x7F80, 0xFF80, B.NAN16
        ob, lse = B.run_forward(q, cu, T, hq, hkv, hd, causal)
        if dirty:
            ob[bad], lse[:hq * T].reshape(hq, T)[:, bad] = B.NAN16, np.inf
        qd, c, o, do, ls = dev_u16(q), B.i32(cu), dev_u16(ob[:T]), dev_u16(d), dev_f32(lse[:hq * T])
        scratch = torch.zeros(sp.spk_attention_packed_bwd_scratch_bytes(T, hq), dtype=torch.uint8, device=DEV)
        dx = torch.zeros_like(qd)
        assert sp.spk_attention_packed_bwd(stream_ptr(), ptr(qd), ptr(c), ptr(o), ptr(do), ptr(ls), ptr(scratch), ptr(dx), n, T, hq, hkv, hd,
                                           causal) == sp.SP_OK
        torch.cuda.synchronize()
        outs.append((ob[:T], lse[:hq * T].reshape(hq, T).T, host_u16(dx)))
    for clean, dirty, name in zip(*outs, ("o", "lse", "dqkv")):
        for rows in (slice(0, 70), slice(110, 240)):
            assert np.array_equal(clean[rows], dirty[rows]), (name, rows)
            assert np.all(np.isfinite(bf16_vals(clean[rows]) if name != "lse" else clean[rows])), name
    assert not np.any(np.isfinite(bf16_vals(outs[1][2][bad].reshape(40, -1, hd)[:, 0])))


HOSTILE = {"back": [0, 150, 60, 200], "far": [-5, 10, 2 ** 31 - 1, 40], "end": [200] * 4, "down": [90, 80, 70, 60],
           "extremes": [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, -2 ** 31], "past": [0, 5000, 3, 200]}


@pytest.mark.parametrize("name", list(HOSTILE) + ["many_down", "many_mixed", "many_past"])
@pytest.mark.parametrize("hq,hkv,hd", [(2, 1, 64), (200, 100, 64), (40, 20, 80), (90, 90, 80), (2, 1, 128), (110, 110, 128)])
def test_starts_that_do_not_ascend_stay_inside(name, hq, hkv, hd):
    """Fewer than 64 requests and more, whatever the starts: nothing outside the outputs and the scratch is written."""
    rng = np.random.default_rng(6)
    many = {"many_down": np.arange(99, -1, -1) * 2, "many_mixed": rng.integers(-300, 700, 100), "many_past": np.arange(100) * 7 - 20}
    cu = np.array(HOSTILE[name] if name in HOSTILE else many[name])
    T, n = 200, len(cu) - 1
    print(f"starts {name} heads {hq}/{hkv} hd={hd}", flush=True)
    q, do = dev_u16(rand_bf16(rng, (T, (hq + 2 * hkv) * hd))[0]), dev_u16(rand_bf16(rng, (T, hq * hd), 0.5)[0])
    c, need = B.i32(cu), sp.spk_attention_packed_bwd_scratch_bytes(T, hq)
    o, dx = (torch.full((T + 2, w * hd), 7, dtype=torch.int16, device=DEV) for w in (hq, hq + 2 * hkv))
    lse = torch.full((hq * T + 2,), 7.0, device=DEV)
    scratch = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    assert sp.spk_attention_packed(stream_ptr(), ptr(q), ptr(c), ptr(o[1:]), ptr(lse[1:]), n, T, hq, hkv, hd, 1) == sp.SP_OK
    torch.cuda.synchronize()
    assert sp.spk_attention_packed_bwd(stream_ptr(), ptr(q), ptr(c), ptr(o[1:]), ptr(do), ptr(lse[1:]), ptr(scratch[128:]), ptr(dx[1:]), n, T, hq,
                                       hkv, hd, 1) == sp.SP_OK
    torch.cuda.synchronize()
    for t in (o, dx):
        assert bool((t[0] == 7).all()) and bool((t[-1] == 7).all())
    assert lse[0] == 7 and lse[-1] == 7 and bool((scratch[:128] == 0xA5).all()) and bool((scratch[128 + need:] == 0xA5).all())


@pytest.mark.parametrize("hq,hkv,hd", [(2, 1, 64), (40, 20, 64), (2, 1, 80), (24, 12, 80), (2, 1, 128), (40, 20, 128)])
def test_scores_that_are_all_minus_infinity(hq, hkv, hd):
    """A query with an infinite element on keys of one sign: 0 / 0 and log 0; of the other sign: infinite.  Nobody else notices."""
    rng = np.random.default_rng(hq)
    lens = [300, 45, 200]
    T, cu = 545, B.sums(lens)
    bits, _ = rand_bf16(rng, (T, (hq + 2 * hkv) * hd))
    x = bits.reshape(T, -1, hd)
    x[:, hq:hq + hkv, 3] |= 0x8000                          # negative, and none is zero
    x[:, hq:hq + hkv, 3] |= 0x0080
    clean, clean_lse = B.run_forward(bits, cu, T, hq, hkv, hd, 1)
    rows = [0, 31, 100, 299, 310, 544]
    x[rows, 1, 3] = 0x7F80                                   # head 1: scores of -inf
    x[rows, 0, 3] = 0xFF80                                   # head 0: of +inf
    ob, lse = B.run_forward(bits, cu, T, hq, hkv, hd, 1)
    got, lse = bf16_vals(ob[:T]).reshape(T, hq, hd), lse[:hq * T].reshape(hq, T)
    assert np.all(np.isnan(got[rows][:, :2])) and np.all(lse[1, rows] == -np.inf) and not np.any(np.isfinite(lse[0, rows]))
    others = np.setdiff1d(np.arange(T), rows)
    assert np.array_equal(ob[others], clean[others]) and np.array_equal(lse[:, others], clean_lse[:hq * T].reshape(hq, T)[:, others])
    assert np.array_equal(ob[:T].reshape(T, hq, hd)[:, 2:], clean[:T].reshape(T, hq, hd)[:, 2:])


@pytest.mark.parametrize("hq,hkv,hd", [(24, 6, 64), (32, 16, 80), (40, 40, 128)])
def test_many_heads_without_log_sum_exp_on_two_streams_and_captured(hq, hkv, hd):
    """Blocks of 128 queries: the same bits without a place for the log-sum-exp, beside another batch on another stream, and from a
    captured step that is replayed on other lengths with eager work and synchronizations in between."""
    rng = np.random.default_rng(hd)
    T, n, s0 = 923, 4, stream_ptr()
    q, do = dev_u16(rand_bf16(rng, (T, (hq + 2 * hkv) * hd))[0]), dev_u16(rand_bf16(rng, (T, hq * hd), 0.5)[0])
    cu = B.i32(B.sums([700, 0, 190, 33]))
    need = sp.spk_attention_packed_bwd_scratch_bytes(T, hq)

    def arrays():
        return dict(o=torch.full_like(do, 7), dx=torch.full_like(q, 7), lse=torch.zeros((hq, T), device=DEV),
                    scratch=torch.zeros(need, dtype=torch.uint8, device=DEV))

    def step(b, cu, s):
        assert sp.spk_attention_packed(s, ptr(q), ptr(cu), ptr(b["o"]), ptr(b["lse"]), n, T, hq, hkv, hd, 1) == sp.SP_OK
        assert sp.spk_attention_packed_bwd(s, ptr(q), ptr(cu), ptr(b["o"]), ptr(do), ptr(b["lse"]), ptr(b["scratch"]), ptr(b["dx"]), n, T, hq, hkv,
                                           hd, 1) == sp.SP_OK
    alone = arrays()
    step(alone, cu, s0)
    bare = torch.full_like(do, 7)
    assert sp.spk_attention_packed(s0, ptr(q), ptr(cu), ptr(bare), None, n, T, hq, hkv, hd, 1) == sp.SP_OK
    torch.cuda.synchronize()
    assert torch.equal(bare, alone["o"])
    pair = [(arrays(), torch.cuda.Stream()) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for b, st in pair:
            step(b, cu, st.cuda_stream)
    torch.cuda.synchronize()
    for b, _ in pair:
        assert torch.equal(b["o"], alone["o"]) and torch.equal(b["dx"], alone["dx"]) and torch.equal(b["lse"], alone["lse"])
    cap, where = arrays(), cu.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(cap, where, stream_ptr())
    torch.cuda.current_stream().wait_stream(side)
    for lens in ([923, 0, 0, 0], [1, 400, 2, 33], [200, 200, 200, 200], [700, 0, 190, 33]):
        where.copy_(B.i32(B.sums(lens)))
        for name in ("o", "dx"):
            cap[name].fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        eager = arrays()
        step(eager, where, s0)
        torch.cuda.synchronize()
        for name in ("o", "dx"):
            assert torch.equal(eager[name], cap[name]) and bool((cap[name][sum(lens):] == 7).all()), (lens, name)


def test_arrays_of_no_bytes_overlap_nothing():
    """A scratch that the call does not need and an empty free list may point anywhere, also into arrays of the call."""
    rng = np.random.default_rng(3)
    hq, hkv, hd, bs = 2, 1, 64, 16
    k8, v8, sc = B.filled(rng, 4, hkv, bs, hd)
    q, k, v, s = dev_u16(rand_bf16(rng, (2, 4 * hd))[0]), B.u8(k8), B.u8(v8), dev_f32(sc)
    t, n, o = B.i32([[0, 1], [2, 3]]), B.i32([20, 32]), torch.zeros((2, hq * hd), dtype=torch.int16, device=DEV)
    assert sp.spk_kv8_attention_scratch_bytes(2, 2, bs, hq, hkv, hd) == 0
    outs = []
    for scratch in (None, ptr(q[1:]), ptr(o.reshape(-1)[64:])):
        o.zero_()
        assert sp.spk_kv8_attention(stream_ptr(), ptr(q), ptr(k), ptr(v), ptr(s), ptr(t), ptr(n), ptr(o), scratch, 2, 4, bs, 2, hq, hkv, hd) == sp.SP_OK
        torch.cuda.synchronize()
        outs.append(o.clone())
    assert bool(outs[0].any()) and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    lens, cached, cu, kv, slots, info = (B.i32(x) for x in ([1, 2], [3, 4], [0] * 3, [0] * 2, [0] * 3, [0] * 4))
    assert sp.spk_batch_plan(stream_ptr(), ptr(lens), ptr(cached), ptr(t[1:]), 0, ptr(t), 2, ptr(cu), ptr(kv), ptr(slots), 3, ptr(info), 2, bs) == sp.SP_OK
    torch.cuda.synchronize()
    assert slots.tolist() == [3, 2 * bs + 4, 2 * bs + 5] and kv.tolist() == [4, 6]


@pytest.mark.parametrize("e", [-126, -125, -124, -60, 0, 119, 120])
def test_cache_attention_of_every_code(e):
    """One position of weight 1: code * scale itself, rounded to multiples of 2^-133 and infinite from 2^128 on."""
    k8, v8, sc = np.full((4, 1, 16, 64), 0x38, np.uint8), np.full((4, 1, 64, 16), 0x7F, np.uint8), np.ones((4, 1, 2), np.float32)
    v8[:, 0, :, 0] = np.arange(256).reshape(4, 64)
    sc[:, :, 1] = 2.0 ** e
    q = rand_bf16(np.random.default_rng(1), (4, 3 * 64))[0]
    got = B.run_cache_attention(q, k8, v8, sc, np.arange(4).reshape(4, 1), np.ones(4, int), 16, 1, 1, 64).reshape(256)
    want = np.round(P.E4M3 * 2.0 ** e * 2.0 ** 133) * 2.0 ** -133
    want[np.abs(want) >= 2.0 ** 128] *= np.inf
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("n", [2, 300])
def test_cache_attention_of_the_largest_values(n):
    """The largest bf16 values through append and attention, the first position with all the weight: 248 * 2^120 and more are stored as
    2^128 and count as infinite, NaN where they weigh nothing; under that the element is what the first position holds."""
    hd, bs, blocks = 64, 16, 20
    bits = np.zeros((n, 3 * hd), np.uint16)
    x = bits.reshape(n, 3, hd)
    x[0, 1], x[1:, 1] = 0x4100, 0xC100                        # keys 8 and -8
    x[:, 2] = 0x3F80                                          # values 1
    x[1, 2, :8] = [0x7F60, 0x7F70, 0x7F77, 0x7F78, 0x7F7F, 0xFF7F, 0xFF77, 0x7F00]
    k8, v8, sc = B.run_append(bits, np.arange(n), *B.filled(np.random.default_rng(2), blocks, 1, bs, hd), bs, 1, 1, hd)
    q = np.full((1, 3 * hd), 0x4100, np.uint16)
    got = B.run_cache_attention(q, k8, v8, sc, np.arange(blocks).reshape(1, -1), np.array([n]), bs, 1, 1, hd)[0, 0]
    assert sc[0, 0, 1] == 2.0 ** 120 and list(v8[0, 0, 3:6, 1]) == [0x78, 0x78, 0xF8]
    assert np.all(np.isnan(got[3:6]))
    assert not np.any(got[[0, 1, 2, 6, 7]]) and not np.any(got[8:])      # 1 is code 0 at that scale
