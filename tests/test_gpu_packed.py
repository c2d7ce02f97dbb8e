"""Operators over packed batches (requests of different lengths) on the GPU, through the C ABI, against
the 64-bit oracle.

Bounds.  The kernels round to bf16 (at most half a step, 2^-8 relative) the probabilities, in the
backward pass dS and P, and what they store; everything else is fp32.  With A = sum_j p_ij |v_j| an
output is therefore off by at most 2^-8 (A + |o|), and by the fp32 parts: a score of hd products
has an error of hd 2^-24 sum |q k| / sqrt(hd), under 1e-4 for the inputs here, which changes p by
as much relative to itself: 1e-4 A."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import packed_oracle as P  # noqa: E402
from paper_2410_08791_amd import binding as sp  # noqa: E402
from tests.gpu_util import DEV, bf16_vals, dev_f32, dev_u16, host_u16, ptr, rand_bf16, stream_ptr  # noqa: E402

STEP = 2.0 ** -8          # half a step of bf16, relative
FP32 = 1e-4
NAN16 = 0x7FC1


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def u8(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.uint8)).to(DEV)


def sums(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


# ---- plan ------------------------------------------------------------------------------------------

def plan(lens, cached, free, table, max_tokens, bs, null_cached=False):
    n, width = table.shape
    d = [i32(a) for a in (lens, cached, free if len(free) else [0], table)]
    cu, kv = torch.full((n + 2,), 77, dtype=torch.int32, device=DEV), torch.full((n + 1,), 77, dtype=torch.int32, device=DEV)
    slots, info = torch.full((max_tokens + 1,), 77, dtype=torch.int32, device=DEV), torch.full((5,), 77, dtype=torch.int32, device=DEV)
    rc = sp.spk_batch_plan(stream_ptr(), ptr(d[0]), None if null_cached else ptr(d[1]), ptr(d[2]) if len(free) else None, len(free), ptr(d[3]),
                           width, ptr(cu), ptr(kv), ptr(slots), max_tokens, ptr(info), n, bs)
    assert rc == sp.SP_OK
    torch.cuda.synchronize()
    assert cu[n + 1] == 77 and kv[n] == 77 and slots[max_tokens] == 77 and info[4] == 77
    return [t.cpu().numpy() for t in (cu[:n + 1], kv[:n], slots[:max_tokens], d[3], info[:4])]


def same_plan(got, want):
    for a, b, name in zip(got, want, ("cu", "kv_len", "slots", "table", "info")):
        assert np.array_equal(a, b), name


def make_tables(rng, cached, width, bs, blocks, unowned=7):
    """Rows with the blocks of the cached positions, `unowned` in the entries that no one owns; the free blocks."""
    order = rng.permutation(blocks).astype(np.int32)
    table = np.full((len(cached), width), unowned, np.int32)
    at = 0
    for r, c in enumerate(cached):
        held = -(-c // bs)
        table[r, :held] = order[at:at + held]
        at += held
    return table, order[at:]


@pytest.mark.parametrize("n,most_new,most_cached,bs", [
    (1, 1, 0, 16), (1, 100, 17, 16), (3, 1, 64, 32), (64, 1, 500, 16), (65, 40, 0, 64), (513, 9, 70, 32), (4096, 3, 40, 16), (7, 5000, 300, 64),
])
def test_plan(n, most_new, most_cached, bs):
    rng = np.random.default_rng(n + most_new)
    lens, cached = rng.integers(0, most_new + 1, n), rng.integers(0, most_cached + 1, n)
    lens[rng.integers(n)] = most_new
    if n > 2:
        cached[0], lens[0] = bs, bs              # a request that ends with a block, and the next begins one
        lens[n - 1] = 0
    width = -(-(most_new + most_cached + 2 * bs) // bs)
    need = int(sum(-(-(c + v) // bs) for c, v in zip(cached, lens)))
    table, free = make_tables(rng, cached, width, bs, need + 3)
    for spare in (0, 5):
        got = plan(lens, cached, free, table, int(lens.sum()) + spare or 1, bs)
        same_plan(got, P.batch_plan(lens, cached, free, table, int(lens.sum()) + spare or 1, bs))


def test_plan_without_cached_positions_or_free_blocks():
    table = np.full((3, 2), 9, np.int32)
    same_plan(plan([3, 0, 20], [0, 0, 0], [5, 6, 7], table, 23, 16, null_cached=True), P.batch_plan([3, 0, 20], [0, 0, 0], [5, 6, 7], table, 23, 16))
    table = np.array([[4, 9], [2, 3]], np.int32)
    same_plan(plan([3, 1], [2, 30], [], table, 6, 16), P.batch_plan([3, 1], [2, 30], [], table, 6, 16))
    same_plan(plan([0, 0], [2, 30], [], table, 1, 16), P.batch_plan([0, 0], [2, 30], [], table, 1, 16))


def test_plan_of_entries_that_are_no_blocks():
    """Rows that would go to them have no slot."""
    table = np.array([[2 ** 28 + 1, 9], [-3, 9], [2 ** 31 - 1, 9], [2 ** 27 - 1, 9]], np.int32)
    got = plan([2, 2, 20, 2], [3, 3, 3, 3], [2 ** 27, 0], table, 26, 16)
    slots = np.full(26, -1)
    slots[24:] = (2 ** 27 - 1) * 16 + np.array([3, 4])
    assert np.array_equal(got[2], slots) and list(got[4]) == [26, 1, 20, 0] and got[3][2, 1] == 2 ** 27


@pytest.mark.parametrize("lens,cached,n_free,max_tokens,why", [
    ([5, 20], [0, 0], 3, 24, 1), ([5, 20], [0, 0], 2, 25, 2), ([5, 20], [0, 40], 9, 25, 4), ([5, -1], [0, 0], 9, 25, 8), ([5, 1], [-2, 0], 9, 25, 8),
    ([2 ** 31 - 1, 2 ** 31 - 1], [0, 0], 2, 9, 7), ([5, 20], [2 ** 31 - 1, 0], 9, 25, 4),
])
def test_plan_that_does_not_fit_is_not_carried_out(lens, cached, n_free, max_tokens, why):
    table, free = np.full((2, 3), 7, np.int32), np.arange(n_free)
    got = plan(lens, cached, free, table, max_tokens, 16)
    assert got[4][3] == why
    assert not got[0].any() and np.array_equal(got[1], np.array(cached)) and np.all(got[2] == -1) and np.array_equal(got[3], table)
    if max(lens) < 2 ** 30:
        same_plan(got, P.batch_plan(lens, cached, free, table, max_tokens, 16))


# ---- packed attention --------------------------------------------------------------------------------

def prompt_inputs(rng, lens, spare, hq, hkv, hd, scale=1.0):
    """Rows of the requests, then `spare` rows of NaN."""
    T = int(sum(lens))
    bits, vals = rand_bf16(rng, (T + spare, (hq + 2 * hkv) * hd), scale)
    bits[T:], vals[T:] = NAN16, 0.0
    return bits, vals


def run_forward(bits, cu, T, hq, hkv, hd, causal, with_lse=True):
    q, c = dev_u16(bits), i32(cu)
    o = torch.full((T + 1, hq * hd), 7, dtype=torch.int16, device=DEV)
    lse = torch.full((hq * T + 1,), 7.0, device=DEV) if with_lse else None
    assert sp.spk_attention_packed(stream_ptr(), ptr(q), ptr(c), ptr(o), ptr(lse), len(cu) - 1, T, hq, hkv, hd, causal) == sp.SP_OK
    torch.cuda.synchronize()
    return host_u16(o), lse.cpu().numpy() if with_lse else None


def check_forward(lens, spare, hq, hkv, hd, causal, scale=1.0, seed=0):
    rng = np.random.default_rng(sum(lens) + hq + seed)
    bits, vals = prompt_inputs(rng, lens, spare, hq, hkv, hd, scale)
    T, used, cu = bits.shape[0], int(sum(lens)), sums(lens)
    print(f"packed attention lens={lens} spare={spare} heads {hq}/{hkv} hd={hd} causal={causal}", flush=True)
    ob, lse = run_forward(bits, cu, T, hq, hkv, hd, causal)
    want, want_lse, weight = P.attention_packed(vals, cu, hq, hkv, hd, causal)
    assert np.all(ob[used:] == 7) and np.all(lse[hq * T:] == 7) and np.all(lse[:hq * T].reshape(hq, T)[:, used:] == 7)
    got = bf16_vals(ob[:used]).reshape(used, hq, hd)
    off = np.abs(got - want[:used]) - (STEP * (weight[:used] + np.abs(want[:used])) + FP32 * weight[:used])
    assert off.max(initial=-1) <= 0, float(off.max())
    # log-sum-exp: a score's error (the header of this file, on the largest sum of products), 100 additions of the tile sums and the logarithm
    x = np.abs(vals.reshape(T, hq + 2 * hkv, hd))
    big = hd * 2.0 ** -24 * max((x[a:b, h] @ x[a:b, hq + h // (hq // hkv)].T).max() for a, b in zip(cu[:-1], cu[1:]) if b > a
                                for h in range(hq)) / np.sqrt(hd)
    assert np.max(np.abs(lse[:hq * T].reshape(hq, T)[:, :used] - want_lse[:, :used]), initial=0) <= big + 2e-5
    return ob


@pytest.mark.parametrize("lens,spare,hq,hkv,hd", [
    ([1], 0, 1, 1, 64), ([1, 1, 1], 2, 2, 1, 128), ([0, 5, 0, 0, 3], 1, 4, 2, 64), ([33], 0, 2, 2, 80), ([64, 63, 65], 0, 4, 4, 128),
    ([127, 128, 129, 1, 300], 3, 4, 2, 64), ([257, 31], 0, 2, 2, 80), ([500, 0, 12], 9, 8, 1, 128), ([1030, 77], 0, 6, 2, 64),
    ([3] * 70 + [200] + [0] * 3 + [9] * 60, 4, 2, 2, 64),
])
@pytest.mark.parametrize("causal", [1, 0])
def test_packed_attention(lens, spare, hq, hkv, hd, causal):
    check_forward(lens, spare, hq, hkv, hd, causal)


@pytest.mark.parametrize("lens,hq,hkv,hd,causal", [
    ([2100, 515, 33], 64, 8, 128, 1),        # more work-groups than the chip holds at once
    ([1025, 900], 48, 48, 64, 1), ([577, 300, 257, 50], 32, 32, 80, 0), ([700, 2], 40, 40, 128, 0),
])
def test_packed_attention_large(lens, hq, hkv, hd, causal):
    check_forward(lens, 3, hq, hkv, hd, causal)


@pytest.mark.parametrize("lens,spare,hq,hkv,hd", [
    ([127, 128, 129, 1, 300, 0, 31], 3, 24, 6, 64), ([33, 257, 576, 0, 64], 0, 12, 4, 80), ([1030, 77, 1], 5, 18, 2, 128), ([1, 2, 3], 0, 200, 1, 128),
    ([3] * 70 + [200] + [0] * 3 + [9] * 60, 4, 8, 8, 64),
])
@pytest.mark.parametrize("causal", [1, 0])
def test_packed_attention_of_many_heads(lens, spare, hq, hkv, hd, causal):
    """Blocks of 128 queries, which small batches do not take."""
    check_forward(lens, spare, hq, hkv, hd, causal)


def test_packed_attention_of_many_requests():
    rng = np.random.default_rng(9)
    lens = rng.integers(0, 6, 4096)
    lens[777] = 200
    check_forward([int(v) for v in lens], 0, 2, 1, 64, 1)


@pytest.mark.parametrize("hd", [64, 80, 128])
def test_packed_attention_of_one_length_is_the_dense_attention(hd):
    """Peaked scores, whose running maximum moves in later tiles; also without a place for the log-sum-exp."""
    B, S, hq, hkv = 3, 190, 4, 2
    ob = check_forward([S] * B, 0, hq, hkv, hd, 1, scale=3.0, seed=1)
    rng = np.random.default_rng(S * B + hq + 1)
    bits, vals = prompt_inputs(rng, [S] * B, 0, hq, hkv, hd, 3.0)
    again, _ = run_forward(bits, sums([S] * B), S * B, hq, hkv, hd, 1, with_lse=False)
    assert np.array_equal(ob, again)
    q = dev_u16(bits)
    o = torch.zeros((B * S, hq * hd), dtype=torch.int16, device=DEV)
    assert sp.spk_attention(stream_ptr(), ptr(q), ptr(o), None, B, S, hq, hkv, hd, 1) == sp.SP_OK
    torch.cuda.synchronize()
    _, _, weight = P.attention_packed(vals, sums([S] * B), hq, hkv, hd, True)
    assert np.all(np.abs(bf16_vals(host_u16(o)) - bf16_vals(ob[:B * S])) <= 4 * STEP * weight.reshape(B * S, -1) + 2 * FP32 * weight.reshape(B * S, -1))


def test_packed_attention_keeps_requests_apart():
    """Infinite and NaN rows of one request leave the others' bits alone; the lengths are clamped to the buffer."""
    rng = np.random.default_rng(4)
    lens, hq, hkv, hd = [70, 40, 130], 2, 1, 128
    bits, _ = prompt_inputs(rng, lens, 0, hq, hkv, hd)
    cu = sums(lens)
    clean, _ = run_forward(bits, cu, 240, hq, hkv, hd, 1)
    bad = bits.copy()
    bad[70:110, ::3], bad[70:110, 1::3] = NAN16, 0x7F80
    dirty, _ = run_forward(bad, cu, 240, hq, hkv, hd, 1)
    assert np.array_equal(clean[:70], dirty[:70]) and np.array_equal(clean[110:240], dirty[110:240])
    assert not np.any(np.isfinite(bf16_vals(dirty[109])))
    # the last request reaches past the buffer: it ends with it
    past, _ = run_forward(bits, np.array([0, 70, 110, 5000]), 240, hq, hkv, hd, 1)
    assert np.array_equal(clean[:240], past[:240])


def test_packed_attention_lengths_that_do_not_ascend_stay_inside():
    rng = np.random.default_rng(6)
    bits, _ = prompt_inputs(rng, [200], 0, 2, 1, 64)
    for cu in ([0, 150, 60, 200], [-5, 10, 2 ** 31 - 1, 40], [200, 200, 200, 200], [90, 80, 70, 60]):
        ob, lse = run_forward(bits, np.array(cu), 200, 2, 1, 64, 1)
        assert np.all(ob[200] == 7) and lse[400] == 7


def check_backward(lens, spare, hq, hkv, hd, causal, seed=0):
    rng = np.random.default_rng(sum(lens) + hq + seed)
    bits, vals = prompt_inputs(rng, lens, spare, hq, hkv, hd)
    T, used, cu = bits.shape[0], int(sum(lens)), sums(lens)
    db, dv = rand_bf16(rng, (T, hq * hd), 0.5)
    db[used:], dv[used:] = NAN16, 0.0
    print(f"packed attention backward lens={lens} spare={spare} heads {hq}/{hkv} hd={hd} causal={causal}", flush=True)
    ob, lse = run_forward(bits, cu, T, hq, hkv, hd, causal)
    ob = ob[:T].copy()
    ob[used:] = NAN16
    q, c, o, d, ls = dev_u16(bits), i32(cu), dev_u16(ob), dev_u16(db), dev_f32(lse[:hq * T])
    scratch = torch.full((sp.spk_attention_packed_bwd_scratch_bytes(T, hq) + 4,), 0xFF, dtype=torch.uint8, device=DEV)
    dx = torch.full((T + 1, bits.shape[1]), 7, dtype=torch.int16, device=DEV)
    assert sp.spk_attention_packed_bwd(stream_ptr(), ptr(q), ptr(c), ptr(o), ptr(d), ptr(ls), ptr(scratch), ptr(dx), len(lens), T, hq, hkv,
                                       hd, causal) == sp.SP_OK
    torch.cuda.synchronize()
    out = host_u16(dx)
    assert np.all(out[used:] == 7) and bool((scratch[-4:] == 0xFF).all())
    got = bf16_vals(out[:used]).reshape(used, -1, hd)
    o64 = bf16_vals(ob).reshape(T, hq, hd)
    o64[used:] = 0
    want, rounded, entering = P.attention_packed_bwd(vals, cu, o64, dv, lse[:hq * T].reshape(hq, T).astype(np.float64), hq, hkv, hd, causal)
    tol = STEP * (rounded + np.abs(want)) + FP32 * entering
    off = np.abs(got - want[:used]) - tol[:used]
    assert off.max(initial=-1) <= 0, float(off.max())
    return vals, dv, got, tol[:used]


@pytest.mark.parametrize("lens,spare,hq,hkv,hd", [
    ([1], 0, 1, 1, 64), ([1, 0, 2], 2, 2, 1, 128), ([64, 63, 65], 0, 4, 4, 128), ([127, 128, 129, 1, 300], 3, 4, 2, 64), ([33, 257], 0, 2, 2, 80),
    ([500, 0, 12], 9, 8, 1, 128), ([3] * 70 + [200] + [0] * 3 + [9] * 20, 4, 2, 2, 64),
])
@pytest.mark.parametrize("causal", [1, 0])
def test_packed_attention_backward(lens, spare, hq, hkv, hd, causal):
    check_backward(lens, spare, hq, hkv, hd, causal)


@pytest.mark.parametrize("lens,spare,hq,hkv,hd", [
    ([127, 128, 129, 1, 300], 3, 32, 16, 64), ([1, 31, 32, 33, 64, 65, 127, 128, 129, 130] * 2, 1, 32, 32, 64),
    ([3] * 70 + [200] + [0] * 3 + [9] * 60, 4, 5, 5, 64), ([33, 257, 96], 0, 40, 20, 80), ([33, 257, 0, 130], 2, 20, 20, 80),
    ([500, 0, 12, 129], 9, 48, 24, 128), ([257, 0, 12, 129], 2, 60, 60, 128), ([130, 1, 70, 0, 0, 9], 0, 140, 70, 128),
])
@pytest.mark.parametrize("causal", [1, 0])
def test_packed_attention_backward_of_many_heads(lens, spare, hq, hkv, hd, causal):
    """Work-groups of more keys, which small batches do not take."""
    check_backward(lens, spare, hq, hkv, hd, causal)


@pytest.mark.parametrize("hd", [64, 128])
def test_packed_attention_behind_four_gigabytes(hd):
    """Rows, outputs and gradients whose offsets in bytes pass 32 bits: the last request of a long buffer, the rows in front of
    it belonging to nobody."""
    hq, hkv, n, far = 24, 24, 150, 2 ** 32 // (72 * hd * 2) + 3
    rng, T = np.random.default_rng(hd), far + n
    bits, vals = rand_bf16(rng, (n, 72 * hd))
    db, dv = rand_bf16(rng, (n, hq * hd), 0.5)
    qkv, do, o, dx = (torch.zeros((T, w * hd), dtype=torch.int16, device=DEV) for w in (72, hq, hq, 72))
    qkv[far:], do[far:] = dev_u16(bits), dev_u16(db)
    lse, cu = torch.zeros((hq, T), device=DEV), i32([far, T])
    scratch = torch.zeros(sp.spk_attention_packed_bwd_scratch_bytes(T, hq), dtype=torch.uint8, device=DEV)
    assert sp.spk_attention_packed(stream_ptr(), ptr(qkv), ptr(cu), ptr(o), ptr(lse), 1, T, hq, hkv, hd, 1) == sp.SP_OK
    assert sp.spk_attention_packed_bwd(stream_ptr(), ptr(qkv), ptr(cu), ptr(o), ptr(do), ptr(lse), ptr(scratch), ptr(dx), 1, T, hq, hkv,
                                       hd, 1) == sp.SP_OK
    torch.cuda.synchronize()
    assert not bool(o[:far].any()) and not bool(dx[:far].any())
    got, got_dx = bf16_vals(host_u16(o[far:])).reshape(n, hq, hd), bf16_vals(host_u16(dx[far:])).reshape(n, -1, hd)
    want, _, weight = P.attention_packed(vals, [0, n], hq, hkv, hd, True)
    assert np.all(np.abs(got - want) <= STEP * (weight + np.abs(want)) + FP32 * weight)
    want, rounded, entering = P.attention_packed_bwd(vals, [0, n], got, dv, lse[:, far:].cpu().numpy().astype(np.float64), hq, hkv, hd, True)
    assert np.all(np.abs(got_dx - want) <= STEP * (rounded + np.abs(want)) + FP32 * entering)


def test_packed_attention_backward_large():
    check_backward([1100, 400, 33], 0, 32, 8, 64, 1)
    check_backward([900, 5], 0, 24, 24, 128, 1)


def test_packed_attention_of_the_most_heads():
    """16384 query heads on one key/value head."""
    check_forward([1, 2], 0, 16384, 1, 64, 1)
    check_backward([1, 2], 0, 16384, 1, 64, 1)


def test_packed_attention_on_two_streams():
    """Two batches on two streams at once, several times over: the bits of each alone, forward and backward."""
    rng = np.random.default_rng(14)
    calls = []
    for lens, hq, hkv, hd in (([400, 33, 700], 8, 2, 128), ([90, 1, 513, 64], 8, 8, 64)):
        T, cu = sum(lens), i32(sums(lens))
        q, do = dev_u16(rand_bf16(rng, (T, (hq + 2 * hkv) * hd))[0]), dev_u16(rand_bf16(rng, (T, hq * hd), 0.5)[0])
        o, dx, lse = torch.zeros_like(do), torch.zeros_like(q), torch.zeros((hq, T), device=DEV)
        scratch = torch.zeros(sp.spk_attention_packed_bwd_scratch_bytes(T, hq), dtype=torch.uint8, device=DEV)

        def call(s, q=q, cu=cu, o=o, lse=lse, do=do, scratch=scratch, dx=dx, n=len(lens), T=T, hq=hq, hkv=hkv, hd=hd):
            assert sp.spk_attention_packed(s, ptr(q), ptr(cu), ptr(o), ptr(lse), n, T, hq, hkv, hd, 1) == sp.SP_OK
            assert sp.spk_attention_packed_bwd(s, ptr(q), ptr(cu), ptr(o), ptr(do), ptr(lse), ptr(scratch), ptr(dx), n, T, hq, hkv, hd, 1) == sp.SP_OK
        call(stream_ptr())
        torch.cuda.synchronize()
        calls.append((call, o, dx, o.clone(), dx.clone(), torch.cuda.Stream()))
    for _, o, dx, _, _, _ in calls:
        o.zero_(), dx.zero_()
    torch.cuda.synchronize()
    for _ in range(6):
        for call, *_, stream in calls:
            call(stream.cuda_stream)
    torch.cuda.synchronize()
    for _, o, dx, o1, dx1, _ in calls:
        assert torch.equal(o, o1) and torch.equal(dx, dx1)


def test_packed_attention_gradient_against_differences():
    """The kernels' gradient along a direction against differences of the 64-bit forward; the bound is the gradient's own,
    element by element, along that direction, and that of the o and lse which it was given (each off by its rounding:
    delta by at most 2 STEP sum |dO| A)."""
    lens, hq, hkv, hd = [19, 1, 40], 4, 2, 64
    vals, dv, got, tol = check_backward(lens, 0, hq, hkv, hd, 1, seed=3)
    rng = np.random.default_rng(8)
    cu, w = sums(lens), dv.reshape(-1, hq, hd)
    _, _, weight = P.attention_packed(vals, cu, hq, hkv, hd, True)
    x = np.abs(vals.reshape(60, -1, hd))
    for _ in range(3):
        u = rng.standard_normal(vals.shape)
        h = 1e-5
        loss = [(P.attention_packed(vals + s * h * u, cu, hq, hkv, hd, True)[0] * w).sum() for s in (1, -1)]
        along = np.abs(u).reshape(60, -1, hd)
        # dS = p (dP - delta) f: an error of delta reaches q through sum p |k| and k through sum p |q|, both under max |x| * sum p
        delta = (2 * STEP + FP32) * (np.abs(w) * weight).sum(-1).max() / np.sqrt(hd)
        reach = delta * x.max() * (along[:, :hq].sum() + along[:, hq:hq + hkv].sum() * hq // hkv)
        assert abs((loss[0] - loss[1]) / (2 * h) - (got * u.reshape(got.shape)).sum()) <= (tol * along).sum() + reach


# ---- the cache -----------------------------------------------------------------------------------------

def run_append(bits, slots, k8, v8, scales, bs, hq, hkv, hd, guard=True):
    T, blocks = len(slots), k8.shape[0]
    q, s = dev_u16(bits), i32(slots)
    pad = np.full(64, 0xA5, np.uint8)
    k, v = u8(np.concatenate([k8.reshape(-1), pad])), u8(np.concatenate([v8.reshape(-1), pad]))
    sc = dev_f32(np.concatenate([scales.reshape(-1), [7.0, 7.0]]))
    assert sp.spk_kv8_append(stream_ptr(), ptr(q), ptr(s), ptr(k), ptr(v), ptr(sc), T, blocks, bs, hq, hkv, hd) == sp.SP_OK
    torch.cuda.synchronize()
    k, v, sc = k.cpu().numpy(), v.cpu().numpy(), sc.cpu().numpy()
    assert np.all(k[-64:] == 0xA5) and np.all(v[-64:] == 0xA5) and np.all(sc[-2:] == 7)
    return k[:-64].reshape(k8.shape), v[:-64].reshape(v8.shape), sc[:-2].reshape(scales.shape)


def filled(rng, blocks, hkv, bs, hd):
    """A pool in use: every code but NaN, scales of several magnitudes."""
    k8 = rng.integers(0, 127, (blocks, hkv, bs, hd)) | (rng.integers(0, 2, (blocks, hkv, bs, hd)) << 7)
    v8 = rng.integers(0, 127, (blocks, hkv, hd, bs)) | (rng.integers(0, 2, (blocks, hkv, hd, bs)) << 7)
    return k8.astype(np.uint8), v8.astype(np.uint8), (2.0 ** rng.integers(-14, 2, (blocks, hkv, 2))).astype(np.float32)


def check_append(rng, bits, vals, slots, bs, hq, hkv, hd, blocks):
    k8, v8, sc = filled(rng, blocks, hkv, bs, hd)
    got = run_append(bits, slots, k8, v8, sc, bs, hq, hkv, hd)
    with np.errstate(invalid="ignore"):
        want = P.kv8_append(vals, slots, k8, v8, sc, bs, hq, hkv, hd)
    for a, b, name in zip(got, want, ("k8", "v8", "scales")):
        assert np.array_equal(a, b), (name, int((a != b).sum()), a.size)
    return got


@pytest.mark.parametrize("bs", [16, 32, 64])
@pytest.mark.parametrize("hd,hq,hkv", [(64, 4, 2), (128, 3, 3), (128, 8, 1)])
def test_append(bs, hd, hq, hkv):
    """Prompts from one token to several blocks, requests that go on inside a block, single tokens, rows without a slot."""
    rng = np.random.default_rng(bs + hd + hq)
    lens = np.array([1, bs, 3 * bs + 5, 0, 1, 2 * bs - 1, 7, 1])
    cached = np.array([0, 0, 0, 9, bs - 1, 5, 3 * bs, bs + 2])
    width = 8
    table, free = make_tables(rng, cached, width, bs, 60)
    T = int(lens.sum()) + 3
    _, _, slots, _, info = P.batch_plan(lens, cached, free, table, T, bs)
    assert info[3] == 0
    bits, vals = rand_bf16(rng, (T, (hq + 2 * hkv) * hd), 2.0)
    mag = 2.0 ** rng.integers(-6, 4, (T, hq + 2 * hkv))
    bits_f = (vals.reshape(T, -1, hd) * mag[..., None]).astype(np.float32)
    from paper_2410_08791_amd import synth
    bits = synth.f32_to_bf16_bits(bits_f).reshape(T, -1)
    check_append(rng, bits, bf16_vals(bits), slots, bs, hq, hkv, hd, 60)


@pytest.mark.parametrize("T,hkv,hd,bs", [(40, 32, 128, 16), (300, 32, 64, 32), (1200, 8, 128, 64)])
def test_append_many_tokens(T, hkv, hd, bs):
    """Few and many rows per wave; slots outside the pool are skipped."""
    rng = np.random.default_rng(T)
    blocks = -(-T // bs) + 4
    slots = (bs // 2 + np.arange(T)).astype(np.int32)
    slots[T // 2:] += bs                                    # a block is left out
    slots[5], slots[T - 1] = -1, blocks * bs
    slots[T // 3] = -2 ** 31
    bits, vals = rand_bf16(rng, (T, (hkv + 2 * hkv) * hd))
    check_append(rng, bits, vals, slots, bs, hkv, hkv, hd, blocks)


def test_append_runs_of_one_block_are_stored_in_order():
    """The same slot twice, slots that go back, rows of other blocks and skipped rows in between: one after the other."""
    rng = np.random.default_rng(6)
    slots = np.array([3, 4, 4, 5, 20, -1, 6, 2, 3, 21, 22, 9, 40, 41, 9, 9] + [-1] * 40 + [23, 42, 10, 43])
    slots = np.concatenate([slots, [-1] * 62, [11, 44], 48 + np.arange(16), 48 + np.arange(4)]).astype(np.int32)
    for hkv in (1, 40):                                     # one row and several rows per wave
        bits, _ = rand_bf16(rng, (len(slots), 3 * hkv * 64))
        vals = bf16_vals(bits) * 2.0 ** rng.integers(-3, 4, (len(slots), 1))
        from paper_2410_08791_amd import synth
        bits = synth.f32_to_bf16_bits(vals.astype(np.float32))
        check_append(rng, bits, bf16_vals(bits), slots, 16, hkv, hkv, 64, 4)


@pytest.mark.parametrize("hd,bs", [(64, 16), (128, 64), (128, 32)])
def test_append_single_tokens_of_many_requests(hd, bs):
    """A row per request at any place of its block, with so many heads that work-groups take 64 rows; blocks in no order."""
    rng = np.random.default_rng(hd + bs)
    T, hkv, blocks = 230, 40, 260
    slots = (rng.permutation(blocks)[:T] * bs + rng.integers(0, bs, T)).astype(np.int32)
    slots[::50] = -1
    bits, _ = rand_bf16(rng, (T, 3 * hkv * hd))
    check_append(rng, bits, bf16_vals(bits), slots, bs, hkv, hkv, hd, blocks)


def test_append_runs_of_one_block_with_many_heads():
    """The runs above by work-groups of 64 rows: few blocks (all waves work a run together) and many (each wave its own)."""
    rng = np.random.default_rng(16)
    runs = np.array([3, 4, 4, 5, 20, -1, 6, 2, 3, 21, 22, 9, 40, 41, 9, 9] + [-1] * 40 + [23, 42, 10, 43] + [-1] * 62 + [11, 44])
    many = np.concatenate([runs, 48 + np.arange(16), [70, 80, 96, 112, 71, 81, 97, 113, 72, 82], [60] * 3, 128 + np.arange(48), [83]])
    few = np.concatenate([[3, 4, 4, 5], [-1] * 30, [6, 7, 7, 2, 3], [-1] * 62, [4, 5], 16 + np.arange(16), [-1] * 50, 30 + np.arange(20)])
    for slots in (many, few):
        bits, _ = rand_bf16(rng, (len(slots), 3 * 64 * 64))
        check_append(rng, bits, bf16_vals(bits), slots.astype(np.int32), 16, 64, 64, 64, 14)


def test_append_edge_values():
    """Zeros, the smallest and largest bf16 values, ties between codes, infinities and NaN."""
    rng = np.random.default_rng(2)
    hq = hkv = 1
    hd, bs, T = 64, 16, 16 * 9
    bits, _ = rand_bf16(rng, (T, 3 * hd))
    bits[0:16] = 0
    bits[16:32] &= 0x807F                                   # subnormal bf16
    bits[32:48] = (bits[32:48] & 0x80FF) | 0x7F00           # the largest binade
    bits[48:64, :] = rng.choice(np.array([0x7F80, 0xFF80, 0x7FC1], np.uint16), (16, 3 * hd))      # nothing finite
    bits[64:80, ::5] = 0x7F80
    bits[80, 3], bits[85, 100] = 0x7FC1, 0xFF80
    bits[96:112] = (bits[96:112] & 0x8008) | 0x43E0         # 448 = 0x43E0 and 464: next to the border of a scale
    bits[112:128] = (bits[112:128] & 0x800F) | 0x3F80       # values between codes, many ties
    bits[128:144, 1:] &= 0x83FF                             # one large value, the others far below the normal codes
    slots = np.arange(T, dtype=np.int32)
    got = check_append(rng, bits, bf16_vals(bits), slots, bs, hq, hkv, hd, 9)
    assert got[2][0, 0, 0] == 2.0 ** -126


def test_append_one_by_one_grows_the_scale():
    """Single tokens of rising magnitude into the same blocks: every step re-codes what was there."""
    rng = np.random.default_rng(3)
    hq, hkv, hd, bs = 2, 2, 64, 16
    k8, v8, sc = filled(rng, 4, hkv, bs, hd)
    want = (k8, v8, sc.astype(np.float64))
    for step in range(bs + 3):
        slots = np.array([step, 3 * bs - 1 if step == 2 else -1, 32 + step if step < bs else -1], np.int32)
        bits, _ = rand_bf16(rng, (3, 6 * hd))
        from paper_2410_08791_amd import synth
        bits = synth.f32_to_bf16_bits((bf16_vals(bits) * 1.7 ** rng.integers(0, step + 1)).astype(np.float32))
        if step == 2:
            slots[2] = -1
        k8, v8, sc = run_append(bits, slots, k8, v8, sc, bs, hq, hkv, hd)
        want = P.kv8_append(bf16_vals(bits), slots, *want, bs, hq, hkv, hd)
        for a, b in zip((k8, v8, sc), want):
            assert np.array_equal(a, b), step


def run_cache_attention(qbits, k8, v8, scales, table, kv_len, bs, hq, hkv, hd):
    B, blocks = len(kv_len), k8.shape[0]
    mb = table.shape[1]
    q, k, v, sc, t, n = dev_u16(qbits), u8(k8), u8(v8), dev_f32(scales), i32(table), i32(kv_len)
    need = sp.spk_kv8_attention_scratch_bytes(B, mb, bs, hq, hkv, hd)
    scratch = torch.full((need + 16,), 0xFF, dtype=torch.uint8, device=DEV)
    o = torch.full((B + 1, hq * hd), 7, dtype=torch.int16, device=DEV)
    assert sp.spk_kv8_attention(stream_ptr(), ptr(q), ptr(k), ptr(v), ptr(sc), ptr(t), ptr(n), ptr(o), ptr(scratch) if need else None, B,
                                blocks, bs, mb, hq, hkv, hd) == sp.SP_OK
    torch.cuda.synchronize()
    assert bool((scratch[need:] == 0xFF).all())
    out = host_u16(o)
    assert np.all(out[B] == 7)
    return bf16_vals(out[:B]).reshape(B, hq, hd)


def check_cache_attention(lens, bs, hq, hkv, hd, extra_width=0, seed=0, bad=()):
    rng = np.random.default_rng(sum(lens) + hq + bs + seed)
    width = max(-(-max(lens) // bs), 1) + extra_width
    blocks = sum(-(-v // bs) for v in lens) + 3
    table, _ = make_tables(rng, lens, width, bs, blocks, unowned=2 ** 31 - 1)
    k8, v8, sc = filled(rng, blocks, hkv, bs, hd)
    sc = (2.0 ** rng.integers(-9, -6, sc.shape)).astype(np.float32)       # codes up to 448: values around 1
    for r, v in enumerate(lens):                                          # NaN behind a request's last position
        if v % bs:
            k8[table[r, v // bs], :, v % bs:], v8[table[r, v // bs], :, :, v % bs:] = 0x7F, 0xFF
    for r, j, value in bad:
        table[r, j] = value
    print(f"cache attention lens={lens[:8]} bs={bs} heads {hq}/{hkv} hd={hd}", flush=True)
    qbits, q = rand_bf16(rng, (len(lens), (hq + 2 * hkv) * hd), 0.3)
    got = run_cache_attention(qbits, k8, v8, sc, table, lens, bs, hq, hkv, hd)
    want, weight = P.kv8_attention(q[:, :hq * hd].reshape(-1, hq, hd), k8, v8, sc.astype(np.float64), table, lens, bs)
    off = np.abs(got - want) - (STEP * (weight + np.abs(want)) + FP32 * weight)
    assert off.max() <= 0, float(off.max())
    return got


@pytest.mark.parametrize("bs", [16, 32, 64])
@pytest.mark.parametrize("hq,hkv,hd", [(2, 2, 64), (4, 1, 128), (16, 1, 64), (17, 1, 128), (6, 2, 128), (40, 1, 64), (8, 8, 128)])
def test_cache_attention(bs, hq, hkv, hd):
    check_cache_attention([1, 15, 16, 17, 0, 63, 64, 65, 200, 255, 257], bs, hq, hkv, hd)


@pytest.mark.parametrize("lens,bs,hq,hkv,hd,extra", [
    ([5000, 3], 16, 8, 2, 128, 0), ([700, 4099, 0, 1], 64, 4, 4, 64, 90), ([20000], 32, 2, 1, 128, 0), ([300] * 40, 16, 8, 8, 64, 40),
    ([1, 1025, 511, 512, 513], 32, 64, 8, 128, 7),
    ([900, 1, 64] * 24, 16, 8, 8, 64, 7),                        # heads and requests enough: no pieces
    ([767, 768, 769, 1] * 10, 64, 16, 8, 128, 60),
])
def test_cache_attention_in_pieces(lens, bs, hq, hkv, hd, extra):
    """Positions shared out over work-groups; pieces that nobody fills."""
    check_cache_attention(lens, bs, hq, hkv, hd, extra)


def test_cache_attention_of_the_most_requests():
    """65535 requests of at most 20 positions, which share blocks; some of the rows against the oracle."""
    rng = np.random.default_rng(65)
    B, bs, blocks = 65535, 16, 50
    table, lens = rng.integers(0, blocks, (B, 2)).astype(np.int32), rng.integers(0, 21, B)
    k8, v8, sc = filled(rng, blocks, 1, bs, 64)
    sc[:] = 2.0 ** -8
    qbits, q = rand_bf16(rng, (B, 4 * 64), 0.3)
    got = run_cache_attention(qbits, k8, v8, sc, table, lens, bs, 2, 1, 64)
    some = np.concatenate([np.arange(40), rng.integers(0, B, 100), B - 1 - np.arange(40)])
    want, weight = P.kv8_attention(q[some, :128].reshape(-1, 2, 64), k8, v8, sc.astype(np.float64), table[some], lens[some], bs)
    assert np.all(np.abs(got[some] - want) <= STEP * (weight + np.abs(want)) + FP32 * weight)


def test_cache_behind_four_gigabytes():
    """Blocks whose offsets in bytes pass 32 bits, in both halves of the cache."""
    hq, hkv, hd, bs = 8, 8, 128, 64
    block = hkv * bs * hd
    blocks = 2 ** 32 // block + 5
    k8, v8 = (torch.zeros(blocks * block, dtype=torch.uint8, device=DEV) for _ in range(2))
    scales = torch.zeros(blocks * hkv * 2, device=DEV)
    table = np.array([[blocks - 1, 3], [blocks - 3, blocks - 2]])
    lens = np.array([70, 128])
    _, _, slots, _, _ = P.batch_plan(lens, [0, 0], table.reshape(-1), np.zeros((2, 2)), 198, bs)
    rng = np.random.default_rng(5)
    bits, vals = rand_bf16(rng, (198, (hq + 2 * hkv) * hd))
    q, s = dev_u16(bits), i32(slots)
    assert sp.spk_kv8_append(stream_ptr(), ptr(q), ptr(s), ptr(k8), ptr(v8), ptr(scales), 198, blocks, bs, hq, hkv, hd) == sp.SP_OK
    torch.cuda.synchronize()
    used = [int(b) for b in table.reshape(-1)]
    near = {b: i for i, b in enumerate(used)}
    z = np.zeros((4, hkv, bs, hd), np.uint8), np.zeros((4, hkv, hd, bs), np.uint8), np.zeros((4, hkv, 2))
    want = P.kv8_append(vals, np.array([near[v // bs] * bs + v % bs for v in map(int, slots)]), *z, bs, hq, hkv, hd)
    for pool, w in zip((k8, v8, scales), want):
        for b, i in near.items():
            assert np.array_equal(pool.reshape(blocks, -1)[b].cpu().numpy(), w[i].reshape(-1)), b
        assert not bool(pool.reshape(blocks, -1)[4:blocks - 4].any())
    qbits, qv = rand_bf16(rng, (2, (hq + 2 * hkv) * hd), 0.3)
    o = torch.zeros((2, hq * hd), dtype=torch.int16, device=DEV)
    x, t, n = dev_u16(qbits), i32(table), i32(lens)
    assert sp.spk_kv8_attention_scratch_bytes(2, 2, bs, hq, hkv, hd) == 0
    assert sp.spk_kv8_attention(stream_ptr(), ptr(x), ptr(k8), ptr(v8), ptr(scales), ptr(t), ptr(n), ptr(o), None, 2, blocks, bs, 2, hq, hkv,
                                hd) == sp.SP_OK
    torch.cuda.synchronize()
    ref, weight = P.kv8_attention(qv[:, :hq * hd].reshape(2, hq, hd), *want, np.array([[0, 1], [2, 3]]), lens, bs)
    got = bf16_vals(host_u16(o)).reshape(2, hq, hd)
    assert np.all(np.abs(got - ref) <= STEP * (weight + np.abs(ref)) + FP32 * weight)


def test_cache_attention_without_positions_and_bad_entries():
    """Blocks outside the pool weigh nothing; a request that is left with nothing gives zeros."""
    got = check_cache_attention([40, 0, 70, 33], 16, 4, 2, 64, extra_width=2, bad=[(0, 1, -1), (2, 0, 10 ** 6), (2, 4, -2 ** 31), (3, 0, -7), (3, 1, 99),
                                                                                  (3, 2, 2 ** 31 - 1)])
    assert not got[1].any() and not got[3].any() and got[0].any() and got[2].any()
    rng = np.random.default_rng(1)
    k8, v8, sc = filled(rng, 3, 1, 16, 64)
    qbits, _ = rand_bf16(rng, (2, 3 * 64))
    assert not run_cache_attention(qbits, k8, v8, sc, np.zeros((2, 4), np.int32), np.array([0, -3]), 16, 1, 1, 64).any()
    # more positions than the table has entries: those of the table
    a = run_cache_attention(qbits, k8, v8, sc, np.array([[0, 1], [2, 0]]), np.array([32, 32]), 16, 1, 1, 64)
    b = run_cache_attention(qbits, k8, v8, sc, np.array([[0, 1], [2, 0]]), np.array([33, 2 ** 31 - 1]), 16, 1, 1, 64)
    assert np.array_equal(a, b)


def test_cache_attention_nan_stays_with_its_request():
    rng = np.random.default_rng(12)
    k8, v8, sc = filled(rng, 8, 2, 16, 64)
    sc[:] = 2.0 ** -8
    table = np.arange(8).reshape(2, 4)
    qbits, _ = rand_bf16(rng, (2, 8 * 64), 0.3)
    clean = run_cache_attention(qbits, k8, v8, sc, table, np.array([50, 60]), 16, 4, 2, 64)
    v8[1, 0, 7, 3] = 0x7F                                    # a value of request 0, kv head 0, element 7
    got = run_cache_attention(qbits, k8, v8, sc, table, np.array([50, 60]), 16, 4, 2, 64)
    assert np.all(np.isnan(got[0, :2, 7]))
    got[0, :2, 7] = clean[0, :2, 7]
    assert np.array_equal(got, clean)
    k8[1, 1, 3, 7] = 0xFF
    got = run_cache_attention(qbits, k8, v8, sc, table, np.array([50, 60]), 16, 4, 2, 64)
    assert np.all(np.isnan(got[0, 2:])) and np.array_equal(got[1], clean[1])


@pytest.mark.parametrize("hd,hq,hkv,n,bs,width", [
    (64, 4, 2, 40, 16, 4),              # one piece
    (128, 4, 2, 900, 64, 16),           # pieces, added up by a wave per head
    (128, 4, 1, 5000, 64, 80),          # by four
])
def test_cache_attention_of_scores_that_are_all_minus_infinity(hd, hq, hkv, n, bs, width):
    """An infinite query on keys of one sign: 0 / 0, as the definition has it.  Requests without positions give zeros whatever their
    query is; a stretch of scores of -inf, longer than a piece, weighs nothing beside finite ones."""
    rng = np.random.default_rng(n)
    lens, per = [n, n, 0, n], -(-n // bs)
    table = np.zeros((4, width), np.int32)
    table[:, :per] = np.arange(4 * per).reshape(4, per)
    table[0, per:] = -1
    k8, v8, sc = filled(rng, 4 * per, hkv, bs, hd)
    sc[:] = 2.0 ** -8
    k8[:, :, :, 0] = 0xFE                                    # -448: the largest code
    k8[table[3, per - 1], :, :, 0] = 0                       # request 3: but the last block's
    qbits, q = rand_bf16(rng, (4, (hq + 2 * hkv) * hd), 0.3)
    qbits.reshape(4, -1, hd)[:3, 1, 0] = 0x7F80              # head 1 of the others
    qbits.reshape(4, -1, hd)[3, :hq, 0] = 0x7F7F             # sums that pass fp32: finite in 64 bits, and their weight is 0 there too
    got = run_cache_attention(qbits, k8, v8, sc, table, lens, bs, hq, hkv, hd)
    want, weight = P.kv8_attention(bf16_vals(qbits)[:, :hq * hd].reshape(4, hq, hd)[[0, 1, 3]], k8, v8, sc.astype(np.float64), table[[0, 1, 3]],
                                   [n] * 3, bs)
    assert not got[2].any()
    got = got[[0, 1, 3]]
    assert np.all(np.isnan(got[:2, 1])) and np.all(np.isnan(want[:2, 1]))
    got[:2, 1] = want[:2, 1] = weight[:2, 1] = 0
    off = np.abs(got - want) - (STEP * (weight + np.abs(want)) + FP32 * weight)
    assert off.max() <= 0, float(off.max())


def test_arrays_side_by_side():
    """Inputs and outputs that share one allocation, end to end, are no overlap: the bits of arrays of their own."""
    rng = np.random.default_rng(17)
    lens, hq, hkv, hd, bs, blocks = [70, 1, 57], 4, 2, 64, 16, 12
    T, cu, n = 128, i32(sums(lens)), 3
    bits, db = rand_bf16(rng, (T, 8 * hd))[0], rand_bf16(rng, (T, hq * hd), 0.5)[0]
    sizes = [("qkv", bits.nbytes), ("o", db.nbytes), ("dO", db.nbytes), ("lse", 4 * hq * T), ("scratch", 4 * hq * T), ("dqkv", bits.nbytes),
             ("slots", 4 * T), ("k8", blocks * bs * hkv * hd), ("v8", blocks * bs * hkv * hd), ("scales", blocks * hkv * 8), ("table", 64), ("kv_len", 16),
             ("step", n * hq * hd * 2)]
    outs = []
    for gap in (0, 256):
        pool = torch.zeros(sum(v + gap for _, v in sizes), dtype=torch.uint8, device=DEV)
        at, a = 0, {}
        for name, size in sizes:
            a[name] = pool[at:at + size]
            at += size + gap
        for name, v in (("qkv", bits), ("dO", db), ("slots", np.concatenate([np.arange(70), [80], 96 + np.arange(57)]).astype(np.int32)),
                        ("table", np.array([[0, 1, 2, 3, 4], [5] * 5, [6, 7, 8, 9, 6]], np.int32)), ("kv_len", np.array([70, 1, 57], np.int32))):
            v = torch.from_numpy(np.ascontiguousarray(v).view(np.uint8).reshape(-1)).to(DEV)
            a[name][:v.numel()] = v
        p = {k: ptr(v) for k, v in a.items()}
        assert sp.spk_attention_packed(stream_ptr(), p["qkv"], ptr(cu), p["o"], p["lse"], n, T, hq, hkv, hd, 1) == sp.SP_OK
        assert sp.spk_attention_packed_bwd(stream_ptr(), p["qkv"], ptr(cu), p["o"], p["dO"], p["lse"], p["scratch"], p["dqkv"], n, T, hq, hkv,
                                           hd, 1) == sp.SP_OK
        assert sp.spk_kv8_append(stream_ptr(), p["qkv"], p["slots"], p["k8"], p["v8"], p["scales"], T, blocks, bs, hq, hkv, hd) == sp.SP_OK
        assert sp.spk_kv8_attention_scratch_bytes(n, 5, bs, hq, hkv, hd) == 0
        assert sp.spk_kv8_attention(stream_ptr(), p["qkv"], p["k8"], p["v8"], p["scales"], p["table"], p["kv_len"], p["step"], None, n, blocks, bs,
                                    5, hq, hkv, hd) == sp.SP_OK
        torch.cuda.synchronize()
        outs.append({k: v.clone() for k, v in a.items()})
    for name, _ in sizes:
        assert torch.equal(outs[0][name], outs[1][name]) and bool(outs[0][name].any()), name


# ---- together --------------------------------------------------------------------------------------------

class Server:
    """Requests through one layer's cache, step by step: plan, attention over the prompts, append, attention over the cache."""

    def __init__(self, n, width, bs, hq, hkv, hd, blocks, max_tokens):
        self.n, self.width, self.bs, self.hq, self.hkv, self.hd, self.blocks, self.rows = n, width, bs, hq, hkv, hd, blocks, max_tokens
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
        self.table, self.cu, self.slots, self.info, self.lens = z(n, width) - 1, z(n + 1), z(max_tokens), z(4), z(n)
        self.kv = [z(n), z(n)]
        self.k8, self.v8 = (torch.full((blocks * hkv * bs * hd,), 0x7F, dtype=torch.uint8, device=DEV) for _ in range(2))
        self.scales = torch.full((blocks * hkv * 2,), float("nan"), device=DEV)
        self.free = torch.arange(blocks - 1, -1, -1, dtype=torch.int32, device=DEV)
        self.taken = 0
        self.o = torch.zeros((max_tokens, hq * hd), dtype=torch.int16, device=DEV)
        self.scratch = torch.zeros(sp.spk_kv8_attention_scratch_bytes(n, width, bs, hq, hkv, hd) + 16, dtype=torch.uint8, device=DEV)

    def step(self, qkv, decode):
        s = stream_ptr()
        old, new = self.kv
        free = self.free[self.taken:]
        assert sp.spk_batch_plan(s, ptr(self.lens), ptr(old), ptr(free), free.numel(), ptr(self.table), self.width, ptr(self.cu), ptr(new),
                                 ptr(self.slots), self.rows, ptr(self.info), self.n, self.bs) == sp.SP_OK
        assert sp.spk_kv8_append(s, ptr(qkv), ptr(self.slots), ptr(self.k8), ptr(self.v8), ptr(self.scales), self.rows, self.blocks, self.bs,
                                 self.hq, self.hkv, self.hd) == sp.SP_OK
        if decode:
            assert sp.spk_kv8_attention(s, ptr(qkv), ptr(self.k8), ptr(self.v8), ptr(self.scales), ptr(self.table), ptr(new), ptr(self.o),
                                        ptr(self.scratch), self.n, self.blocks, self.bs, self.width, self.hq, self.hkv, self.hd) == sp.SP_OK
        else:
            assert sp.spk_attention_packed(s, ptr(qkv), ptr(self.cu), ptr(self.o), None, self.n, self.rows, self.hq, self.hkv, self.hd, 1) == sp.SP_OK
        self.kv.reverse()


def test_requests_of_different_lengths_generate_together():
    """Prompts, then tokens one by one, on a stream of its own; every output against attention over the values that the cache
    holds for what was appended, and the whole again from a captured graph, replayed with eager work in between."""
    hq, hkv, hd, bs, lens = 6, 2, 64, 16, [1, 37, 16, 90]
    n, T, steps = len(lens), sum(lens), 20
    rng = np.random.default_rng(21)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sv = Server(n, 8, bs, hq, hkv, hd, 40, T)
        bits, vals = rand_bf16(rng, (T, (hq + 2 * hkv) * hd))
        sv.lens.copy_(i32(lens))
        sv.step(dev_u16(bits), False)
        cu = sums(lens)
        want, _, weight = P.attention_packed(vals, cu, hq, hkv, hd, True)
        got = bf16_vals(host_u16(sv.o)).reshape(T, hq, hd)
        assert np.all(np.abs(got - want) <= STEP * (weight + np.abs(want)) + FP32 * weight)
        held = P.kv8_append(vals, sv.slots.cpu().numpy(), np.full((40, hkv, bs, hd), 0x7F, np.uint8), np.full((40, hkv, hd, bs), 0x7F, np.uint8),
                            np.full((40, hkv, 2), np.nan), bs, hq, hkv, hd)
        sv.taken += int(sv.info[1])
        sv.lens.fill_(1)
        sv.rows = n
        for step in range(steps):
            bits, vals = rand_bf16(rng, (n, (hq + 2 * hkv) * hd))
            sv.step(dev_u16(bits), True)
            assert list(sv.info.cpu())[0::3] == [n, 0]
            sv.taken += int(sv.info[1])
            kv = sv.kv[0].cpu().numpy()
            assert np.array_equal(kv, np.array(lens) + step + 1)
            held = P.kv8_append(vals, sv.slots.cpu().numpy()[:n], *held, bs, hq, hkv, hd)
            want, weight = P.kv8_attention(vals[:, :hq * hd].reshape(n, hq, hd), *held, sv.table.cpu().numpy(), kv, bs)
            got = bf16_vals(host_u16(sv.o[:n])).reshape(n, hq, hd)
            assert np.all(np.abs(got - want) <= STEP * (weight + np.abs(want)) + FP32 * weight), step
        used = sorted(int(b) for r in range(n) for b in sv.table[r, :-(-int(kv[r]) // bs)])
        assert len(set(used)) == len(used) == sv.taken
        assert np.array_equal(sv.k8.cpu().numpy().reshape(held[0].shape)[used], held[0][used])


def test_captured_step_is_the_eager_step():
    """One decode step (plan, append, attention in pieces) captured and replayed on new tokens and lengths, with eager work and
    synchronizations between the replays."""
    hq, hkv, hd, bs, n = 8, 2, 128, 32, 5
    rng = np.random.default_rng(33)
    kv0 = np.array([700, 1, 64, 1023, 400], np.int32)
    servers = []
    for _ in range(2):
        sv = Server(n, 40, bs, hq, hkv, hd, 90, n)
        sv.lens.fill_(1)
        sv.kv[0].copy_(i32(kv0))
        at = 0
        for r in range(n):
            held = -(-int(kv0[r]) // bs)
            sv.table[r, :held] = sv.free[at:at + held]
            at += held
        sv.taken = at
        k8, v8, _ = filled(np.random.default_rng(1), 90, hkv, bs, hd)
        sv.k8.copy_(u8(k8.reshape(-1)))
        sv.v8.copy_(u8(v8.reshape(-1)))
        sv.scales.fill_(2.0 ** -8)
        servers.append(sv)
    eager, cap = servers
    qkv = torch.zeros((n, (hq + 2 * hkv) * hd), dtype=torch.int16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            cap.step(qkv, True)
    torch.cuda.current_stream().wait_stream(side)
    old, new = cap.kv[1], cap.kv[0]                    # what the captured step reads and writes
    for step in range(4):
        bits, _ = rand_bf16(rng, (n, (hq + 2 * hkv) * hd))
        x = dev_u16(bits)
        qkv.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        eager.step(x, True)
        torch.cuda.synchronize()
        for name in ("cu", "slots", "info", "table", "k8", "v8", "o"):
            assert torch.equal(getattr(eager, name), getattr(cap, name)), (name, step)
        assert torch.equal(eager.scales.view(torch.int32), cap.scales.view(torch.int32)) and torch.equal(eager.kv[0], new)
        taken = int(eager.info[1])
        # the next step's free blocks: the captured call reads the same list from its front
        eager.free = torch.cat([eager.free[:eager.taken], eager.free[eager.taken + taken:], eager.free[eager.taken:eager.taken + taken]])
        cap.free.copy_(eager.free)
        old.copy_(new)


def test_captured_training_step_takes_other_lengths():
    """Forward and backward captured once, replayed on other lengths and rows, with eager work and synchronizations between the
    replays: the eager bits."""
    hq, hkv, hd, T, n = 8, 2, 128, 700, 5
    rng = np.random.default_rng(44)
    buf = {}
    for who in ("eager", "captured"):
        z = lambda *shape, dtype=torch.int16: torch.zeros(shape, dtype=dtype, device=DEV)  # noqa: E731
        buf[who] = dict(qkv=z(T, 12 * hd), do=z(T, hq * hd), o=z(T, hq * hd), dx=z(T, 12 * hd), lse=z(hq, T, dtype=torch.float32), cu=z(n + 1, dtype=torch.int32),
                        scratch=z(sp.spk_attention_packed_bwd_scratch_bytes(T, hq), dtype=torch.uint8))

    def step(b):
        assert sp.spk_attention_packed(stream_ptr(), ptr(b["qkv"]), ptr(b["cu"]), ptr(b["o"]), ptr(b["lse"]), n, T, hq, hkv, hd, 1) == sp.SP_OK
        assert sp.spk_attention_packed_bwd(stream_ptr(), ptr(b["qkv"]), ptr(b["cu"]), ptr(b["o"]), ptr(b["do"]), ptr(b["lse"]), ptr(b["scratch"]),
                                           ptr(b["dx"]), n, T, hq, hkv, hd, 1) == sp.SP_OK
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(buf["captured"])
    torch.cuda.current_stream().wait_stream(side)
    for lens in ([700, 0, 0, 0, 0], [1, 300, 2, 33, 64], [100, 100, 100, 100, 100], [0, 0, 0, 0, 1]):
        q, d = dev_u16(rand_bf16(rng, (T, 12 * hd))[0]), dev_u16(rand_bf16(rng, (T, hq * hd), 0.5)[0])
        for b in buf.values():
            b["qkv"].copy_(q), b["do"].copy_(d), b["cu"].copy_(i32(sums(lens)))
            for name in ("o", "dx"):
                b[name].fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        step(buf["eager"])
        torch.cuda.synchronize()
        used = sum(lens)
        for name in ("o", "dx"):
            a, b = buf["eager"][name], buf["captured"][name]
            assert torch.equal(a, b) and bool((a[used:] == 7).all()) and bool((a[:used] != 7).any()), (lens, name)
