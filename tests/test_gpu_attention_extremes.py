"""The attention half of a layer at the ends of what its arguments may be: steps beyond fp16, scores far beyond what a softmax
needs, against 64-bit numpy."""
import numpy as np
import pytest

from tests import attention_plain as plain
from tests import test_gpu_attention as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2603_27914_amd import binding

    binding.lib()
    return torch, binding


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---- append


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("normed", [False, True])
def test_rows_far_beyond_the_largest_step_keep_their_signs(gpu, D, normed):
    """Steps stop at 65504, digits at -8 and 7: rows of 1e12 to 1e24 beside ordinary ones, in one wavefront with them, as they come (fp32)
    or by their norm's weights (fp16 keys)."""
    torch, binding = gpu
    rng = np.random.default_rng(D)
    T, H = 48, 3
    size = np.where(rng.random((2, T, H, 1)) < 0.3, 1.0, 10.0 ** rng.uniform(12, 24, (2, T, H, 1)))
    size[0, 0], size[1, :8] = 1e16, 1e16  # whole wavefronts of them
    k, v = (rng.standard_normal((2, T, H, D)) * size).astype(np.float32)
    weight = None
    if normed:
        k, weight = rng.standard_normal((T, H, D)).astype(np.float16), (10.0 ** rng.uniform(14, 18, D)).astype(np.float32)
        v = k
    cache = binding.alloc_cache(2, 32, H, D)
    slots = rng.permutation(64)[:T].astype(np.int64)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.itq3s_cache_append(None, dev(torch, k.reshape(T, -1)), dev(torch, v.reshape(T, -1)), None, None, cache, dev(torch, slots), k_norm=dev(torch, weight) if normed else None, status_flags=flags)
    want = plain.PlainCache(2, 32, H, D)
    want.write(slots, plain.rotated(k.reshape(T, -1), D, weight).reshape(T, H, D), v.astype(np.float64))
    assert np.array_equal(cache.data.cpu().numpy(), want.data)
    assert int(flags.item()) == binding.FLAG_SCALE_SAT


@pytest.mark.parametrize("kind", ["turned", "normed"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_keys_in_fp16_are_rounded_once(gpu, D, kind):
    """Products of fp32 keys and an fp32 factor are exact in 64 bits, and one in 2^14 lies so near a border of fp16 that a rounding to
    fp32 on the way would move it there.  Every value is the 64-bit one's nearest."""
    torch, binding = gpu
    rng = np.random.default_rng(D)
    T, H = 4096, 512 // D
    k = rng.standard_normal((T, H * D)).astype(np.float32)
    if kind == "turned":  # by no angle, with a gain
        gain = np.float32(1.2345678)
        _, got = binding.itq3s_cache_append(None, dev(torch, k), None, torch.zeros(T, dtype=torch.int32, device="cuda"), binding.itq3s_rope_frequencies(D).cuda(), head_dim=D, gain=float(gain))
        want = k.astype(np.float64) * np.float64(gain)
    else:  # rows of +-1, whose norm is 1 with no eps
        k = np.where(k > 0, 1, -1).astype(np.float16)
        weight = (rng.standard_normal(D) * 2.0 ** rng.integers(-20, 15, D)).astype(np.float32)
        tie = (1 + (2 * rng.integers(0, 1024, D) + 1) * 2.0**-11) * 2.0 ** rng.integers(-10, 10, D)
        weight[::2] = tie[::2]  # to even
        weight[:8] = 65520, 65519.996, 1e30, np.inf, 2.0**-25, 2.0**-25 * (1 + 2.0**-23), 1e-30, 0.0  # its ends
        _, got = binding.itq3s_cache_append(None, dev(torch, k), None, head_dim=D, k_norm=dev(torch, weight), eps=0.0)
        want = (k.reshape(T, H, D) * weight.astype(np.float64)).reshape(T, H * D)
    with np.errstate(over="ignore"):
        assert np.array_equal(got.cpu().numpy(), want.astype(np.float16))


# ---- scores of every size


SCALES = [1e4, -1e6, 1e9, 2.0**40]


def check_row(got, q, k, v, scale, reach, slack):
    """One row over the tokens that it sees, where scores may be of any size: 1 if it could be checked.

    A score may be off by `slack` of its reach (operands' roundings, sums).  Where all scores are small that is what bound() prices.  Where
    the largest leads by more than both scores may be off, and by 50 beside that (e^-50 is below any rounding), it alone has weight, with those
    equal to it bit for bit (equal keys): their weights are the same number, so no error of the score enters."""
    s = k @ q
    if abs(scale) * reach <= 500:
        o, weight, _ = plain.attend(q, k, v, scale)
        assert np.linalg.norm(got - o) <= plain.bound(o, weight, abs(scale) * reach)
        return 1
    s = s * np.sign(scale)
    same = (k == k[s.argmax()]).all(axis=1)
    if len(k) > same.sum() and s.max() - s[~same].max() <= 2 * slack * reach + 50 / abs(scale):
        return 0
    o, weight = v[same].mean(axis=0), float(np.sqrt((v[same] ** 2).sum(axis=1)).mean())
    assert np.linalg.norm(got - o) <= plain.bound(o, weight, 0.0), (s.max() * abs(scale), np.linalg.norm(got - o))
    return 1


def big_rows(rng, T, heads, D):
    """Rows of which some are 2^10 and 2^20 times smaller"""
    return (rng.standard_normal((T, heads, D)) * 2.0 ** rng.choice([0, 0, 0, -10, -20], (T, heads, 1))).astype(np.float16)


PROMPTS = [
    # q_heads, kv_heads, lengths, causal: two wavefronts a workgroup, two that share rows' tokens, four
    (4, 2, [1, 2, 33, 70], True),
    (2, 2, [300], True),
    (4, 1, [250, 40], False),
    (64, 8, [530, 12, 300], True),
]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads,lens,causal", PROMPTS)
def test_prompt_scores_of_every_size(gpu, q_heads, kv_heads, lens, causal, D, scale):
    torch, binding = gpu
    rng = np.random.default_rng(D + q_heads)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T, G = int(starts[-1]), q_heads // kv_heads
    q, k, v = big_rows(rng, T, q_heads, D), rng.standard_normal((T, kv_heads, D)).astype(np.float16), rng.standard_normal((T, kv_heads, D)).astype(np.float16)
    k[rng.permutation(T)[: T // 3]] = k[rng.integers(0, T, T // 3)]  # equal keys
    got = binding.itq3s_prompt_attention(*(dev(torch, x.reshape(T, -1)) for x in (q, k, v)), D, dev(torch, starts), causal=causal, scale=scale)
    got, q, k, v = (x.astype(np.float64) for x in (got.cpu().numpy().reshape(T, q_heads, D), q, k, v))
    done = []
    for a, b in zip(starts[:-1], starts[1:]):
        for i in range(a, b) if b - a < 80 else sorted({int(a), int(b) - 1, *(int(x) for x in rng.integers(a, b, 30))}):
            end = i + 1 if causal else b
            for h in range(q_heads) if q_heads < 10 else rng.choice(q_heads, 4, replace=False):
                kk = k[a:end, h // G]
                # products of fp16 are exact; D sums of fp32, cut or rounded
                done.append(check_row(got[i, h], q[i, h], kk, v[a:end, h // G], scale, float((np.abs(kk) @ np.abs(q[i, h])).max()), D * 2.0**-23))
    assert np.mean(done) > 0.6


@pytest.mark.parametrize("factor", [3000.0, 8000.0, 20000.0])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_prompts_of_one_token_give_its_value(gpu, D, factor):
    """The default scale, q and k as large as fp16 has them: scores of 2^27 to 2^37."""
    torch, binding = gpu
    rng = np.random.default_rng(int(factor))
    T, H = 200, 2
    q = (rng.standard_normal((T, H * D)) * factor).clip(-65504, 65504).astype(np.float16)
    q[0], q[1] = 8000.0, -factor
    k, v = np.where(rng.random((T, 1)) < 0.5, 1, -1).astype(np.float16) * q, rng.standard_normal((T, H * D)).astype(np.float16)
    got = binding.itq3s_prompt_attention(*(dev(torch, x) for x in (q, k, v)), D, dev(torch, np.arange(T + 1, dtype=np.int32)), max_len=1).double().cpu().numpy()
    v = v.astype(np.float64)
    # one weight, rounded to fp16, against itself in fp32, and the result's rounding
    assert np.all(np.abs(got - v) <= 2.02 * 2.0**-11 * np.abs(v) + 2.0**-25)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("scale", [0.25, 0.5, 1.0, 2.0, 4.0])
@pytest.mark.parametrize("T,heads", [(60, 1), (400, 1), (200, 64)])
def test_prompt_scores_that_are_large_and_close(gpu, T, heads, scale, sign):
    """Scores 2^23 + j times the scale, j from 0 to 5, which are exact in fp32: the weights are e^(j scale) all the same."""
    torch, binding = gpu
    rng = np.random.default_rng(T)
    D = 64
    q, k, v = np.zeros((T, heads, D)), np.zeros((T, 1, D)), rng.standard_normal((T, 1, D)).astype(np.float16)
    q[..., 0], q[..., 1], k[..., 0], k[..., 1] = 2048.0 * sign, 1.0, 4096.0, rng.integers(0, 6, (T, 1))
    got = binding.itq3s_prompt_attention(*(dev(torch, x.reshape(T, -1).astype(np.float16)) for x in (q, k, v)), D, dev(torch, np.array([0, T], dtype=np.int32)), scale=scale)
    got, v = got.double().cpu().numpy().reshape(T, heads, D), v.astype(np.float64)
    for i in range(T):
        o, weight, _ = plain.attend(q[i, 0], k[: i + 1, 0], v[: i + 1, 0], scale)
        assert np.linalg.norm(got[i] - o, axis=1).max() <= plain.bound(o, weight, 0.0)


WAYS = [
    # q_heads, kv_heads, rows, tokens: sixteen wavefronts a sequence, parts of one, tiles of 16 rows in parts, two tiles a workgroup, rows of their own
    (8, 2, [1, 1, 1], [200, 1, 77]),
    (8, 1, [1], [6000]),
    (8, 2, [3, 1, 4], [1500, 31, 600]),
    (8, 1, [4, 3], [900, 500]),
    (64, 8, [300, 40], [1400, 60]),
]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads,n,lens", WAYS)
def test_cache_scores_of_every_size(gpu, q_heads, kv_heads, n, lens, D, scale):
    torch, binding = gpu
    rng = np.random.default_rng(D + q_heads + len(n))
    page, G, S, total = 64, q_heads // kv_heads, len(lens), sum(lens)
    starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    T, counts, first = int(starts[-1]), [-(-x // page) for x in lens], np.concatenate([[0], np.cumsum(lens)])
    table, at = np.zeros((S, max(counts)), dtype=np.int32), 0
    for s in range(S):
        table[s, : counts[s]], at = np.arange(at, at + counts[s]), at + counts[s]
    slots = np.concatenate([table[s, np.arange(lens[s]) // page].astype(np.int64) * page + np.arange(lens[s]) % page for s in range(S)])
    k, v = rng.standard_normal((total, kv_heads, D)), rng.standard_normal((total, kv_heads, D)) * 10.0 ** rng.uniform(-2, 2, (total, 1, 1))
    k[rng.permutation(total)[: total // 3]] = k[rng.integers(0, total, total // 3)]  # equal keys
    cache = binding.alloc_cache(at, page, kv_heads, D)
    binding.itq3s_cache_append(None, *(dev(torch, x.reshape(total, -1).astype(np.float32)) for x in (k, v)), None, None, cache, dev(torch, slots))
    k, v = (x.double().cpu().numpy().reshape(total, kv_heads, D) for x in binding.itq3s_cache_read(cache, dev(torch, slots), dtype=torch.float32))
    q = big_rows(rng, T, q_heads, D)
    out = binding.itq3s_cache_attention(dev(torch, q.reshape(T, -1)), cache, dev(torch, starts), dev(torch, np.array(lens, dtype=np.int32)), dev(torch, table), scale=scale, max_q=max(n), max_kv=max(lens))
    got, q = out.double().cpu().numpy().reshape(T, q_heads, D), q.astype(np.float64)
    done = []
    for s in range(S):
        for i in sorted({0, n[s] - 1, *(int(x) for x in rng.integers(0, n[s], 12))}):
            see = max(0, lens[s] - n[s] + i + 1)
            for h in range(q_heads) if q_heads < 10 else rng.choice(q_heads, 6, replace=False):
                kk, vv = k[first[s] : first[s] + see, h // G], v[first[s] : first[s] + see, h // G]
                reach = float((np.abs(plain.turned(kk)) @ np.abs(plain.turned(q[starts[s] + i, h]))).max()) if see else 0.0
                if see:
                    # H q rounds to fp16 once where rows are a wavefront's own
                    done.append(check_row(got[starts[s] + i, h], q[starts[s] + i, h], kk, vv, scale, reach, 1.02 * 2.0**-11))
                else:
                    assert not got[starts[s] + i, h].any()
    assert np.mean(done) > 0.6


@pytest.mark.parametrize("factor", [3000.0, 20000.0])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows_of_one", [1, 40])
def test_cached_sequences_of_one_token_give_its_value(gpu, rows_of_one, D, factor):
    """The default scale, q and k as large as fp16 has them.  (Forty rows of a sequence of one token: all but the last see nothing.)"""
    torch, binding = gpu
    rng = np.random.default_rng(D)
    S, G = 30, 4
    k = (rng.standard_normal((S, 1, D)) * factor).clip(-65504, 65504).astype(np.float16)
    v = (rng.standard_normal((S, D)) * 10.0 ** rng.uniform(-3, 3, (S, 1))).astype(np.float16)
    q = np.where(rng.random((S, G, 1)) < 0.5, 1, -1).astype(np.float16) * k
    cache, slots = binding.alloc_cache(S, 32, 1, D), np.arange(S, dtype=np.int64) * 32
    binding.itq3s_cache_append(None, dev(torch, k[:, 0]), dev(torch, v), None, None, cache, dev(torch, slots))
    v = binding.itq3s_cache_read(cache, dev(torch, slots), dtype=torch.float32)[1].double().cpu().numpy()
    all_q = np.ones((S, rows_of_one, G * D), dtype=np.float16)
    all_q[:, -1] = q.reshape(S, -1)
    starts = np.arange(S + 1, dtype=np.int32) * rows_of_one
    got = binding.itq3s_cache_attention(dev(torch, all_q.reshape(-1, G * D)), cache, dev(torch, starts), dev(torch, np.ones(S, dtype=np.int32)), dev(torch, np.arange(S, dtype=np.int32)[:, None]), max_q=rows_of_one, max_kv=32)
    got = got.double().cpu().numpy().reshape(S, rows_of_one, G, D)
    assert not got[:, :-1].any()
    for s in range(S):
        most = plain.bound(v[s], float(np.linalg.norm(v[s])), 0.0)
        assert np.all(np.linalg.norm(got[s, -1] - v[s], axis=1) <= most)


# ---- row starts that fall or leave the rows


STARTS = [
    # starts of a tensor of 8 rows, the rows of every sequence that they are cut to
    ([4, 2, -7, 3, 900], [(4, 4), (2, 2), (0, 3), (3, 8)]),
    ([900, 4, 5, -2], [(8, 8), (4, 5), (5, 5)]),
    ([-2147483648, 2147483647], [(0, 8)]),
    ([5, 5, 8, 2147483647], [(5, 5), (5, 8), (8, 8)]),
]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("max_q", [1, 8])
@pytest.mark.parametrize("starts,cut", STARTS)
def test_cache_attention_cuts_starts_to_the_rows(gpu, starts, cut, max_q, D):
    torch, binding = gpu
    rng = np.random.default_rng(D)
    T, H, G = 8, 2, 16
    lens = [40 + 7 * s for s in range(len(cut))]
    c, table, slots = base.fill(rng, lens, 32, H, D)
    q = base.rows(rng, T, H * G, D, "f16")
    out = torch.full((T, H * G * D), 2.0, dtype=torch.float16, device="cuda")
    binding.itq3s_cache_attention(dev(torch, q), binding.Cache(dev(torch, c.data), 32, H, D), dev(torch, np.array(starts, dtype=np.int32)), dev(torch, np.array(lens, dtype=np.int32)), dev(torch, table), out=out, max_q=max_q)
    got = out.double().cpu().numpy().reshape(T, H * G, D)
    for s, (a, b) in enumerate(cut):
        base.check_cache_attention(c, [slots[s]], q.reshape(T, H * G, D)[a:b], [0, b - a], [lens[s]], D**-0.5, got[a:b], G)
    nobody = [i for i in range(T) if not any(a <= i < b for a, b in cut)]
    assert np.all(got[nobody] == 2.0)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("starts,cut", STARTS)
def test_prompt_attention_cuts_starts_to_the_rows(gpu, starts, cut, causal, D):
    torch, binding = gpu
    rng = np.random.default_rng(D)
    T, H, G = 8, 2, 16
    q, k, v = base.rows(rng, T, H * G, D, "f16", outliers=False), base.rows(rng, T, H, D, "f16"), base.rows(rng, T, H, D, "f16")
    out = torch.full((T, H * G * D), 2.0, dtype=torch.float16, device="cuda")
    binding.itq3s_prompt_attention(dev(torch, q), dev(torch, k), dev(torch, v), D, dev(torch, np.array(starts, dtype=np.int32)), causal=causal, out=out)
    got, q, k, v = (x.astype(np.float64).reshape(T, -1, D) for x in (out.cpu().numpy(), q, k, v))
    for a, b in cut:
        for i in range(a, b):
            for h in range(H * G):
                end = i + 1 if causal else b
                o, weight, reach = plain.attend(q[i, h], k[a:end, h // G], v[a:end, h // G], D**-0.5)
                assert np.linalg.norm(got[i, h] - o) <= plain.bound(o, weight, reach)
    nobody = [i for i in range(T) if not any(a <= i < b for a, b in cut)]
    assert np.all(got[nobody] == 2.0)


# ---- sums of digits


@pytest.mark.parametrize("G", [8, 32])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_sums_of_values_that_cancel_are_exact(gpu, D, G):
    """Weights that are powers of two, 1 to 2^4 and, of two tokens of each block whose values are opposite, 2^15 (but for some 2^-21 of them, which
    fp16 rounds away): sums of weights times digits have 24 bits at most, so fp32 holds them however much they cancel (few rows, where
    the blocks are shared).  The transform's eight sums at most, the sum of weights and the last factor round to fp32, some twelve
    times what is added; the result rounds once."""
    torch, binding = gpu
    rng = np.random.default_rng(D)
    n = 2016
    c = plain.PlainCache(63, 32, 1, D)
    digits, power = rng.integers(-7, 8, (n, D)), rng.integers(-8, -3, n)
    for b in range(0, n, 32):
        i, j = b + rng.choice(32, 2, replace=False)
        power[[i, j]], digits[j] = 7, -digits[i]
    for t in range(n):
        c.put(t, 0, False, np.full(D, power[t]), np.float16(0.125))  # in channel 0: 0.125 sqrt(D) times the power
        c.put(t, 0, True, digits[t], np.float16(4096.0))
    q = np.zeros((1, G, D), dtype=np.float16)
    q[..., 0] = 1.0
    out = binding.itq3s_cache_attention(dev(torch, q.reshape(1, -1)), binding.Cache(dev(torch, c.data), 32, 1, D), dev(torch, np.array([0, 1], dtype=np.int32)), dev(torch, np.array([n], dtype=np.int32)),
                                        dev(torch, np.arange(63, dtype=np.int32)[None]), max_q=1, max_kv=n, scale=float(np.log(2) / (0.125 * np.sqrt(D))))
    weight = 2.0**power
    total = weight @ digits
    want, unit = plain.turned(total) * 4096 / weight.sum(), 4096 / weight.sum() / np.sqrt(D)
    got = out.double().cpu().numpy().reshape(G, D)
    assert np.all(np.abs(got - want) <= 1.01 * 2.0**-11 * np.abs(want) + 12 * 2.0**-24 * unit * np.abs(total).sum() + 2.0**-25), np.abs(got - want).max() / np.abs(want).max()


# ---- what is not finite, where a row does not see it


@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads,lens", [(4, 2, [70, 33, 2]), (2, 2, [300]), (8, 1, [250, 40]), (64, 8, [530, 12, 300]), (7, 1, [100, 41]), (5, 1, [500, 260])])
def test_what_is_not_finite_stays_behind_the_mask(gpu, q_heads, kv_heads, lens, D, what):
    """A NaN or an infinity in a token of a prompt is NaN in the rows that see it and in no other, of that head's group alone."""
    torch, binding = gpu
    rng = np.random.default_rng(D + q_heads)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T, G = int(starts[-1]), q_heads // kv_heads
    x = {"q": base.rows(rng, T, q_heads, D, "f16", outliers=False), "k": base.rows(rng, T, kv_heads, D, "f16"), "v": base.rows(rng, T, kv_heads, D, "f16")}
    clean = {n: x[n].astype(np.float64).reshape(T, -1, D) for n in "kv"}
    first = np.full((len(lens), kv_heads), 10**9)
    for s, n in enumerate(lens):
        for h in range(kv_heads):
            if n > 1 and (s + h) % 3 != 2:
                bad = int(rng.integers(1, n))
                first[s, h] = bad
                for t in {bad, *(int(i) for i in rng.integers(bad, n, 3))}:
                    x[what][starts[s] + t, h * D + rng.integers(0, D)] = rng.choice([np.nan, np.inf, -np.inf])
                if what == "k":  # an infinite key is an infinite score, or one of minus infinity: not a number whatever the query
                    x[what][starts[s] + bad, h * D : h * D + 2] = np.inf, -np.inf
                    x["q"].reshape(T, -1, D)[starts[s] + bad :, h * G : (h + 1) * G, :2] = 1.0
    clean["q"] = x["q"].astype(np.float64).reshape(T, -1, D)
    got = binding.itq3s_prompt_attention(*(dev(torch, x[n]) for n in "qkv"), D, dev(torch, starts)).double().cpu().numpy().reshape(T, q_heads, D)
    for s, (a, b) in enumerate(zip(starts[:-1], starts[1:])):
        for h in rng.choice(q_heads, min(q_heads, 6), replace=False):
            bad = first[s, h // G]
            for i in range(b - a):
                if i >= bad:
                    # a value's infinity stays one where only that reached the row
                    assert np.isnan(got[a + i, h]).all() if what == "k" else not np.isfinite(got[a + i, h]).all()
                elif b - a < 100 or bad - i < 40 or i % 16 == 0:
                    o, weight, reach = plain.attend(clean["q"][a + i, h], clean["k"][a : a + i + 1, h // G], clean["v"][a : a + i + 1, h // G], D**-0.5)
                    assert np.linalg.norm(got[a + i, h] - o) <= plain.bound(o, weight, reach), (s, h, i, bad)
