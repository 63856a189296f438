"""The attention half of a layer against 64-bit numpy: norm, rotation and codes bit for bit, rows read back, attention over the cache
and over prompts, at the sizes and masks where it can go wrong, and all of it together with the packed products."""
import numpy as np
import pytest

from tests import attention_plain as plain

pytestmark = pytest.mark.gpu

F = {"f16": np.float16, "f32": np.float32}


@pytest.fixture(scope="module")
def gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2603_27914_amd import binding

    binding.lib()
    return torch, binding


def dev(torch, a, pad=0):
    """On the device; with `pad`, as columns of a wider buffer."""
    a = np.ascontiguousarray(a)
    if not pad:
        return torch.from_numpy(a).cuda()
    wide = np.full((a.shape[0], a.shape[1] + pad), 7, dtype=a.dtype)
    wide[:, : a.shape[1]] = a
    return torch.from_numpy(wide).cuda()[:, : a.shape[1]]


def rows(rng, T, heads, D, kind, outliers=True):
    x = rng.standard_normal((T, heads, D))
    if outliers:
        x[:, :, rng.integers(0, D, 2)] *= 8.0
    return x.reshape(T, heads * D).astype(F[kind])


def flag(torch):
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ---- append


APPEND = [
    # T, q_heads, kv_heads, D, page, in, out, rot, interleaved, norm, pad
    (1, 32, 8, 128, 64, "f16", "f16", 128, False, False, 0),
    (1, 1, 1, 64, 32, "f32", "f32", 64, True, True, 0),
    (3, 7, 1, 64, 32, "f16", "f32", 32, False, True, 8),
    (5, 12, 3, 256, 128, "f16", "f16", 256, True, True, 16),
    (37, 6, 2, 128, 32, "f32", "f16", 48, False, True, 8),
    (33, 4, 4, 256, 64, "f32", "f32", 96, False, False, 4),
    (70, 5, 5, 64, 32, "f16", "f16", 0, False, True, 0),
    (2111, 16, 2, 128, 64, "f16", "f16", 128, False, True, 8),   # neighbouring tokens share a wavefront
    (1027, 8, 8, 64, 256, "f32", "f16", 64, True, False, 0),
    (1100, 2, 2, 256, 32, "f16", "f32", 64, False, True, 8),
]


@pytest.mark.parametrize("T,q_heads,kv_heads,D,page,kind,out,rot,interleaved,norm,pad", APPEND)
def test_append_matches_the_definition(gpu, T, q_heads, kv_heads, D, page, kind, out, rot, interleaved, norm, pad):
    torch, binding = gpu
    rng = np.random.default_rng(T * D + rot)
    q, k, v = rows(rng, T, q_heads, D, kind), rows(rng, T, kv_heads, D, kind), rows(rng, T, kv_heads, D, kind)
    pages = T // page + 3
    slots = rng.permutation(pages * page)[:T].astype(np.int64) if T < 1000 else np.arange(T, dtype=np.int64) + 5
    slots[T // 2] = -1 if T > 1 else slots[T // 2]
    pos = rng.integers(0, 200000, T).astype(np.int32)
    freq = binding.itq3s_rope_frequencies(rot, 500000.0) if rot else None
    qn, kn = (rng.uniform(0.5, 1.5, D).astype(np.float32) for _ in range(2)) if norm else (None, None)
    cache = binding.alloc_cache(pages, page, kv_heads, D)
    cache.data.fill_(0x5A)
    flags = flag(torch)
    odt = {"f16": torch.float16, "f32": torch.float32}[out]
    q_out, k_out = (torch.full((T, h * D + pad), 3.0, dtype=odt, device="cuda") for h in (q_heads, kv_heads))
    binding.itq3s_cache_append(dev(torch, q, pad), dev(torch, k, pad), dev(torch, v, pad), dev(torch, pos), freq.cuda() if rot else None, cache, dev(torch, slots), interleaved=interleaved, gain=1.25,
                               q_norm=dev(torch, qn) if norm else None, k_norm=dev(torch, kn) if norm else None, eps=1e-5, q_out=q_out[:, : q_heads * D], k_out=k_out[:, : kv_heads * D],
                               status_flags=flags)
    args = dict(eps=1e-5, positions=pos, freq=freq.numpy() if rot else None, interleaved=interleaved, gain=1.25)
    ke = plain.rotated(k, D, kn, **args)
    for x, got, heads, w in ((q, q_out, q_heads, qn), (k, k_out, kv_heads, kn)):
        want = plain.rotated(x, D, w, **args)
        # the rounding to the output's type, and for queries arithmetic in fp32: some sixteen roundings of a pair's magnitude
        size = np.abs(plain.rotated(x, D, w, eps=1e-5)).reshape(T, heads, D)
        pair = 1.25 * (size + np.roll(size, 1, axis=2)) if interleaved else 1.25 * size
        if rot:
            n = rot // 2
            at = np.arange(rot)
            mate = at ^ 1 if interleaved else (at + n) % rot
            pair = size.copy()
            pair[..., :rot] = 1.25 * (size[..., :rot] + size[..., mate])
        else:
            pair = size
        g = got.double().cpu().numpy()
        assert np.all(g[:, heads * D :] == 3.0)
        assert np.all(np.abs(g[:, : heads * D] - want) <= plain.HALF[out] * np.abs(want) + 16 * 2.0**-24 * pair.reshape(T, -1) + 2.0**-25)
    assert int(flags.item()) == 0
    want = plain.PlainCache(pages, page, kv_heads, D, fill=0x5A)
    want.write(slots, ke.reshape(T, kv_heads, D), v.astype(np.float64).reshape(T, kv_heads, D))
    assert np.array_equal(cache.data.cpu().numpy(), want.data)  # digits, steps, and every byte that is nobody's


def test_append_in_place_and_its_optional_parts(gpu):
    torch, binding = gpu
    rng = np.random.default_rng(5)
    T, D = 41, 128
    q, k, v = rows(rng, T, 6, D, "f16"), rows(rng, T, 2, D, "f16"), rows(rng, T, 2, D, "f16")
    pos, freq = dev(torch, np.arange(T, dtype=np.int32)), binding.itq3s_rope_frequencies(D).cuda()
    slots = dev(torch, np.arange(T, dtype=np.int64))
    cache = binding.alloc_cache(2, 32, 2, D)
    qo, ko = binding.itq3s_cache_append(dev(torch, q), dev(torch, k), dev(torch, v), pos, freq, cache, slots)
    assert ko is None
    qi, ki = dev(torch, q), dev(torch, k)
    other = binding.alloc_cache(2, 32, 2, D)
    binding.itq3s_cache_append(qi, ki, dev(torch, v), pos, freq, other, slots, q_out=qi, k_out=ki)
    q2, k2 = binding.itq3s_cache_append(dev(torch, q), dev(torch, k), None, pos, freq, head_dim=D)
    assert torch.equal(qo, qi) and torch.equal(qo, q2) and torch.equal(ki, k2) and torch.equal(cache.data, other.data)
    q3, k3 = binding.itq3s_cache_append(None, dev(torch, k), None, pos, freq, head_dim=D)
    q4, k4 = binding.itq3s_cache_append(dev(torch, q), None, None, pos, freq, head_dim=D)
    assert q3 is None and k4 is None and torch.equal(k3, ki) and torch.equal(q4, qo)
    third = binding.alloc_cache(2, 32, 2, D)
    binding.itq3s_cache_append(None, dev(torch, k), dev(torch, v), pos, freq, third, slots)
    assert torch.equal(third.data, cache.data)


def test_append_of_rows_that_do_not_fit(gpu):
    """NaN, infinities, zeros, values beyond and below the range of steps, ties, slots behind the cache."""
    torch, binding = gpu
    rng = np.random.default_rng(6)
    T, D = 12, 64
    k, v = rng.standard_normal((T, D)).astype(np.float32), rng.standard_normal((T, D)).astype(np.float32)
    k[0, 3], v[1, 5], v[2, 7] = np.nan, np.inf, -np.inf
    k[3], v[4] = 0.0, 0.0
    v[5] *= 1e30
    v[6] *= 1e-9
    v[7] *= 3e-7   # a step below fp16's normal range
    v[8] = np.where(plain.hadamard(D)[11] > 0, 4.0, -4.0)  # one channel after the transform
    v[9, :] = 0
    v[9, 0] = 60.0  # |w| = 7.5: step 1, every digit at a tie
    slots = np.arange(T, dtype=np.int64)
    slots[10], slots[11] = 64, -5
    cache = binding.alloc_cache(2, 32, 1, D)
    flags = flag(torch)
    binding.itq3s_cache_append(None, dev(torch, k), dev(torch, v), None, None, cache, dev(torch, slots), status_flags=flags)
    want = plain.PlainCache(2, 32, 1, D)
    want.write(slots, k[:, None].astype(np.float64), v[:, None].astype(np.float64))
    assert np.array_equal(cache.data.cpu().numpy(), want.data)
    assert int(flags.item()) == binding.FLAG_NONFINITE | binding.FLAG_SCALE_SAT | binding.FLAG_BAD_SLOT


# ---- read


@pytest.mark.parametrize("T,heads,D,page,kind,pad", [(1, 1, 64, 32, "f16", 0), (31, 3, 128, 64, "f32", 4), (77, 2, 256, 32, "f16", 8), (100, 5, 64, 128, "f32", 0), (129, 8, 128, 32, "f16", 0)])
def test_read_gives_what_rows_stand_for(gpu, T, heads, D, page, kind, pad):
    torch, binding = gpu
    rng = np.random.default_rng(T)
    pages = 3 + T // page
    want = plain.PlainCache(pages, page, heads, D, fill=0x11)
    have = rng.permutation(pages * page)[: T // 2 + 1]
    k, v = (rng.standard_normal((len(have), heads, D)) * rng.choice([0.01, 1.0, 300.0], (len(have), heads, 1)) for _ in range(2))
    want.write(have, k, v)
    slots = rng.choice(have, T).astype(np.int64)  # any order, some twice
    if T > 2:
        slots[1], slots[T - 1] = -1, pages * page
    cache = binding.Cache(dev(torch, want.data), page, heads, D)
    flags = flag(torch)
    dt = {"f16": torch.float16, "f32": torch.float32}[kind]
    ko, vo = (torch.full((T, heads * D + pad), 9.0, dtype=dt, device="cuda") for _ in range(2))
    binding.itq3s_cache_read(cache, dev(torch, slots), k_out=ko[:, : heads * D], v_out=vo[:, : heads * D], status_flags=flags)
    assert int(flags.item()) == (binding.FLAG_BAD_SLOT if T > 2 else 0)
    live = (slots >= 0) & (slots < pages * page)
    for got, value in ((ko, False), (vo, True)):
        g = got.double().cpu().numpy()
        assert np.all(g[:, heads * D :] == 9.0) and np.all(g[~live, : heads * D] == 0.0)
        for h in range(heads):
            w = plain.stands_for(*want.rows(slots[live], h, value))
            # the step times 1 / sqrt(D), the constant itself and the product round to fp32, then the result to its type
            tol = (3 * 2.0**-24 + plain.HALF[kind]) * np.abs(w) + (2.0**-25 if kind == "f16" else 0.0)
            assert np.all(np.abs(g[live, h * D : (h + 1) * D] - w) <= tol)


def test_append_then_read_is_the_code_of_the_input(gpu):
    torch, binding = gpu
    rng = np.random.default_rng(8)
    T, H, D = 600, 2, 128
    k, v = rows(rng, T, H, D, "f16"), rows(rng, T, H, D, "f16")
    cache = binding.alloc_cache(20, 32, H, D)
    slots = dev(torch, rng.permutation(640)[:T].astype(np.int64))
    binding.itq3s_cache_append(None, dev(torch, k), dev(torch, v), None, None, cache, slots)
    for got, x in zip(binding.itq3s_cache_read(cache, slots, dtype=torch.float32), (k, v)):
        x = x.astype(np.float64).reshape(T, H, D)
        g = got.double().cpu().numpy().reshape(T, H, D)
        step = np.abs(plain.turned(x)).max(axis=2) / 7.5
        # no value is clipped by more than the rounding of the step: half a step a value, D of them after the transform
        assert np.all(np.linalg.norm(g - x, axis=2) <= np.sqrt(D) * step * (0.5 + 8 * 2.0**-11))


# ---- attention over the cache


def fill(rng, lens, page, heads, D, garbage=True, v_scale=None):
    """A cache with lens[s] tokens of every sequence in shuffled pages: PlainCache, table, slots of every sequence.  Whatever is not a
    token's is NaN and odd digits."""
    counts = [-(-n // page) for n in lens]
    pool = sum(counts) + 2
    order = rng.permutation(pool)
    table = np.full((len(lens), max(1, max(counts))), 0x7FFFFFF0, dtype=np.int32)  # never read
    at, slots = 0, []
    c = plain.PlainCache(pool, page, heads, D, fill=0xFE if garbage else 0)
    for s, n in enumerate(lens):
        table[s, : counts[s]] = order[at : at + counts[s]]
        at += counts[s]
        j = np.arange(n)
        mine = table[s, j // page].astype(np.int64) * page + j % page
        scale = 1.0 if v_scale is None else v_scale(n)[:, None, None]
        k = rng.standard_normal((n, heads, D))
        k[:, :, rng.integers(0, D, 1)] *= 6.0
        c.write(mine, k, scale * rng.standard_normal((n, heads, D)))
        slots.append(mine)
    return c, table, slots


def check_cache_attention(plain_cache, slots, q, starts, lens, scale, got, group, dead=()):
    """got [T, q_heads, D] against the rows of the cache; dead: slots that nobody sees"""
    H, D = plain_cache.heads, plain_cache.D
    for s, n_kv in enumerate(lens):
        a, b = starts[s], starts[s + 1]
        for h in range(H):
            k, v = (plain.turned(x * st.astype(np.float64)[:, None]) for x, st in (plain_cache.rows(slots[s], h, w) for w in (False, True)))
            ok = np.array([sl not in dead for sl in slots[s]], dtype=bool)
            for i in range(b - a):
                see = max(0, n_kv - (b - a) + i + 1)
                kk, vv = k[:see][ok[:see]], v[:see][ok[:see]]
                for g in range(group):
                    x = q[a + i, h * group + g].astype(np.float64)
                    o, weight, _ = plain.attend(x, kk, vv, scale)
                    # the products are formed in the turned domain: the roundings are of H q
                    reach = abs(scale) * (np.abs(plain.turned(kk)) @ np.abs(plain.turned(x))).max() if len(kk) else 0.0
                    most = plain.bound(o, weight, reach)
                    # what an error of `most` takes beyond fp16's largest value, 65504, may be infinite; it cannot be small
                    y = got[a + i, h * group + g]
                    out = np.abs(o) + most >= 65504
                    assert np.all(y[out] * np.sign(o[out]) >= np.abs(o[out]).clip(max=65504) - most - 32)
                    err = np.linalg.norm((y - o)[~out])
                    assert err <= most, (s, h, i, g, err, most)


CACHE_ATTENTION = [
    # q_heads, kv_heads, D, page, [(tokens, rows)], scale factor, max_q, max_kv
    (4, 1, 64, 32, [(1, 1)], 1.0, None, None),
    (8, 2, 128, 64, [(0, 1), (1, 1), (31, 1), (32, 1), (33, 1), (65, 1)], 1.0, None, None),
    (8, 8, 128, 32, [(40, 2), (2, 5), (0, 3), (129, 1)], 1.0, None, None),        # rows that see nothing
    (6, 2, 256, 32, [(50, 3), (97, 7)], 1.0, None, None),
    (7, 1, 64, 128, [(300, 4), (12, 12)], 2.0, None, None),                       # prompts from their first token
    (16, 1, 128, 32, [(1500, 1)], 1.0, None, None),                               # split
    (32, 1, 64, 64, [(900, 1), (70, 2)], 1.0, None, None),                        # two column tiles
    (4, 2, 128, 32, [(200, 150)], 1.0, None, None),                               # rows of their own a wavefront
    (5, 1, 256, 64, [(333, 60)], 1.0, None, None),
    (2, 1, 64, 32, [(700, 500), (30, 30)], 1.0, None, None),
    (8, 2, 128, 32, [(1000, 9), (400, 40)], 1.0, 1, 32),                          # cut up for less than there is
    (8, 2, 64, 32, [(100, 40), (3, 2)], 1.0, 17, 10**9),                          # ... and for more
    (4, 2, 64, 32, [(90, 3)], 0.0, None, None),
    (4, 2, 64, 32, [(90, 3), (64, 40)], -1.0, None, None),
]


@pytest.mark.parametrize("q_heads,kv_heads,D,page,seqs,factor,max_q,max_kv", CACHE_ATTENTION)
def test_cache_attention(gpu, q_heads, kv_heads, D, page, seqs, factor, max_q, max_kv):
    torch, binding = gpu
    rng = np.random.default_rng(D + q_heads + len(seqs))
    lens, n = [s[0] for s in seqs], [s[1] for s in seqs]
    c, table, slots = fill(rng, lens, page, kv_heads, D)
    starts = np.concatenate([[1], 1 + np.cumsum(n)]).astype(np.int32)  # a row of nobody's in front, two behind
    T = int(starts[-1]) + 2
    q = rows(rng, T, q_heads, D, "f16", outliers=False)
    scale = factor / np.sqrt(D)
    out = torch.full((T, q_heads * D + 8), 5.0, dtype=torch.float16, device="cuda")
    flags = flag(torch)
    args = (dev(torch, q, 16), binding.Cache(dev(torch, c.data), page, kv_heads, D), dev(torch, starts), dev(torch, np.array(lens, dtype=np.int32)), dev(torch, table))
    ws = None
    if max_kv is not None:  # a workspace of just its size, which the call may not overrun
        need = binding.itq3s_cache_attention_workspace_bytes(T, len(lens), q_heads, kv_heads, D, max_q, max_kv)
        ws = torch.full((need + 256,), 0x77, dtype=torch.uint8, device="cuda")
    binding.itq3s_cache_attention(*args, scale=scale, max_q=max_q, max_kv=max_kv, out=out[:, : q_heads * D], workspace=ws[:need] if ws is not None else None, status_flags=flags)
    assert int(flags.item()) == 0
    if ws is not None:
        assert bool((ws[need:] == 0x77).all())
    g = out.double().cpu().numpy()
    assert np.all(g[:, q_heads * D :] == 5.0) and np.all(g[0] == 5.0) and np.all(g[-2:] == 5.0)
    check_cache_attention(c, slots, q.reshape(T, q_heads, D), starts, lens, scale, g[:, : q_heads * D].reshape(T, q_heads, D), q_heads // kv_heads)
    again = torch.full_like(out, 5.0)
    binding.itq3s_cache_attention(*args, scale=scale, max_q=max_q, max_kv=max_kv, out=again[:, : q_heads * D])
    assert torch.equal(again, out)  # no order of summation that changes


def test_cache_attention_with_steps_of_every_size(gpu):
    """Values whose steps run over fp16's whole range within one row, and zeros among them: the weights' reference follows."""
    torch, binding = gpu
    rng = np.random.default_rng(3)
    D, n = 128, 700
    for v_scale in (lambda n: 10.0 ** rng.uniform(-5, 4.5, n), lambda n: np.where(rng.random(n) < 0.9, 0.0, 1e-3), lambda n: np.linspace(-4, 4, n)[::-1] ** 9 / 10 + 1e-4, lambda n: np.full(n, 2e-6)):
        c, table, slots = fill(rng, [n], 64, 1, D, v_scale=v_scale)
        for T in (1, 30):
            q = rows(rng, T, 8, D, "f16", outliers=False)
            starts = np.array([0, T], dtype=np.int32)
            out = binding.itq3s_cache_attention(dev(torch, q), binding.Cache(dev(torch, c.data), 64, 1, D), dev(torch, starts), dev(torch, np.array([n], dtype=np.int32)), dev(torch, table), scale=0.3)
            check_cache_attention(c, slots, q.reshape(T, 8, D), starts, [n], np.float64(np.float32(0.3)), out.double().cpu().numpy().reshape(T, 8, D), 8)


def test_cache_attention_of_queries_of_every_size(gpu):
    """The largest and smallest fp16 values, zeros, and a row with a NaN or an infinity, which stays that row's."""
    torch, binding = gpu
    rng = np.random.default_rng(4)
    D, n = 64, 100
    c, table, slots = fill(rng, [n], 32, 1, D)
    q = rng.standard_normal((6, 1, D)).astype(np.float16)
    q[0] = np.sign(q[0]) * np.float16(60000)
    q[1] *= np.float16(1e-5)
    q[2] = 0
    q[3, 0, 7], q[4, 0, 9] = np.nan, np.inf
    starts, lens = np.array([0, 6], dtype=np.int32), np.array([n], dtype=np.int32)
    out = binding.itq3s_cache_attention(dev(torch, q.reshape(6, D)), binding.Cache(dev(torch, c.data), 32, 1, D), dev(torch, starts), dev(torch, lens), dev(torch, table), scale=1e-3)
    g = out.double().cpu().numpy().reshape(6, 1, D)
    assert np.isnan(g[3]).all() and np.isnan(g[4]).all()
    keep = np.where(np.isfinite(q), q, 0)
    g[3:5] = 0
    for i in (0, 1, 2, 5):
        s1 = np.array([0, 1])
        check_cache_attention(c, [slots[0][: n - 5 + i]], keep[i : i + 1], s1, [n - 5 + i], np.float64(np.float32(1e-3)), g[i : i + 1], 1)


def test_cache_attention_of_pages_and_lengths_that_are_not_there(gpu):
    """Pages before and behind the pool are tokens that nobody sees; lengths beyond the table are cut, negative ones empty."""
    torch, binding = gpu
    rng = np.random.default_rng(9)
    D = 64
    c, table, slots = fill(rng, [100, 96, 40], 32, 2, D)
    table[0, 1], table[1, 0], table[1, 2] = c.pages, -3, 0x7FFFFFFF
    lens = np.array([100, 500, -7], dtype=np.int32)
    q = rows(rng, 6, 4, D, "f16")
    starts = np.array([0, 2, 4, 6], dtype=np.int32)
    flags = flag(torch)
    out = binding.itq3s_cache_attention(dev(torch, q), binding.Cache(dev(torch, c.data), 32, 2, D), dev(torch, starts), dev(torch, lens), dev(torch, table[:, :3].copy()), status_flags=flags)
    assert int(flags.item()) == binding.FLAG_BAD_SLOT
    dead = set(slots[0][32:64].tolist()) | set(slots[1][:32].tolist()) | set(slots[1][64:].tolist())
    # the first sequence's fourth page lies behind the table's three: 96 tokens
    check_cache_attention(c, [slots[0][:96], slots[1], slots[2][:0]], q.reshape(6, 4, D), starts, [96, 96, 0], D**-0.5, out.double().cpu().numpy().reshape(6, 4, D), 2, dead)
    # starts that fall or leave the rows
    bad = dev(torch, np.array([-5, 2, 1, 900], dtype=np.int32))
    out = torch.full((6, 4 * D), 2.0, dtype=torch.float16, device="cuda")
    binding.itq3s_cache_attention(dev(torch, q), binding.Cache(dev(torch, c.data), 32, 2, D), bad, dev(torch, np.array([50, 40, 30], dtype=np.int32)), dev(torch, table), out=out)
    torch.cuda.synchronize()


def test_captured_decode_follows_lengths_pages_and_slots(gpu):
    """Two graphs that share a workspace, replayed as the sequences grow, against eager calls."""
    torch, binding = gpu
    rng = np.random.default_rng(10)
    D, H, G, S, page, most = 128, 2, 4, 3, 32, 1024
    cache = binding.alloc_cache(S * most // page, page, H, D)
    pages = dev(torch, rng.permutation(S * most // page).astype(np.int32).reshape(S, -1))
    freq = binding.itq3s_rope_frequencies(D).cuda()
    q, k, v = (torch.zeros((S, h * D), dtype=torch.float16, device="cuda") for h in (H * G, H, H))
    pos, lens, slots = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int64, device="cuda")
    starts = dev(torch, np.arange(S + 1, dtype=np.int32))
    ws = torch.empty(binding.itq3s_cache_attention_workspace_bytes(S, S, H * G, H, D, 1, most), dtype=torch.uint8, device="cuda")
    qr, outs = torch.empty_like(q), [torch.empty_like(q) for _ in range(2)]

    def step(out, workspace, target):
        binding.itq3s_cache_append(q, k, v, pos, freq, target, slots, q_out=qr)
        binding.itq3s_cache_attention(qr, target, starts, lens, pages, max_q=1, max_kv=most, out=out, workspace=workspace)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(outs[0], ws, binding.Cache(cache.data.clone(), page, H, D))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for out in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(out, ws, cache)
        graphs.append(g)
    eager = binding.Cache(cache.data.clone(), page, H, D)
    at = np.array([0, 30, 400], dtype=np.int64)
    for i in range(6):
        q.copy_(dev(torch, rows(rng, S, H * G, D, "f16")))
        k.copy_(dev(torch, rows(rng, S, H, D, "f16")))
        v.copy_(dev(torch, rows(rng, S, H, D, "f16")))
        pos.copy_(dev(torch, at.astype(np.int32)))
        lens.copy_(dev(torch, (at + 1).astype(np.int32)))
        slots.copy_(torch.gather(pages.long(), 1, dev(torch, at // page)[:, None])[:, 0] * page + dev(torch, at % page))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        want = torch.empty_like(q)
        step(want, torch.empty_like(ws), eager)
        assert torch.equal(outs[i % 2], want) and torch.equal(cache.data, eager.data)
        at += np.array([1, 3, 100])


def test_calls_run_on_the_current_stream(gpu):
    torch, binding = gpu
    rng = np.random.default_rng(11)
    T, D = 300, 64
    x = dev(torch, rows(rng, T, 6, D, "f16"))
    starts = dev(torch, np.array([0, T], dtype=np.int32))
    want = binding.itq3s_prompt_attention(x[:, : 4 * D], x[:, 4 * D : 5 * D], x[:, 5 * D :], D, starts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = torch.empty_like(x)
        for _ in range(20):
            y.copy_(x)
        got = binding.itq3s_prompt_attention(y[:, : 4 * D], y[:, 4 * D : 5 * D], y[:, 5 * D :], D, starts)
    side.synchronize()
    assert torch.equal(got, want)


# ---- attention over prompts


PROMPT = [
    # q_heads, kv_heads, D, lengths, causal, scale factor, max_len
    (1, 1, 64, [1], True, 1.0, None),
    (4, 2, 128, [1, 2, 31, 32, 33, 64, 65, 0, 200], True, 1.0, None),
    (4, 4, 64, [129, 77, 5], False, 1.0, None),
    (8, 1, 128, [150, 3], True, 2.0, None),
    (7, 1, 64, [100, 41], True, 1.0, 7),
    (6, 2, 256, [97, 33, 1], True, 1.0, None),
    (2, 2, 256, [70], False, 1.0, None),
    (64, 8, 128, [530, 12, 300], True, 1.0, None),       # 64 rows a wavefront
    (32, 32, 64, [700], False, 1.0, None),
    (2, 1, 64, [60], True, -1.0, None),
    (2, 1, 128, [60], True, 0.0, None),
]


@pytest.mark.parametrize("q_heads,kv_heads,D,lens,causal,factor,max_len", PROMPT)
def test_prompt_attention(gpu, q_heads, kv_heads, D, lens, causal, factor, max_len):
    torch, binding = gpu
    rng = np.random.default_rng(D + q_heads + len(lens))
    starts = np.concatenate([[3], 3 + np.cumsum(lens)]).astype(np.int32)  # three rows of nobody's in front, two behind
    T, G = int(starts[-1]) + 2, q_heads // kv_heads
    q, k, v = rows(rng, T, q_heads, D, "f16", outliers=False), rows(rng, T, kv_heads, D, "f16"), rows(rng, T, kv_heads, D, "f16")
    for x in (q, k, v):
        x[:3], x[-2:] = np.nan, np.inf
    scale = factor / np.sqrt(D)
    out = torch.full((T, q_heads * D + 8), 5.0, dtype=torch.float16, device="cuda")
    binding.itq3s_prompt_attention(dev(torch, q, 8), dev(torch, k, 16), dev(torch, v, 24), D, dev(torch, starts), max_len=max_len, causal=causal, scale=scale, out=out[:, : q_heads * D])
    g = out.double().cpu().numpy()
    assert np.all(g[:, q_heads * D :] == 5.0) and np.all(g[:3] == 5.0) and np.all(g[-2:] == 5.0)
    q, k, v, g = (x[:, : h * D].astype(np.float64).reshape(T, h, D) for x, h in ((q, q_heads), (k, kv_heads), (v, kv_heads), (g, q_heads)))
    heads = range(q_heads) if q_heads * max(lens) < 3000 else rng.choice(q_heads, 5, replace=False)
    for a, b in zip(starts[:-1], starts[1:]):
        for i in range(a, b) if b - a < 200 else sorted(rng.choice(np.arange(a, b), 60, replace=False)):
            end = i + 1 if causal else b
            for h in heads:
                o, weight, reach = plain.attend(q[i, h], k[a:end, h // G], v[a:end, h // G], scale)
                err = np.linalg.norm(g[i, h] - o)
                assert err <= plain.bound(o, weight, reach), (a, i, h, err, plain.bound(o, weight, reach))


def test_prompts_do_not_see_each_other(gpu):
    """NaN and infinities in one sequence leave its neighbours' bits as they are."""
    torch, binding = gpu
    rng = np.random.default_rng(12)
    D, lens = 128, [40, 57, 90]
    starts = dev(torch, np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
    x = rows(rng, sum(lens), 4, D, "f16")
    y = x.copy()
    y[40:97] = np.nan
    y[60:70] = np.inf
    a, b = (binding.itq3s_prompt_attention(t[:, : 2 * D], t[:, 2 * D : 3 * D], t[:, 3 * D :], D, starts) for t in (dev(torch, x), dev(torch, y)))
    assert torch.equal(a[:40], b[:40]) and torch.equal(a[97:], b[97:]) and bool(torch.isnan(b[40:97]).all())


@pytest.mark.parametrize("D,q_heads,kv_heads,lens,causal", [(64, 4, 2, [800, 31, 33, 1, 500], True), (64, 4, 1, [333, 300], False), (128, 4, 2, [800, 31, 33, 1, 500], True), (128, 7, 7, [290], False), (256, 4, 2, [600, 64, 1], True), (256, 2, 2, [430], False), (64, 32, 32, [1100, 40], True), (64, 32, 32, [900], False), (256, 16, 8, [2100, 7], True), (256, 8, 8, [1400, 600], False), (128, 8, 8, [3100], True)])
def test_prompt_attention_of_many_rows(gpu, D, q_heads, kv_heads, lens, causal):
    """Rows whose tokens two wavefronts share, and enough of them for workgroups of four with rows of their own, for every head
    dimension; a sample of the rows."""
    torch, binding = gpu
    rng = np.random.default_rng(D + lens[0])
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T, G = int(starts[-1]), q_heads // kv_heads
    q, k, v = rows(rng, T, q_heads, D, "f16", outliers=False), rows(rng, T, kv_heads, D, "f16"), rows(rng, T, kv_heads, D, "f16")
    g = binding.itq3s_prompt_attention(dev(torch, q), dev(torch, k), dev(torch, v), D, dev(torch, starts), max_len=max(lens), causal=causal).double().cpu().numpy()
    q, k, v, g = (x.astype(np.float64).reshape(T, -1, D) for x in (q, k, v, g))
    for a, b in zip(starts[:-1], starts[1:]):
        for i in {int(a), int(b) - 1, *(int(x) for x in rng.integers(a, b, 20))}:
            for h in rng.choice(q_heads, min(q_heads, 4), replace=False):
                end = i + 1 if causal else b
                o, weight, reach = plain.attend(q[i, h], k[a:end, h // G], v[a:end, h // G], D**-0.5)
                assert np.linalg.norm(g[i, h] - o) <= plain.bound(o, weight, reach)


WAYS = [
    # q_heads, kv_heads, rows, tokens: which way the work is cut (a unit's count of the card that decides is 256)
    (8, 2, [1, 1, 1], [400, 130, 77]),        # sixteen wavefronts a sequence
    (8, 2, [1], [9000]),                      # parts of a sequence
    (8, 2, [3, 1, 4], [2500, 31, 6000]),      # tiles of 16 rows in parts, sequences of different lengths
    (8, 1, [4, 3], [3000, 500]),              # two tiles a workgroup
    (8, 1, [12, 2], [2000, 50]),              # several tiles, of 16 rows each
    (64, 8, [300], [2100]),                   # rows of their own, in parts
    (64, 8, [40, 1, 0, 280], [70, 3, 9, 300]),
]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads,n,lens", WAYS)
def test_every_way_of_cutting_up_cache_attention(gpu, q_heads, kv_heads, n, lens, D):
    """A sample of rows against 64 bits on what the cache holds."""
    torch, binding = gpu
    rng = np.random.default_rng(D + sum(lens))
    page, G, S = 64, q_heads // kv_heads, len(lens)
    starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    T, counts = int(starts[-1]), [-(-x // page) for x in lens]
    table, order, at = np.zeros((S, max(counts)), dtype=np.int32), rng.permutation(sum(counts)), 0
    for s in range(S):
        table[s, : counts[s]], at = order[at : at + counts[s]], at + counts[s]
    slots = [table[s, np.arange(lens[s]) // page].astype(np.int64) * page + np.arange(lens[s]) % page for s in range(S)]
    cache, total = binding.alloc_cache(sum(counts), page, kv_heads, D), sum(lens)
    k, v, q = rows(rng, total, kv_heads, D, "f16"), rows(rng, total, kv_heads, D, "f16"), rows(rng, T, q_heads, D, "f16", outliers=False)
    all_slots = dev(torch, np.concatenate(slots))
    binding.itq3s_cache_append(None, dev(torch, k), dev(torch, v), None, None, cache, all_slots)
    K, V = (x.double().cpu().numpy().reshape(total, kv_heads, D) for x in binding.itq3s_cache_read(cache, all_slots, dtype=torch.float32))
    args = (dev(torch, q), cache, dev(torch, starts), dev(torch, np.array(lens, dtype=np.int32)), dev(torch, table))
    out = binding.itq3s_cache_attention(*args, max_q=max(n), max_kv=max(lens))
    assert torch.equal(out, binding.itq3s_cache_attention(*args, max_q=max(n), max_kv=max(lens)))
    g, q = out.double().cpu().numpy().reshape(T, q_heads, D), q.astype(np.float64).reshape(T, q_heads, D)
    first = np.concatenate([[0], np.cumsum(lens)])
    for s in range(S):
        for i in sorted({0, n[s] - 1, *(int(x) for x in rng.integers(0, max(n[s], 1), 12))} & set(range(n[s]))):
            see = max(0, lens[s] - n[s] + i + 1)
            for h in rng.choice(q_heads, min(q_heads, 6), replace=False):
                kk, vv, x = K[first[s] : first[s] + see, h // G], V[first[s] : first[s] + see, h // G], q[starts[s] + i, h]
                o, weight, _ = plain.attend(x, kk, vv, D**-0.5)
                reach = D**-0.5 * float((np.abs(plain.turned(kk)) @ np.abs(plain.turned(x))).max()) if see else 0.0
                assert np.linalg.norm(g[starts[s] + i, h] - o) <= plain.bound(o, weight, reach), (s, i, h)


def test_positions_at_their_ends(gpu):
    """Angles of positions up to 2^31 - 1, negative ones, frequencies above 1."""
    torch, binding = gpu
    rng = np.random.default_rng(31)
    D, T = 128, 9
    pos = np.array([0, 1, -1, 2**31 - 1, -(2**31), 10**9 + 7, -12345678, 2**24 + 1, 131071], dtype=np.int32)
    x = rows(rng, T, 2, D, "f32")
    for interleaved in (False, True):
        freq = np.concatenate([binding.itq3s_rope_frequencies(2 * 60, 1e6).numpy(), [3.0, 0.0, 1e-300, 0.7853981633974483]])
        got, _ = binding.itq3s_cache_append(dev(torch, x), None, None, dev(torch, pos), dev(torch, freq), head_dim=D, interleaved=interleaved, dtype=torch.float32)
        want = plain.rotated(x, D, positions=pos, freq=freq, interleaved=interleaved)
        pair = np.abs(x.astype(np.float64)).max()
        # cosine and sine round to fp32, two products and a sum: four roundings of a pair's magnitude
        assert np.abs(got.double().cpu().numpy() - want).max() <= 4 * 2.0**-24 * 2 * pair


# ---- sizes at their ends


def test_pages_of_more_than_two_gib(gpu):
    """One page of 65536 tokens of 128 heads of 256 is 2.2e9 bytes: the second page against the same rows in small pages."""
    torch, binding = gpu
    rng = np.random.default_rng(21)
    T, H, D, page = 70, 128, 256, 65536
    k, v, q = (dev(torch, rows(rng, T, H, D, "f16")) for _ in range(3))
    small, large = binding.alloc_cache(2, 64, H, D), binding.alloc_cache(2, page, H, D)
    assert large.data.numel() > 2**32
    here = dev(torch, np.arange(T, dtype=np.int64))
    binding.itq3s_cache_append(None, k, v, None, None, small, here)
    flags = flag(torch)
    for at in (page, 2 * page - T):
        binding.itq3s_cache_append(None, k, v, None, None, large, here + at, status_flags=flags)
        for a, b in zip(binding.itq3s_cache_read(small, here), binding.itq3s_cache_read(large, here + at, status_flags=flags)):
            assert torch.equal(a, b)
    starts, lens = dev(torch, np.array([0, 1], dtype=np.int32)), dev(torch, np.array([T], dtype=np.int32))
    for n in (1, 3, T):  # rows alone, in shared tiles, and in tiles of their own
        starts[1] = n
        a = binding.itq3s_cache_attention(q[:n], small, starts, lens, dev(torch, np.array([[0, 1]], dtype=np.int32)), max_kv=T)
        b = binding.itq3s_cache_attention(q[:n], large, starts, lens, dev(torch, np.array([[1]], dtype=np.int32)), max_kv=T, status_flags=flags)
        assert torch.equal(a, b)
    assert int(flags.item()) == 0


def test_many_sequences_and_estimates_far_too_high(gpu):
    """Rows of two sequences among 2^15 of none, and as many rows expected of each as there are in all: tiles by the million.  Attention
    is cut up in another way then than for the two, so each is held against 64 bits."""
    torch, binding = gpu
    rng = np.random.default_rng(22)
    S, T, D, Hq, H, page = 2**15, 512, 64, 128, 8, 32
    q, k, v = dev(torch, rows(rng, T, Hq, D, "f16")), dev(torch, rows(rng, T, H, D, "f16")), dev(torch, rows(rng, T, H, D, "f16"))
    few = np.array([0, 500, T], dtype=np.int32)
    many = np.zeros(S + 1, dtype=np.int32)
    many[8:], many[30000:] = 500, T
    few, many = dev(torch, few), dev(torch, many)
    prompts = [binding.itq3s_prompt_attention(q, k, v, D, x).double().cpu().numpy().reshape(T, Hq, D) for x in (few, many)]
    Q, K, V = (x.double().cpu().numpy().reshape(T, -1, D) for x in (q, k, v))
    for at, end in ((0, 500), (500, T)):
        for i in sorted(rng.choice(np.arange(at, end), 12, replace=False)):
            for h in rng.choice(Hq, 16, replace=False):
                o, weight, reach = plain.attend(Q[i, h], K[at : i + 1, h // 16], V[at : i + 1, h // 16], D**-0.5)
                assert all(np.linalg.norm(p[i, h] - o) <= plain.bound(o, weight, reach) for p in prompts)
    cache = binding.alloc_cache(17, page, H, D)
    slots = np.concatenate([np.arange(500), 512 + np.arange(12)])
    binding.itq3s_cache_append(None, k, v, None, None, cache, dev(torch, slots))
    table, lens = np.zeros((2, 16), dtype=np.int32), np.array([500, 12], dtype=np.int32)
    table[0], table[1, 0] = np.arange(16), 16
    all_tables, all_lens = np.zeros((S, 16), dtype=np.int32), np.zeros(S, dtype=np.int32)
    all_tables[7], all_tables[29999], all_lens[7], all_lens[29999] = table[0], table[1], 500, 12
    a = binding.itq3s_cache_attention(q, cache, few, dev(torch, lens), dev(torch, table), max_kv=512)
    b = binding.itq3s_cache_attention(q, cache, many, dev(torch, all_lens), dev(torch, all_tables), max_kv=512)
    K, V = (x.double().cpu().numpy().reshape(T, H, D) for x in binding.itq3s_cache_read(cache, dev(torch, slots), dtype=torch.float32))
    Q, A, B = (x.double().cpu().numpy().reshape(T, Hq, D) for x in (q, a, b))
    for at, end in ((0, 500), (500, T)):
        for i in sorted(rng.choice(np.arange(at, end), 12, replace=False)):
            for h in rng.choice(Hq, 16, replace=False):
                k, v = K[at : i + 1, h // 16], V[at : i + 1, h // 16]
                o, weight, _ = plain.attend(Q[i, h], k, v, D**-0.5)
                most = plain.bound(o, weight, D**-0.5 * float((np.abs(plain.turned(k)) @ np.abs(plain.turned(Q[i, h]))).max()))
                assert np.linalg.norm(A[i, h] - o) <= most and np.linalg.norm(B[i, h] - o) <= most


def test_read_of_rows_far_apart_with_others_that_are_not_there(gpu):
    """Every listed row in another block, and among them padding and slots behind the cache."""
    torch, binding = gpu
    rng = np.random.default_rng(23)
    H, D, page, pages = 2, 128, 32, 40
    k, v = (dev(torch, rows(rng, page * pages, H, D, "f16")) for _ in range(2))
    cache = binding.alloc_cache(pages, page, H, D)
    binding.itq3s_cache_append(None, k, v, None, None, cache, dev(torch, np.arange(page * pages, dtype=np.int64)))
    K, V = binding.itq3s_cache_read(cache, dev(torch, np.arange(page * pages, dtype=np.int64)))  # (neighbours)
    slots = np.concatenate([rng.permutation(pages) * page + rng.integers(0, page, pages) for _ in range(3)])
    slots[rng.permutation(len(slots))[:50]] = rng.choice([-1, -(2**62), page * pages, 2**62], 50)
    slots[:32] = np.where(np.arange(32) % 3 == 0, slots[:32], -1)
    live = dev(torch, (slots >= 0) & (slots < page * pages))
    at = dev(torch, slots.clip(0, page * pages - 1))
    for got, all_rows in zip(binding.itq3s_cache_read(cache, dev(torch, slots)), (K, V)):
        assert torch.equal(got, torch.where(live[:, None], all_rows[at], torch.zeros_like(got)))


# ---- together


def test_a_layer_s_attention_from_products_to_product(gpu):
    """q/k/v product over packed weights, norm and rotation into the cache, attention over the prompt, output product; then two decode
    steps over the cache.  Every operator against 64 bits on what the one before it gave."""
    torch, binding = gpu
    rng = np.random.default_rng(13)
    width, D, Hq, H, page = 512, 64, 8, 2, 32
    packed = {}
    for name, n in (("q", Hq * D), ("k", H * D), ("v", H * D), ("o", width)):
        w = torch.from_numpy(rng.standard_normal((n, width)).astype(np.float32) / np.float32(np.sqrt(width))).cuda()
        packed[name] = binding.itq3s_quantize(w) + (n,)
    norm = [rng.uniform(0.5, 1.5, D).astype(np.float32) for _ in range(2)]
    freq = binding.itq3s_rope_frequencies(D, 10000.0, 4.0, 32, 1.0, 4.0)
    lens = np.array([50, 33])
    pages = rng.permutation(6).astype(np.int32).reshape(2, 3)
    cache, model = binding.alloc_cache(6, page, H, D), plain.PlainCache(6, page, H, D)
    past = np.zeros(2, dtype=np.int64)
    for n in (lens, np.array([1, 1]), np.array([2, 1])):
        starts = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        T = int(starts[-1])
        x = torch.from_numpy(rng.standard_normal((T, width)).astype(np.float16)).cuda()
        q, k, v = binding.itq3s_matmul_grouped([packed[i] for i in "qkv"], width, x, dtype=torch.float16)
        pos = np.concatenate([p + np.arange(m) for p, m in zip(past, n)])
        seq = np.repeat(np.arange(2), n)
        slots = pages[seq, pos // page].astype(np.int64) * page + pos % page
        qr, kr = binding.itq3s_cache_append(q, k, v, dev(torch, pos.astype(np.int32)), freq.cuda(), cache, dev(torch, slots), q_norm=dev(torch, norm[0]), k_norm=dev(torch, norm[1]),
                                            k_out=torch.empty_like(k))
        past = past + n
        args = dict(positions=pos, freq=freq.numpy())
        want_q, want_k = (plain.rotated(t.cpu().numpy(), D, w, **args) for t, w in ((q, norm[0]), (k, norm[1])))
        assert np.allclose(qr.double().cpu().numpy(), want_q, rtol=2.0**-11 + 2.0**-18, atol=2.0**-18)
        model.write(slots, want_k.reshape(T, H, D), v.double().cpu().numpy().reshape(T, H, D))
        assert np.array_equal(cache.data.cpu().numpy(), model.data)
        if n is lens:
            out = binding.itq3s_prompt_attention(qr, kr, v, D, dev(torch, starts))
            q64, k64, v64, o64 = (t.double().cpu().numpy().reshape(T, -1, D) for t in (qr, kr, v, out))
            for a, b in zip(starts[:-1], starts[1:]):
                for i in range(a, b):
                    for h in range(Hq):
                        o, weight, reach = plain.attend(q64[i, h], k64[a : i + 1, h // 4], v64[a : i + 1, h // 4], D**-0.5)
                        assert np.linalg.norm(o64[i, h] - o) <= plain.bound(o, weight, reach)
        else:
            out = binding.itq3s_cache_attention(qr, cache, dev(torch, starts), dev(torch, past.astype(np.int32)), dev(torch, pages))
            all_slots = [pages[s, np.arange(past[s]) // page].astype(np.int64) * page + np.arange(past[s]) % page for s in range(2)]
            check_cache_attention(model, all_slots, qr.double().cpu().numpy().reshape(T, Hq, D), starts, past, D**-0.5, out.double().cpu().numpy().reshape(T, Hq, D), 4)
        y = binding.itq3s_matmul(*packed["o"], width, out)
        w_hat = binding.itq3s_dequantize(*packed["o"], width).double().cpu().numpy()
        want = out.double().cpu().numpy() @ w_hat.T
        assert np.linalg.norm(y.double().cpu().numpy() - want) <= 2e-3 * np.linalg.norm(want)
