"""Windowed attention against its definition in 64 bits (tests/encoder_ref.py), forward and gradients."""
import math

import pytest
import torch

import encoder_ref as R

pytestmark = pytest.mark.gpu
DT = R.DT


def draw(seed, dt, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(DT[dt]).cuda()


def ints(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def run(q, k, v, do=None, lengths=None, starts=None, **kw):
    from paper_2607_21271_amd.attention import window_attention
    if do is None:
        return {"o": window_attention(q, k, v, lengths=ints(lengths), starts=ints(starts), **kw)}
    q, k, v = (t.detach().requires_grad_() for t in (q, k, v))
    o = window_attention(q, k, v, lengths=ints(lengths), starts=ints(starts), **kw)
    dq, dk, dv = torch.autograd.grad(o, (q, k, v), do)
    return {"o": o, "dq": dq, "dk": dk, "dv": dv}


def compare(q, k, v, do=None, **kw):
    got = run(q, k, v, do, **kw)
    torch.cuda.synchronize()
    want = R.attention(q, k, v, do, **kw)
    for n, t in got.items():
        R.within(n, t, *want[n])
    return got


# B, Lq, Lk, H, Hkv, D, window
TRAIN = [
    (1, 1, 1, 1, 1, 64, {}),                                            # one token
    (2, 2, 2, 3, 1, 32, dict(left=0, right=0)),                         # every token sees itself
    (2, 33, 33, 2, 2, 64, dict(right=0)),
    (1, 64, 64, 2, 1, 64, {}),                                          # whole tiles
    (2, 65, 65, 2, 1, 64, dict(left=7, right=3)),
    (1, 129, 129, 4, 2, 128, dict(left=20, right=0, sinks=4)),
    (1, 200, 200, 3, 3, 96, dict(left=0, right=70, sinks=1)),
    (3, 197, 197, 2, 2, 64, {}),
    (1, 300, 300, 6, 2, 40, dict(left=64, right=64, sinks=70)),         # sinks past a tile
    (1, 517, 517, 2, 1, 16, dict(left=31, right=-1, sinks=5)),
    (1, 130, 130, 3, 1, 8, dict(left=-1, right=5)),
    (1, 600, 600, 1, 1, 80, dict(left=15, right=0, sinks=3)),           # sink tiles in parts
    (1, 50, 180, 4, 1, 72, dict(left=100, right=0, sinks=2)),           # the last 50 of 180
    (1, 700, 700, 7, 1, 64, dict(left=40, right=10)),                   # seven heads share one
]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", TRAIN, ids=lambda c: "x".join(map(str, c[:6])))
def test_forward_and_gradients(case, dt):
    B, Lq, Lk, H, Hkv, D, kw = case
    compare(draw(1, dt, B, Lq, H, D), draw(2, dt, B, Lk, Hkv, D), draw(3, dt, B, Lk, Hkv, D), draw(4, dt, B, Lq, H, D), **kw)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_ragged_lengths_and_garbage_past_them(dt):
    """Padding holds infinities and NaN in every input; lengths of 0 and 1, a length past Lk, negative starts."""
    B, L, H, Hkv, D = 6, 150, 4, 2, 64
    lengths, starts = [0, 1, 64, 97, 150, 999], [0, 0, 0, 0, 0, -3]
    q, k, v, do = draw(5, dt, B, L, H, D), draw(6, dt, B, L, Hkv, D), draw(7, dt, B, L, Hkv, D), draw(8, dt, B, L, H, D)
    for b, n in enumerate(lengths):
        for t, bad in ((q, math.nan), (k, math.inf), (v, math.nan), (do, -math.inf)):
            t[b, n:] = bad
    got = compare(q, k, v, do, lengths=lengths, starts=starts, left=30, right=12, sinks=4)
    for n in ("o", "dq", "dk", "dv"):
        assert torch.isfinite(got[n]).all(), n
        for b in range(4):
            assert (got[n][b, lengths[b]:] == 0).all(), (n, b)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kw", [dict(left=10, right=0, sinks=2), dict(left=3, right=40), dict(left=-1, right=0)])
def test_nonfinite_token_touches_only_who_sees_it(kw, dt):
    """One token of NaN and infinities in the middle of finite ones: rows and keys that do not see it stay as they are."""
    L, D, bad = 170, 64, 77
    q, k, v, do = (draw(s, dt, 1, L, 1, D) for s in (11, 12, 13, 14))
    seen = R.visible(L, L, L, 0, kw.get("left", -1), kw.get("right", -1), kw.get("sinks", 0))
    clean = run(q, k, v, do, **kw)
    for which, value in (("k", math.nan), ("v", math.inf), ("v", math.nan), ("q", math.nan), ("do", math.inf)):
        t = {"q": q.clone(), "k": k.clone(), "v": v.clone(), "do": do.clone()}
        t[which][0, bad] = value
        got = run(t["q"], t["k"], t["v"], t["do"], **kw)
        rows = ~seen[:, bad] if which in "kv" else torch.arange(L) != bad
        if which == "do":
            assert torch.equal(got["o"], clean["o"])
        assert torch.equal(got["o"][0, rows.cuda()], clean["o"][0, rows.cuda()]), which
        assert torch.equal(got["dq"][0, rows.cuda()], clean["dq"][0, rows.cuda()]), which
        # a key's gradient depends on the rows that see it, and through them on every key they see
        touched = seen[:, bad] if which in "kv" else torch.arange(L) == bad
        keys = ~(seen & touched[:, None]).any(0)
        assert keys.any() or kw["left"] == -1
        assert torch.equal(got["dk"][0, keys.cuda()], clean["dk"][0, keys.cuda()]), which
        assert torch.equal(got["dv"][0, keys.cuda()], clean["dv"][0, keys.cuda()]), which
        seers = seen[:, bad].cuda()
        if which == "v":
            assert not torch.isfinite(got["o"][0, seers]).any()


# B, Lq, Lk, H, Hkv, D, lengths, window
DECODE = [
    (1, 1, 1, 1, 1, 64, None, {}),
    (3, 1, 700, 4, 1, 64, [700, 1, 0], dict(right=0)),                        # one sequence is empty
    (2, 1, 5000, 3, 3, 128, [5000, 2049], dict(left=1023, right=0, sinks=4)),
    (1, 1, 9000, 8, 2, 64, [8765], dict(right=0)),                           # split along the keys
    (2, 5, 333, 6, 2, 40, [333, 5], dict(left=50, right=0, sinks=17)),
    (1, 16, 2000, 6, 2, 96, [1999], dict(left=300, right=0)),
    (2, 40, 900, 2, 1, 32, [900, 40], dict(right=0)),
    (1, 3, 3000, 1, 1, 8, [2999], dict(left=2000, right=0, sinks=100)),
]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "x".join(map(str, c[:6])))
def test_new_tokens_over_a_cache(case, dt):
    """The last Lq places of a filled cache; what lies past a sequence's length is garbage."""
    B, Lq, Lk, H, Hkv, D, lengths, kw = case
    q, k, v = draw(21, dt, B, Lq, H, D), draw(22, dt, B, Lk, Hkv, D), draw(23, dt, B, Lk, Hkv, D)
    if lengths:
        for b, n in enumerate(lengths):
            k[b, n:], v[b, n:] = math.nan, math.inf
        kw = dict(kw, lengths=lengths, starts=[n - Lq for n in lengths])
    compare(q, k, v, **kw)


def test_evicted_places_of_a_cache_may_hold_anything():
    q, k, v = draw(31, "f16", 1, 1, 2, 64), draw(32, "f16", 1, 400, 1, 64), draw(33, "f16", 1, 400, 1, 64)
    k[:, 3:300], v[:, 3:300] = math.nan, math.nan
    compare(q, k, v, left=99, right=0, sinks=3)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_large_scores(dt):
    """Scores of a few hundred: the running maximum moves in every tile, one key takes all."""
    q, k, v, do = (draw(s, dt, 1, 260, 2, 64, scale=c) for s, c in ((41, 6.0), (42, 6.0), (43, 1.0), (44, 1.0)))
    got = run(q, k, v, do, right=0)
    want = R.attention(q, k, v, do, right=0)
    # scores of up to ~400 carry fp32 errors of 400 * 2^-24 * a few in the exponent
    for n in got:
        R.within(n, got[n], want[n][0], want[n][1] * 4 + 400 * 2.0 ** -21 * want[n][0].abs().max())


def test_strides_views_and_alignment():
    """Packed views, permuted storage and unaligned rows give the same bits as contiguous tensors."""
    B, L, H, Hkv, D = 2, 90, 4, 2, 64
    qkv, do = draw(51, "f16", B, L, H + 2 * Hkv, D), draw(52, "f16", B, L, H, D)
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
    want = run(q.contiguous(), k.contiguous(), v.contiguous(), do, left=20, right=4, sinks=2)
    odd = torch.zeros(B, L, H, D + 1, dtype=torch.float16, device="cuda")
    odd[..., 1:] = q
    heads_first = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)
    for got in (run(q, k, v, do, left=20, right=4, sinks=2),
                run(odd[..., 1:], heads_first(k), heads_first(v), heads_first(do), left=20, right=4, sinks=2),
                run(q.permute(3, 2, 1, 0).contiguous().permute(3, 2, 1, 0), k, v, do, left=20, right=4, sinks=2)):
        for n in want:
            assert torch.equal(got[n], want[n]), n
    one = do[:1, :1, :1].expand(B, L, H, D)  # a broadcast gradient
    a, b = run(q, k, v, one, left=20), run(q, k, v, one.contiguous(), left=20)
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_reproducible_other_stream_and_graph():
    q, k, v = draw(61, "bf16", 2, 1, 4, 128), draw(62, "bf16", 2, 3000, 2, 128), draw(63, "bf16", 2, 3000, 2, 128)
    from paper_2607_21271_amd.attention import window_attention
    want = window_attention(q, k, v)
    assert torch.equal(window_attention(q, k, v), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = window_attention(q, k, v)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = window_attention(q, k, v)
    for step in range(3):
        q.copy_(draw(70 + step, "bf16", 2, 1, 4, 128))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, window_attention(q, k, v)), step
    qt, kt, vt, do = (draw(s, "f16", 1, 700, 2, 64) for s in (81, 82, 83, 84))
    a, b = (run(qt, kt, vt, do, left=50, right=0, sinks=4) for _ in range(2))
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_offsets_past_32_bits():
    """The last sequence and last tokens of caches of more than 2^32 bytes and 2^31 elements."""
    B, Lk, Hkv, D = 2, 1 << 20, 8, 128
    k = torch.zeros(B, Lk, Hkv, D, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    q = draw(91, "f16", B, 1, Hkv, D)
    k[1, -200:], v[1, -200:] = draw(92, "f16", 200, Hkv, D), draw(93, "f16", 200, Hkv, D)
    from paper_2607_21271_amd.attention import window_attention
    got = window_attention(q, k, v, left=199, right=0)
    want = R.attention(q[1:], k[1:, -200:], v[1:, -200:], left=199, right=0)
    R.within("o", got[1:], *want["o"])


def test_gradient_against_differences():
    """Directional derivatives of the kernel's own fp32 forward."""
    q, k, v, do = (draw(s, "f32", 1, 70, 2, 32) for s in (101, 102, 103, 104))
    k, v = k[:, :, :1].contiguous(), v[:, :, :1].contiguous()
    kw = dict(left=20, right=3, sinks=2)
    got = run(q, k, v, do, **kw)
    h = 1e-2
    for i, n in enumerate(("dq", "dk", "dv")):
        base = [q, k, v]
        d = draw(110 + i, "f32", *base[i].shape)
        f = []
        for s in (h, -h):
            t = list(base)
            t[i] = base[i] + s * d
            f.append((run(*t, **kw)["o"].double() * do.double()).sum())
        diff = ((f[0] - f[1]) / (2 * h)).item()
        dot = (got[n].double() * d.double()).sum().item()
        # central difference: h^2 / 6 times a third derivative of order |dot|'s terms, and 2^-22 / h of the outputs' sizes
        size = (got[n].double().abs() * d.double().abs()).sum().item()
        assert abs(diff - dot) <= (h * h + 2.0 ** -22 / h) * size + 1e-3, (n, diff, dot)


@pytest.mark.parametrize("power", [-12, 9])
def test_fp16_gradients_far_from_one(power):
    """Gradients of 2^-12 and 2^9 times as large are the same numbers up to the result's own rounding: no product in
    between loses bits to fp16's range."""
    L, D = 300, 64
    q, k, v, do = (draw(s, "f16", 1, L, 2, D) for s in (141, 142, 143, 144))
    k, v = k[:, :, :1].contiguous(), v[:, :, :1].contiguous()
    do = do.clamp(-4, 4)
    a, b = run(q, k, v, do, right=0), run(q, k, v, (do.double() * 2.0 ** power).half(), right=0)
    for n in ("dq", "dk", "dv"):
        x, y = a[n].double(), b[n].double() * 2.0 ** -power
        # the scaled do is exact (or rounded by 2^-25 where it is subnormal: that error passes on like do's own size);
        # either result is rounded once, the smaller one by 2^-25 at least
        scale = x.abs().max()
        bound = 2 * 2.0 ** -11 * x.abs() + 2.0 ** (-25 - min(power, 0)) * 4 + 2.0 ** -14 * scale
        assert ((x - y).abs() <= bound).all(), (n, ((x - y).abs() - bound).max())


def test_packed_attention_with_positions():
    """Rotary and attention in one call on a packed buffer against the two operators apart, with its gradient."""
    from paper_2607_21271_amd import attention, rotary
    B, H, Hkv, dh, T = 2, 4, 2, 8, 4
    sections, D = (1, 2, 1), 32
    pos = rotary.grid_positions((2, 5, 6), prefix=3, device="cuda")
    L = pos.shape[0]
    freqs = rotary.axis_frequencies(sections, device="cuda")
    qkv, do = draw(121, "f32", B, L, H + 2 * Hkv, D), draw(122, "f32", B, L, H, D)
    kw = dict(left=20, right=20, sinks=3)
    lengths = ints([L, L - 9])
    x = qkv.clone().requires_grad_()
    o = attention.packed_window_attention(x, Hkv, pos, freqs, sections, T, lengths=lengths, **kw)
    (gx,) = torch.autograd.grad(o, (x,), do)
    y = qkv.clone().requires_grad_()
    qk = rotary.rotary_axes(y[:, :, :H + Hkv], pos, freqs, sections, T)
    o2 = attention.window_attention(qk[:, :, :H], qk[:, :, H:], y[:, :, H + Hkv:], lengths=lengths,
                                    starts=torch.zeros(B, dtype=torch.int32, device="cuda"), **kw)
    (gy,) = torch.autograd.grad(o2, (y,), do)
    assert torch.equal(o, o2) and torch.equal(gx, gy)
    with torch.no_grad():
        assert torch.equal(attention.packed_window_attention(qkv, Hkv, pos, freqs, sections, T, lengths=lengths, **kw), o)
    plain = attention.packed_window_attention(qkv, Hkv, **kw)
    assert torch.equal(plain, attention.window_attention(qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:], **kw))


def test_empty_sizes():
    from paper_2607_21271_amd.attention import window_attention
    z = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")
    assert window_attention(z(0, 3, 2, 64), z(0, 3, 2, 64), z(0, 3, 2, 64)).shape == (0, 3, 2, 64)
    assert window_attention(z(2, 0, 2, 64), z(2, 3, 2, 64), z(2, 3, 2, 64)).shape == (2, 0, 2, 64)
    q = draw(131, "f16", 2, 3, 2, 64)
    assert (window_attention(q, z(2, 0, 2, 64), z(2, 0, 2, 64)) == 0).all()  # no keys at all
    k = draw(132, "f16", 2, 5, 2, 64).requires_grad_()
    o = window_attention(z(2, 0, 2, 64).requires_grad_(), k, k)
    assert (torch.autograd.grad(o.sum(), k)[0] == 0).all()
