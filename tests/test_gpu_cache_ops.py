"""Operators around a bounded KV cache on the GPU, against plain 64-bit implementations: rotary append, attention that totals the
keys' weights, eviction -- and a run of them together behind the INT4 projection."""
import numpy as np
import pytest

import gen

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def mb():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_18655_b200 import binding
    binding.lib()
    return binding


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(a):
    return dev(np.asarray(a, dtype=np.int32))


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ rotary append
def rotated(x, pos, freq, gain, rotary, interleaved):
    """x float64 [rows][heads][hd]; also what the roundings scale with: |a| + |b| of a pair"""
    a_at = np.arange(rotary // 2) * (2 if interleaved else 1)
    b_at = a_at + (1 if interleaved else rotary // 2)
    ang = pos.astype(np.float64)[:, None, None] * freq
    c, s = np.cos(ang) * gain, np.sin(ang) * gain
    out, size = x.copy(), np.abs(x)
    a, b = x[..., a_at], x[..., b_at]
    out[..., a_at], out[..., b_at] = a * c - b * s, b * c + a * s
    size[..., a_at] = size[..., b_at] = (np.abs(a) + np.abs(b)) * gain
    return out, size


def close_fp16(got, want, size):
    """A rounding to fp16 (half a step, 2^-11, or 2^-25 below the normal range) of a value from 32-bit products: cos and sin good to
    2^-22 (an angle to 2^-22 and half a step), two products and a sum: 2^-20 of |a| + |b| covers them."""
    got = got.double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0**-11 * np.abs(want) + 2.0**-20 * size + 2.0**-25).all()


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("n,T,Hq,Hkv,hd,rotary,inter,base", [
    (1, 1, 32, 8, 64, 64, False, 512), (8, 1, 24, 8, 128, 128, False, 0), (3, 5, 8, 2, 64, 16, True, 70000),
    (2, 33, 6, 6, 128, 96, True, 1000003), (2, 7, 5, 1, 64, 48, False, -9), (1, 1300, 4, 2, 128, 112, False, 4000000),
    (1, 1300, 3, 1, 64, 32, True, 12345), (65, 1, 1, 1, 128, 80, True, 3)])
def test_rope_append(mb, fp32, n, T, Hq, Hkv, hd, rotary, inter, base):
    rng = np.random.default_rng(n * 1000 + T + hd)
    lens = [int(x) for x in rng.integers(0, 20, n)]
    cap, rows, W = max(lens) + T + 3, n * T, (Hq + 2 * Hkv) * hd
    f = np.float32 if fp32 else np.float16
    # rows of one matrix with room at the end, as a wider fused projection has it
    x = rng.standard_normal((rows, W + 16)).astype(f)
    xd = dev(x)
    q, k, v = xd[:, :Hq * hd], xd[:, Hq * hd:(Hq + Hkv) * hd], xd[:, (Hq + Hkv) * hd:W]
    pos = (base + np.arange(rows) * 3).astype(np.int32)
    freq, gain = mb.mlora_rope_frequencies(rotary, 1e4, "ramp", 4.0, 4096.0, 1.0, 32.0)
    own = rng.standard_normal((2, n, Hkv, cap, hd)).astype(np.float16)
    ok, ov = dev(own[0]), dev(own[1])
    wt, ps = torch.full((n, Hkv, cap), 7.0, device="cuda"), torch.full((n, Hkv, cap), -5, dtype=torch.int32, device="cuda")
    qo, st = torch.full((rows, Hq, hd), NAN, dtype=torch.float16, device="cuda"), status()
    mb.mlora_rope_append(q, k, v, dev(pos), freq.cuda(), qo, ok, ov, i32(lens), st, gain=gain, interleaved=inter, own_weight=wt, own_position=ps)
    assert int(st.item()) == 0
    x = x.astype(np.float64)
    fr = freq.numpy()
    close_fp16(qo, *rotated(x[:, :Hq * hd].reshape(rows, Hq, hd), pos, fr, gain, rotary, inter))
    wk, sk = rotated(x[:, Hq * hd:(Hq + Hkv) * hd].reshape(rows, Hkv, hd), pos, fr, gain, rotary, inter)
    wv = x[:, (Hq + Hkv) * hd:W].reshape(rows, Hkv, hd).astype(np.float16)
    for s in range(n):
        at, new = lens[s], slice(lens[s], lens[s] + T)
        mine = slice(s * T, (s + 1) * T)
        close_fp16(ok[s, :, new], wk[mine].transpose(1, 0, 2), sk[mine].transpose(1, 0, 2))
        assert np.array_equal(ov[s, :, new].cpu().numpy(), wv[mine].transpose(1, 0, 2))
        assert bool((wt[s, :, new] == 0).all()) and np.array_equal(ps[s, :, new].cpu().numpy(), np.broadcast_to(pos[mine], (Hkv, T)))
        for t, was in ((ok, own[0]), (ov, own[1])):                     # nothing else is written
            assert np.array_equal(t[s, :, :at].cpu().numpy(), was[s, :, :at]) and np.array_equal(t[s, :, at + T:].cpu().numpy(), was[s, :, at + T:])
        assert bool((wt[s, :, :at] == 7).all()) and bool((wt[s, :, at + T:] == 7).all()) and bool((ps[s, :, at + T:] == -5).all())


def test_rope_parts_alone_and_in_place(mb):
    """q alone, K/V alone, q in place: the same bits as all at once; K/V of a prompt straight into a prefix."""
    rng = np.random.default_rng(5)
    n, T, Hq, Hkv, hd, cap = 2, 9, 4, 2, 64, 40
    q, k, v = (dev(rng.standard_normal((n * T, h, hd)).astype(np.float16)) for h in (Hq, Hkv, Hkv))
    pos, lens = i32(np.arange(n * T) + 100), i32([4, 0])
    freq = mb.mlora_rope_frequencies(32, 1e4)[0].cuda()
    new = lambda: torch.zeros(n, Hkv, cap, hd, dtype=torch.float16, device="cuda")  # noqa: E731
    st, qo, k1, v1, k2, v2 = status(), torch.empty_like(q), new(), new(), new(), new()
    mb.mlora_rope_append(q, k, v, pos, freq, qo, k1, v1, lens, st)
    mb.mlora_rope_append(None, k, v, pos, freq, None, k2, v2, lens, st)
    assert torch.equal(k1, k2) and torch.equal(v1, v2)
    qi = q.clone()
    mb.mlora_rope_append(qi, None, None, pos, freq, qi, None, None, None, None)
    assert torch.equal(qi, qo)
    pk, pv = (torch.zeros(1, Hkv, n * T, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    mb.mlora_rope_append(None, k, v, pos, freq, None, pk, pv, i32([0]), st)
    assert torch.equal(pk[0, :, :T], k1[0, :, 4:4 + T]) and torch.equal(pv[0, :, T:], v1[1, :, :T])
    assert int(st.item()) == 0


def test_rope_special_values_stay_in_their_pair(mb):
    """inf, NaN and values beyond fp16 reach only their own pair; a row that does not fit appends nothing and says so"""
    hd, cap = 64, 8
    q = torch.zeros(3, 1, hd, device="cuda")
    q[0, 0, 5], q[1, 0, 0], q[2, 0, 40] = NAN, float("inf"), 1e6
    kv = torch.ones(3, 1, hd, device="cuda")
    freq = mb.mlora_rope_frequencies(32, 1e4)[0].cuda()
    qo, st = torch.empty(3, 1, hd, dtype=torch.float16, device="cuda"), status()
    k, v = (torch.zeros(3, 1, cap, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    mb.mlora_rope_append(q, kv, kv, i32([1, 2, 3]), freq, qo, k, v, i32([8, -1, 7]), st)
    assert int(st.item()) == -3
    bad = ~torch.isfinite(qo[:, 0])
    assert bad.nonzero().tolist() == [[0, 5], [0, 21], [1, 0], [1, 16], [2, 40]]
    assert not k[:2].any() and not v[:2].any() and bool((v[2, 0, 7] == 1).all()) and not v[2, 0, :7].any()


# ------------------------------------------------------------------ attention with totals
def scored_case(mb, n, T, Hq, Hkv, hd, P, lens, seed, parents=None, slack=3, bound=None, ws_off=0):
    """Random inputs, everything behind a stream's rows NaN; runs the call twice on one workspace and checks it."""
    rng = np.random.default_rng(seed)
    cap = max(lens) + T + slack
    bound = max(lens) if bound is None else bound
    G = Hq // Hkv
    q = rng.standard_normal((n * T, Hq, hd)).astype(np.float16)
    pk, pv = (rng.standard_normal((Hkv, P, hd)).astype(np.float16) for _ in range(2))
    ok, ov = (rng.standard_normal((n, Hkv, cap, hd)).astype(np.float16) for _ in range(2))
    for s in range(n):
        ok[s, :, lens[s] + T:], ov[s, :, lens[s] + T:] = np.nan, np.nan
    w0, p0 = rng.random((n, Hkv, cap)).astype(np.float32), rng.random((Hkv, P)).astype(np.float32)
    for s in range(n):
        w0[s, :, lens[s] + T:] = np.nan
    ws = torch.full((mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, P, bound) + ws_off,), 255, dtype=torch.uint8, device="cuda")[ws_off:]
    st, res = status(), []
    dq, dpk, dpv, dok, dov = dev(q), dev(pk) if P else None, dev(pv) if P else None, dev(ok), dev(ov)
    for _ in range(2):
        out = torch.full((n * T, Hq, hd), NAN, dtype=torch.float16, device="cuda")
        wt, pw = dev(w0), dev(p0) if P else None
        mb.mlora_attention_scored(dq, dpk, dpv, dok, dov, i32(lens), bound, None if parents is None else i32(parents), out, wt, pw, ws, st)
        res.append((out, wt, pw))
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    out, wt, pw = res[0]
    assert torch.equal(out, res[1][0]) and torch.equal(wt.nan_to_num(-1), res[1][1].nan_to_num(-1)) and (pw is None or torch.equal(pw, res[1][2]))
    out, wt = out.double().cpu().numpy(), wt.double().cpu().numpy()
    d = lambda a: torch.from_numpy(a).cuda().double()  # noqa: E731
    pre = np.zeros((Hkv, P))
    pre_tol = np.zeros(Hkv)
    for s in range(n):
        L = lens[s] + T
        see = np.zeros((T, P + L), dtype=bool)
        see[:, :P + lens[s]] = True
        for t in range(T):
            a = t
            while a >= 0:
                see[t, P + lens[s] + a] = True
                a = (a - 1 if parents is None else parents[s][a])
        for h in range(Hkv):
            k, v = (np.concatenate([a[h], b[s, h, :L]]) for a, b in ((pk, ok), (pv, ov)))
            qs = q[s * T:(s + 1) * T, h * G:(h + 1) * G].reshape(T * G, hd)
            e = (d(qs) @ d(k).T / np.sqrt(hd)).masked_fill(~torch.from_numpy(np.repeat(see, G, axis=0)).cuda(), -np.inf)
            # a score: hd products added in 32 bits (a step of 2^-23 each time), scaled and shifted in powers of two
            delta = float((d(np.abs(qs)) @ d(np.abs(k)).T).max()) / np.sqrt(hd) * (hd + 8) * 2.0**-23
            p = torch.softmax(e, dim=-1)
            want = (p @ d(v)).cpu().numpy()
            # weights: the scores' errors twice (numerator, sum), 2^-20 for exponentials and sums; p as fp16 for the product
            # (2^-11, or 2^-25 of the largest below the normal range), the output as fp16
            size = (p @ d(np.abs(v))).cpu().numpy()
            low = 2.0**-25 * np.abs(v.astype(np.float64)).sum(axis=0)
            got = out[s * T:(s + 1) * T, h * G:(h + 1) * G].reshape(T * G, hd)
            tol = 2.0**-11 * np.abs(want) + (2.0**-11 + 2 * delta + 2.0**-20) * size * (1 + 2.0**-8) + low + 2.0**-25
            assert (np.abs(got - want) <= tol).all(), (s, h, np.abs(got - want).max())
            tot = p.sum(dim=0).cpu().numpy()
            rel = 2 * delta + 2.0**-20 + (T * G) * 2.0**-24
            grown = wt[s, h, :L] - w0[s, h, :L]
            assert (np.abs(grown - tot[P:]) <= rel * tot[P:] + 2.0**-23 * (w0[s, h, :L] + tot[P:])).all()
            pre[h] += tot[:P]
            pre_tol[h] = max(pre_tol[h], rel)
    if P:
        pw = pw.double().cpu().numpy()
        rel = pre_tol[:, None] + n * T * G * 2.0**-24
        assert (np.abs(pw - p0 - pre) <= rel * pre + 2.0**-23 * (p0 + pre)).all()
    for s in range(n):
        assert np.isnan(wt[s, :, lens[s] + T:]).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,Hq,Hkv,P,lens", [
    (1, 32, 8, 512, [64]), (1, 8, 2, 0, [0]), (3, 8, 2, 1, [0, 1, 63]), (2, 4, 4, 64, [64, 65]), (4, 6, 2, 100, [0, 500, 31, 700]),
    (8, 8, 2, 513, [3, 64, 65, 1, 127, 128, 129, 200]), (2, 16, 1, 777, [1500, 4]), (3, 34, 2, 15, [16, 17, 15]), (2, 40, 1, 300, [90, 0]),
    (20, 8, 2, 129, [7 * i for i in range(20)]), (1, 4, 1, 0, [6000]), (2, 8, 8, 2500, [2000, 1])])
def test_scored_one_row_per_stream(mb, hd, n, Hq, Hkv, P, lens):
    scored_case(mb, n, 1, Hq, Hkv, hd, P, lens, seed=hd + n + P)


def tree(rng, T):
    return [-1] + [int(rng.integers(0, i)) for i in range(1, T)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,T,Hq,Hkv,P,lens,kind", [
    (1, 2, 8, 2, 0, [0], "tree"), (2, 16, 8, 2, 300, [63, 130], "tree"), (2, 64, 8, 2, 65, [1, 40], "tree"), (3, 10, 12, 4, 0, [4, 0, 200], "tree"),
    (2, 5, 4, 4, 128, [128, 3], "chain"), (2, 64, 3, 1, 640, [300, 0], "chain"), (8, 30, 8, 2, 512, [16 * i for i in range(8)], "tree"),
    (1, 3, 16, 1, 1, [1000], "tree"), (2, 64, 16, 1, 70, [61, 64], "tree"), (1, 63, 2, 2, 64, [65], "star"), (2, 7, 260, 2, 40, [5, 150], "tree")])
def test_scored_trees(mb, hd, n, T, Hq, Hkv, P, lens, kind):
    rng = np.random.default_rng(T)
    parents = None if kind == "chain" else [[-1] + [0] * (T - 1)] * n if kind == "star" else [tree(rng, T) for _ in range(n)]
    scored_case(mb, n, T, Hq, Hkv, hd, P, lens, seed=T + P, parents=parents)


def test_scored_workspace_of_a_larger_bound_and_any_start(mb):
    scored_case(mb, 3, 1, 8, 2, 64, 100, [5, 900, 0], seed=1, bound=2000, slack=1200, ws_off=7)
    scored_case(mb, 2, 9, 8, 2, 128, 100, [5, 90], seed=1, bound=300, slack=300, ws_off=3, parents=[tree(np.random.default_rng(0), 9)] * 2)


def test_scored_matches_plain_attention_call(mb):
    """out agrees with mlora_attention on the same tensors to their roundings; prefix totals may be left out"""
    rng = np.random.default_rng(3)
    n, T, Hq, Hkv, hd, P, cap = 4, 1, 32, 8, 64, 512, 300
    lens = [0, 20, 150, 299]
    q, pk, pv = (dev(rng.standard_normal(s).astype(np.float16)) for s in ((n, Hq, hd), (Hkv, P, hd), (Hkv, P, hd)))
    ok, ov = (dev(rng.standard_normal((n, Hkv, cap, hd)).astype(np.float16)) for _ in range(2))
    par, st = i32([[-1]] * n), status()
    a, b = (torch.empty(n, Hq, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    ws = torch.empty(mb.mlora_attention_workspace_bytes(n, T, Hq, Hkv, hd, P, cap), dtype=torch.uint8, device="cuda")
    mb.mlora_attention(q, pk, pv, ok, ov, i32(lens), 299, par, a, ws, st)
    ws2 = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, P, 299), dtype=torch.uint8, device="cuda")
    wt = torch.zeros(n, Hkv, cap, device="cuda")
    mb.mlora_attention_scored(q, pk, pv, ok, ov, i32(lens), 299, par, b, wt, None, ws2, st)
    assert int(st.item()) == 0
    # two roundings to fp16 of the output and of the weights each; |v| averages to at most 5 here
    assert float((a.float() - b.float()).abs().max()) <= 4 * 2.0**-11 * 5
    # a row's weights add up to one over prefix and own rows: own totals lie below the heads of a group
    assert float(wt.sum(dim=2).max()) <= Hq // Hkv


def test_scored_reports_bad_trees_and_lengths(mb):
    n, T, Hq, Hkv, hd, cap = 2, 3, 4, 2, 64, 40
    z = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")  # noqa: E731
    ws = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, 16, 30), dtype=torch.uint8, device="cuda")
    for lens, par in (([3, 4], [[-1, 0, 2], [-1, 0, 0]]), ([3, 4], [[-1, 0, 0], [0, 0, 1]]), ([3, 4], [[-1, 0, 0], [-1, -7, 99]]),
                      ([-1, 4], [[-1, 0, 1]] * 2), ([3, 31], [[-1, 0, 1]] * 2)):
        st, wt = status(), torch.zeros(n, Hkv, cap, device="cuda")
        mb.mlora_attention_scored(z(n * T, Hq, hd), z(Hkv, 16, hd), z(Hkv, 16, hd), z(n, Hkv, cap, hd), z(n, Hkv, cap, hd), i32(lens), 30, i32(par),
                                  z(n * T, Hq, hd), wt, None, ws, st)
        assert int(st.item()) == -1


@pytest.mark.parametrize("T", [1, 40])
def test_scored_takes_lengths_as_within_their_bound(mb, T):
    """Lengths far outside 0 .. suffix_bound: reported, and the results of the nearest length inside"""
    n, Hq, Hkv, hd, cap, bound = 4, 8, 2, 64, 400, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(*s, generator=g, device="cuda", dtype=torch.float16) for s in ((n * T, Hq, hd), (n, Hkv, cap, hd), (n, Hkv, cap, hd)))
    ws = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, 0, bound), dtype=torch.uint8, device="cuda")
    res = []
    for lens, code in (([0, 0, bound, bound], 0), ([-2**31, -5, 2**31 - 1, bound + 1], -1)):
        out, w, st = torch.zeros_like(q), torch.zeros(n, Hkv, cap, device="cuda"), status()
        mb.mlora_attention_scored(q, None, None, k, v, i32(lens), bound, None, out, w, None, ws, st)
        assert int(st.item()) == code
        res.append((out, w))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1]) and not res[1][1][:, :, bound + T:].any()


def test_scored_large_scores_and_infinite_keys(mb):
    """Scores far apart, a key of -inf features (weight 0 by the softmax itself) and one that takes all the weight."""
    n, Hq, Hkv, hd, cap = 1, 4, 1, 64, 70
    q = torch.ones(n, Hq, hd, dtype=torch.float16, device="cuda")
    ok = torch.zeros(n, Hkv, cap, hd, dtype=torch.float16, device="cuda")
    ov = torch.arange(cap, device="cuda", dtype=torch.float16).view(1, 1, cap, 1).expand(n, Hkv, cap, hd).contiguous()
    ok[0, 0, 3], ok[0, 0, 17] = -float("inf"), 1000.0
    ok[0, 0, 30] = -65504.0
    out, wt, st = torch.empty(n, Hq, hd, dtype=torch.float16, device="cuda"), torch.zeros(n, Hkv, cap, device="cuda"), status()
    ws = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, 1, Hq, Hkv, hd, 0, 60), dtype=torch.uint8, device="cuda")
    mb.mlora_attention_scored(q, None, None, ok, ov, i32([60]), 60, None, out, wt, None, ws, st)
    assert bool((out == 17).all()) and wt[0, 0].nonzero().flatten().tolist() == [17] and float(wt[0, 0, 17]) == Hq


# ------------------------------------------------------------------ eviction
def evict_reference(w, pos, S, budget, recent, newest):
    """source rows of what is left of one segment, in place order"""
    a = w[:S].astype(np.float64)
    a = np.where(np.isnan(a), -np.inf, a)
    low = np.isnan(w[:S])                           # NaN below -inf
    new = (pos[:S].astype(np.int64) > newest - recent) if recent else np.zeros(S, dtype=bool)
    order = np.lexsort((np.arange(S), low, -a, ~new))
    keep = np.zeros(S, dtype=bool)
    keep[order[:budget]] = True
    src = np.arange(min(S, budget))
    src[~keep[:len(src)]] = np.flatnonzero(keep[budget:]) + budget
    return src


def evict_case(mb, n, Hkv, hd, lens, budget, recent, seed, in_place=False, weights="random", slack=5, ws_off=0, bound=None):
    rng = np.random.default_rng(seed)
    bound = max(lens) if bound is None else bound
    cap = bound + slack
    k, v = (rng.integers(0, 65536, (n, Hkv, cap, hd), dtype=np.uint16).view(np.float16) for _ in range(2))
    if weights == "random":
        w = rng.exponential(size=(n, Hkv, cap)).astype(np.float32)
    elif weights == "ties":
        w = rng.integers(0, 3, (n, Hkv, cap)).astype(np.float32)
    else:
        w = rng.choice(np.array([0.0, -0.0, np.nan, np.inf, -np.inf, 1e-45, -1e-45, 3e38, -1.0], dtype=np.float32), (n, Hkv, cap))
    pos = np.stack([rng.permutation(cap) for _ in range(n * Hkv)]).reshape(n, Hkv, cap).astype(np.int32)
    newest = [max(0, s - 1) for s in lens]
    dk, dv, dw, dp = dev(k.view(np.int16)).view(torch.float16), dev(v.view(np.int16)).view(torch.float16), dev(w), dev(pos)
    ow, op = (dw, dp) if in_place else (torch.full_like(dw, 99.0), torch.full_like(dp, -99))
    ow0, op0 = (w, pos) if in_place else (ow.cpu().numpy(), op.cpu().numpy())
    ol, src, st = torch.full((n,), -1, dtype=torch.int32, device="cuda"), torch.full((n, Hkv, budget), -1, dtype=torch.int32, device="cuda"), status()
    ws = torch.full((mb.mlora_kv_evict_workspace_bytes(n, Hkv, bound, budget) + ws_off,), 255, dtype=torch.uint8, device="cuda")[ws_off:]
    mb.mlora_kv_evict(dk, dv, dw, dp, i32(lens), bound, i32(newest) if recent else None, budget, recent, ow, op, ol, ws, st, out_source=src)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and ol.tolist() == [min(s, budget) for s in lens]
    bits = lambda t: t.view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
    gk, gv, gw, gp, gs = bits(dk), bits(dv), ow.cpu().numpy(), op.cpu().numpy(), src.cpu().numpy()
    for s in range(n):
        for h in range(Hkv):
            want = evict_reference(w[s, h], pos[s, h], lens[s], budget, recent, newest[s])
            m = len(want)
            assert np.array_equal(gs[s, h, :m], want) and (gs[s, h, m:] == -1).all()
            for got, was in ((gk, k.view(np.uint16)), (gv, v.view(np.uint16))):
                assert np.array_equal(got[s, h, :m], was[s, h][want]) and np.array_equal(got[s, h, m:], was[s, h, m:])
            assert np.array_equal(gw[s, h, :m].view(np.uint32), w[s, h][want].view(np.uint32)) and np.array_equal(gp[s, h, :m], pos[s, h][want])
            assert np.array_equal(gw[s, h, m:].view(np.uint32), ow0[s, h, m:].view(np.uint32)) and np.array_equal(gp[s, h, m:], op0[s, h, m:])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("weights", ["random", "ties", "special"])
@pytest.mark.parametrize("n,Hkv,hd,lens,budget,recent", [
    (1, 8, 64, [257], 256, 32), (1, 1, 64, [2], 1, 0), (2, 2, 128, [0, 1], 1, 1), (3, 2, 64, [100, 101, 140], 100, 100), (2, 3, 128, [1023, 1025], 512, 0),
    (4, 2, 64, [1, 33, 64, 2000], 33, 7), (2, 1, 128, [5000, 4096], 4000, 256), (1, 2, 64, [9000], 17, 17), (1, 1, 64, [31], 31, 3),
    (2, 1, 64, [40000, 33000], 30000, 1000), (1, 2, 128, [70001], 35000, 0), (5, 1, 64, [300, 301, 302, 303, 304], 300, 64)])
def test_evict(mb, in_place, weights, n, Hkv, hd, lens, budget, recent):
    evict_case(mb, n, Hkv, hd, lens, budget, recent, seed=sum(lens), in_place=in_place, weights=weights)


def test_evict_any_workspace_start_larger_bound_and_budget_beyond_it(mb):
    evict_case(mb, 2, 2, 64, [50, 80], 40, 8, seed=1, ws_off=5, bound=400)
    evict_case(mb, 2, 2, 64, [50, 80], 500, 8, seed=2, bound=90)


def test_evict_more_new_rows_than_the_budget(mb):
    """positions that repeat: the new rows alone exceed the budget, their totals decide"""
    n, hd, S, B = 1, 64, 64, 8
    rng = np.random.default_rng(0)
    w = rng.permutation(S).astype(np.float32).reshape(1, 1, S)
    pos = np.where(np.arange(S) % 2 == 0, 100, 0).astype(np.int32).reshape(1, 1, S)
    k = dev(np.arange(S * hd).reshape(1, 1, S, hd).astype(np.float16))
    dw, dp, ol, src, st = dev(w), dev(pos), i32([0]), torch.full((1, 1, B), -1, dtype=torch.int32, device="cuda"), status()
    ws = torch.empty(mb.mlora_kv_evict_workspace_bytes(n, 1, S, B), dtype=torch.uint8, device="cuda")
    mb.mlora_kv_evict(k, k.clone(), dw, dp, i32([S]), S, i32([100]), B, 4, dw, dp, ol, ws, st, out_source=src)
    assert src[0, 0].tolist() == evict_reference(w[0, 0], pos[0, 0], S, B, 4, 100).tolist()


def test_evict_without_positions_and_bad_length(mb):
    rng = np.random.default_rng(1)
    n, hd, S, B = 3, 64, 40, 16
    w = rng.random((n, 1, S)).astype(np.float32)
    k = dev(rng.standard_normal((n, 1, S, hd)).astype(np.float16))
    v, k0 = k.clone(), k.cpu().numpy()
    dw, ol, st = dev(w), i32([0] * n), status()
    ws = torch.empty(mb.mlora_kv_evict_workspace_bytes(n, 1, S - 5, B), dtype=torch.uint8, device="cuda")
    mb.mlora_kv_evict(k, v, dw, None, i32([20, -3, S]), S - 5, None, B, 0, dw, None, ol, ws, st)
    assert int(st.item()) == -1 and ol.tolist() == [B, 0, B]             # (bounded: a length of -3 counts as 0, of 40 as 35)
    for s, S_used in ((0, 20), (2, S - 5)):
        want = evict_reference(w[s, 0], np.zeros(S), S_used, B, 0, 0)
        assert np.array_equal(k[s, 0, :B].cpu().numpy(), k0[s, 0][want]) and np.array_equal(v[s, 0, :B].cpu().numpy(), k0[s, 0][want])


# ------------------------------------------------------------------ refusals of the binding, streams, graphs, large offsets
@pytest.mark.parametrize("T", [1, 16])
def test_scored_writes_right_behind_its_rows(mb, T):
    """q and out as the two halves of one buffer; out over q is refused and writes nothing"""
    rng = np.random.default_rng(31)
    n, Hq, Hkv, hd, P, cap = 8, 32, 8, 64, 512, 320
    both = dev(rng.standard_normal((2, n * T, Hq, hd)).astype(np.float16))
    q, out, apart = both[0], both[1], torch.empty(n * T, Hq, hd, dtype=torch.float16, device="cuda")
    pk, pv = (dev(rng.standard_normal((Hkv, P, hd)).astype(np.float16)) for _ in range(2))
    k, v = (dev(rng.standard_normal((n, Hkv, cap, hd)).astype(np.float16)) for _ in range(2))
    lens, st, bound = i32([30 * s for s in range(n)]), status(), 256
    w, w2 = torch.zeros(n, Hkv, cap, device="cuda"), torch.zeros(n, Hkv, cap, device="cuda")
    ws = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, P, bound), dtype=torch.uint8, device="cuda")
    mb.mlora_attention_scored(q, pk, pv, k, v, lens, bound, None, apart, w, None, ws, st)
    mb.mlora_attention_scored(q, pk, pv, k, v, lens, bound, None, out, w2, None, ws, st)
    assert torch.equal(out, apart) and torch.equal(w, w2) and int(st.item()) == 0
    before = q.clone()
    with pytest.raises(mb.MloraError) as e:
        mb.mlora_attention_scored(q, pk, pv, k, v, lens, bound, None, q, w2, None, ws, st)
    assert e.value.code == -1 and torch.equal(q, before) and torch.equal(w, w2)


def test_binding_refuses_wrong_tensors(mb):
    n, T, Hq, Hkv, hd, cap = 2, 1, 4, 2, 64, 32
    f = lambda *s, t=torch.float16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    good = dict(q=f(n, Hq, hd), pk=f(Hkv, 16, hd), pv=f(Hkv, 16, hd), k=f(n, Hkv, cap, hd), v=f(n, Hkv, cap, hd), lens=i32([3, 4]), bound=8,
                par=None, out=f(n, Hq, hd), w=f(n, Hkv, cap, t=torch.float32), pw=None,
                ws=f(mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, 16, 8), t=torch.uint8), st=status())
    mb.mlora_attention_scored(*good.values())
    for bad in (dict(q=f(n, Hq, hd, t=torch.float32)), dict(q=f(n, hd, Hq).transpose(1, 2)), dict(k=f(n, Hkv, cap + 1, hd)), dict(v=f(n, Hkv, cap + 1, hd)),
                dict(lens=f(n, t=torch.int64)), dict(lens=i32([3])), dict(out=f(n, Hq, hd).cpu()), dict(w=f(n, Hkv, cap)), dict(pv=f(Hkv, 15, hd)),
                dict(par=i32([[-1]])), dict(pw=f(Hkv, 15, t=torch.float32)), dict(st=f(1, t=torch.int64))):
        with pytest.raises(mb.MloraError) as e:
            mb.mlora_attention_scored(*{**good, **bad}.values())
        assert e.value.code == -1, bad
    freq = mb.mlora_rope_frequencies(64, 1e4)[0].cuda()
    k1, x = f(n, Hkv, hd), f(n, Hq, hd)
    args = dict(q=x, k=k1, v=k1, pos=i32([0, 1]), freq=freq, qo=f(n, Hq, hd), ok=f(n, Hkv, cap, hd), ov=f(n, Hkv, cap, hd), lens=i32([0, 1]), st=status())
    mb.mlora_rope_append(*args.values())
    for bad in (dict(q=f(n, Hq + 1, hd)), dict(k=f(n, Hkv, hd, t=torch.float32)), dict(q=x.transpose(1, 2)), dict(freq=freq.float()), dict(pos=i32([0, 1, 2])),
                dict(q=x.bfloat16()), dict(ov=f(n, Hkv, cap, hd).cpu()), dict(k=None), dict(qo=None, q=None, k=None, v=None, ok=None, ov=None)):
        with pytest.raises((mb.MloraError, AttributeError)):
            mb.mlora_rope_append(*{**args, **bad}.values())
    ev = dict(k=f(n, Hkv, cap, hd), v=f(n, Hkv, cap, hd), w=f(n, Hkv, cap, t=torch.float32), p=f(n, Hkv, cap, t=torch.int32), lens=i32([9, 3]), bound=16,
              newest=i32([8, 2]), budget=8, recent=2, ow=f(n, Hkv, cap, t=torch.float32), op=f(n, Hkv, cap, t=torch.int32), ol=i32([0, 0]),
              ws=f(mb.mlora_kv_evict_workspace_bytes(n, Hkv, 16, 8), t=torch.uint8), st=status())
    mb.mlora_kv_evict(*ev.values())
    for bad in (dict(v=f(n, Hkv, cap, 128)), dict(w=f(n, Hkv, cap)), dict(p=f(n, Hkv, cap, t=torch.int64)), dict(ow=f(n, Hkv, cap - 1, t=torch.float32)),
                dict(ol=ev["lens"]), dict(op=None), dict(recent=9), dict(ws=f(8, t=torch.uint8))):
        with pytest.raises(mb.MloraError):
            mb.mlora_kv_evict(*{**ev, **bad}.values())


class Loop:
    """A bounded stream's step at kernel level: q, k, v rows in, rotate and append, attend, drop what exceeds the budget."""

    def __init__(self, mb, n, T, Hq, Hkv, hd, P, budget, recent, seed, kept=0):
        rng = np.random.default_rng(seed)
        self.mb, self.n, self.T, self.budget, self.recent, self.bound = mb, n, T, budget, recent, budget + T
        cap = budget + T
        r16 = lambda *s: dev(rng.standard_normal(s).astype(np.float16))  # noqa: E731
        self.pk, self.pv = r16(Hkv, P, hd), r16(Hkv, P, hd)
        self.k, self.v = r16(n, Hkv, cap, hd), r16(n, Hkv, cap, hd)
        self.w = dev(rng.random((n, Hkv, cap)).astype(np.float32))
        self.p = dev(np.broadcast_to(P + np.arange(cap, dtype=np.int32), (n, Hkv, cap)))
        self.pw = torch.zeros(Hkv, P, device="cuda")
        self.lens, self.with_new, self.newest = i32([kept] * n), i32([0] * n), i32([0] * n)
        self.pos = i32([[P + kept + t for t in range(T)]] * n).view(-1)
        self.freq = mb.mlora_rope_frequencies(hd, 1e4)[0].cuda()
        self.q, self.out = torch.empty(n * T, Hq, hd, dtype=torch.float16, device="cuda"), torch.empty(n * T, Hq, hd, dtype=torch.float16, device="cuda")
        self.ws = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, P, budget), dtype=torch.uint8, device="cuda")
        self.ws2 = torch.empty(mb.mlora_kv_evict_workspace_bytes(n, Hkv, self.bound, budget), dtype=torch.uint8, device="cuda")
        self.src = torch.full((n, Hkv, budget), -1, dtype=torch.int32, device="cuda")
        self.st = status()

    def step(self, q, k, v):
        mb = self.mb
        mb.mlora_rope_append(q, k, v, self.pos, self.freq, self.q, self.k, self.v, self.lens, self.st, own_weight=self.w, own_position=self.p)
        mb.mlora_attention_scored(self.q, self.pk, self.pv, self.k, self.v, self.lens, self.budget, None, self.out, self.w, self.pw, self.ws, self.st)
        torch.add(self.lens, self.T, out=self.with_new)
        self.newest.copy_(self.pos.view(self.n, self.T)[:, -1])
        mb.mlora_kv_evict(self.k, self.v, self.w, self.p, self.with_new, self.bound, self.newest, self.budget, self.recent, self.w, self.p, self.lens,
                          self.ws2, self.st, out_source=self.src)
        self.pos += self.T

    def state(self):
        return [t.clone() for t in (self.out, self.k, self.v, self.w, self.p, self.pw, self.lens, self.src)]


def rows(seed, steps, n, T, W):
    return [dev(np.random.default_rng([seed, i]).standard_normal((n * T, W)).astype(np.float32)) for i in range(steps)]


def split(x, Hq, Hkv, hd):
    return x[:, :Hq * hd], x[:, Hq * hd:(Hq + Hkv) * hd], x[:, (Hq + Hkv) * hd:]


@pytest.mark.parametrize("T", [1, 5])
def test_steps_replayed_from_a_graph_match_direct_steps(mb, T):
    """The same twelve steps: directly; on another stream; captured once and replayed, next to a second loop's graph."""
    n, Hq, Hkv, hd, P, B = 3, 8, 2, 64, 70, 24
    xs = rows(1, 12, n, T, (Hq + 2 * Hkv) * hd)
    ref = Loop(mb, n, T, Hq, Hkv, hd, P, B, 6, seed=9)
    for x in xs:
        ref.step(*split(x, Hq, Hkv, hd))
    want = ref.state()
    assert int(ref.st.item()) == 0 and ref.lens.tolist() == [B if 12 * T > B else 12 * T] * n
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = Loop(mb, n, T, Hq, Hkv, hd, P, B, 6, seed=9)
        for x in xs:
            other.step(*split(x, Hq, Hkv, hd))
        got = other.state()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    loops = [Loop(mb, n, T, Hq, Hkv, hd, P, B, 6, seed=9) for _ in range(2)]
    buf = torch.empty_like(xs[0])
    graphs = []
    for lp in loops:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            lp.step(*split(buf, Hq, Hkv, hd))
        graphs.append(g)
    for x in xs:
        buf.copy_(x)
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for lp in loops:
        assert all(torch.equal(a, b) for a, b in zip(lp.state(), want))


def test_decode_loop_behind_the_projection(mb):
    """INT4 projection with adapters -> rotate and append -> attention with totals -> eviction, forty steps of a bounded stream, against
    64-bit arithmetic on the GPU's own inputs of each step (projection rows, cache, totals)."""
    n, Hq, Hkv, hd, P, B, K, r = 2, 8, 2, 64, 40, 16, 256, 8
    rng = np.random.default_rng(4)
    W = (Hq + 2 * Hkv) * hd
    qb, sc = gen.quantize_int4(rng.standard_normal((K, W)).astype(np.float32) * 0.1, 64)
    w = mb.mlora_weight_create(dev(qb), dev(sc), K, W, 64)
    Aw, Bw = dev(rng.standard_normal((2, r, K)).astype(np.float16)), dev((rng.standard_normal((2, r, W)) * 0.1).astype(np.float16))
    ptr = lambda m: torch.tensor([m[0].data_ptr(), m[1].data_ptr()], dtype=torch.int64, device="cuda")  # noqa: E731
    pA, pB, scale, pick = ptr(Aw), ptr(Bw), torch.tensor([0.5, 2.0], device="cuda"), i32([1, 0])
    lws = torch.zeros(mb.mlora_linear_workspace_bytes(w, n, r), dtype=torch.uint8, device="cuda")
    lp = Loop(mb, n, 1, Hq, Hkv, hd, P, B, 4, seed=2)
    y = torch.empty(n, W, device="cuda")
    plain = torch.empty(n, Hq, hd, dtype=torch.float16, device="cuda")
    dropped = 0
    for i in range(40):
        x = dev(rng.standard_normal((n, K)).astype(np.float16))
        mb.mlora_linear(w, x, y, lws, pick, pA, pB, scale, r)
        before_w, before_p, S = lp.w.clone(), lp.p.clone(), lp.lens.tolist()
        lp.step(*split(y, Hq, Hkv, hd))
        assert lp.lens.tolist() == [min(s + 1, B) for s in S] and int(lp.st.item()) == 0
        src, p_now, w_now = lp.src.cpu().numpy(), lp.p.cpu().numpy(), lp.w.cpu().numpy()
        before_p = before_p.cpu().numpy()
        for s in range(n):
            for h in range(Hkv):
                m = min(S[s] + 1, B)
                pos = before_p[s, h].copy()
                pos[S[s]] = P + i
                assert np.array_equal(p_now[s, h, :m], pos[src[s, h, :m]])
                assert len(set(p_now[s, h, :m])) == m and all(P + j in p_now[s, h, :m] for j in range(max(0, i - 3), i + 1))
                if S[s] + 1 > B:                    # the row that went had the smallest total of those that were not new
                    gone = (set(range(S[s] + 1)) - set(src[s, h, :m])).pop()
                    assert pos[gone] <= P + i - 4
                    dropped += 1
        # every row's own weight over the cache: totals of a stream grow by at most the heads of a group, and only grow
        assert bool((lp.w[:, :, :min(S[0] + 1, B)] >= 0).all())
    mb.mlora_weight_destroy(w)
    assert dropped == n * Hkv * (40 - B)
    # the cache that is left, attended to by the plain call: the rows are there, in whatever order
    ws = torch.empty(mb.mlora_attention_workspace_bytes(n, 1, Hq, Hkv, hd, P, B + 1), dtype=torch.uint8, device="cuda")
    st = status()
    mb.mlora_attention(lp.q, lp.pk, lp.pv, lp.k, lp.v, i32([B - 1] * n), B - 1, i32([[-1]] * n), plain, ws, st)
    k = torch.cat([lp.pk.expand(n, -1, -1, -1), lp.k[:, :, :B]], dim=2).double()
    v = torch.cat([lp.pv.expand(n, -1, -1, -1), lp.v[:, :, :B]], dim=2).double()
    q = lp.q.double().view(n, Hkv, Hq // Hkv, hd)
    want = torch.softmax(q @ k.transpose(2, 3) / hd**0.5, dim=-1) @ v
    assert float((plain.double().view_as(want) - want).abs().max()) <= 1e-2 * float(want.abs().max())


def test_offsets_beyond_32_bits(mb):
    """Segments whose elements are counted beyond 2^31: append, attend and evict in the last stream and head"""
    n, Hq, Hkv, hd, cap = 2, 18, 9, 64, 1 << 21
    S, B = [5, cap - 7], cap - 40
    assert n * Hkv * cap * hd > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn(n, Hkv, cap, hd, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    w, p = torch.rand(n, Hkv, cap, generator=g, device="cuda"), torch.arange(cap, dtype=torch.int32, device="cuda").repeat(n, Hkv, 1)
    x = torch.randn(n, (Hq + 2 * Hkv) * hd, generator=g, device="cuda")
    lens, st, freq = i32(S), status(), mb.mlora_rope_frequencies(hd, 1e4)[0].cuda()
    q, out = (torch.empty(n, Hq, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    mb.mlora_rope_append(*split(x, Hq, Hkv, hd), lens, freq, q, k, v, lens, st, own_weight=w, own_position=p)
    assert torch.equal(v[1, :, S[1]], x[1, (Hq + Hkv) * hd:].view(Hkv, hd).half()) and not w[1, :, S[1]].any()
    w0 = w[1, 8].double()
    ws = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, 1, Hq, Hkv, hd, 0, S[1]), dtype=torch.uint8, device="cuda")
    mb.mlora_attention_scored(q, None, None, k, v, lens, S[1], None, out, w, None, ws, st)
    pr = torch.softmax(q[1, 16:].double() @ k[1, 8, :S[1] + 1].double().T / hd**0.5, dim=-1)
    want = pr @ v[1, 8, :S[1] + 1].double()
    assert float((out[1, 16:].double() - want).abs().max()) <= 2.0**-10 * float((pr @ v[1, 8, :S[1] + 1].double().abs()).max())
    grown = w[1, 8, :S[1] + 1].double() - w0[:S[1] + 1]
    assert float((grown - pr.sum(dim=0)).abs().max()) <= 2.0**-23       # (totals below 1 in 32 bits; weights of a millionth)
    kh, vh, wh = k[1, 8].clone(), v[1, 8].clone(), w[1, 8].cpu().numpy()
    lens1, ol = lens + 1, i32([0, 0])
    ws = torch.empty(mb.mlora_kv_evict_workspace_bytes(n, Hkv, cap, B), dtype=torch.uint8, device="cuda")
    src = torch.empty(n, Hkv, B, dtype=torch.int32, device="cuda")
    mb.mlora_kv_evict(k, v, w, p, lens1, cap, lens, B, 10, w, p, ol, ws, st, out_source=src)
    ref = dev(evict_reference(wh, np.arange(cap, dtype=np.int32), S[1] + 1, B, 10, S[1]))
    assert ol.tolist() == [6, B] and int(st.item()) == 0
    assert torch.equal(src[1, 8].long(), ref) and torch.equal(k[1, 8, :B], kh[ref]) and torch.equal(v[1, 8, :B], vh[ref])


@pytest.mark.parametrize("n,T,Hq,Hkv,hd,P,bound", [(2, 1, 8, 2, 64, 100, 3000), (20, 1, 24, 8, 128, 5500, 2500), (2, 9, 32, 8, 64, 700, 1500), (3, 20, 6, 2, 128, 64, 700), (1, 64, 16, 1, 64, 0, 9000)])
def test_scored_workspace_serves_every_smaller_bound(mb, n, T, Hq, Hkv, hd, P, bound):
    """One workspace of the largest bound's size, filled with NaN; the call sizes its chunks (and picks its kernels) by each bound."""
    g = torch.Generator(device="cuda").manual_seed(0)
    r16 = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float16)  # noqa: E731
    cap = bound + T
    q, k, v = r16(n * T, Hq, hd), r16(n, Hkv, cap, hd), r16(n, Hkv, cap, hd)
    pk, pv = (r16(Hkv, P, hd), r16(Hkv, P, hd)) if P else (None, None)
    need = mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, P, bound)
    ws, st = torch.full((need,), 255, dtype=torch.uint8, device="cuda"), status()
    lens = i32([7] * n)
    first = None
    for b in sorted({7, 8, 63, 64, 127, 128, bound // 7, bound // 3, bound // 2, 2 * bound // 3, bound - 1, bound} | set(range(100, bound, bound // 23))):
        out, w = torch.empty_like(q), torch.zeros(n, Hkv, cap, device="cuda")
        ws.fill_(255)
        mb.mlora_attention_scored(q, pk, pv, k, v, lens, b, None, out, w, None, ws, st)
        if first is None:
            first = (out.float(), w)
        # the same keys in other chunks: rounding of weights to fp16 and of the output, sums in another order
        assert float((out.float() - first[0]).abs().max()) <= 4 * 2.0**-11 * float(first[0].abs().max()) + 2.0**-9
        assert float((w - first[1]).abs().max()) <= 2.0**-17 * float(first[1].max())
    assert int(st.item()) == 0


def test_evict_few_rows_too_many_in_every_place(mb):
    """One to four rows over the budget: found one by one, as decoding at the budget does it"""
    for over in (1, 2, 3, 4, 5):
        for seed in range(6):
            evict_case(mb, 2, 3, 64, [40 + over, 38], 40, [0, 5, 40][seed % 3], seed=seed, weights=["random", "ties", "special"][seed // 2], in_place=seed % 2 == 0)
    evict_case(mb, 1, 2, 128, [3], 1, 1, seed=3)
    evict_case(mb, 1, 2, 64, [4], 1, 0, seed=4, weights="ties")
    evict_case(mb, 2, 1, 64, [5002, 5001], 5000, 100, seed=5, weights="ties", bound=7000)


def test_scored_many_streams_behind_a_long_prefix(mb):
    """One row a stream, by the tensor-memory kernels where prefix rows are many and own segments short, by the others around that"""
    scored_case(mb, 34, 1, 16, 4, 128, 5000, [(7 * i) % 100 for i in range(34)], seed=5)
    scored_case(mb, 32, 1, 32, 8, 64, 6001, [(13 * i) % 130 for i in range(32)], seed=6)
    scored_case(mb, 32, 1, 32, 8, 64, 6001, [0] * 31 + [700], seed=7, bound=900, slack=300)
    scored_case(mb, 34, 1, 16, 4, 128, 2050, [(7 * i) % 100 for i in range(34)], seed=8)


@pytest.mark.parametrize("n,T,Hq,Hkv,hd,P,lens", [(4, 32, 32, 8, 64, 1000, [700, 3, 1023, 512]), (3, 60, 24, 8, 128, 300, [500, 0, 129]), (32, 1, 32, 8, 64, 6001, list(range(32)))])
def test_scored_large_passes_replayed_from_two_graphs(mb, n, T, Hq, Hkv, hd, P, lens):
    """Passes of the tensor-memory kernels, captured twice with a workspace each and replayed side by side: the bits of direct calls"""
    g = torch.Generator(device="cuda").manual_seed(3)
    r16 = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float16)  # noqa: E731
    bound = max(lens)
    cap = bound + T + 5
    pk, pv, k, v = r16(Hkv, P, hd), r16(Hkv, P, hd), r16(n, Hkv, cap, hd), r16(n, Hkv, cap, hd)
    par, dl, qs = i32([tree(np.random.default_rng(T), T)] * n), i32(lens), [r16(n * T, Hq, hd) for _ in range(3)]
    need = mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, P, bound)

    def make():
        return dict(q=torch.empty_like(qs[0]), out=torch.empty_like(qs[0]), w=torch.zeros(n, Hkv, cap, device="cuda"), pw=torch.zeros(Hkv, P, device="cuda"),
                    ws=torch.empty(need, dtype=torch.uint8, device="cuda"), st=status())

    def call(s):
        mb.mlora_attention_scored(s["q"], pk, pv, k, v, dl, bound, par, s["out"], s["w"], s["pw"], s["ws"], s["st"])

    direct, outs = make(), []
    for q in qs:
        direct["q"].copy_(q)
        call(direct)
        outs.append(direct["out"].clone())
    states, graphs, streams = [make(), make()], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in states:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(s)
        graphs.append(gr)
    torch.cuda.synchronize()
    for i, q in enumerate(qs):
        for s, gr, sm in zip(states, graphs, streams):
            with torch.cuda.stream(sm):
                s["q"].copy_(q)
                gr.replay()
        torch.cuda.synchronize()
        for s in states:
            assert torch.equal(s["out"], outs[i])
    for s in states:
        assert torch.equal(s["w"], direct["w"]) and torch.equal(s["pw"], direct["pw"]) and int(s["st"].item()) == 0


def test_two_loops_on_two_streams_at_once(mb):
    """Nothing is shared between calls: steps of two loops enqueued alternately on two streams, against each alone"""
    n, T, Hq, Hkv, hd, P, B = 4, 3, 8, 2, 128, 200, 300
    xs = rows(7, 10, n, T, (Hq + 2 * Hkv) * hd)
    want = []
    for seed in (1, 2):
        lp = Loop(mb, n, T, Hq, Hkv, hd, P, B, 20, seed=seed, kept=B - 4)
        for x in xs:
            lp.step(*split(x, Hq, Hkv, hd))
        want.append(lp.state())
    torch.cuda.synchronize()
    loops = [Loop(mb, n, T, Hq, Hkv, hd, P, B, 20, seed=seed, kept=B - 4) for seed in (1, 2)]
    streams = [torch.cuda.Stream() for _ in loops]
    torch.cuda.synchronize()
    for x in xs:
        for lp, sm in zip(loops, streams):
            with torch.cuda.stream(sm):
                lp.step(*split(x, Hq, Hkv, hd))
    torch.cuda.synchronize()
    for lp, w in zip(loops, want):
        assert all(torch.equal(a, b) for a, b in zip(lp.state(), w))


def test_evict_long_segments_replayed_from_a_graph(mb):
    """A cluster's selection and the kernel that moves the rows, captured: two replays after one another cut once and then nothing"""
    g = torch.Generator(device="cuda").manual_seed(0)
    n, Hkv, hd, S, B = 2, 2, 64, 50000, 20000
    k, v = (torch.randn(n, Hkv, S, hd, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    w = torch.rand(n, Hkv, S, generator=g, device="cuda")
    k0, w0 = k.clone(), w.cpu().numpy()
    lens, ol, st = i32([S, S - 777]), i32([0, 0]), status()
    src = torch.full((n, Hkv, B), -1, dtype=torch.int32, device="cuda")
    ws = torch.empty(mb.mlora_kv_evict_workspace_bytes(n, Hkv, S, B), dtype=torch.uint8, device="cuda")
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        mb.mlora_kv_evict(k, v, w, None, lens, S, None, B, 0, w, None, ol, ws, st, out_source=src)
        lens.copy_(ol)
    gr.replay()
    torch.cuda.synchronize()
    kept = src.clone()
    for s, m in ((0, S), (1, S - 777)):
        for h in range(Hkv):
            want = evict_reference(w0[s, h], np.zeros(S), m, B, 0, 0)
            assert np.array_equal(kept[s, h].cpu().numpy(), want) and torch.equal(k[s, h, :B], k0[s, h][dev(want)])
    k1 = k.clone()
    gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(k, k1) and lens.tolist() == [B, B] and torch.equal(src, torch.arange(B, dtype=torch.int32, device="cuda").expand(n, Hkv, B))
    assert int(st.item()) == 0
