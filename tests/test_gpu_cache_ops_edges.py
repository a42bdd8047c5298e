"""Operators around a bounded KV cache on the GPU: calls at the edges of what their documentation allows."""
import numpy as np
import pytest

from tests.test_gpu_cache_ops import Loop, close_fp16, dev, evict_case, evict_reference, i32, mb, rotated, rows, split, status  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def arena(sizes):
    """tensors (shape, type) that lie right behind each other in one buffer, in this order"""
    count = [int(np.prod(s)) * torch.empty((), dtype=t).element_size() for s, t in sizes]
    assert all(c % 16 == 0 for c in count)
    buf, at, out = torch.zeros(sum(count), dtype=torch.uint8, device="cuda"), 0, []
    for (s, t), c in zip(sizes, count):
        out.append(buf[at:at + c].view(t).view(s))
        at += c
    return out


def test_rope_append_between_tensors_that_touch(mb):  # noqa: F811
    """Everything that is read and written in one buffer without a gap: taken, with the bits of a call on tensors of their own"""
    n, T, Hq, Hkv, hd, cap = 2, 4, 8, 2, 64, 16
    f16, f32, i4, f8 = torch.float16, torch.float32, torch.int32, torch.float64
    rows = n * T
    q, qo, k, ok, v, ov, w, pos, p, freq = arena([
        ((rows, Hq, hd), f16), ((rows, Hq, hd), f16), ((rows, Hkv, hd), f16), ((n, Hkv, cap, hd), f16), ((rows, Hkv, hd), f16), ((n, Hkv, cap, hd), f16),
        ((n, Hkv, cap), f32), ((rows,), i4), ((n, Hkv, cap), i4), ((hd // 2,), f8)])
    g = torch.Generator(device="cuda").manual_seed(0)
    for t in (q, k, v, ok, ov, w):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    pos.copy_(torch.arange(rows, device="cuda") + 50)
    freq.copy_(mb.mlora_rope_frequencies(hd, 1e4)[0])
    lens, st = i32([3, 12]), status()
    apart = [t.clone() for t in (q, k, v, pos, freq, qo, ok, ov, w, p)]
    mb.mlora_rope_append(q, k, v, pos, freq, qo, ok, ov, lens, st, own_weight=w, own_position=p)
    mb.mlora_rope_append(*apart[:5], *apart[5:8], lens, st, own_weight=apart[8], own_position=apart[9])
    assert int(st.item()) == 0
    assert all(torch.equal(a, b) for a, b in zip((q, k, v, pos, freq, qo, ok, ov, w, p), apart))


@pytest.mark.parametrize("T", [1, 20])
def test_scored_between_tensors_that_touch(mb, T):  # noqa: F811
    """As above, the workspace among them, of the queried size to the byte; and no prefix totals where there is no prefix"""
    n, Hq, Hkv, hd, cap, P, bound = 2, 8, 2, 64, 64, 32, 40
    f16, f32, i4 = torch.float16, torch.float32, torch.int32
    need = mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, P, bound)
    ws, q, pk, out, pv, ok, w, ov, pw, ws2 = arena([
        (((need + 15) // 16 * 16,), torch.uint8), ((n * T, Hq, hd), f16), ((Hkv, P, hd), f16), ((n * T, Hq, hd), f16), ((Hkv, P, hd), f16),
        ((n, Hkv, cap, hd), f16), ((n, Hkv, cap), f32), ((n, Hkv, cap, hd), f16), ((Hkv, P), f32), ((4096,), torch.uint8)])
    g = torch.Generator(device="cuda").manual_seed(0)
    for t in (q, pk, pv, ok, ov, w, pw):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    ws.fill_(255), ws2.fill_(7)
    lens, st = i32([40, 3]), status()
    par = i32([[-1] + [i // 2 for i in range(T - 1)]] * n)
    apart = [t.clone() for t in (q, pk, pv, ok, ov, out, w, pw)]
    mb.mlora_attention_scored(q, pk, pv, ok, ov, lens, bound, par, out, w, pw, ws[:need], st)
    mb.mlora_attention_scored(*apart[:5], lens, bound, par, *apart[5:], torch.empty(need, dtype=torch.uint8, device="cuda"), st)
    assert int(st.item()) == 0 and bool((ws2 == 7).all())
    assert all(torch.equal(a, b) for a, b in zip((q, pk, pv, ok, ov, out, w, pw), apart))
    mb.mlora_attention_scored(q, None, None, ok, ov, lens, bound, par, out, w, torch.empty(Hkv, 0, device="cuda"), ws[:need], st)
    assert int(st.item()) == 0


@pytest.mark.parametrize("recent,in_place", [(0, False), (4, False), (4, True)])
def test_evict_between_tensors_that_touch(mb, recent, in_place):  # noqa: F811
    """As above; newest may be out_len where no row is kept for being new: it is not read then"""
    n, Hkv, hd, cap, B = 4, 2, 64, 64, 32
    f16, f32, i4 = torch.float16, torch.float32, torch.int32
    need = mb.mlora_kv_evict_workspace_bytes(n, Hkv, cap, B)
    lens, k, w, p, v, ow, op, ol, src, newest, ws = arena([
        ((n,), i4), ((n, Hkv, cap, hd), f16), ((n, Hkv, cap), f32), ((n, Hkv, cap), i4), ((n, Hkv, cap, hd), f16), ((n, Hkv, cap), f32), ((n, Hkv, cap), i4),
        ((n,), i4), ((n, Hkv, B), i4), ((n,), i4), (((need + 15) // 16 * 16,), torch.uint8)])
    g = torch.Generator(device="cuda").manual_seed(0)
    for t in (k, v, w):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    p.copy_(torch.arange(cap, device="cuda"))
    lens.copy_(i32([64, 50, 33, 7])), newest.copy_(lens - 1)
    st = status()
    apart = [t.clone() for t in (k, v, w, p, lens, newest, ow, op, ol, src)]
    if in_place:
        ow, op = w, p
        apart[6:8] = apart[2:4]
    mb.mlora_kv_evict(k, v, w, p, lens, cap, newest if recent else ol, B, recent, ow, op, ol, ws[:need], st, out_source=src)
    mb.mlora_kv_evict(*apart[:5], cap, apart[5], B, recent, *apart[6:9], torch.empty(need, dtype=torch.uint8, device="cuda"), st, out_source=apart[9])
    assert int(st.item()) == 0 and ol.tolist() == [32, 32, 32, 7]
    assert all(torch.equal(a, b) for a, b in zip((k, v, w, p, lens, newest, ow, op, ol, src), apart))


# n, T, Hq, Hkv, hd, P: by the kernels for few rows, by those on tensor memory, one row a stream by both
@pytest.mark.parametrize("n,T,Hq,Hkv,hd,P", [(2, 1, 8, 2, 64, 16), (2, 1, 8, 8, 128, 0), (2, 3, 4, 2, 64, 16), (2, 40, 32, 8, 64, 500), (2, 64, 24, 8, 128, 600),
                                            (32, 1, 32, 8, 64, 6001)])
def test_scored_reports_every_malformed_parent(mb, n, T, Hq, Hkv, hd, P):  # noqa: F811
    """One wrong entry of the last stream, whatever kernels the sizes pick: a root that has a parent, a node whose parent is itself, a later
    node, none or out of range"""
    z = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")  # noqa: E731
    bound, cap = 30, 30 + T
    q, out, pk, pv, k, v = z(n * T, Hq, hd), z(n * T, Hq, hd), z(Hkv, P, hd), z(Hkv, P, hd), z(n, Hkv, cap, hd), z(n, Hkv, cap, hd)
    w = torch.zeros(n, Hkv, cap, device="cuda")
    ws = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, T, Hq, Hkv, hd, P, bound), dtype=torch.uint8, device="cuda")
    good = [[-1] + [(i - 1) // 2 for i in range(1, T)] for _ in range(n)]
    wrong = [(0, x) for x in (0, 7, -2, -2**31)] + ([(T - 1, x) for x in (T - 1, T, -1, 2**31 - 1)] + [(1, 1)] if T > 1 else [])
    for lens in ([0] * n, [bound] * n):
        for node, value in [(0, -1)] + wrong:
            par = [list(r) for r in good]
            par[-1][node] = value
            st = status()
            mb.mlora_attention_scored(q, pk if P else None, pv if P else None, k, v, i32(lens), bound, i32(par), out, w, None, ws, st)
            assert int(st.item()) == (0 if (node, value) == (0, -1) else -1), (lens[0], node, value)


def test_readme_example_runs(mb):  # noqa: F811
    """The example that README gives, as it stands there: what is ahead of the projection once, the rest every step, until the streams are at their budget"""
    import os

    import gen
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        text = f.read()
    blocks = [b.split("```")[0] for b in text.split("```python\n")[1:]]
    blocks = [b for b in blocks if "mlora_kv_evict" in b]
    assert len(blocks) == 1
    once, step = blocks[0].split("mb.mlora_linear(", 1)
    step = "mb.mlora_linear(" + step
    n, Hq, Hkv, head_dim, P, budget, recent, K, rank = 2, 8, 2, 64, 40, 16, 4, 256, 8
    cap, nq, nkv = budget + 1, Hq * head_dim, Hkv * head_dim
    rng = np.random.default_rng(0)
    qb, sc = gen.quantize_int4(rng.standard_normal((K, nq + 2 * nkv)).astype(np.float32) * 0.1, 64)
    r16 = lambda *s: dev(rng.standard_normal(s).astype(np.float16))  # noqa: E731
    low = [r16(rank, K), r16(rank, nq + 2 * nkv)]
    e = dict(torch=torch, mb=mb, head_dim=head_dim, nq=nq, nkv=nkv, budget=budget, recent=recent, rank=rank, status=status(),
             w_qkv=mb.mlora_weight_create(dev(qb), dev(sc), K, nq + 2 * nkv, 64), x=r16(n, K), qkv=torch.empty(n, nq + 2 * nkv, device="cuda"),
             adapters=i32([0] * n), A=torch.tensor([low[0].data_ptr()], dtype=torch.int64, device="cuda"),
             B=torch.tensor([low[1].data_ptr()], dtype=torch.int64, device="cuda"), scale=torch.ones(1, device="cuda"),
             pos=i32([P] * n), q=torch.empty(n, Hq, head_dim, dtype=torch.float16, device="cuda"), own_k=r16(n, Hkv, cap, head_dim),
             own_v=r16(n, Hkv, cap, head_dim), lens=i32([0] * n), lens_new=i32([0] * n), weight=torch.zeros(n, Hkv, cap, device="cuda"),
             position=torch.zeros(n, Hkv, cap, dtype=torch.int32, device="cuda"), prefix_k=r16(Hkv, P, head_dim), prefix_v=r16(Hkv, P, head_dim),
             out=torch.empty(n, Hq, head_dim, dtype=torch.float16, device="cuda"))
    e["linear_ws"] = torch.zeros(mb.mlora_linear_workspace_bytes(e["w_qkv"], n, rank), dtype=torch.uint8, device="cuda")
    e["attn_ws"] = torch.empty(mb.mlora_attention_scored_workspace_bytes(n, 1, Hq, Hkv, head_dim, P, budget), dtype=torch.uint8, device="cuda")
    e["evict_ws"] = torch.empty(mb.mlora_kv_evict_workspace_bytes(n, Hkv, budget + 1, budget), dtype=torch.uint8, device="cuda")
    exec(once, e)
    for i in range(budget + 5):
        e["x"].copy_(r16(n, K))
        exec(step, e)
    torch.cuda.synchronize()
    mb.mlora_weight_destroy(e["w_qkv"])
    assert int(e["status"].item()) == 0 and e["lens"].tolist() == [budget] * n and e["pos"].tolist() == [P + budget + 5] * n
    newest = sorted(range(P + budget + 5))[-recent:]
    for row in e["position"][:, :, :budget].reshape(-1, budget).tolist():
        assert len(set(row)) == budget and set(newest) <= set(row)


def test_rotate_only_ignores_lengths_and_status(mb):  # noqa: F811
    """q alone, with the lengths (of fewer streams than rows) and the status of the call that appends left in place"""
    n, T, Hq, hd = 2, 5, 4, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    q = torch.randn(n * T, Hq, hd, generator=g, device="cuda", dtype=torch.float16)
    pos, freq, st = i32(np.arange(n * T)), mb.mlora_rope_frequencies(hd, 1e4)[0].cuda(), status()
    a, b = torch.empty_like(q), torch.empty_like(q)
    mb.mlora_rope_append(q, None, None, pos, freq, a, None, None, None, None)
    mb.mlora_rope_append(q, None, None, pos, freq, b, None, None, i32([99, -7]), st)
    assert torch.equal(a, b) and int(st.item()) == 0
    with pytest.raises(mb.MloraError):             # totals and positions belong to appended rows
        mb.mlora_rope_append(q, None, None, pos, freq, b, None, None, None, None, own_weight=torch.zeros(n, 2, 8, device="cuda"))


@pytest.mark.parametrize("pos", [2**31 - 1, -2**31, 2**31 - 12345, 2**30 + 77, -2**30 - 1, 1 << 24, -12345])
def test_rope_angles_of_far_positions(mb, pos):  # noqa: F811
    """Angles next to a quarter turn, so that the rotated 1 is a small number that fp16 resolves: off by 2^-22 at most (the angle), by half a
    step of fp16 below 2^-13 (2^-25), and by the 1 in 2^24 that products and sums of 32 bits round by.  Reference in 64-bit mantissas."""
    L, hd = np.longdouble, 128
    if np.finfo(L).nmant < 63:
        pytest.skip("long double is no longer than double here")
    two_pi = L("6.283185307179586476925286766559005768")
    rng = np.random.default_rng(pos % 1000)
    k = rng.integers(int(abs(pos) * 0.5 / 6.2832), int(abs(pos) * 0.999 / 6.2832) + 1, hd // 2)
    f = ((k + L("0.25") + L(2.0)**-17 * (rng.random(hd // 2) - 0.5)) * two_pi / abs(pos)).astype(np.float64)
    angle = L(pos) * f.astype(L)
    want = np.cos(angle).astype(np.float64)
    assert (np.abs(want) < 2.0**-13).all() and (f < 1.01).all()
    q = torch.zeros(1, 1, hd, device="cuda")
    q[0, 0, :hd // 2] = 1.0
    out = torch.empty(1, 1, hd, dtype=torch.float16, device="cuda")
    mb.mlora_rope_append(q, None, None, i32([pos]), dev(f), out, None, None, None, None)
    got = out[0, 0].double().cpu().numpy()
    assert (np.abs(got[:hd // 2] - want) <= 2.0**-22 + 2.0**-25 + 2.0**-24 * np.abs(want)).all(), np.log2(np.abs(got[:hd // 2] - want).max())
    assert (got[hd // 2:] == np.sign(np.sin(angle))).all()


@pytest.mark.parametrize("n,Hq,Hkv,hd,P,B,recent", [(2, 8, 2, 64, 40, 16, 4), (3, 6, 3, 128, 0, 21, 1)])
def test_every_step_of_a_bounded_stream_against_64_bits(mb, n, Hq, Hkv, hd, P, B, recent):  # noqa: F811
    """INT4 projection -> rotate and append -> attention with totals -> eviction, until well past the budget.  Every step is computed in 64 bits
    from what the GPU had before it (the projection's rows, cache, totals): rotated rows, output, totals, and which row goes."""
    import gen
    rng = np.random.default_rng(hd)
    K, r, G, W, R = 256, 8, Hq // Hkv, (Hq + 2 * Hkv) * hd, hd
    qb, sc = gen.quantize_int4(rng.standard_normal((K, W)).astype(np.float32) * 0.1, 64)
    w = mb.mlora_weight_create(dev(qb), dev(sc), K, W, 64)
    low = [dev(rng.standard_normal((r, K)).astype(np.float16)), dev((rng.standard_normal((r, W)) * 0.1).astype(np.float16))]
    pA, pB = (torch.tensor([m.data_ptr()], dtype=torch.int64, device="cuda") for m in low)
    scale, pick = torch.ones(1, device="cuda"), i32([0] * n)
    lws = torch.zeros(mb.mlora_linear_workspace_bytes(w, n, r), dtype=torch.uint8, device="cuda")
    lp, y = Loop(mb, n, 1, Hq, Hkv, hd, P, B, recent, seed=hd), torch.empty(n, W, device="cuda")
    if not P:
        lp.pk = lp.pv = lp.pw = None
    freq, dropped = lp.freq.cpu().numpy(), 0
    for i in range(B + 12):
        mb.mlora_linear(w, dev(rng.standard_normal((n, K)).astype(np.float16)), y, lws, pick, pA, pB, scale, r)
        S, pos = lp.lens.tolist(), lp.pos.cpu().numpy()
        was = [t.clone() for t in (lp.k, lp.v, lp.w, lp.p)]
        pw = lp.pw.double().clone() if P else None
        lp.step(*split(y, Hq, Hkv, hd))
        assert lp.lens.tolist() == [min(s + 1, B) for s in S] and int(lp.st.item()) == 0
        x = y.double().cpu().numpy()
        close_fp16(lp.q, *rotated(x[:, :Hq * hd].reshape(n, Hq, hd), pos, freq, 1.0, R, False))
        new_k, size_k = rotated(x[:, Hq * hd:(Hq + Hkv) * hd].reshape(n, Hkv, hd), pos, freq, 1.0, R, False)
        new_v = x[:, (Hq + Hkv) * hd:].astype(np.float16).reshape(n, Hkv, hd)
        grown_p, grown_tol = (torch.zeros(Hkv, P, dtype=torch.float64, device="cuda"), 0.0) if P else (None, 0.0)
        for s in range(n):
            L = S[s] + 1
            for h in range(Hkv):
                src = lp.src[s, h, :min(L, B)].tolist()
                place = src.index(S[s])            # (the new row stays: it is among the `recent` ones)
                k, v, t, p = (a[s, h, :L].clone() for a in was)
                k[S[s]], v[S[s]], t[S[s]], p[S[s]] = lp.k[s, h, place], lp.v[s, h, place], 0.0, int(pos[s])
                close_fp16(k[S[s]], new_k[s, h], size_k[s, h])
                assert np.array_equal(v[S[s]].cpu().numpy(), new_v[s, h])
                ks, vs = (torch.cat([a[h], b]).double() for a, b in ((lp.pk, k), (lp.pv, v))) if P else (k.double(), v.double())
                q = lp.q[s, h * G:(h + 1) * G].double()
                pr = torch.softmax(q @ ks.T / np.sqrt(hd), dim=-1)
                # a score: hd products added in 32 bits; a weight: scores' errors twice, 2^-20 for exponentials and sums; weights as fp16 for the
                # product (2^-11, or 2^-25 of the largest below the normal range), the output as fp16
                delta = float((q.abs() @ ks.abs().T).max()) / np.sqrt(hd) * (hd + 8) * 2.0**-23
                want, size = pr @ vs, pr @ vs.abs()
                tol = 2.0**-11 * want.abs() + (2.0**-11 + 2 * delta + 2.0**-20) * size * (1 + 2.0**-8) + 2.0**-25 * vs.abs().sum(dim=0) + 2.0**-25
                assert bool(((lp.out[s, h * G:(h + 1) * G].double() - want).abs() <= tol).all()), (i, s, h)
                rel = 2 * delta + 2.0**-20 + G * 2.0**-24
                add = pr.sum(dim=0)
                total = t.double() + add[P:]
                # (an exponential below the smallest normal number of 32 bits, 2^-126 of the row's largest, counts as zero: so much is lost a row,
                # a weight being an exponential divided by a sum of at least one)
                total_tol = rel * add[P:] + 2.0**-23 * total + G * 2.0**-126
                assert bool(((lp.w[s, h, :len(src)].double() - total[src]).abs() <= total_tol[src]).all()), (i, s, h)
                assert torch.equal(lp.p[s, h, :len(src)], p[src]) and torch.equal(lp.k[s, h, :len(src)], k[src]) and torch.equal(lp.v[s, h, :len(src)], v[src])
                if P:
                    grown_p[h] += add[:P]
                    grown_tol = max(grown_tol, rel)
                if L > B:                          # the smallest total of the rows that are not new, but for what the totals round by
                    (gone,) = set(range(L)) - set(src)
                    old = p <= int(pos[s]) - recent
                    assert bool(old[gone]) and float(total[gone] - total_tol[gone]) <= float((total + total_tol)[old].min())
                    dropped += 1
        if P:
            assert bool(((lp.pw.double() - pw - grown_p).abs() <= (grown_tol + n * G * 2.0**-24) * grown_p + 2.0**-23 * (pw + grown_p) + n * G * 2.0**-126).all())
    mb.mlora_weight_destroy(w)
    assert dropped == n * Hkv * 12


@pytest.mark.parametrize("T", [1, 20])
def test_nan_totals_go_from_the_attention_into_the_eviction(mb, T):  # noqa: F811
    """A cached key of NaN: its stream's outputs and totals become NaN, and eviction keeps the new rows and then the first ones; the other
    streams come out with the bits that they have without it"""
    n, Hq, Hkv, hd, P, B, recent = 3, 8, 2, 64, 70, 60, 25
    xs = rows(3, 3, n, T, (Hq + 2 * Hkv) * hd)
    ref, lp = (Loop(mb, n, T, Hq, Hkv, hd, P, B, recent, seed=4, kept=B - 3) for _ in range(2))
    lp.k[1, 0, 0, 5] = float("nan")
    for x in xs:
        ref.step(*split(x, Hq, Hkv, hd))
        before_p, S = lp.p.cpu().numpy(), lp.lens.tolist()[1]
        before_p[1, 0, S:S + T] = lp.pos.view(n, T)[1].cpu().numpy()
        lp.step(*split(x, Hq, Hkv, hd))
        newest = int(lp.newest[1])
        want = evict_reference(np.full(S + T, np.nan, dtype=np.float32), before_p[1, 0], S + T, B, recent, newest)
        assert lp.src[1, 0, :len(want)].tolist() == want.tolist()
        assert bool(lp.w[1, 0, :min(S + T, B)].isnan().all()) and bool(lp.out.view(n, T, Hq, hd)[1, :, :Hq // Hkv].isnan().all())
    assert int(lp.st.item()) == 0 and bool(lp.pw[0].isnan().all())
    keep = [0, 2]
    for a, b in zip((lp.out.view(n, -1), lp.k, lp.v, lp.w, lp.p, lp.src), (ref.out.view(n, -1), ref.k, ref.v, ref.w, ref.p, ref.src)):
        assert torch.equal(a[keep], b[keep])
    assert torch.equal(lp.w[1, 1], ref.w[1, 1]) and torch.equal(lp.src[1, 1], ref.src[1, 1]) and torch.equal(lp.pw[1], ref.pw[1])


@pytest.mark.parametrize("n,Hkv,hd,S,B", [(8, 8, 64, 16384, 8192), (16, 8, 128, 8192, 4096)])
def test_evict_more_than_l2_holds(mb, n, Hkv, hd, S, B):  # noqa: F811
    """Moves of over 100 MB: what is read is marked to leave L2 first too, the moving kernel (64 segments) has twice the blocks; and 128
    segments, moved by the selecting blocks"""
    assert n * Hkv * B * hd * 4 > 100000000
    evict_case(mb, n, Hkv, hd, [S - 331 * (s % 5) for s in range(n)], B, 100, seed=n, in_place=n == 8)
