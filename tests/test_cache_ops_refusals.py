"""Operators around a bounded KV cache, host side: refusals of the C calls (made before anything touches a device), workspace
sizes, and the frequencies of rotary positions against their formulas.  No GPU."""
import ctypes as C
import math

import numpy as np
import pytest

ARG, CAPACITY, UNSUPPORTED = -1, -3, -6
A = 1 << 20                                        # stands for an aligned address; a refused call reads none


@pytest.fixture(scope="module")
def mb():
    from paper_2604_18655_b200 import binding, build
    build.build()
    binding.lib()
    return binding


# ------------------------------------------------------------------ frequencies
def expected(d, theta, scaling, factor, length, low, high):
    out = []
    if scaling == "base" and d > 2:
        theta = theta * factor ** (d / (d - 2))
    pair_of = lambda turns: d * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    for i in range(d // 2):
        f = theta ** (-2 * i / d)
        turns = length * f / (2 * math.pi) if length else 0.0
        if scaling == "linear":
            f /= factor
        elif scaling == "waves":
            if turns <= low:
                f /= factor
            elif turns < high:
                w = (turns - low) / (high - low)
                f = (1 - w) * f / factor + w * f
        elif scaling == "ramp":
            a, b = max(math.floor(pair_of(high)), 0), min(math.ceil(pair_of(low)), d - 1)
            w = min(max((i - a) / max(b - a, 1e-3), 0.0), 1.0)
            f = w * f / factor + (1 - w) * f
        out.append(f)
    return np.array(out)


@pytest.mark.parametrize("d", [2, 16, 64, 96, 128])
@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "waves", "ramp"])
def test_frequencies_follow_their_formulas(mb, d, scaling):
    args = (5e5, scaling, 8.0, 8192.0, 1.0, 4.0 if scaling == "waves" else 32.0)
    freq, gain = mb.mlora_rope_frequencies(d, *args)
    # a handful of 64-bit operations, pow within an ulp of its own and its exponent's rounding times the logarithm (13)
    np.testing.assert_allclose(freq.numpy(), expected(d, *args), rtol=64 * 2.0**-53)
    assert gain == (pytest.approx(0.1 * math.log(8.0) + 1, rel=2.0**-23) if scaling == "ramp" else 1.0)


def test_scaled_frequencies_keep_short_waves_and_divide_long_ones(mb):
    plain, _ = mb.mlora_rope_frequencies(128, 1e4)
    for scaling, high in (("waves", 4.0), ("ramp", 32.0)):
        f, _ = mb.mlora_rope_frequencies(128, 1e4, scaling, 4.0, 8192.0, 1.0, high)
        assert f[0] == plain[0] and f[-1] == plain[-1] / 4
        assert bool((f[1:] < f[:-1]).all())


@pytest.mark.parametrize("bad", [
    dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=-2), dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")),
    dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("nan")), dict(scaling="waves", factor=2.0, length=0.0),
    dict(scaling="ramp", factor=2.0, length=100.0, low=4.0, high=4.0), dict(scaling="ramp", factor=float("inf"), length=100.0)])
def test_frequencies_refuse(mb, bad):
    with pytest.raises(mb.MloraError) as e:
        mb.mlora_rope_frequencies(**{**dict(rotary_dim=64, theta=1e4), **bad})
    assert e.value.code == ARG


def test_frequencies_refuse_null_and_unknown(mb):
    L = mb.lib()
    f, g = (C.c_double * 32)(), C.c_float()
    assert L.mlora_rope_frequencies(64, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None, C.byref(g)) == ARG
    assert L.mlora_rope_frequencies(64, 1e4, 0, 1.0, 0.0, 0.0, 0.0, f, None) == ARG
    assert L.mlora_rope_frequencies(64, 1e4, 5, 1.0, 0.0, 0.0, 0.0, f, C.byref(g)) == ARG
    assert L.mlora_rope_frequencies(64, 1e4, -1, 1.0, 0.0, 0.0, 0.0, f, C.byref(g)) == ARG


# ------------------------------------------------------------------ refusals
def call(mb, name, good, **change):
    args = {**good, **change}
    assert set(args) == set(good)
    return getattr(mb.lib(), name)(*args.values())


ROPE = dict(q=A, k=A, v=A, in_fp32=0, q_stride=512, k_stride=128, v_stride=128, positions=A, freq=A, gain=1.0, rotary_dim=64,
            interleaved=0, n=2, T=3, Hq=8, Hkv=2, hd=64, q_out=2 * A, own_k=A, own_v=A, cap=16, suffix_len=A, own_weight=None,
            own_position=None, status=A, stream=None)


@pytest.mark.parametrize("code,change", [
    (ARG, dict(positions=None)), (ARG, dict(freq=None)), (ARG, dict(q=None)), (ARG, dict(q_out=None)), (ARG, dict(k=None)),
    (ARG, dict(v=None)), (ARG, dict(own_k=None)), (ARG, dict(own_v=None)), (ARG, dict(suffix_len=None)), (ARG, dict(status=None)),
    (ARG, dict(q=None, q_out=None, k=None, v=None, own_k=None, own_v=None)),
    (ARG, dict(k=None, v=None, own_k=None, own_v=None, own_weight=A)),
    (ARG, dict(n=0)), (ARG, dict(T=0)), (ARG, dict(n=-1)), (ARG, dict(Hq=0)), (ARG, dict(Hkv=0)), (ARG, dict(n=1 << 20, T=1 << 20, cap=1 << 21)),
    (UNSUPPORTED, dict(hd=80)), (UNSUPPORTED, dict(hd=256)), (UNSUPPORTED, dict(rotary_dim=0)), (UNSUPPORTED, dict(rotary_dim=24)),
    (UNSUPPORTED, dict(rotary_dim=80)), (CAPACITY, dict(T=17)),
    (ARG, dict(q_stride=504)), (ARG, dict(q_stride=516)), (ARG, dict(k_stride=132)), (ARG, dict(v_stride=120)), (ARG, dict(q_stride=-512)),
    (ARG, dict(q=A + 8)), (ARG, dict(k=A + 2)), (ARG, dict(v=A + 4)), (ARG, dict(q_out=A + 8)), (ARG, dict(own_k=A + 8)), (ARG, dict(own_v=A + 8)),
    (ARG, dict(q_out=A, in_fp32=1)), (ARG, dict(q_out=A, q_stride=1024)),
])
def test_rope_append_refuses(mb, code, change):
    assert call(mb, "mlora_rope_append", ROPE, **change) == code
    assert b"rope_append" in mb.lib().mlora_last_error(None)


SCORED = dict(q=A, prefix_k=A, prefix_v=A, P=32, own_k=A, own_v=A, cap=64, suffix_len=A, suffix_bound=40, tree_parent=A, n=2, T=3,
              Hq=8, Hkv=2, hd=64, out=A, own_weight=A, prefix_weight=A, workspace=A, workspace_bytes=1 << 40, status=A, stream=None)


@pytest.mark.parametrize("code,change", [
    (ARG, dict(q=None)), (ARG, dict(own_k=None)), (ARG, dict(own_v=None)), (ARG, dict(suffix_len=None)), (ARG, dict(out=None)),
    (ARG, dict(own_weight=None)), (ARG, dict(workspace=None)), (ARG, dict(status=None)), (ARG, dict(prefix_k=None)), (ARG, dict(prefix_v=None)),
    (ARG, dict(n=0)), (ARG, dict(T=0)), (ARG, dict(T=65, cap=200)), (ARG, dict(Hq=7)), (ARG, dict(Hkv=0)), (ARG, dict(P=-1)), (ARG, dict(suffix_bound=-1)),
    (UNSUPPORTED, dict(hd=96)), (CAPACITY, dict(suffix_bound=62)), (CAPACITY, dict(workspace_bytes=64)),
    (ARG, dict(q=A + 8)), (ARG, dict(prefix_k=A + 8)), (ARG, dict(own_v=A + 2)), (ARG, dict(out=A + 8)),
])
def test_attention_scored_refuses(mb, code, change):
    assert call(mb, "mlora_attention_scored", SCORED, **change) == code
    assert b"attention_scored" in mb.lib().mlora_last_error(None)


@pytest.mark.parametrize("out", [A, A + 2 * 3 * 8 * 64 * 2 - 16, A - 16])
def test_attention_scored_refuses_out_over_q(mb, out):
    assert call(mb, "mlora_attention_scored", SCORED, out=out) == ARG
    assert b"overlaps" in mb.lib().mlora_last_error(None)


@pytest.mark.parametrize("change", [dict(q_out=A + 16), dict(q_out=A + 2 * 3 * 512 * 2 - 16), dict(q_out=A - 16), dict(q_stride=1024, q_out=A + 5 * 1024 * 2),
                                    dict(in_fp32=1, q_out=A + 2 * 3 * 512 * 4 - 16)])
def test_rope_append_refuses_q_out_over_q(mb, change):
    assert call(mb, "mlora_rope_append", ROPE, **change) == ARG
    assert b"overlaps" in mb.lib().mlora_last_error(None)


EVICT = dict(own_k=A, own_v=A, own_weight=A, own_position=A, cap=64, suffix_len=A, suffix_bound=40, newest=A, budget=32, recent=4, n=2,
             Hkv=2, hd=64, out_weight=A, out_position=A, out_len=2 * A, out_source=None, workspace=A, workspace_bytes=1 << 30, status=A,
             stream=None)


@pytest.mark.parametrize("code,change", [
    (ARG, dict(own_k=None)), (ARG, dict(own_v=None)), (ARG, dict(own_weight=None)), (ARG, dict(suffix_len=None)), (ARG, dict(out_weight=None)),
    (ARG, dict(out_len=None)), (ARG, dict(workspace=None)), (ARG, dict(status=None)), (ARG, dict(own_position=None)), (ARG, dict(out_position=None)),
    (ARG, dict(newest=None)), (ARG, dict(own_position=None, out_position=None)), (ARG, dict(recent=33)), (ARG, dict(recent=-1)),
    (ARG, dict(budget=0)), (ARG, dict(n=0)), (ARG, dict(Hkv=0)), (ARG, dict(n=70000)), (ARG, dict(suffix_bound=-1)), (ARG, dict(out_len=A)),
    (UNSUPPORTED, dict(hd=32)), (CAPACITY, dict(suffix_bound=65)), (CAPACITY, dict(workspace_bytes=32)), (ARG, dict(own_k=A + 8)), (ARG, dict(own_v=A + 2)),
])
def test_kv_evict_refuses(mb, code, change):
    assert call(mb, "mlora_kv_evict", EVICT, **change) == code
    assert b"kv_evict" in mb.lib().mlora_last_error(None)


@pytest.mark.parametrize("change", [dict(out_len=A + 4), dict(out_len=A - 4), dict(suffix_len=4 * A, out_len=A), dict(suffix_len=4 * A, out_len=A + 4),
                                    dict(out_weight=A + 256), dict(out_weight=A - 4), dict(out_position=A + 2 * 2 * 64 * 4 - 4)])
def test_kv_evict_refuses_overlaps(mb, change):
    assert call(mb, "mlora_kv_evict", EVICT, **change) == ARG
    assert b"overlap" in mb.lib().mlora_last_error(None)


# ------------------------------------------------------------------ workspaces
@pytest.mark.parametrize("n,T,Hq,Hkv,hd,P", [(1, 1, 32, 8, 64, 512), (8, 1, 24, 8, 128, 0), (3, 7, 8, 2, 64, 100), (8, 32, 24, 8, 128, 2048)])
def test_scored_workspace_covers_every_smaller_bound(mb, n, T, Hq, Hkv, hd, P):
    need = mb.mlora_attention_scored_workspace_bytes
    last = 0
    for bound in [0, 1, 63, 64, 65, 500, 1000, 1999, 2000, 4000, 8191, 16384, 40000, 131072]:
        b = need(n, T, Hq, Hkv, hd, P, bound)
        assert b >= last > -1
        last = b
        # the call itself takes what the query says for this bound
        assert call(mb, "mlora_attention_scored", SCORED, n=n, T=T, Hq=Hq, Hkv=Hkv, hd=hd, P=P, suffix_bound=bound, cap=1 << 20,
                    workspace_bytes=16) == CAPACITY
    assert need(0, T, Hq, Hkv, hd, P, 5) == 0 and need(n, T, Hq, Hkv, 96, P, 5) == 0 and need(n, 65, Hq, Hkv, hd, P, 5) == 0


def test_evict_workspace_grows_with_the_bound(mb):
    need = mb.mlora_kv_evict_workspace_bytes
    sizes = [need(4, 8, bound, 256) for bound in (0, 100, 256, 257, 300, 512, 513, 100000)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert need(4, 8, 256, 256) < need(4, 8, 257, 256) and need(4, 8, 512, 256) == need(4, 8, 100000, 256)
    assert need(0, 8, 5, 5) == 0 and need(4, 8, 5, 0) == 0


# ------------------------------------------------------------------ the binding's own checks that need no GPU
def test_binding_refuses_host_tensors_and_other_objects(mb):
    import torch
    z = lambda *s, t=torch.float16: torch.zeros(*s, dtype=t)  # noqa: E731
    i = lambda *s: z(*s, t=torch.int32)  # noqa: E731
    own, row = z(1, 2, 8, 64), z(1, 2, 64)
    calls = [
        lambda: mb.mlora_rope_append(row, row, row, i(1), z(32, t=torch.float64), row, own, own, i(1), i(1)),
        lambda: mb.mlora_rope_append(None, None, None, i(1), z(32, t=torch.float64), None, None, None, None, None),
        lambda: mb.mlora_rope_append(row, None, row, i(1), z(32, t=torch.float64), row, own, own, i(1), i(1)),
        lambda: mb.mlora_rope_append(row, row, row, 5, z(32, t=torch.float64), row, own, own, i(1), i(1)),
        lambda: mb.mlora_attention_scored(row, None, None, own, own, i(1), 7, None, row, z(1, 2, 8), None, i(9), i(1)),
        lambda: mb.mlora_attention_scored([1], None, None, own, own, i(1), 7, None, row, z(1, 2, 8), None, i(9), i(1)),
        lambda: mb.mlora_attention_scored(row, None, None, row, own, i(1), 7, None, row, z(1, 2, 8), None, i(9), i(1)),
        lambda: mb.mlora_kv_evict(own, own, z(1, 2, 8), i(1, 2, 8), i(1), 8, i(1), 4, 0, z(1, 2, 8), i(1, 2, 8), i(1), i(99), i(1)),
        lambda: mb.mlora_kv_evict(row, own, z(1, 2, 8), i(1, 2, 8), i(1), 8, i(1), 4, 0, z(1, 2, 8), i(1, 2, 8), i(1), i(99), i(1)),
        lambda: mb.mlora_kv_evict(None, own, None, None, None, 8, None, 4, 0, None, None, None, None, None),
    ]
    for call in calls:
        with pytest.raises(mb.MloraError) as e:
            call()
        assert e.value.code == ARG and len(str(e.value)) > 20
