"""Refusals of the calls around a bounded KV cache, each by the check that is meant: tensors that lie over each other, and the rest.  The
base arguments of every call are apart, so that one change is one fault.  No GPU."""
import pytest

ARG = -1
STEP = 1 << 32                                     # stands for aligned addresses that are far apart; a refused call reads none
A = [STEP * (i + 1) for i in range(16)]


@pytest.fixture(scope="module")
def mb():
    from paper_2604_18655_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def refused(mb, name, good, change):
    assert set(change) <= set(good)
    assert getattr(mb.lib(), name)(*{**good, **change}.values()) == ARG
    return mb.lib().mlora_last_error(None).decode()


# two streams of three rows, 8 query heads and 2 KV heads of 64, segments of 16 rows
ROPE = dict(q=A[0], k=A[1], v=A[2], in_fp32=0, q_stride=512, k_stride=128, v_stride=128, positions=A[3], freq=A[4], gain=1.0, rotary_dim=64,
            interleaved=0, n=2, T=3, Hq=8, Hkv=2, hd=64, q_out=A[5], own_k=A[6], own_v=A[7], cap=16, suffix_len=A[8], own_weight=A[9],
            own_position=A[10], status=A[11], stream=None)
SEG, ROWS_KV, ROWS_Q = 2 * 2 * 16 * 64 * 2, 6 * 128 * 2, 6 * 512 * 2


@pytest.mark.parametrize("change", [
    dict(own_k=A[1]), dict(own_v=A[2]), dict(own_k=A[2]), dict(own_v=A[1] + ROWS_KV - 16), dict(own_k=A[1] - SEG + 16),
    dict(own_v=A[0]), dict(own_k=A[0] + ROWS_Q - 16), dict(own_v=A[6]), dict(own_v=A[6] + SEG - 16),
    dict(q_out=A[1]), dict(q_out=A[2] + ROWS_KV - 16), dict(q_out=A[1] - ROWS_Q + 16), dict(q_out=A[6]), dict(q_out=A[7] + SEG - 16),
    dict(own_weight=A[3]), dict(own_position=A[3] + 5 * 4), dict(own_weight=A[4] + 31 * 8), dict(own_position=A[8] + 4), dict(own_position=A[9]),
    dict(own_k=A[8]), dict(own_weight=A[6]), dict(own_position=A[2]),
    # strided rows reach as far as their last one; fp32 rows twice as far
    dict(k_stride=384, own_k=A[1] + 5 * 384 * 2 + 128 * 2 - 16), dict(in_fp32=1, own_v=A[2] + 2 * ROWS_KV - 16),
    # append only, rotate only
    dict(q=None, q_out=None, own_k=A[1]), dict(k=None, v=None, own_k=None, own_v=None, own_weight=None, own_position=None, q_out=A[3]),
    # a segment's own rows as the rows to append: a later row's source is an earlier one's place
    dict(q=None, q_out=None, Hkv=1, k_stride=64, k=A[6] + 64 * 2)])
def test_rope_append_refuses_outputs_over_what_it_reads(mb, change):
    assert "overlaps" in refused(mb, "mlora_rope_append", ROPE, change)


# two streams of three rows, 8 query heads and 2 KV heads of 64 behind 32 keys, segments of 64 rows
SCORED = dict(q=A[0], prefix_k=A[1], prefix_v=A[2], P=32, own_k=A[3], own_v=A[4], cap=64, suffix_len=A[5], suffix_bound=40, tree_parent=A[6], n=2, T=3,
              Hq=8, Hkv=2, hd=64, out=A[7], own_weight=A[8], prefix_weight=A[9], workspace=A[10], workspace_bytes=STEP, status=A[11], stream=None)
PREFIX, OWN, TOTALS = 2 * 32 * 64 * 2, 2 * 2 * 64 * 64 * 2, 2 * 2 * 64 * 4


@pytest.mark.parametrize("change", [
    dict(out=A[0]), dict(out=A[1]), dict(out=A[2] + PREFIX - 16), dict(out=A[3] - ROWS_Q + 16), dict(out=A[4] + OWN - 16), dict(own_weight=A[1]),
    dict(own_weight=A[5] + 4), dict(own_weight=A[6] + 5 * 4), dict(own_weight=A[7] + ROWS_Q - 4), dict(prefix_weight=A[8] + TOTALS - 4),
    dict(prefix_weight=A[4]), dict(prefix_weight=A[7]), dict(prefix_weight=A[8] - 2 * 32 * 4 + 4), dict(own_weight=A[0]),
    dict(workspace=A[0]), dict(workspace=A[3] + OWN - 16), dict(workspace=A[8]), dict(workspace=A[9] + 2 * 32 * 4 - 4), dict(workspace=A[7]), dict(workspace=A[6] - 64),
    dict(P=0, prefix_k=None, prefix_v=None, prefix_weight=None, out=A[3])])
def test_attention_scored_refuses_outputs_over_what_it_reads(mb, change):
    assert "overlaps" in refused(mb, "mlora_attention_scored", SCORED, change)


# two streams of 2 KV heads of 64, segments of 64 rows cut to 32
EVICT = dict(own_k=A[0], own_v=A[1], own_weight=A[2], own_position=A[3], cap=64, suffix_len=A[4], suffix_bound=40, newest=A[5], budget=32, recent=4, n=2,
             Hkv=2, hd=64, out_weight=A[6], out_position=A[7], out_len=A[8], out_source=A[9], workspace=A[10], workspace_bytes=STEP, status=A[11], stream=None)
SOURCE = 2 * 2 * 32 * 4
IN_PLACE = dict(out_weight=A[2], out_position=A[3])


@pytest.mark.parametrize("change", [
    dict(own_v=A[0]), dict(own_v=A[0] + OWN - 16), dict(own_k=A[2]), dict(own_weight=A[1] + OWN - 4), dict(out_weight=A[3]), dict(out_position=A[2] + TOTALS - 4),
    dict(out_weight=A[7]), dict(out_weight=A[0]), dict(out_position=A[1] + OWN - 4), dict(out_len=A[2]), dict(out_len=A[6] + TOTALS - 4), dict(out_len=A[4] + 4),
    dict(out_len=A[5]), dict(out_weight=A[4]), dict(out_position=A[5] - TOTALS + 4), dict(out_source=A[2]), dict(out_source=A[3] + TOTALS - 4), dict(out_source=A[7]),
    dict(out_source=A[8]), dict(out_source=A[4] - SOURCE + 4), dict(workspace=A[0]), dict(workspace=A[2]), dict(workspace=A[7] + TOTALS - 16), dict(workspace=A[4]),
    dict(workspace=A[9] + SOURCE - 16), dict(workspace=A[8]), dict(out_weight=A[2] + 4), dict(out_position=A[3] - 4),
    {**IN_PLACE, "out_len": A[2]}, {**IN_PLACE, "out_source": A[3]}, {**IN_PLACE, "own_v": A[3]}, dict(out_weight=A[3], out_position=A[2])])
def test_kv_evict_refuses_outputs_over_what_it_reads(mb, change):
    assert "overlap" in refused(mb, "mlora_kv_evict", EVICT, change)


# ------------------------------------------------------------------ the other refusals, each by its own check
UNSUPPORTED, CAPACITY = -6, -3


def each(fragment, *changes, code=ARG):
    return [pytest.param(code, fragment, c, id=f"{fragment}-{'-'.join(f'{k}={v}' for k, v in c.items())}".replace(" ", "_")) for c in changes]


def by_its_own_check(mb, name, good, code, fragment, change):
    assert set(change) <= set(good)
    assert getattr(mb.lib(), name)(*{**good, **change}.values()) == code
    assert fragment in mb.lib().mlora_last_error(None).decode()


NO_KV = dict(k=None, v=None, own_k=None, own_v=None)


@pytest.mark.parametrize("code,fragment,change", [
    *each("null argument", dict(positions=None), dict(freq=None)),
    *each("q and q_out go together", dict(q=None), dict(q_out=None)),
    *each("k, v, own_k and own_v go together", dict(k=None), dict(v=None), dict(own_k=None), dict(own_v=None)),
    *each("nothing to do", dict(q=None, q_out=None, **NO_KV)),
    *each("null suffix_len or status", dict(suffix_len=None), dict(status=None)),
    *each("belong to appended rows", dict(own_position=None, **NO_KV), dict(own_weight=None, **NO_KV)),
    *each("bad shape", dict(n=0), dict(n=-1), dict(T=0), dict(Hq=0), dict(Hkv=0), dict(Hkv=-2), dict(Hq=1 << 14), dict(n=1 << 20, T=1 << 20, cap=1 << 21)),
    *each("head_dim", dict(hd=80), dict(hd=256), dict(hd=0), code=UNSUPPORTED),
    *each("rotary_dim", dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=80), dict(rotary_dim=-16), code=UNSUPPORTED),
    *each("exceeds own_capacity", dict(cap=2), dict(cap=0), dict(cap=-1), code=CAPACITY),
    *each("row strides", dict(q_stride=504), dict(q_stride=516), dict(q_stride=-512), dict(k_stride=132), dict(k_stride=120), dict(v_stride=0), dict(in_fp32=1, v_stride=130)),
    *each("aligned", *[{k: ROPE[k] + 8} for k in ("q", "k", "v", "q_out", "own_k", "own_v")]),
    *each("in place only", dict(q_out=A[0], in_fp32=1), dict(q_out=A[0], q_stride=1024))])
def test_rope_append_refuses_by_the_check_that_is_meant(mb, code, fragment, change):
    by_its_own_check(mb, "mlora_rope_append", ROPE, code, fragment, change)


@pytest.mark.parametrize("code,fragment,change", [
    *each("null argument", *[{k: None} for k in ("q", "own_k", "own_v", "suffix_len", "out", "own_weight", "workspace", "status")]),
    *each("null prefix", dict(prefix_k=None), dict(prefix_v=None)),
    *each("bad shape", dict(n=0), dict(n=-1), dict(T=0), dict(T=65, cap=200), dict(Hq=7), dict(Hq=0), dict(Hkv=0), dict(Hkv=-2), dict(P=-1), dict(suffix_bound=-1),
          dict(P=1 << 28), dict(suffix_bound=1 << 28, cap=(1 << 28) + 3), dict(Hq=1 << 17, Hkv=1 << 17), dict(n=1 << 27)),
    *each("head_dim", dict(hd=96), dict(hd=256), code=UNSUPPORTED),
    *each("exceeds own_capacity", dict(suffix_bound=62), dict(cap=42), dict(cap=-1), code=CAPACITY),
    *each("workspace too small", dict(workspace_bytes=0), dict(workspace_bytes=64), code=CAPACITY),
    *each("aligned", *[{k: SCORED[k] + 8} for k in ("q", "prefix_k", "prefix_v", "own_k", "own_v", "out")])])
def test_attention_scored_refuses_by_the_check_that_is_meant(mb, code, fragment, change):
    by_its_own_check(mb, "mlora_attention_scored", SCORED, code, fragment, change)


@pytest.mark.parametrize("code,fragment,change", [
    *each("null argument", *[{k: None} for k in ("own_k", "own_v", "own_weight", "suffix_len", "out_weight", "out_len", "workspace", "status")]),
    *each("go together", dict(own_position=None), dict(out_position=None)),
    *each("bad shape", dict(n=0), dict(n=-1), dict(Hkv=0), dict(n=40000), dict(suffix_bound=-1), dict(budget=0), dict(budget=-3)),
    *each("recent needs", dict(newest=None), dict(own_position=None, out_position=None), dict(recent=33), dict(recent=-1)),
    *each("head_dim", dict(hd=32), dict(hd=96), code=UNSUPPORTED),
    *each("exceeds own_capacity", dict(suffix_bound=65), dict(cap=39), code=CAPACITY),
    *each("workspace too small", dict(workspace_bytes=0), dict(workspace_bytes=64), code=CAPACITY),
    *each("aligned", dict(own_k=A[0] + 8), dict(own_v=A[1] + 2))])
def test_kv_evict_refuses_by_the_check_that_is_meant(mb, code, fragment, change):
    by_its_own_check(mb, "mlora_kv_evict", EVICT, code, fragment, change)
