"""Operators around a bounded KV cache on the GPU: calls at the edges of what their documentation allows."""
import numpy as np
import pytest

from tests.test_gpu_cache_ops import dev, i32, mb, status  # noqa: F401

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
