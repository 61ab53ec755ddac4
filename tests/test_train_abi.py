"""Host side of the training calls (no GPU): what they refuse, the frequencies of rotary positions, the table of gradients."""
import ctypes
import math
import struct

import pytest
import torch

from paper_2604_15408_amd import binding

FAKE = 0x10000          # non-null, 16-byte aligned; never dereferenced because validation fails first
NULL, SHAPE, UNSUPPORTED, CAPACITY = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    if not binding.LIB_PATH.exists():
        from paper_2604_15408_amd import build
        build.build()
    return binding.load()


def test_rope_validation(lib):
    def call(q=FAKE, k=FAKE, qo=FAKE * 2, ko=FAKE * 3, rows=8, rd=None, hq=2, hk=1, d=64, qs=128, ks=64, qos=128, kos=64, co=FAKE, nc=8,
             axes=1, ix=None, fr=FAKE, pairs=32, layout=0, amp=1.0, inv=0, dt=0):
        return lib.ragged_rope(q, k, qo, ko, rows, rd, hq, hk, d, qs, ks, qos, kos, co, nc, axes, ix, fr, pairs, layout, amp, inv, dt, None)
    for null in ("q", "qo", "co", "fr", "k", "ko"):
        assert call(**{null: None}) == NULL
    for bad in (dict(rows=0), dict(rows=1 << 31), dict(hq=0), dict(hk=0), dict(d=0), dict(pairs=0), dict(pairs=33), dict(axes=0),
                dict(axes=3), dict(nc=0), dict(nc=1 << 31), dict(qs=120), dict(ks=56), dict(qos=127), dict(kos=0), dict(qs=1 << 31),
                dict(hq=1 << 17, qs=1 << 23, qos=1 << 23), dict(qo=FAKE, qos=136), dict(ko=FAKE, kos=72)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(dt=2), dict(d=60, pairs=30), dict(d=520, qs=1040, qos=1040, ks=520, kos=520), dict(layout=2), dict(inv=2),
                dict(amp=float("nan")), dict(qs=132), dict(kos=68), dict(q=FAKE + 8), dict(ko=FAKE + 2), dict(fr=FAKE + 4), dict(co=FAKE + 2),
                dict(ix=FAKE + 1), dict(rd=FAKE + 2), dict(k=FAKE * 2), dict(q=FAKE * 3), dict(ko=FAKE * 2)):
        assert call(**bad) == UNSUPPORTED, bad


def test_attn_lse_validation(lib):
    def call(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, cu=FAKE, B=2, ms=8, H=2, D=64, si=384, so=128, scale=0.125, dt=0):
        return lib.ragged_attn_lse(q, k, v, o, lse, cu, B, ms, H, D, si, so, scale, dt, None)
    for null in ("q", "k", "v", "o", "lse", "cu"):
        assert call(**{null: None}) == NULL
    for bad in (dict(B=0), dict(ms=0), dict(si=127), dict(so=64), dict(si=(1 << 23) + 8), dict(so=1 << 31)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(D=32), dict(si=132), dict(so=132), dict(dt=2), dict(scale=float("inf")), dict(lse=FAKE + 2), dict(o=FAKE + 8)):
        assert call(**bad) == UNSUPPORTED, bad


def test_attn_backward_validation(lib):
    def call(q=FAKE, k=FAKE, v=FAKE, o=FAKE, do=FAKE, lse=FAKE, dq=2 * FAKE, dk=3 * FAKE, dv=4 * FAKE, cu=FAKE, B=2, ms=8, H=2, D=64, si=384,
             so=128, sg=384, scale=0.125, dt=0):
        return lib.ragged_attn_backward(q, k, v, o, do, lse, dq, dk, dv, cu, B, ms, H, D, si, so, sg, scale, dt, None)
    for null in ("q", "k", "v", "o", "do", "lse", "dq", "dk", "dv", "cu"):
        assert call(**{null: None}) == NULL
    for bad in (dict(B=0), dict(H=0), dict(ms=0), dict(ms=64 * 32767 + 1), dict(ms=(1 << 31) - 1), dict(B=1 << 16, H=16, ms=1 << 16),
                dict(si=127), dict(so=64), dict(sg=120), dict(so=(1 << 23) + 8), dict(sg=1 << 31)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(D=128, si=768, so=256, sg=768), dict(si=132), dict(so=132), dict(sg=132), dict(dt=2), dict(scale=float("nan")),
                dict(lse=FAKE + 2), dict(do=FAKE + 8), dict(dq=FAKE + 2), dict(dk=FAKE + 4), dict(dv=FAKE + 8), dict(dq=FAKE),
                dict(dk=FAKE), dict(dv=FAKE), dict(o=5 * FAKE, dv=5 * FAKE), dict(dk=2 * FAKE), dict(dv=3 * FAKE)):
        assert call(**bad) == UNSUPPORTED, bad


def test_layernorm_backward_validation(lib):
    def call(x=FAKE, g=FAKE, dy=FAKE, r=None, dx=FAKE * 2, dg=FAKE, db=FAKE, ws=FAKE, rows=16, rd=None, C=768, eps=1e-6, dt=0):
        return lib.ragged_layernorm_backward(x, g, dy, r, dx, dg, db, ws, rows, rd, C, eps, dt, None)
    for null in ("x", "g", "dy", "dx", "dg", "db", "ws"):
        assert call(**{null: None}) == NULL
    for bad in (dict(rows=0), dict(rows=1 << 31), dict(C=0)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(C=100), dict(C=4096), dict(eps=-1.0), dict(eps=float("nan")), dict(dt=2), dict(dx=FAKE), dict(dy=FAKE + 8),
                dict(r=FAKE + 2), dict(dg=FAKE + 2), dict(db=FAKE + 1), dict(ws=FAKE + 8), dict(rd=FAKE + 2)):
        assert call(**bad) == UNSUPPORTED, bad
    need = lib.ragged_layernorm_backward_workspace
    assert need(0, 64) == need(8, 12) == need(8, 4096) == need(1 << 31, 64) == 0
    assert need(1, 8) >= 2 * 8 * 4 and need(1 << 20, 2048) >= need(1, 2048)
    with pytest.raises(ValueError):
        binding.layernorm_backward_workspace(8, 12)


def test_grad_clip_validation(lib):
    def call(table=FAKE, chunks=1, scale=1.0, most=1.0, ws=FAKE, norm=FAKE):
        return lib.ragged_grad_clip(table, chunks, scale, most, ws, norm, None)
    for null in ("table", "ws", "norm"):
        assert call(**{null: None}) == NULL
    assert call(chunks=-1) == SHAPE and call(chunks=1 << 31) == SHAPE
    for bad in (dict(scale=float("inf")), dict(scale=float("nan")), dict(most=0.0), dict(most=-1.0), dict(most=float("nan")),
                dict(table=FAKE + 8), dict(ws=FAKE + 8), dict(norm=FAKE + 4)):
        assert call(**bad) == UNSUPPORTED, bad


def _plan(lib, tensors, table=None, capacity=0):
    entries = (binding._GradTensor * max(1, len(tensors)))(*[binding._GradTensor(*t) for t in tensors])
    chunks = ctypes.c_int64(-1)
    return lib.ragged_grad_plan(ctypes.addressof(entries), len(tensors), table, capacity, ctypes.addressof(chunks)), chunks.value


def test_grad_plan_refuses(lib):
    good = (FAKE, FAKE * 2, 100, 2, 2)
    chunks = ctypes.c_int64()
    assert lib.ragged_grad_plan(None, 1, None, 0, ctypes.addressof(chunks)) == NULL
    assert lib.ragged_grad_plan(FAKE, 0, None, 0, ctypes.addressof(chunks)) == SHAPE
    assert _plan(lib, [good]) == (0, 1)
    for bad, status in (((None, FAKE, 100, 2, 2), NULL), ((FAKE, FAKE, -1, 2, 2), SHAPE), ((FAKE, FAKE * 2, 1 << 50, 2, 2), SHAPE),
                        ((FAKE, FAKE * 2, 8, 3, 2), UNSUPPORTED), ((FAKE, FAKE * 2, 8, 2, 0), UNSUPPORTED), ((FAKE, FAKE * 2, 8, 0, 1), UNSUPPORTED),
                        ((FAKE, FAKE, 8, 0, 2), UNSUPPORTED), ((FAKE + 2, FAKE * 2, 8, 2, 2), UNSUPPORTED), ((FAKE, FAKE + 1, 8, 0, 0), UNSUPPORTED)):
        assert _plan(lib, [good, bad])[0] == status, bad
    table = ctypes.create_string_buffer(64)
    assert _plan(lib, [good, good, good], ctypes.addressof(table), 64)[0] == CAPACITY


def test_grad_plan_covers_every_value_once(lib):
    tensors = [(FAKE, FAKE * 8, 5, 2, 2), (None, None, 0, 0, 0), (FAKE * 2, FAKE * 16, 40000, 0, 2), (FAKE * 3 + 2, None, 16384, 1, 1),
               (FAKE * 4, FAKE * 4, 16385, 1, 1)]
    status, chunks = _plan(lib, tensors)
    assert status == 0
    size = binding.GRAD_CHUNK_BYTES
    table = ctypes.create_string_buffer(chunks * size)
    assert _plan(lib, tensors, ctypes.addressof(table), chunks * size) == (0, chunks)
    at = 0
    bytes_of = {0: 2, 1: 2, 2: 4}
    for src, dst, numel, src_dt, dst_dt in tensors:
        done = 0
        while done < numel:
            s, d, n, sdt, ddt, _ = struct.unpack_from("<QQiiii", table, at)
            at += size
            assert 0 < n <= numel - done and (sdt, ddt) == (src_dt, dst_dt)
            assert s == src + done * bytes_of[src_dt] and d == (0 if dst is None else dst + done * bytes_of[dst_dt])
            done += n
    assert at == chunks * size


def test_grad_plan_of_a_tensor_beyond_32_bits(lib):
    numel = (1 << 33) + 5
    status, chunks = _plan(lib, [(FAKE, FAKE << 20, numel, 2, 2)])
    assert status == 0
    size = binding.GRAD_CHUNK_BYTES
    table = ctypes.create_string_buffer(chunks * size)
    assert _plan(lib, [(FAKE, FAKE << 20, numel, 2, 2)], ctypes.addressof(table), chunks * size) == (0, chunks)
    s, d, n, *_ = struct.unpack_from("<QQiiii", table, (chunks - 1) * size)
    assert s + 4 * n == FAKE + 4 * numel and d + 4 * n == (FAKE << 20) + 4 * numel


def test_rope_frequencies(lib):
    for pairs, base in ((1, 10000.0), (10, 100.0), (32, 10000.0)):
        want = torch.tensor([base ** (-p / pairs) for p in range(pairs)], dtype=torch.float64)
        close = lambda got, w: torch.allclose(got, w, rtol=1e-14, atol=0)
        assert close(binding.rope_frequencies(pairs, base), want)
        assert close(binding.rope_frequencies(2 * pairs, base, axes=2), want.repeat(2))
        assert close(binding.rope_frequencies(pairs, base, scaling="linear", factor=8.0), want / 8)
        longer = binding.rope_frequencies(pairs, base, scaling="base", factor=8.0)
        assert longer[0] == 1.0 and (pairs == 1 or abs(longer[-1] / (want[-1] / 8) - 1) < 1e-12)
        parts = binding.rope_frequencies(pairs, base, scaling="parts", factor=8.0, original_length=4096.0)
        share = ((4096.0 * want / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        assert close(parts, want * share + want / 8 * (1 - share))
    out = (ctypes.c_double * 4)()
    call = lambda p=FAKE, n=4, base=10.0, s=0, f=1.0, length=1.0, fast=2.0, slow=1.0: lib.ragged_rope_frequencies(p, n, base, s, f, length, fast, slow)
    assert call(p=None) == NULL and call(n=0) == SHAPE
    for bad in (dict(s=4), dict(s=-1), dict(base=0.0), dict(base=float("inf")), dict(f=0.0), dict(f=float("nan")), dict(s=3, length=0.0),
                dict(s=3, fast=1.0), dict(s=3, slow=float("nan"))):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(p=ctypes.addressof(out), length=0.0) == 0
    with pytest.raises(ValueError):
        binding.rope_frequencies(5, axes=2)


def test_native_checks_of_rows_and_devices(lib):
    native = binding._native()
    t = torch.zeros(4, 2, 64, dtype=torch.float16)
    for other in (t, torch.nn.Parameter(t), None, 3):
        assert native.rows(other, None, None) is None
    assert native.here(-1, t, None) and not native.here(0, t) and not native.here(-1, t, "x") and native.here(0)
    with pytest.raises(TypeError):
        native.rows(t)


def test_grad_outputs_that_overlap_are_refused(monkeypatch):
    """Two tensors that would be written to the same place, or one over another's gradient (addresses stand in for GPU tensors)."""
    monkeypatch.setattr(binding, "_dev", lambda t, *rest: t.data_ptr())
    flat = torch.zeros(100)
    for grads, outs in (([flat[:50], flat[:50]], None), ([flat[:60], flat[50:]], None), ([flat[:50], flat[50:]], [flat[:50], flat[:50]]),
                        ([flat[:50], flat[50:]], [flat[50:], None]), ([flat[:50]], [flat[1:51]])):
        with pytest.raises(ValueError, match="overlap"):
            binding.GradPlan(grads, outs)
    binding.GradPlan([flat[:50], flat[:50]], [None, None])     # (nothing is written)
    binding.GradPlan([flat[:50], flat[50:]])
    binding.GradPlan([flat[:0], flat[:50]], [flat[:0], torch.zeros(50)])


def test_binding_refuses_before_the_library():
    t = torch.zeros(4, 2, 64, dtype=torch.float16)
    with pytest.raises(TypeError, match="q must be a GPU tensor"):
        binding.ragged_rope(t, None, t, None, torch.zeros(4, 1), torch.zeros(32, dtype=torch.float64), stream=0)
    with pytest.raises(ValueError, match="come together"):
        binding.ragged_rope(t, t, t, None, torch.zeros(4, 1), torch.zeros(32, dtype=torch.float64), stream=0)
    with pytest.raises(TypeError, match="q must be a GPU tensor"):
        binding.ragged_attn_backward(t, t, t, t, t, t, t, t, t, torch.zeros(2, dtype=torch.int32), 4, 0.125, stream=0)
    with pytest.raises(ValueError, match="bytes"):
        x = torch.zeros(4, 64, dtype=torch.float16)
        binding.ragged_layernorm_backward(x, x[0], x, x, x[0], x[0], torch.zeros(8, dtype=torch.uint8), stream=0)
    with pytest.raises(TypeError, match="grad must be a GPU tensor"):
        binding.GradPlan([torch.zeros(4)])
    with pytest.raises(ValueError):
        binding.GradPlan([])
