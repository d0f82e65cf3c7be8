"""The memory's operators refuse what their kernels could not use safely, before any
device work: host tensors stand in for device ones (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2607_26005_amd import memory, pictura

B, T, C = 2, 5, 6


@pytest.fixture(autouse=True)
def host_is_device(request, monkeypatch):
    if "device" not in request.node.name:
        monkeypatch.setattr(pictura, "_check_device", lambda t, name, ctx: None)


def _raises(match, fn, *a, **k):
    with pytest.raises(pictura.PicturaError, match=match) as e:
        fn(*a, **k)
    assert e.value.status == pictura.EINVAL


z = torch.zeros


@pytest.mark.parametrize("match, bad", [
    ("gates: expected a torch tensor", dict(gates=[[0.0]])),
    ("inputs: expected a torch tensor", dict(inputs=None)),
    ("gates: shape", dict(gates=z(T, C))),
    ("inputs: shape", dict(inputs=z(T, C))),
    ("gates: dtype", dict(gates=z(B, T, C).double(), inputs=z(B, T, C).double())),
    ("gates: shape", dict(gates=z(B, T, 0), inputs=z(B, T, 0))),
    ("gates: strides", dict(gates=z(B, C, T).transpose(1, 2))),
    ("gates: expected a plain", dict(gates=torch._neg_view(z(B, T, C)))),
    ("inputs: dtype", dict(inputs=z(B, T, C).half())),
    ("inputs: shape", dict(inputs=z(B, T + 1, C))),
    ("inputs: strides", dict(inputs=z(B, T, 2 * C)[..., ::2])),
    ("state: ", dict(state=z(B, C).half())),
    ("state: ", dict(state=z(B, C + 1))),
    ("state: ", dict(state=z(C, B).t())),
    ("state: expected a torch tensor", dict(state=0.0)),
    ("resets: dtype", dict(resets=z(B, T))),
    ("resets: shape", dict(resets=z(B, T + 1, dtype=torch.bool))),
    ("resets: shape", dict(resets=z(T, dtype=torch.bool))),
])
def test_scan_refuses(match, bad):
    _raises(match, memory.gated_scan, **dict(dict(gates=z(B, T, C), inputs=z(B, T, C)), **bad))
    if "inputs" not in bad:   # and where a gradient is wanted
        _raises(match, memory.gated_scan, **dict(dict(gates=z(B, T, C), inputs=z(B, T, C, requires_grad=True)), **bad))


@pytest.mark.parametrize("match, bad", [
    ("gates: shape", dict(gates=z(B, T, C))),
    ("inputs: dtype", dict(inputs=z(B, C).half())),
    ("inputs: expected a torch tensor", dict(inputs=None)),
    ("state: ", dict(state=z(B, C).half())),
    ("state: ", dict(state=z(B, 2 * C)[:, :C])),
    ("resets: shape", dict(resets=z(B, T, dtype=torch.bool))),
    ("out: dtype", dict(out=z(B, C).half())),
    ("out: shape", dict(out=z(B + 1, C))),
    ("out: strides", dict(out=z(1, C).expand(B, C))),
])
def test_step_refuses(match, bad):
    _raises(match, memory.gated_step, **dict(dict(gates=z(B, C), inputs=z(B, C), state=z(B, C)), **bad))


def test_a_step_refuses_to_lose_a_gradient():
    for name in ("gates", "inputs", "state"):
        a = dict(gates=z(B, C), inputs=z(B, C), state=z(B, C))
        a[name].requires_grad_()
        _raises("no gradient", memory.gated_step, **a)


def test_a_step_into_what_wants_a_gradient():
    """An `out` with a graph would keep that of what the step replaced."""
    for out in (z(B, C, requires_grad=True), z(B, C, requires_grad=True) * 2):
        _raises("no gradient", memory.gated_step, z(B, C), z(B, C), z(B, C), out=out)
        with torch.no_grad():   # (the next check)
            _raises("expected the HIP device", memory.gated_step, z(B, C), z(B, C), z(B, C), out=out)


def _steps():
    """What a step may write over, and what not: (match or None, arguments)."""
    both, half, held, row = z(4, 48), z(4, 48, dtype=torch.bfloat16), z(5, 16), z(64)
    a = dict(gates=both[:, :16], inputs=both[:, 16:32], state=z(4, 16))
    b = dict(gates=z(4, 16, dtype=torch.bfloat16), inputs=half[:, 16:32], state=z(4, 16))
    flat, last = both.view(-1), both.view(torch.bool).view(4, -1)[:, -1]
    for out in (None, a["gates"], a["inputs"], both[:, 32:], a["state"], z(4, 16)):   # its own rows, or rows between
        yield None, dict(a, out=out)
    yield None, dict(a, inputs=a["state"])
    yield None, dict(a, resets=last)
    yield "out: overlaps the gates", dict(a, out=both[:, 8:24])                            # shifted
    yield "out: overlaps the gates", dict(a, out=both[:, 1:17])
    yield "out: overlaps the inputs", dict(a, out=both[:, 31:47])
    yield "out: overlaps the gates", dict(a, out=flat[:64].view(4, 16))                   # another stride
    yield "out: overlaps the gates", dict(a, out=flat[-65:-1].view(4, 16))   # (the inputs too)
    yield "out: overlaps the gates", dict(a, gates=row[:16].expand(4, 16), out=row.view(4, 16))
    yield "out: overlaps the state", dict(a, state=held[:4], out=held[1:])
    yield "out: overlaps the state", dict(b, out=b["state"].view(torch.bfloat16)[:, :16])
    yield "state: overlaps the gates", dict(a, gates=held[1:], state=held[:4])
    yield "state: overlaps the inputs", dict(a, inputs=flat[8:72].view(4, 16), state=flat[:64].view(4, 16), gates=z(4, 16))
    yield "state: overlaps the inputs", dict(b, state=half.view(-1)[:128].view(torch.float32).view(4, 16))
    yield "out: overlaps the resets", dict(a, out=both[:, 32:], resets=last)
    yield "state: overlaps the resets", dict(a, resets=a["state"].view(torch.bool)[:, 3])


def test_a_step_writes_over_its_own_operands_alone():
    """Threads run in any order: what one writes over another's operands is right or wrong by chance."""
    for match, a in _steps():
        _raises(match or "expected the HIP device", memory.gated_step, **a)
        if match:
            _raises(match, pictura.pictura_gated_step, **dict(dict(out=z(4, 16, dtype=a["gates"].dtype)), **a))


def test_the_step_entry_refuses_the_same():
    L, ref = pictura._lib, ctypes.byref
    q = lambda **k: ref(_q(**dict(dict(steps=1, batch=4, channels=16, gates=4096, inputs=4096 + 64, gates_batch=48, inputs_batch=48), **k)))
    step = lambda out=1 << 16, stride=16, state=1 << 20, **k: L.pictura_gated_step(q(**k), out, stride, state, None)
    for k in (dict(out=4096 + 4, stride=48), dict(out=4096, stride=16), dict(out=4096 - 252), dict(out=4096 + 3 * 192 + 60),
              dict(state=4096), dict(state=4096 + 640 - 4), dict(out=(1 << 20) + 4), dict(out=(1 << 20) - 252, stride=16),
              dict(resets=(1 << 16) + 252, resets_batch=1), dict(resets=(1 << 20) - 3, resets_batch=1), dict(dtype=1, out=1 << 20)):
        assert step(**k) == pictura.EINVAL, k


def test_overlap_is_exact(tmp_path):
    """pictura_overlap.h against every byte of small regions."""
    import os
    import subprocess
    source = tmp_path / "overlap.cpp"
    source.write_text(r"""
#include <cstdio>
#include <set>
#include "pictura_overlap.h"
using namespace pictura;
int main()
{
    int both = 0, wrong = 0;
    std::set<uintptr_t> held;
    for (int64_t ra = 1; ra < 5; ++ra) for (int64_t na = 1; na < 4; ++na) for (int64_t sa = 0; sa < 9; ++sa) {
        const Region a{100, ra, na, sa};
        held.clear();
        for (int64_t i = 0; i < ra; ++i) for (int64_t j = 0; j < na; ++j) held.insert(100 + i * sa + j);
        for (uintptr_t at = 70; at < 140; ++at) for (int64_t rb = 1; rb < 5; ++rb) for (int64_t nb = 1; nb < 4; ++nb)
            for (int64_t sb = 0; sb < 9; ++sb) {
                bool want = false;
                for (int64_t i = 0; i < rb && !want; ++i) for (int64_t j = 0; j < nb; ++j) want = want || held.count(at + i * sb + j);
                both += want;
                wrong += want != overlap(a, Region{at, rb, nb, sb});
            }
    }
    const Region none{0, 4, 4, 4}, empty{100, 0, 4, 4}, some{100, 4, 4, 4};
    wrong += overlap(none, some) + overlap(empty, some) + overlap(some, empty) + !same(some, some) + same(some, Region{100, 4, 4, 8});
    printf("%d %d\n", both, wrong);
}
""")
    csrc = os.path.join(os.path.dirname(pictura.__file__), "csrc")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-I", csrc, str(source), "-o", str(tmp_path / "overlap")])
    both, wrong = map(int, subprocess.check_output([str(tmp_path / "overlap")]).split())
    assert both > 10000 and wrong == 0


def test_outputs_of_the_scan_are_checked():
    ok = lambda: dict(gates=z(B, T, C), inputs=z(B, T, C), out=z(B, T, C), last_state=z(B, C))
    _raises("out: shape", pictura.pictura_gated_scan, **dict(ok(), out=z(B, T, C + 1)))
    _raises("last_state: ", pictura.pictura_gated_scan, **dict(ok(), last_state=z(B)))
    _raises("saved: ", pictura.pictura_gated_scan, **dict(ok(), saved=z(2, B, C)))
    _raises("out: strides .* overlap", pictura.pictura_gated_scan, **dict(ok(), out=z(B, 1, C).expand(B, T, C)))
    _raises("out: strides .* overlap", pictura.pictura_gated_scan, **dict(ok(), out=z(20 * C).as_strided((B, T, C), (C, C, 1))))
    g = lambda **k: dict(dict(gates=z(B, T, C), inputs=z(B, T, C), saved=z(1, B, C), dout=z(B, T, C), dlast=z(B, C),
                              dgates=z(B, T, C), dinputs=z(B, T, C), dstate=z(B, C)), **k)
    _raises("dout: dtype", pictura.pictura_gated_scan_gradient, **g(dout=z(B, T, C).half()))
    _raises("dlast: ", pictura.pictura_gated_scan_gradient, **g(dlast=z(B, C + 1)))
    _raises("dgates: shape", pictura.pictura_gated_scan_gradient, **g(dgates=z(B, C)))
    _raises("dinputs: strides .* overlap", pictura.pictura_gated_scan_gradient, **g(dinputs=z(1, T, C).expand(B, T, C)))
    _raises("dstate: ", pictura.pictura_gated_scan_gradient, **g(dstate=z(B, C).half()))


def test_host_tensors_are_refused_for_their_device():
    _raises("expected the HIP device", memory.gated_scan, z(B, T, C), z(B, T, C))
    _raises("expected the HIP device", memory.gated_step, z(B, C), z(B, C), z(B, C))


# --- the C entries themselves: bad arguments come back as a status, before any launch

class _Sequences(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("gates", "inputs", "state", "resets")] + \
               [(n, ctypes.c_int64) for n in ("gates_batch", "gates_step", "inputs_batch", "inputs_step", "resets_batch",
                                              "resets_step", "batch", "steps")] + \
               [("channels", ctypes.c_int32), ("dtype", ctypes.c_int32)]


def _q(**over):
    q = _Sequences(64, 64, None, None, T * C, C, T * C, C, 0, 0, B, T, C, 0)
    for k, v in over.items():
        setattr(q, k, v)
    return q


def test_c_entries_refuse():
    L, ref = pictura._lib, ctypes.byref
    scan = lambda q=None, out=64, ob=T * C, os_=C, last=64, saved=64, ws=256, n=1 << 40: \
        L.pictura_gated_scan(ref(q or _q()), out, ob, os_, last, saved, ws, n, None)
    grad = lambda q=None, saved=64, dout=64, db=T * C, dlast=64, dg=64, gb=T * C, dx=64, xs=C, ds=64, ws=256, n=1 << 40: \
        L.pictura_gated_scan_gradient(ref(q or _q()), saved, dout, db, C, dlast, dg, gb, C, dx, T * C, xs, ds, ws, n, None)
    step = lambda q=None, out=64, ob=C, state=64: L.pictura_gated_step(ref(q or _q(steps=1)), out, ob, state, None)
    sizes = [dict(dtype=3), dict(batch=-1), dict(steps=-1), dict(steps=1 << 31), dict(channels=0), dict(batch=1 << 31)]
    inputs = [dict(gates=None), dict(inputs=None), dict(gates=66), dict(inputs=65), dict(state=66), dict(gates_step=-1),
              dict(inputs_batch=-1), dict(resets_step=-1)]
    for over in sizes + inputs:
        assert scan(_q(**over)) == pictura.EINVAL, over
        assert grad(_q(**over)) == pictura.EINVAL, over
        assert step(_q(**dict(dict(steps=1), **over))) == pictura.EINVAL, over
    for k in (dict(out=None), dict(out=66), dict(ob=T * C - 1), dict(os_=C - 1), dict(last=66), dict(saved=66), dict(ws=None),
              dict(ws=128), dict(n=8)):
        assert scan(**k) == pictura.EINVAL, k
    for k in (dict(saved=None), dict(saved=66), dict(dout=None), dict(dout=66), dict(db=-1), dict(dlast=66), dict(dg=None), dict(dg=66),
              dict(gb=T * C - 1), dict(dx=None), dict(xs=0), dict(ds=66), dict(ws=None), dict(n=8)):
        assert grad(**k) == pictura.EINVAL, k
    for k in (dict(out=None), dict(out=66), dict(ob=C - 1), dict(state=None), dict(state=66), dict(q=_q())):
        assert step(**k) == pictura.EINVAL, k
    assert L.pictura_gated_scan(None, 64, T * C, C, 64, 64, 256, 1 << 40, None) == pictura.EINVAL
    out = ctypes.c_uint64()
    assert L.pictura_gated_scan_workspace(None, ctypes.addressof(out)) == pictura.EINVAL
    assert L.pictura_gated_scan_workspace(ref(_q()), None) == pictura.EINVAL
    assert scan(_q(batch=0, gates=None)) == pictura.OK


def test_c_entries_of_no_steps_have_nothing_to_write():
    """Without steps all that a scan or its gradient could write is the state's side."""
    L, q = pictura._lib, ctypes.byref(_q(steps=0, gates=None, inputs=None))
    assert L.pictura_gated_scan(q, None, 0, 0, None, None, None, 0, None) == pictura.OK
    assert L.pictura_gated_scan_gradient(q, None, None, 0, 0, 64, None, 0, 0, None, 0, 0, None, None, 0, None) == pictura.OK
    assert L.pictura_gated_scan(q, None, 0, 0, 66, None, None, 0, None) == pictura.EINVAL
    assert L.pictura_gated_scan_gradient(q, None, None, 0, 0, 66, None, 0, 0, None, 0, 0, None, None, 0, None) == pictura.EINVAL


def test_workspace_covers_every_split():
    """However the steps are cut, maps of all segments and groups fit."""
    L = pictura._lib
    need = ctypes.c_uint64()
    for batch, steps, channels in ((1, 1, 1), (1, 10 ** 6, 1), (1, 65521, 1024), (3, 8191, 331), (2048, 128, 512),
                                   (1, 2 ** 31 - 1, 2), (2 ** 20, 3, 2047)):
        q = _q(batch=batch, steps=steps, channels=channels)
        assert L.pictura_gated_scan_workspace(ctypes.byref(q), ctypes.addressof(need)) == pictura.OK
        assert need.value <= 256 + (512 + 32) * 8 * max(batch * channels, 64 * 4096)


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("channels", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 8])
def test_as_many_channels_as_there_may_be(channels, dtype):
    """Their count of threads does not leave 32 bits: such scans are not cut, and need no words for tiles."""
    need = ctypes.c_uint64()
    q = _q(batch=1, steps=1 << 20, channels=channels, dtype=dtype)
    assert pictura._lib.pictura_gated_scan_workspace(ctypes.byref(q), ctypes.addressof(need)) == pictura.OK
    assert need.value == 256


def test_a_workspace_holds_the_words_of_its_tiles():
    """Pairs of channels of 16 bits are cut into tiles of 128 steps, single channels into tiles of 256; each tile
    tells a word of 8 bytes a channel, and every 16 of them one more, behind 256 bytes for the tickets."""
    need = ctypes.c_uint64()
    for dtype, batch, steps, channels in ((0, 1, 65521, 1024), (1, 1, 65521, 1024), (2, 3, 8191, 331), (0, 3, 8191, 331), (1, 5, 512, 1),
                                          (1, 1, 2 ** 31 - 1, 2), (0, 1, 511, 8), (0, 1, 512, 8), (1, 1, 255, 8), (1, 1, 256, 8)):
        q = _q(batch=batch, steps=steps, channels=channels, dtype=dtype)
        assert pictura._lib.pictura_gated_scan_workspace(ctypes.byref(q), ctypes.addressof(need)) == pictura.OK
        pair, tile = (2, 128) if dtype and channels > 1 else (1, 256)
        threads, tiles = batch * -(-channels // pair), -(-steps // tile)
        cut = steps >= 2 * tile and (threads + 63) // 64 * tiles <= 1 << 21
        assert need.value == 256 + (8 * threads * pair * (tiles + -(-tiles // 16)) if cut else 0), (dtype, batch, steps, channels)


# --- the norm ---------------------------------------------------------------------

N, W = 4, 6


@pytest.mark.parametrize("match, bad", [
    ("x: expected a torch tensor", dict(x=[[0.0]])),
    ("x: expected a torch tensor", dict(x=torch.zeros(()))),
    ("x: dtype", dict(x=z(N, W).double())),
    ("x: shape", dict(x=z(N, 0))),
    ("x: shape", dict(x=z(1, 65537), weight=z(65537))),
    ("x: expected a plain", dict(x=torch._neg_view(z(N, W)))),
    ("weight: expected a torch tensor", dict(weight=1.0)),
    ("weight: ", dict(weight=z(W + 1))),
    ("weight: ", dict(weight=z(1, W))),
    ("weight: ", dict(weight=z(2 * W)[::2])),
    ("weight: ", dict(weight=z(W).half())),
    ("weight: dtype", dict(weight=z(W).double())),
    ("residual: expected a torch tensor", dict(residual=0)),
    ("residual: dtype", dict(residual=z(N, W).half())),
    ("residual: shape", dict(residual=z(N + 1, W))),
    ("eps: ", dict(eps=-1.0)),
    ("eps: ", dict(eps=float("nan"))),
    ("eps: ", dict(eps=float("inf"))),
    ("eps: ", dict(eps="small")),
])
def test_norm_refuses(match, bad):
    a = dict(dict(x=z(N, W), weight=z(W)), **bad)
    _raises(match, memory.rms_norm, **a)
    _raises(match, memory.rms_norm_8bit, **a)
    if "weight" not in bad:
        _raises(match, memory.rms_norm, **dict(a, weight=z(W, requires_grad=True)))


def test_the_norms_other_arguments_are_checked():
    x, w, f, s = z(N, W), z(W), z(N), pictura
    _raises("dtype: ", memory.rms_norm_8bit, x, w, dtype=torch.uint8)
    _raises("out: shape", s.pictura_rms_norm, x, w, z(N, W + 1))
    _raises("out: dtype", s.pictura_rms_norm, x, w, z(N, W).half())
    _raises("out: strides", s.pictura_rms_norm, x, w, z(1, W).expand(N, W))
    _raises("out: strides", s.pictura_rms_norm, x, w, z(W, N).t())
    _raises("sum: shape", s.pictura_rms_norm, x, w, x, z(N, W + 1))
    _raises("sum: strides", s.pictura_rms_norm, x, w, x, z(1, W).expand(N, W))
    _raises("factors: ", s.pictura_rms_norm, x, w, x, None, None, 1e-6, z(N + 1))
    _raises("codes: dtype", s.pictura_rms_norm_codes, x, w, z(N, W), f)
    _raises("codes: shape", s.pictura_rms_norm_codes, x, w, z(N, W + 1, dtype=torch.int8), f)
    _raises("scales: ", s.pictura_rms_norm_codes, x, w, z(N, W, dtype=torch.int8), z(N).half())
    _raises("dout: shape", s.pictura_rms_norm_gradient, x, w, f, z(N, W + 1), x, w)
    _raises("dsum: dtype", s.pictura_rms_norm_gradient, x, w, f, x, x, w, x.half())
    _raises("dx: strides", s.pictura_rms_norm_gradient, x, w, f, x, z(1, W).expand(N, W), w)
    _raises("dweight: ", s.pictura_rms_norm_gradient, x, w, f, x, x, w.half())
    _raises("codes: dtype", s.pictura_row_values, x, f, x)
    _raises("out: dtype", s.pictura_row_values, z(N, W, dtype=torch.int8), f, x.half())
    _raises("out: shape", s.pictura_row_values, z(N, W, dtype=torch.int8), f, z(N, W + 1))
    _raises("scales: shape", s.pictura_row_values, z(N, W, dtype=torch.int8), z(N + 1), x)
    _raises("out: expected a contiguous", memory.RowCodes(z(N, W, dtype=torch.int8), f, None).values, z(W, N).t())


def test_values_are_apart_from_their_codes():
    out = z(4, 16)
    codes = out.view(torch.int8)
    for c in (codes[:, :16], codes[:, 48:], codes.view(-1)[100:164].view(4, 16)):
        _raises("out: overlaps the codes", memory.RowCodes(c, z(4), None).values, out)
    _raises("out: overlaps the scales", memory.RowCodes(z(4, 16, dtype=torch.int8), out.view(-1)[3:7], None).values, out)
    held = z(5, 16)   # beside one another
    _raises("expected the HIP device", memory.RowCodes(held.view(torch.int8)[:4, :16], held[4, :4], None).values, z(4, 16))
    _raises("expected the HIP device", memory.RowCodes(held.view(torch.int8)[4:, :16], held[4, 15:], None).values, held[3:4])
    values = lambda c=1 << 16, cs=16, s=1 << 20, out=4096, os_=16: pictura._lib.pictura_row_values(c, cs, s, 0, 4, 16, out, os_, None)
    for k in (dict(c=4096 + 240), dict(c=4096 - 63), dict(s=4096 + 252), dict(s=4096 - 12)):
        assert values(**k) == pictura.EINVAL, k


def test_values_refuse_to_lose_a_gradient():
    codes, scales, out = z(N, W, dtype=torch.int8), z(N), z(N, W)
    _raises("out: hands on no gradient", memory.RowCodes(codes, scales.requires_grad_(), None).values, out)
    _raises("out: hands on no gradient", memory.RowCodes(codes, z(N), None).values, z(N, W, requires_grad=True))
    with torch.no_grad():   # (the next check)
        _raises("expected the HIP device", memory.RowCodes(codes, scales, None).values, out)


def test_the_norm_refuses_host_tensors_for_their_device():
    _raises("expected the HIP device", memory.rms_norm, z(N, W), z(W))
    _raises("expected the HIP device", memory.rms_norm_8bit, z(N, W), z(W))


class _Norm(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "residual", "weight")] + \
               [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride", "rows")] + \
               [(n, ctypes.c_int32) for n in ("width", "dtype", "weight_dtype")] + [("eps", ctypes.c_float)]


def test_the_norms_c_entries_refuse():
    L, ref = pictura._lib, ctypes.byref

    def q(**over):
        n = _Norm(64, None, 64, W, W, N, W, 0, 0, 1e-6)
        for k, v in over.items():
            setattr(n, k, v)
        return n

    norm = lambda n=None, sum=None, ss=W, out=64, os_=W, f=None: L.pictura_rms_norm(ref(n or q()), sum, ss, out, os_, f, None)
    codes = lambda n=None, kind=0, sum=None, ss=W, c=64, cs=W, s=64: \
        L.pictura_rms_norm_codes(ref(n or q()), kind, sum, ss, c, cs, s, None)
    grad = lambda n=None, f=64, dy=64, dys=W, ds=None, dss=W, dx=64, dxs=W, dw=64, ws=256, size=1 << 30: \
        L.pictura_rms_norm_gradient(ref(n or q()), f, dy, dys, ds, dss, dx, dxs, dw, ws, size, None)
    sizes = [dict(dtype=3), dict(weight_dtype=1), dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=65537), dict(eps=-1.0),
             dict(eps=float("nan")), dict(eps=float("inf"))]
    operands = [dict(x=None), dict(x=66), dict(weight=None), dict(weight=66), dict(x_stride=-1)]
    for over in sizes + operands:
        assert norm(q(**over)) == codes(q(**over)) == grad(q(**over)) == pictura.EINVAL, over
    for over in (dict(residual=66), dict(residual=64, residual_stride=-1)):
        assert norm(q(**over)) == codes(q(**over)) == pictura.EINVAL, over
    for k in (dict(out=None), dict(out=66), dict(os_=W - 1), dict(sum=66), dict(sum=64, ss=W - 1), dict(f=66)):
        assert norm(**k) == pictura.EINVAL, k
    for k in (dict(kind=2), dict(c=None), dict(cs=W - 1), dict(s=None), dict(s=66), dict(sum=66)):
        assert codes(**k) == pictura.EINVAL, k
    for k in (dict(n=q(residual=64)), dict(f=None), dict(f=66), dict(dy=None), dict(dy=66), dict(dys=-1), dict(ds=66), dict(ds=64, dss=-1),
              dict(dx=None), dict(dxs=0), dict(dw=None), dict(dw=66), dict(ws=None), dict(ws=128), dict(size=8)):
        assert grad(**k) == pictura.EINVAL, k
    values = lambda c=64, cs=W, s=64, kind=0, rows=N, width=W, out=64, os_=W: \
        L.pictura_row_values(c, cs, s, kind, rows, width, out, os_, None)
    for k in (dict(c=None), dict(cs=-1), dict(s=None), dict(s=66), dict(kind=2), dict(rows=-1), dict(width=0), dict(out=None), dict(out=66),
              dict(os_=W - 1)):
        assert values(**k) == pictura.EINVAL, k
    assert norm(q(rows=0, x=None)) == codes(q(rows=0)) == values(rows=0) == pictura.OK
    out = ctypes.c_uint64()
    assert L.pictura_rms_norm_gradient_workspace(None, ctypes.addressof(out)) == pictura.EINVAL
    assert L.pictura_rms_norm_gradient_workspace(ref(q()), None) == pictura.EINVAL


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_weights_in_8_bits(dtype):
    """Codes stand for the weights to half a step of e4m3, rows of zeros and of the smallest numbers too."""
    layer = memory.MemoryLayer(32)
    w = torch.randn(64, 32, generator=torch.Generator().manual_seed(1))
    w[3], w[5], w[7] = 0, w[5] * 2.0 ** -20, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    with torch.no_grad():
        layer.project.weight.copy_(w)
    layer = layer.to(dtype)
    w = layer.project.weight.detach().double()
    codes, scales = layer.quantized()
    assert codes.shape == (64, 32) and scales.shape == (1, 64) and scales.dtype == torch.float32 and (scales > 0).all()
    values, half = codes.double() * scales.double().t(), torch.maximum(w.abs() * 2.0 ** -4, scales.double().t() * 2.0 ** -10)
    # (a row whose largest magnitude is below 1e-30 is taken for zeros; the quotient is rounded to fp32)
    held = w.abs().amax(1) >= 1e-30
    assert ((values - w).abs() <= half * (1 + 2.0 ** -20))[held].all() and (values[~held].abs() <= 1e-30).all() and (values[3] == 0).all()
