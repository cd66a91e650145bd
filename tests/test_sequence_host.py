"""The behaviour-sequence operators and AdamW refuse bad arguments before touching the GPU (runs without one)."""
import ctypes

import numpy as np
import pytest

import seq_reference as ref
from paper_2606_21101_amd import dpi

P = 0x10000   # an address that is never read: every call here ends on the host
INV, UNS, MIS, SMALL = (dpi.DPI_ERR_INVALID_ARG, dpi.DPI_ERR_UNSUPPORTED, dpi.DPI_ERR_MISALIGNED,
                        dpi.DPI_ERR_WORKSPACE_TOO_SMALL)


def embed(**kw):
    a = dict(table=P, tdt=0, rows=10, dim=8, ids=P, n=4, pad=-1, out=P, odt=0, stride=8, status=None, **{})
    a.update(kw)
    return dpi.load().dpi_embed_forward(a["table"], a["tdt"], a["rows"], a["dim"], a["ids"], a["n"], 1.0, a["pad"],
                                        a["out"], a["odt"], a["stride"], a["status"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(n=0, ids=None, out=None, table=None), dpi.DPI_OK), (dict(n=-1), INV), (dict(rows=-1), INV), (dict(dim=0), INV),
    (dict(tdt=3), INV), (dict(odt=-1), INV), (dict(stride=7), INV), (dict(ids=None), INV), (dict(table=None), INV),
    (dict(out=None), INV), (dict(dim=65537, stride=65537), UNS), (dict(rows=1 << 31), UNS), (dict(n=1 << 31), UNS),
    (dict(stride=1 << 62), UNS), (dict(table=P + 2), MIS), (dict(tdt=2, table=P + 1), MIS), (dict(out=P + 1, odt=1), MIS),
    (dict(ids=P + 2), MIS), (dict(status=P + 1), MIS)])
def test_embedding_refusals(kw, want):
    assert embed(**kw) == want


def embed_grad(**kw):
    a = dict(dout=P, ddt=0, stride=8, ids=P, n=4, grad=P, gdt=0, rows=10, dim=8, ws=P, bytes=1 << 20, status=None)
    a.update(kw)
    return dpi.load().dpi_embed_backward(a["dout"], a["ddt"], a["stride"], a["ids"], a["n"], 1.0, -1, a["grad"], a["gdt"],
                                         a["rows"], a["dim"], a["ws"], a["bytes"], a["status"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(n=0, rows=0, grad=None, dout=None, ids=None, ws=None, bytes=0), dpi.DPI_OK), (dict(n=-1), INV), (dict(dim=0), INV),
    (dict(ddt=9), INV), (dict(gdt=9), INV), (dict(stride=7), INV), (dict(dout=None), INV), (dict(ids=None), INV),
    (dict(grad=None), INV), (dict(ws=None), INV), (dict(ws=P + 8), MIS), (dict(dout=P + 2), MIS), (dict(grad=P + 2), MIS),
    (dict(ids=P + 1), MIS), (dict(bytes=16), SMALL), (dict(n=1 << 31), UNS), (dict(status=P + 2), MIS)])
def test_embedding_gradient_refusals(kw, want):
    assert embed_grad(**kw) == want


def test_embedding_workspace_query():
    assert dpi.dpi_embed_workspace_bytes(-1, 4, 4) == 0 and dpi.dpi_embed_workspace_bytes(1, 0, 4) == 0
    a, b = dpi.dpi_embed_workspace_bytes(1000, 64, 1000), dpi.dpi_embed_workspace_bytes(1000, 64, 100_000)
    assert 0 < a < b


def desc(**kw):
    a = dict(num_tokens=100, num_seqs=4, dim=8, dtype=0, max_len=0, offsets=P, x=P, gate=P, x_stride=8, gate_stride=8, h0=None)
    a.update(kw)
    return dpi.dpi_glr_desc(*[a[n] for n, _ in dpi.dpi_glr_desc._fields_])


DESC = [(dict(num_tokens=-1), INV), (dict(num_seqs=-1), INV), (dict(num_seqs=0), INV), (dict(max_len=-1), INV),
        (dict(dim=0), INV), (dict(dtype=3), INV), (dict(dim=65537, x_stride=1 << 17, gate_stride=1 << 17), UNS),
        (dict(num_tokens=1 << 31), UNS), (dict(num_seqs=(1 << 31) - 1), UNS), (dict(offsets=None), INV), (dict(offsets=P + 2), MIS),
        (dict(x=None), INV), (dict(x=P + 2), MIS), (dict(gate=None), INV), (dict(x_stride=7), INV), (dict(gate_stride=7), INV),
        (dict(h0=P + 2), MIS)]


@pytest.mark.parametrize("kw,want", DESC)
def test_recurrence_refuses_bad_descriptions(kw, want):
    d = desc(**kw)
    stride = max(8, d.dim)
    lib = dpi.load()
    assert lib.dpi_glr_forward(ctypes.byref(d), P, stride, P, P, P, 1 << 30, None, None) == want
    assert lib.dpi_glr_backward(ctypes.byref(d), P, P, stride, P, P, stride, P, stride, P, P, 1 << 30, None, None) == want


def test_recurrence_refuses_bad_operands():
    lib, d = dpi.load(), desc()

    def fwd(h=P, stride=8, last=P, entry=P, ws=P, size=1 << 30, status=None):
        return lib.dpi_glr_forward(ctypes.byref(d), h, stride, last, entry, ws, size, status, None)

    def bwd(entry=P, dh=P, ds=8, dl=P, dx=P, xs=8, dg=P, gs=8, d0=P, ws=P, size=1 << 30):
        return lib.dpi_glr_backward(ctypes.byref(d), entry, dh, ds, dl, dx, xs, dg, gs, d0, ws, size, None, None)

    assert lib.dpi_glr_forward(None, P, 8, P, P, P, 64, None, None) == INV
    assert [fwd(h=None), fwd(stride=7), fwd(ws=None), fwd(h=P + 1), fwd(last=P + 2), fwd(entry=P + 2), fwd(ws=P + 4),
            fwd(status=P + 1), fwd(size=0)] == [INV, INV, INV, MIS, MIS, MIS, MIS, MIS, SMALL]
    assert [bwd(entry=None), bwd(ds=7), bwd(dx=None), bwd(xs=7), bwd(dg=None), bwd(gs=7), bwd(dh=P + 2), bwd(dl=P + 1),
            bwd(d0=P + 3), bwd(size=0)] == [INV] * 6 + [MIS] * 3 + [SMALL]
    assert dpi.dpi_glr_entry_bytes(desc(dim=0)) == 0 == dpi.dpi_glr_workspace_bytes(desc(dtype=7))
    assert dpi.dpi_glr_entry_bytes(desc()) > 0 and dpi.dpi_glr_workspace_bytes(desc()) >= 16


def test_step_refusals():
    def step(x=P, xs=8, g=P, gs=8, dt=0, batch=4, dim=8, state=P, slots=9, which=P, h=P, hs=8, status=None):
        return dpi.load().dpi_glr_step(x, xs, g, gs, dt, batch, dim, state, slots, which, h, hs, status, None)
    assert step(batch=0) == dpi.DPI_OK
    assert [step(batch=-1), step(slots=-1), step(dim=0), step(dt=4), step(xs=7), step(gs=7), step(hs=7), step(x=None),
            step(g=None), step(h=None), step(state=None)] == [INV] * 11
    assert [step(x=P + 2), step(state=P + 2), step(which=P + 2), step(status=P + 2)] == [MIS] * 4
    assert step(slots=1 << 31) == UNS


def adam_tensor(**kw):
    a = dict(param=P, master=None, m=P, v=P, m_scale=None, v_scale=None, count=10, param_dtype=0, grad_dtype=0)
    a.update(kw)
    return dpi.dpi_adamw_tensor(*[a[n] for n, _ in dpi.dpi_adamw_tensor._fields_])


@pytest.mark.parametrize("kw,bits,want", [
    (dict(count=-1), 32, INV), (dict(param=None), 32, INV), (dict(m=None), 32, INV), (dict(v=None), 32, INV),
    (dict(param_dtype=3), 32, INV), (dict(grad_dtype=-1), 32, INV), (dict(), 16, INV), (dict(), 8, INV),
    (dict(param=P + 2), 32, MIS), (dict(m=P + 1), 32, MIS), (dict(master=P + 2), 32, MIS), (dict(count=1 << 43), 32, UNS),
    (dict(m_scale=P + 2, v_scale=P), 8, MIS)])
def test_adamw_refuses_bad_tensors(kw, bits, want):
    lib, out = dpi.load(), ctypes.c_void_p()
    arr = (dpi.dpi_adamw_tensor * 1)(adam_tensor(**kw))
    assert lib.dpi_adamw_create(arr, 1, bits, P, 1 << 30, ctypes.byref(out)) == want
    assert lib.dpi_adamw_workspace_bytes(arr, 1, bits) == 0 and not out.value


def test_adamw_refuses_bad_calls():
    lib, out = dpi.load(), ctypes.c_void_p()
    arr = (dpi.dpi_adamw_tensor * 1)(adam_tensor())
    assert lib.dpi_adamw_create(arr, 0, 32, P, 1 << 20, ctypes.byref(out)) == INV
    assert lib.dpi_adamw_create(None, 1, 32, P, 1 << 20, ctypes.byref(out)) == INV
    assert lib.dpi_adamw_create(arr, 1, 32, P, 1 << 20, None) == INV
    assert lib.dpi_adamw_create(arr, 1, 32, None, 1 << 20, ctypes.byref(out)) == INV
    assert lib.dpi_adamw_create(arr, 1, 32, P + 4, 1 << 20, ctypes.byref(out)) == MIS
    assert lib.dpi_adamw_create(arr, 1, 32, P, 8, ctypes.byref(out)) == SMALL
    assert lib.dpi_adamw_step(None, None, None, None) == INV
    lib.dpi_adamw_destroy(None)


def test_older_entry_points_still_refuse_bf16():
    lib = dpi.load()
    assert lib.dpi_fm_second_order(P, dpi.DPI_BF16, 2, 3, 4, 12, P, None) == INV


# --------------------------------------------------------- the plain forms pin themselves
def test_reference_gradient_against_differences():
    """The 64-bit gradients of the recurrence against central differences of its 64-bit forward form."""
    rng = np.random.default_rng(0)
    off = np.array([0, 3, 3, 10, 11])
    z = [rng.standard_normal(s) for s in ((11, 2), (11, 2), (4, 2))]
    dh, dl = rng.standard_normal((11, 2)), rng.standard_normal((4, 2))

    def loss(x, g, h0):
        h, last, _ = ref.recur(x, g, off, h0)
        return (h * dh).sum() + (last * dl).sum()

    grads = ref.recur_grad(z[0], z[1], off, dh, dl, z[2])
    for k in range(3):
        for at in np.ndindex(z[k].shape):
            d = [np.zeros_like(a) for a in z]
            d[k][at] = 1e-6
            slope = (loss(*[a + b for a, b in zip(z, d)]) - loss(*[a - b for a, b in zip(z, d)])) / 2e-6
            assert abs(slope - grads[k][at]) < 1e-8, (k, at)


def test_reference_codes():
    """Every code decodes to what rounding its own value gives back; neighbours are chosen with the right frequency."""
    codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    vals = ref.decode(codes)
    assert vals.max() == 448 and vals[1] == 2.0 ** -9
    block = np.zeros(256, np.float32)
    block[: len(codes)] = vals
    back, scale = ref.store8(block, np.zeros(256, np.int64), False)
    assert scale[0] == 1 and np.array_equal(ref.decode(back[: len(codes)]), vals)
    x = np.full(256 * 400, 0.3, np.float32)
    x[::256] = 448
    rm, _ = ref.random_bits(len(x), 1, 2, 3)
    back, scale = ref.store8(x, rm, False)
    got = ref.decode(back)[np.arange(len(x)) % 256 != 0]
    assert set(np.unique(got)) == {0.28125, 0.3125} and abs(got.mean() - 0.3) < 5 * 0.016 / 320
