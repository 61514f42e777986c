"""What the calls of a training step around the sampled layers refuse, on the host, before anything is enqueued.  Needs no GPU."""
import ctypes as C
import math

import pytest
import torch

import plain_training as plain
from paper_2101_07706_amd import csgs

Z, P = C.c_void_p(0), C.c_void_p(4096)     # null; an aligned address that the host never dereferences


def test_struct_layouts_match_the_header():
    assert C.sizeof(csgs.AdamwTensor) == 144 and csgs.AdamwTensor.rows.offset == 72 and csgs.AdamwTensor.weight_decay.offset == 132
    assert C.sizeof(csgs.AdamwArgs) == 88 and csgs.AdamwArgs.lr.offset == 24 and csgs.AdamwArgs.clip.offset == 48 and csgs.AdamwArgs.norm.offset == 72
    assert C.sizeof(csgs.AdamwList) == 32 and csgs.AdamwList.n.offset == 24


def adam(**kw):
    t = dict(p=4096, copy=0, g=8192, m=12288, v=16384, m_exp=0, v_exp=0, ids=0, n_dev=0, rows=3, cols=5, n=3, ldp=5, ldcopy=0, ldg=5, p_dtype=0, g_dtype=0, state=0,
             weight_decay=0.0, lr_scale=1.0, reserved=0)
    t.update(kw)
    return csgs.AdamwTensor(*[t[k] for k, _ in csgs.AdamwTensor._fields_])


def test_adamw_lists():
    L = csgs.lib()
    size = L.csgs_adamw_list_bytes
    one = (csgs.AdamwTensor * 1)(adam())
    need = size(one, 1)
    assert need > 0 and need % 256 == 0 and size(None, 1) == 0 and size(one, 0) == 0 and size(one, (1 << 20) + 1) == 0
    assert size((csgs.AdamwTensor * 1)(adam(state=1, m_exp=4100, v_exp=4200)), 1) > 0
    bads = [(dict(p=0), "EINVAL"), (dict(g=0), "EINVAL"), (dict(m=0), "EINVAL"), (dict(v=0), "EINVAL"), (dict(rows=0, n=0), "EINVAL"), (dict(cols=0), "EINVAL"),
            (dict(n=2), "EINVAL"), (dict(n=0, ids=4096), "EINVAL"), (dict(ldp=4), "EINVAL"), (dict(ldg=4), "EINVAL"), (dict(copy=4100, ldcopy=4), "EINVAL"),
            (dict(copy=4096, ldcopy=5), "EINVAL"), (dict(m=16384), "EINVAL"), (dict(m=4096), "EINVAL"), (dict(v=4096), "EINVAL"), (dict(g=4096), "EINVAL"),
            (dict(m_exp=4096), "EINVAL"), (dict(state=1), "EINVAL"), (dict(state=1, m_exp=4096), "EINVAL"), (dict(state=1, m_exp=4096, v_exp=4096), "EINVAL"),
            (dict(weight_decay=-1.0), "EINVAL"), (dict(weight_decay=math.nan), "EINVAL"), (dict(lr_scale=-1.0), "EINVAL"), (dict(lr_scale=math.nan), "EINVAL"),
            (dict(p_dtype=2), "EUNSUPPORTED"), (dict(g_dtype=-1), "EUNSUPPORTED"), (dict(state=2), "EUNSUPPORTED"), (dict(rows=1 << 40, n=1 << 40), "EUNSUPPORTED"),
            (dict(ids=4096, rows=1 << 31), "EUNSUPPORTED"), (dict(ids=4096, n=1 << 31), "EUNSUPPORTED")]
    for bad, code in bads:
        ts = (csgs.AdamwTensor * 1)(adam(**bad))
        assert size(ts, 1) == 0, bad
        l = csgs.AdamwList(4096, 1 << 40, 0, 0, 0)
        assert L.csgs_adamw_list_init(C.byref(l), ts, 1, Z) == getattr(csgs, code) and l.ready == 0, bad
    for l, code in ((csgs.AdamwList(0, need, 0, 0, 0), "EINVAL"), (csgs.AdamwList(4100, need, 0, 0, 0), "EINVAL"), (csgs.AdamwList(4096, need - 1, 0, 0, 0), "EWORKSPACE")):
        assert L.csgs_adamw_list_init(C.byref(l), one, 1, Z) == getattr(csgs, code)
    assert L.csgs_adamw_list_init(None, one, 1, Z) == csgs.EINVAL


def test_adamw_step():
    L = csgs.lib()
    ready, raw = csgs.AdamwList(4096, 1 << 20, 1, 1, 1), csgs.AdamwList(4096, 1 << 20, 0, 0, 0)
    grads = csgs.GradList(4096, 1 << 20, 1, 1, 1)

    def call(l=ready, **kw):
        a = dict(beta1=0.9, beta2=0.999, eps=1e-8, lr=0.1, max_norm=1.0, lr_dev=0, step=4096, clip=None, total=0, kind=0, reserved=0, norm=0, status=0)
        a.update(kw)
        if a["clip"] is not None:
            a["clip"] = C.pointer(a["clip"])
        return L.csgs_adamw(None if l is None else C.byref(l), C.byref(csgs.AdamwArgs(*[a[k] for k, _ in csgs.AdamwArgs._fields_])), Z)
    assert call(l=None) == csgs.EINVAL and call(l=raw) == csgs.EINVAL and L.csgs_adamw(C.byref(ready), None, Z) == csgs.EINVAL
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta1=math.nan), dict(beta2=math.nan), dict(eps=-1.0), dict(eps=math.nan), dict(lr=-1.0),
                dict(lr=math.nan), dict(norm=4096), dict(clip=grads, total=4096), dict(clip=grads, max_norm=0.0), dict(total=4096, max_norm=math.nan),
                dict(clip=grads, kind=3), dict(total=4096, kind=-1), dict(clip=csgs.GradList(4096, 1, 0, 0, 0))):
        assert call(**bad) == csgs.EINVAL, bad


def test_states():
    L = csgs.lib()

    def read(codes=P, exps=P, which=0, rows=3, cols=5, values=P, ld=5):
        return L.csgs_state_read(codes, exps, which, rows, cols, values, ld, Z)

    def write(codes=P, exps=P, which=0, rows=3, cols=5, values=P, ld=5):
        return L.csgs_state_write(values, ld, which, rows, cols, codes, exps, Z)
    for f in (read, write):
        for bad in (dict(codes=Z), dict(exps=Z), dict(values=Z), dict(which=2), dict(which=-1), dict(rows=0), dict(cols=0), dict(ld=4)):
            assert f(**bad) == csgs.EINVAL, bad
        assert f(rows=1 << 40) == csgs.EUNSUPPORTED


def test_binding_refuses_what_it_cannot_describe():
    """Wrong types, strides and sizes end in Python (the tensors are CPU tensors: nothing here reaches a kernel)."""
    p, ids, step = torch.zeros(4, 6), torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    f32, b8 = csgs.adamw_states(p), csgs.adamw_states(p, 8)
    entry = csgs.adamw_entry
    shared = torch.zeros(4, 6)
    for bad in (lambda: entry(p.half(), p, **f32), lambda: entry(p, p.half(), **f32), lambda: entry(p, torch.zeros(4, 5), **f32), lambda: entry(p, torch.zeros(3, 6), **f32),
                lambda: entry(p, torch.zeros(3, 6), **f32, ids=ids), lambda: entry(p, p, f32["m"], b8["v"]), lambda: entry(p, p, b8["m"], b8["v"]),
                lambda: entry(p, p, **f32, m_exp=b8["m_exp"], v_exp=b8["v_exp"]), lambda: entry(p, p, **{**b8, "m_exp": b8["m_exp"][:3]}),
                lambda: entry(p, p, **f32, copy=torch.zeros(4, 6)), lambda: entry(p, p, torch.zeros(4, 7)[:, :6], f32["v"]), lambda: entry(p, p, **f32, ids=ids.long()),
                lambda: entry(p.t().contiguous().t(), p, **f32), lambda: csgs.adamw_states(p, 16), lambda: csgs.make_adamw_list([]),
                lambda: csgs.make_adamw_list([entry(shared, p, **f32), entry(shared, p, **csgs.adamw_states(p))]),
                lambda: csgs.make_adamw_list([entry(p, shared, **f32), entry(torch.zeros(4, 6), shared, **f32)]),
                lambda: csgs.csgs_adamw(csgs.AdamwList(), 0.1, step.long()), lambda: csgs.csgs_adamw(csgs.AdamwList(), 0.1, step, total=torch.zeros(1)),
                lambda: csgs.csgs_state_read(b8["m"], b8["m_exp"], 0, torch.zeros(4, 5)), lambda: csgs.csgs_state_write(p.double(), 0, b8["m"], b8["m_exp"]),
                lambda: csgs.csgs_state_read(b8["m"], b8["m_exp"][:2], 0, p)):
        with pytest.raises((AssertionError, TypeError)):
            bad()


def test_plain_codes():
    """The tables of the 8-bit states, against the ways to write them down."""
    e4m3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    first = plain.first_values()
    assert torch.equal(first.isnan(), e4m3.isnan()) and torch.equal(first[~first.isnan()], e4m3[~e4m3.isnan()])
    second = plain.second_values()
    assert second[0] == 0 and second[1] == 1.25 * 2.0 ** -31 and second[255] == 2 and second[247] == 1 and bool((second[1:] > second[:-1]).all())
    # a value is its own code's, and what lies between two goes to the nearer
    for second_state, table in ((False, first[:120]), (True, second)):
        x = (table / (256 if not second_state else 1)).float().reshape(1, -1)[:, :250]
        top = float(x.max())
        codes, exps = plain.encode(x, second_state)
        assert torch.equal(plain.decode(codes, exps, second_state).float(), x) or second_state
        back = plain.decode(codes, exps, second_state)
        assert float((back - x.double()).abs().max()) <= 2.0 ** -16 * top
