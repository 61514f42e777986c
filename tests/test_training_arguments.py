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


@pytest.mark.parametrize("theirs", ["p", "copy", "m", "v", "m_exp", "v_exp"])
def test_what_a_step_writes_belongs_to_one_tensor(theirs):
    L = csgs.lib()
    one = dict(p=1 << 20, copy=2 << 20, ldcopy=5, m=3 << 20, v=4 << 20, m_exp=5 << 20, v_exp=6 << 20, state=1)
    other = {k: v if k in ("ldcopy", "state") else v + (8 << 20) for k, v in one.items()}
    pair = lambda **kw: (csgs.AdamwTensor * 2)(adam(**one), adam(**{**other, **kw}))  # noqa: E731
    assert L.csgs_adamw_list_bytes(pair(), 2) > 0
    for mine in ("p", "copy", "m", "v", "m_exp", "v_exp"):
        ts = pair(**{theirs: one[mine]})
        l = csgs.AdamwList(4096, 1 << 40, 0, 0, 0)
        assert L.csgs_adamw_list_bytes(ts, 2) == 0 and L.csgs_adamw_list_init(C.byref(l), ts, 2, Z) == csgs.EINVAL and l.ready == 0


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


def linear(**kw):
    p = dict(M=4, K=6, N=5, act=0, M_dev=0, a=4096, w=8192, bias=12288, r=16384, lda=6, ldw=5, ldr=5, dtype=0, y_dtype=0, alpha=1.0, beta=1.0)
    p.update(kw)
    return csgs.LinearArgs(*[p[k] for k, _ in csgs.LinearArgs._fields_])


def gated(**kw):
    p = dict(M=4, K=6, N=5, act=3, M_dev=0, x=4096, wg=8192, wu=12288, bg=16384, bu=16384, ldx=6, ldwg=5, ldwu=5, dtype=0, reserved=0)
    p.update(kw)
    return csgs.GatedArgs(*[p[k] for k, _ in csgs.GatedArgs._fields_])


def test_product_struct_layouts_match_the_header():
    assert C.sizeof(csgs.LinearArgs) == 96 and csgs.LinearArgs.lda.offset == 56 and csgs.LinearArgs.alpha.offset == 88
    assert C.sizeof(csgs.GatedArgs) == 96 and csgs.GatedArgs.ldx.offset == 64 and csgs.GatedArgs.dtype.offset == 88
    assert csgs._linear_layout.size == 96 and csgs._gated_layout.size == 96


BAD_LINEAR = [(dict(M=0), "EINVAL"), (dict(K=0), "EINVAL"), (dict(N=-1), "EINVAL"), (dict(a=0), "EINVAL"), (dict(w=0), "EINVAL"), (dict(lda=5), "EINVAL"), (dict(ldw=4), "EINVAL"),
              (dict(ldr=4), "EINVAL"), (dict(act=5), "EINVAL"), (dict(act=-1), "EINVAL"), (dict(dtype=0, y_dtype=1), "EUNSUPPORTED"), (dict(dtype=2, y_dtype=2), "EUNSUPPORTED")]
BAD_GATED = [(dict(M=0), "EINVAL"), (dict(K=-2), "EINVAL"), (dict(N=0), "EINVAL"), (dict(x=0), "EINVAL"), (dict(wg=0), "EINVAL"), (dict(wu=0), "EINVAL"), (dict(ldx=5), "EINVAL"),
             (dict(ldwg=4), "EINVAL"), (dict(ldwu=4), "EINVAL"), (dict(act=5), "EINVAL"), (dict(act=-1), "EINVAL"), (dict(dtype=2), "EUNSUPPORTED")]
ptr = C.c_void_p


def test_linear():
    L = csgs.lib()

    def call(p, y=ptr(1 << 20), ldy=5):
        return L.csgs_linear(C.byref(p), y, ldy, Z)
    assert L.csgs_linear(None, P, 5, Z) == csgs.EINVAL
    for bad, code in BAD_LINEAR:
        assert call(linear(**bad)) == getattr(csgs, code), bad
    for bad in (dict(y=Z), dict(ldy=4), dict(y=ptr(4096)), dict(y=ptr(8192)), dict(y=ptr(16384), ldy=6)):
        assert call(linear(), **bad) == csgs.EINVAL, bad


def test_linear_gradient():
    L = csgs.lib()
    need = csgs.csgs_linear_grad_scratch_bytes(4, 6, 5, csgs.F32)
    full = dict(dy=ptr(1 << 20), lddy=5, da=ptr(2 << 20), ldda=6, dw=ptr(3 << 20), lddw=5, db=ptr(4 << 20), dr=ptr(5 << 20), lddr=5, scratch=ptr(6 << 20), nbytes=need)

    def call(p, **kw):
        a = {**full, **kw}
        return L.csgs_linear_grad(None if p is None else C.byref(p), a["dy"], a["lddy"], a["da"], a["ldda"], a["dw"], a["lddw"], a["db"], a["dr"], a["lddr"], a["scratch"], a["nbytes"], Z)
    assert call(None) == csgs.EINVAL
    for bad, code in BAD_LINEAR:
        assert call(linear(**bad)) == getattr(csgs, code), bad
    for bad in (dict(dy=Z), dict(lddy=4), dict(ldda=5), dict(lddw=4), dict(lddr=4), dict(da=Z, dw=Z, db=Z, dr=Z), dict(dr=ptr(1 << 20), lddr=6), dict(da=ptr(1 << 20)),
                dict(dw=ptr(1 << 20)), dict(scratch=Z), dict(scratch=ptr(4224))):
        assert call(linear(), **bad) == csgs.EINVAL, bad
    assert call(linear(bias=0)) == csgs.EINVAL and call(linear(r=0)) == csgs.EINVAL
    assert call(linear(), nbytes=need - 1) == csgs.EWORKSPACE


def test_gated():
    L = csgs.lib()

    def call(p, h=ptr(1 << 20), ldh=5):
        return L.csgs_gated(C.byref(p), h, ldh, Z)
    assert L.csgs_gated(None, P, 5, Z) == csgs.EINVAL
    for bad, code in BAD_GATED:
        assert call(gated(**bad)) == getattr(csgs, code), bad
    for bad in (dict(h=Z), dict(ldh=4), dict(h=ptr(4096)), dict(h=ptr(8192)), dict(h=ptr(12288))):
        assert call(gated(), **bad) == csgs.EINVAL, bad


def test_gated_gradient():
    L = csgs.lib()
    need = csgs.csgs_gated_grad_scratch_bytes(4, 6, 5, csgs.F32)
    full = dict(dh=ptr(1 << 20), lddh=5, dx=ptr(2 << 20), lddx=6, dwg=ptr(3 << 20), lddwg=5, dwu=ptr(4 << 20), lddwu=5, dbg=ptr(5 << 20), dbu=ptr(6 << 20), scratch=ptr(7 << 20), nbytes=need)

    def call(p, **kw):
        a = {**full, **kw}
        return L.csgs_gated_grad(None if p is None else C.byref(p), a["dh"], a["lddh"], a["dx"], a["lddx"], a["dwg"], a["lddwg"], a["dwu"], a["lddwu"], a["dbg"], a["dbu"], a["scratch"],
                                 a["nbytes"], Z)
    assert call(None) == csgs.EINVAL
    for bad, code in BAD_GATED:
        assert call(gated(**bad)) == getattr(csgs, code), bad
    for bad in (dict(dh=Z), dict(lddh=4), dict(lddx=5), dict(lddwg=4), dict(lddwu=4), dict(dx=Z, dwg=Z, dwu=Z, dbg=Z, dbu=Z), dict(dx=ptr(1 << 20)), dict(dwg=ptr(1 << 20)),
                dict(dwu=ptr(1 << 20)), dict(scratch=Z), dict(scratch=ptr(4224))):
        assert call(gated(), **bad) == csgs.EINVAL, bad
    assert call(gated(bg=0)) == csgs.EINVAL and call(gated(bu=0)) == csgs.EINVAL
    assert call(gated(), nbytes=need - 1) == csgs.EWORKSPACE


def test_products_whose_outputs_lie_on_inputs_or_each_other():
    L = csgs.lib()
    inputs, outputs = [4096, 8192, 12288, 1 << 20], [2 << 20, 3 << 20, 4 << 20, 5 << 20]

    def linear_grad(out):
        p = linear(r=24576)
        return L.csgs_linear_grad(C.byref(p), ptr(1 << 20), 5, ptr(out[0]), 6, ptr(out[1]), 5, ptr(out[2]), ptr(out[3]), 5, ptr(6 << 20), 1, Z)

    def gated_grad(out):
        p = gated(bu=20480)
        return L.csgs_gated_grad(C.byref(p), ptr(1 << 20), 5, ptr(out[0]), 6, ptr(out[1]), 5, ptr(out[2]), 5, ptr(out[3]), ptr(out[4]), ptr(6 << 20), 1, Z)
    for call, ins, outs in ((linear_grad, inputs, outputs), (gated_grad, inputs + [16384, 20480], outputs + [7 << 20])):
        assert call(outs) == csgs.EWORKSPACE        # (nothing else is wrong with it)
        for i in range(len(outs)):
            for other in ins + outs[:i]:
                ok = call is linear_grad and i == 3 and other == 1 << 20       # (dr may be dy)
                assert call([*outs[:i], other, *outs[i + 1:]]) == (csgs.EWORKSPACE if ok else csgs.EINVAL), (call, i, other)
    assert L.csgs_linear(C.byref(linear()), ptr(12288), 5, Z) == csgs.EINVAL and L.csgs_gated(C.byref(gated()), ptr(16384), 5, Z) == csgs.EINVAL


def test_products_of_more_blocks_than_a_launch_has():
    L = csgs.lib()
    big = 2 ** 31 - 1
    assert L.csgs_linear(C.byref(linear(M=big, N=129, ldw=129, ldr=129)), ptr(1 << 20), 129, Z) == csgs.EUNSUPPORTED
    assert L.csgs_gated(C.byref(gated(M=big, N=1000, ldwg=1000, ldwu=1000)), ptr(1 << 20), 1000, Z) == csgs.EUNSUPPORTED
    p = linear(M=big, N=1, ldw=1, ldr=1, K=1 << 20, lda=1 << 20)
    assert L.csgs_linear_grad(C.byref(p), ptr(1 << 20), 1, ptr(2 << 20), 1 << 20, Z, 1, Z, Z, 1, ptr(6 << 20), 1 << 62, Z) == csgs.EUNSUPPORTED


@pytest.mark.parametrize("size", [csgs.csgs_linear_grad_scratch_bytes, csgs.csgs_gated_grad_scratch_bytes])
def test_scratch_for_the_largest_product_serves_smaller_ones(size):
    assert size(0, 1, 1, 0) == 0 and size(1, 0, 1, 0) == 0 and size(1, 1, 0, 0) == 0 and size(1, 1, 1, 2) == 0 and size(-1, 1, 1, 0) == 0
    Ms, Ks, Ns = [1, 2, 63, 64, 65, 511, 512, 513, 8192, 8193, 65_536, 131_072, 1 << 24], [1, 7, 64, 512, 513, 1024, 4096, 1 << 20], [1, 5, 64, 512, 513, 1111, 4096, 1 << 20]
    for dtype in (csgs.F32, csgs.BF16):
        for M in Ms:
            for K in Ks:
                row = [size(M, K, N, dtype) for N in Ns]
                assert all(0 < a <= b for a, b in zip(row, row[1:]))
        for M in Ms:
            for N in Ns:
                row = [size(M, K, N, dtype) for K in Ks]
                assert all(a <= b for a, b in zip(row, row[1:]))
        for K in Ks:
            for N in Ns:
                row = [size(M, K, N, dtype) for M in Ms]
                assert all(a <= b for a, b in zip(row, row[1:]))


def test_binding_refuses_products_that_it_cannot_describe():
    a, w, y, b = torch.zeros(4, 6), torch.zeros(6, 5), torch.zeros(4, 5), torch.zeros(5)
    s = torch.zeros(64)
    for bad in (lambda: csgs.csgs_linear(a.half(), w.half(), y), lambda: csgs.csgs_linear(a, w.bfloat16(), y), lambda: csgs.csgs_linear(a, torch.zeros(7, 5), y),
                lambda: csgs.csgs_linear(a, w, torch.zeros(4, 6)), lambda: csgs.csgs_linear(a, w, y, bias=torch.zeros(6)), lambda: csgs.csgs_linear(a, w, y, bias=b.double()),
                lambda: csgs.csgs_linear(a, w, y, r=y.bfloat16()), lambda: csgs.csgs_linear(a, w, y, r=torch.zeros(3, 5)), lambda: csgs.csgs_linear(a.t().contiguous().t(), w, y),
                lambda: csgs.csgs_linear(a, w, y, M_dev=torch.zeros(1)), lambda: csgs.csgs_linear_grad(a, w, y, torch.zeros(4, 5), None, None, None, s),
                lambda: csgs.csgs_linear_grad(a, w, y, None, w.bfloat16(), None, None, s), lambda: csgs.csgs_linear_grad(a, w, y, None, w, torch.zeros(4), None, s),
                lambda: csgs.csgs_linear_grad(a, w, y, None, w, None, None, torch.zeros(8, 8)[:, :4]), lambda: csgs.csgs_gated(a, w, torch.zeros(6, 4), y),
                lambda: csgs.csgs_gated(a, w, w, y.bfloat16()), lambda: csgs.csgs_gated(a, w, w, y, bg=torch.zeros(4)), lambda: csgs.csgs_gated(a.double(), w.double(), w.double(), y),
                lambda: csgs.csgs_gated_grad(a, w, w, y, None, w, torch.zeros(5, 6), None, None, s), lambda: csgs.csgs_gated_grad(a, w, w, torch.zeros(4, 6), a, w, w, None, None, s)):
        with pytest.raises((AssertionError, TypeError)):
            bad()
