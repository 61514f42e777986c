"""What the table's, residual's and clipping calls refuse, on the host, before anything is enqueued.  Needs no GPU."""
import ctypes as C

import pytest
import torch

from paper_2101_07706_amd import csgs

Z, P = C.c_void_p(0), C.c_void_p(4096)     # null; an aligned address that the host never dereferences


def test_struct_layouts_match_the_header():
    assert C.sizeof(csgs.Residual) == 8 + 8 * 4 + 8 * 3 + 8 * 4 + 4 * 8 and csgs.Residual.post_w.offset == 64 and csgs.Residual.eps.offset == 116
    assert C.sizeof(csgs.GradTensor) == 64 and csgs.GradTensor.rows_dev.offset == 48 and csgs.GradTensor.dtype.offset == 56
    assert C.sizeof(csgs.GradList) == 32 and csgs.GradList.n.offset == 24


def test_lookup():
    def call(T=P, ld=8, rows=10, F=8, dtype=0, ids=P, n=5, scale=1.0, out=P, ldo=8, out_dtype=0):
        return csgs.lib().csgs_embed(T, ld, rows, F, dtype, ids, n, Z, scale, out, ldo, out_dtype, Z)
    for bad in (dict(T=Z), dict(ids=Z), dict(out=Z), dict(ld=7), dict(ldo=7), dict(rows=0), dict(F=0), dict(n=0), dict(n=-1)):
        assert call(**bad) == csgs.EINVAL, bad
    for bad in (dict(dtype=2), dict(out_dtype=-1), dict(n=1 << 31)):
        assert call(**bad) == csgs.EUNSUPPORTED, bad


def test_table_gradient():
    size = csgs.csgs_embed_grad_scratch_bytes
    assert size(0, 5, 5) == 0 and size(5, 0, 5) == 0 and size(5, 5, 0) == 0 and size(1 << 31, 5, 5) == 0 and size(5, 1 << 31, 5) == 0
    assert 0 < size(10, 1000, 8) <= size(100_000, 1000, 8) and size(10, 1000, 8) % 256 == 0
    need = size(5, 10, 8)

    def dense(ids=P, n=5, G=P, ldg=8, F=8, gt=0, acc=0, d=P, ldd=8, rows=10, dt=0, scratch=P, nbytes=need):
        return csgs.lib().csgs_embed_grad(ids, n, Z, G, ldg, F, gt, 1.0, acc, d, ldd, rows, dt, scratch, nbytes, Z)

    def rows(uniq=P, n_uniq=P, ids=P, n=5, G=P, ldg=8, F=8, gt=0, d=P, ldd=8, rows=10, dt=0, scratch=P, nbytes=need):
        return csgs.lib().csgs_embed_grad_rows(ids, n, Z, G, ldg, F, gt, 1.0, rows, uniq, n_uniq, d, ldd, dt, scratch, nbytes, Z)
    shared = [(dict(ids=Z), "EINVAL"), (dict(n=0), "EINVAL"), (dict(G=Z), "EINVAL"), (dict(ldg=7), "EINVAL"), (dict(F=0), "EINVAL"), (dict(d=Z), "EINVAL"),
              (dict(ldd=7), "EINVAL"), (dict(rows=0), "EINVAL"), (dict(scratch=Z), "EINVAL"), (dict(scratch=C.c_void_p(4100)), "EINVAL"),
              (dict(nbytes=need - 1), "EWORKSPACE"), (dict(gt=5), "EUNSUPPORTED"), (dict(dt=5), "EUNSUPPORTED"), (dict(n=1 << 31), "EUNSUPPORTED"),
              (dict(rows=1 << 31), "EUNSUPPORTED")]
    for f in (dense, rows):
        for bad, code in shared:
            assert f(**bad) == getattr(csgs, code), (f, bad)
    assert dense(acc=2) == csgs.EINVAL and rows(uniq=Z) == csgs.EINVAL and rows(n_uniq=Z) == csgs.EINVAL


def residual(**kw):
    r = dict(M=4, F=8, M_dev=0, x=4096, h=4096, gate=4096, ldx=8, ldh=8, ldg=8, post_w=4096, post_b=0, pre_w=0, pre_b=0, x_dtype=0, h_dtype=0, post=1, pre=1,
             gate_act=1, eps=1e-5, alpha=1.0, beta=1.0)
    r.update(kw)
    return csgs.Residual(*[r[k] for k, _ in csgs.Residual._fields_])


BAD_RESIDUALS = [(dict(M=0), "EINVAL"), (dict(F=0), "EINVAL"), (dict(x=0, h=0, gate=0), "EINVAL"), (dict(ldx=7), "EINVAL"), (dict(ldh=7), "EINVAL"),
                 (dict(ldg=7), "EINVAL"), (dict(h=0), "EINVAL"), (dict(eps=-1.0), "EINVAL"), (dict(eps=float("nan")), "EINVAL"), (dict(post=3), "EINVAL"),
                 (dict(post=-1), "EINVAL"), (dict(pre=3), "EINVAL"), (dict(gate_act=3), "EINVAL"), (dict(x_dtype=1, h_dtype=0), "EUNSUPPORTED"),
                 (dict(x_dtype=2, h_dtype=2), "EUNSUPPORTED"), (dict(h_dtype=7), "EUNSUPPORTED")]


def test_norm_residual():
    L = csgs.lib()

    def call(r, y=P, ldy=8, u=P, ldu=8):
        return L.csgs_norm_residual(C.byref(r), y, ldy, u, ldu, Z)
    assert L.csgs_norm_residual(None, P, 8, P, 8, Z) == csgs.EINVAL
    for bad, code in BAD_RESIDUALS:
        assert call(residual(**bad)) == getattr(csgs, code), bad
    for bad in (dict(y=Z, u=Z), dict(ldy=7), dict(ldu=7)):
        assert call(residual(), **bad) == csgs.EINVAL, bad
    assert call(residual(pre=0)) == csgs.EINVAL          # u without a norm


def test_norm_residual_gradient():
    L = csgs.lib()
    size = csgs.csgs_norm_residual_grad_scratch_bytes
    assert size(0, 8) == 0 and size(8, 0) == 0 and 0 < size(1, 1) <= size(1, 4096) <= size(100_000, 4096) and size(3, 5) % 256 == 0
    need = size(4, 8)

    def call(r, dy=P, lddy=8, du=P, lddu=8, dx=P, lddx=8, dh=P, lddh=8, dg=P, lddg=8, v=(P, P, P, P), scratch=P, nbytes=need):
        return L.csgs_norm_residual_grad(C.byref(r), dy, lddy, du, lddu, dx, lddx, dh, lddh, dg, lddg, *v, scratch, nbytes, Z)
    for bad, code in BAD_RESIDUALS:
        assert call(residual(**bad)) == getattr(csgs, code), bad
    for bad in (dict(dy=Z, du=Z), dict(lddy=7), dict(lddu=7), dict(lddx=7), dict(lddh=7), dict(lddg=7), dict(scratch=Z), dict(scratch=C.c_void_p(4352 - 128)),
                dict(du=Z)):                              # dpre_w without du
        assert call(residual(), **bad) == csgs.EINVAL, bad
    assert call(residual(), nbytes=need - 1) == csgs.EWORKSPACE
    # outputs whose inputs are absent
    assert call(residual(x=0)) == csgs.EINVAL and call(residual(h=0, gate=0)) == csgs.EINVAL and call(residual(gate=0)) == csgs.EINVAL
    assert call(residual(post=0)) == csgs.EINVAL and call(residual(pre=0)) == csgs.EINVAL


def tensor(**kw):
    t = dict(g=4096, out=8192, rows=3, cols=5, ldg=5, ldo=5, rows_dev=0, dtype=0, reserved=0)
    t.update(kw)
    return csgs.GradTensor(*[t[k] for k, _ in csgs.GradTensor._fields_])


def test_gradient_lists():
    L = csgs.lib()
    size = L.csgs_grad_list_bytes
    one = (csgs.GradTensor * 1)(tensor())
    need = size(one, 1)
    assert need > 0 and need % 256 == 0 and size(None, 1) == 0 and size(one, 0) == 0 and size(one, (1 << 20) + 1) == 0
    bads = [(dict(g=0), "EINVAL"), (dict(rows=0), "EINVAL"), (dict(cols=0), "EINVAL"), (dict(ldg=4), "EINVAL"), (dict(ldo=4), "EINVAL"),
            (dict(out=4096, ldo=6), "EINVAL"), (dict(dtype=2), "EUNSUPPORTED"), (dict(rows=1 << 40, cols=5, ldg=5), "EUNSUPPORTED")]
    for bad, code in bads:
        ts = (csgs.GradTensor * 1)(tensor(**bad))
        assert size(ts, 1) == 0, bad
        l = csgs.GradList(4096, 1 << 30, 0, 0, 0)
        assert L.csgs_grad_list_init(C.byref(l), ts, 1, Z) == getattr(csgs, code) and l.ready == 0, bad
    for l, code in ((csgs.GradList(0, need, 0, 0, 0), "EINVAL"), (csgs.GradList(4100, need, 0, 0, 0), "EINVAL"), (csgs.GradList(4096, need - 1, 0, 0, 0), "EWORKSPACE")):
        assert L.csgs_grad_list_init(C.byref(l), one, 1, Z) == getattr(csgs, code)
    assert L.csgs_grad_list_init(None, one, 1, Z) == csgs.EINVAL
    # lists that no init has filled, kinds, limits
    raw, ready = csgs.GradList(4096, need, 0, 0, 0), csgs.GradList(4096, need, 1, 1, 1)
    assert L.csgs_grad_clip(C.byref(raw), 0, 1.0, P, P, Z) == csgs.EINVAL and L.csgs_grad_norm(C.byref(raw), 0, P, Z) == csgs.EINVAL
    assert L.csgs_grad_clip(None, 0, 1.0, P, P, Z) == csgs.EINVAL
    for kind, limit in ((3, 1.0), (-1, 1.0), (0, 0.0), (0, -1.0), (0, float("nan"))):
        assert L.csgs_grad_clip(C.byref(ready), kind, limit, P, P, Z) == csgs.EINVAL
        assert L.csgs_grad_scale(C.byref(ready), kind, P, limit, P, P, Z) == csgs.EINVAL
    assert L.csgs_grad_norm(C.byref(ready), 0, Z, Z) == csgs.EINVAL and L.csgs_grad_scale(C.byref(ready), 0, Z, 1.0, P, P, Z) == csgs.EINVAL


def test_binding_refuses_what_it_cannot_describe():
    """Wrong types, strides and sizes end in Python (the tensors are CPU tensors: nothing here reaches a kernel)."""
    ids = torch.zeros(4, dtype=torch.int32)
    ok, half = torch.zeros(4, 6), torch.zeros(4, 6, dtype=torch.float16)
    for bad in (lambda: csgs.csgs_embed(half, ids, ok), lambda: csgs.csgs_embed(ok, ids.long(), ok), lambda: csgs.csgs_embed(ok.t().contiguous().t(), ids, ok),
                lambda: csgs.csgs_embed(ok, ids, torch.zeros(3, 6)), lambda: csgs.csgs_embed(ok, ids, torch.zeros(4, 5)),
                lambda: csgs.csgs_norm_residual(ok, torch.zeros(4, 5), ok, ok), lambda: csgs.csgs_norm_residual(ok, half, ok, ok),
                lambda: csgs.csgs_norm_residual(ok, ok, ok, ok, post_w=torch.zeros(5)), lambda: csgs.csgs_norm_residual(ok, ok, ok, ok, gate=torch.zeros(2, 6)),
                lambda: csgs.make_grad_list([half]), lambda: csgs.make_grad_list([]), lambda: csgs.make_grad_list([torch.zeros(8)[::2]]),
                lambda: csgs.make_grad_list([ok], [torch.zeros(4, 5)]), lambda: csgs.make_grad_list([torch.zeros(5)], None, [ids[:1]])):
        with pytest.raises((AssertionError, TypeError)):
            bad()


def test_norm_residual_wider_than_its_indices():
    L = csgs.lib()
    wide = (1 << 31) - 1
    r = dict(F=wide - 100, ldx=wide, ldh=wide, ldg=wide)
    assert L.csgs_norm_residual(C.byref(residual(**r)), P, wide, P, wide, Z) == csgs.EUNSUPPORTED
    assert L.csgs_norm_residual_grad(C.byref(residual(**r)), P, wide, P, wide, P, wide, P, wide, P, wide, P, Z, Z, Z, P, 1 << 60, Z) == csgs.EUNSUPPORTED


def part_doubles_needed(n, F, bf16):
    """What the sums of a call leave for the joins: two rows of F doubles a chunk (the library's share of a group, and lanes that take a row)."""
    most = 16 if F <= 128 else 32 if F <= 256 else 64
    share = 8
    while share < most and n // (2 * share) * F >= 1 << 20:
        share *= 2
    V = 8 if bf16 else 4
    lanes = 16 if F <= 16 * V else 32 if F <= 32 * V else 64
    chunk = share * (256 // lanes)
    return 2 * F * ((n + chunk - 1) // chunk)


@pytest.mark.parametrize("F", [1, 3, 16, 33, 64, 65, 100, 128, 129, 256, 257, 512, 602, 1024, 5000, 1 << 20])
def test_scratch_for_the_largest_table_gradient_serves_smaller_ones(F):
    size = csgs.csgs_embed_grad_scratch_bytes
    around = {1, 2, 7, 2048, 2049, 98_304, 98_305, 1 << 20, (1 << 31) - 1}
    for share in (8, 16, 32):                   # where a share doubles
        n = 2 * share * -(-(1 << 20) // F)
        around |= {n - 1, n, n + 1, n // 2, 3 * n}
    ns = sorted(n for n in around if 0 < n < 1 << 31)
    sizes = [size(n, 1000, F) for n in ns]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])), list(zip(ns, sizes))
    for n in ns:
        assert size(n, 1, F) <= size(n, 1 << 30, F)
        assert size(n, 1000, F) <= size(n, 1000, F + 1), n
        for bf16 in (False, True):
            assert size(n, 1000, F) >= n * 20 + 8 * part_doubles_needed(n, F, bf16), n
    # and no more than the positions and the rows that are summed take
    for n in ns:
        assert size(n, 1000, F) <= 20 * n + (n + 64) * F * 4 + (1 << 20), n
