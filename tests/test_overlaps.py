"""Outputs that lie on inputs, on each other or on the scratch, in whole or in part, are refused on the host.  Needs no GPU: every call below ends in an error."""
import ctypes as C
import subprocess

import pytest

pytest.importorskip("torch")

from paper_2101_07706_amd import build, csgs
from test_training_arguments import gated, linear

ASK = """
#include <cstdio>
#include "apart.hpp"
int main()
{
    using namespace csgs;
    long p[2], rows[2], width[2], step[2];
    while (scanf("%ld %ld %ld %ld %ld %ld %ld %ld", p, rows, width, step, p + 1, rows + 1, width + 1, step + 1) == 8) {
        const Memory a{(void *)p[0], rows[0], width[0], step[0]}, b{(void *)p[1], rows[1], width[1], step[1]};
        printf("%d%d\\n", (int)memory_meets(a, b), (int)memory_meets(b, a));
    }
}
"""


def test_rows_that_meet(tmp_path):
    """Against every byte of both, for all small matrices."""
    (tmp_path / "ask.cpp").write_text(ASK)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, "-o", str(tmp_path / "ask"), str(tmp_path / "ask.cpp")], check=True)
    shapes = [(r, w, w + g) for r in (1, 2, 3, 5) for w in (1, 2, 4) for g in (0, 1, 3, 7)]
    cases = [(100, *a, 100 + d, *b) for a in shapes for b in shapes for d in (-9, -4, -1, 0, 1, 3, 8, 17)]
    out = subprocess.run([str(tmp_path / "ask")], input="\n".join(" ".join(map(str, c)) for c in cases), stdout=subprocess.PIPE, text=True, check=True).stdout.split()
    assert len(out) == len(cases)
    bytes_of = lambda p, r, w, s: {p + i * s + k for i in range(r) for k in range(w)}  # noqa: E731
    meets = 0
    for c, got in zip(cases, out):
        want = bool(bytes_of(*c[:4]) & bytes_of(*c[4:]))
        assert got == ("11" if want else "00"), c
        meets += want
    assert 1000 < meets < len(cases) - 1000


KB = 1 << 10
FORWARD_LINEAR = dict(a=(64 * KB, 6), w=(128 * KB, 5), bias=(192 * KB, 5), r=(256 * KB, 5), M_dev=(320 * KB, 1))
FORWARD_GATED = dict(x=(64 * KB, 6), wg=(128 * KB, 5), wu=(192 * KB, 5), bg=(256 * KB, 5), bu=(320 * KB, 5), M_dev=(384 * KB, 1))
ROWS = dict(a=40, w=6, bias=1, r=40, M_dev=1, x=40, wg=6, wu=6, bg=1, bu=1, y=40, h=40, dy=40, dh=40, da=40, dx=40, dw=6, dwg=6, dwu=6, dbias=1, dbg=1, dbu=1, dr=40)


def places(name, at, cols, ld, size=4):
    """Addresses whose four bytes are the first, a middle row's and the last entry of a matrix."""
    rows = ROWS[name]
    return [at, at + (rows // 2) * ld * size + (cols // 2) * size, at + ((rows - 1) * ld + cols - 1) * size]


def test_forward_outputs_on_part_of_an_input():
    L = csgs.lib()
    M = 40
    p = lambda d: {k: v[0] for k, v in d.items()}  # noqa: E731
    for name, (at, cols) in FORWARD_LINEAR.items():
        for place in places(name, at, cols, 6 if name == "a" else 5):
            for y in (place, place - ((M - 1) * 5 + 4) * 4):            # its first entry there, and its last
                if y != FORWARD_LINEAR["r"][0]:
                    assert L.csgs_linear(C.byref(linear(M=M, **p(FORWARD_LINEAR))), y, 5, None) == csgs.EINVAL, (name, place, y)
    for name, (at, cols) in FORWARD_GATED.items():
        for place in places(name, at, cols, 6 if name == "x" else 5):
            for h in (place, place - ((M - 1) * 5 + 4) * 4):
                assert L.csgs_gated(C.byref(gated(M=M, **p(FORWARD_GATED))), h, 5, None) == csgs.EINVAL, (name, place, h)


def linear_grad(out, scratch=2048 * KB, nbytes=None):
    p = linear(M=40, **{k: v[0] for k, v in FORWARD_LINEAR.items()})
    nbytes = csgs.csgs_linear_grad_scratch_bytes(40, 6, 5, csgs.F32) if nbytes is None else nbytes
    return csgs.lib().csgs_linear_grad(C.byref(p), out["dy"], 5, out["da"], 6, out["dw"], 5, out["dbias"], out["dr"], 5, scratch, nbytes, None)


def gated_grad(out, scratch=2048 * KB, nbytes=None):
    p = gated(M=40, **{k: v[0] for k, v in FORWARD_GATED.items()})
    nbytes = csgs.csgs_gated_grad_scratch_bytes(40, 6, 5, csgs.F32) if nbytes is None else nbytes
    return csgs.lib().csgs_gated_grad(C.byref(p), out["dh"], 5, out["dx"], 6, out["dwg"], 5, out["dwu"], 5, out["dbg"], out["dbu"], scratch, nbytes, None)


@pytest.mark.parametrize("call", [linear_grad, gated_grad])
def test_gradients_on_part_of_something_else(call):
    names = ["dy", "da", "dw", "dbias", "dr"] if call is linear_grad else ["dh", "dx", "dwg", "dwu", "dbg", "dbu"]
    out = {k: (512 + 64 * i) * KB for i, k in enumerate(names)}
    inputs = dict(FORWARD_LINEAR if call is linear_grad else FORWARD_GATED)
    inputs.pop("r", None)                                               # (of r only that there is one counts)
    cols = lambda k: 6 if k in ("a", "x", "da", "dx") else 1 if k == "M_dev" else 5  # noqa: E731
    inputs[names[0]] = (out[names[0]], 5)
    assert call(out, nbytes=1) == csgs.EWORKSPACE                       # (nothing else is wrong with it)
    for k in names[1:]:
        last = ((ROWS[k] - 1) * cols(k) + cols(k) - 1) * 4
        others = {**inputs, **{o: (out[o], cols(o)) for o in names[1:] if o != k}}
        for name, (at, n) in others.items():
            for place in places(name, at, n, n):
                for address in (place, place - last):
                    if (k, name) != ("dr", "dy") or address != at:
                        assert call({**out, k: address}, nbytes=1) == csgs.EINVAL, (k, name, address)
            end = at + ROWS[name] * n * 4
            for address in (end, at - last - 4):                        # beside it
                assert call({**out, k: address}, nbytes=1) == csgs.EWORKSPACE, (k, name, address)
    need = csgs.csgs_linear_grad_scratch_bytes(40, 6, 5, csgs.F32) if call is linear_grad else csgs.csgs_gated_grad_scratch_bytes(40, 6, 5, csgs.F32)
    for name, (at, n) in {**inputs, **{o: (out[o], cols(o)) for o in names[1:]}}.items():
        for scratch in (at, at - (need - 256)):
            assert scratch % 256 == 0 and call(out, scratch=scratch) == csgs.EINVAL, (name, scratch)


def test_columns_of_one_buffer_lie_apart():
    """A row of one buffer holds a row of a, of dy and of da; one entry further on or rows one entry closer, and they meet."""
    L = csgs.lib()

    def call(ld, at=11):
        p = linear(M=40, a=64 * KB, lda=ld, r=0, bias=0, w=512 * KB)
        return L.csgs_linear_grad(C.byref(p), 64 * KB + 6 * 4, ld, 64 * KB + at * 4, ld, 1024 * KB, 5, None, None, 0, 2048 * KB, 1, None)
    assert call(17) == csgs.EWORKSPACE and call(18) == csgs.EWORKSPACE and call(18, at=12) == csgs.EWORKSPACE
    assert call(16) == csgs.EINVAL and call(17, at=10) == csgs.EINVAL and call(17, at=12) == csgs.EINVAL


def test_memory_that_no_device_has():
    L = csgs.lib()
    for kw in (dict(lda=1 << 61), dict(ldw=(1 << 62) + 1), dict(lda=1 << 40)):
        assert L.csgs_linear(C.byref(linear(M=40, **kw)), 1 << 20, 5, None) == csgs.EUNSUPPORTED, kw
    assert L.csgs_linear(C.byref(linear(M=40)), 1 << 20, 1 << 62, None) == csgs.EUNSUPPORTED
    assert L.csgs_gated(C.byref(gated(M=40, ldx=1 << 50)), 1 << 20, 5, None) == csgs.EUNSUPPORTED


WRITTEN = ["p", "copy", "m", "v", "m_exp", "v_exp"]


def tensor(base, **kw):
    """A parameter of 40 x 300 bfloat16 with states in 8 bits, its memory 64 KB apart from `base` on."""
    at = {k: base + 64 * KB * i for i, k in enumerate(WRITTEN + ["g", "ids", "n_dev"])}
    t = dict(at, rows=40, cols=300, n=40, ldp=300, ldcopy=300, ldg=300, p_dtype=1, g_dtype=1, state=1, weight_decay=0.0, lr_scale=1.0, reserved=0)
    t.update(kw)
    return csgs.AdamwTensor(*[t[k] for k, _ in csgs.AdamwTensor._fields_])


SPAN = dict(p=24_000, copy=24_000, m=12_000, v=12_000, m_exp=80, v_exp=80, g=24_000, ids=160, n_dev=4)


def answer(*tensors):
    L = csgs.lib()
    ts = (csgs.AdamwTensor * len(tensors))(*tensors)
    if L.csgs_adamw_list_bytes(ts, len(ts)) > 0:
        return csgs.OK
    l = csgs.AdamwList(4096, 1 << 40, 0, 0, 0)
    rc = L.csgs_adamw_list_init(C.byref(l), ts, len(ts), None)
    assert rc != csgs.OK and l.ready == 0
    return rc


@pytest.mark.parametrize("mine", list(SPAN))
def test_lists_whose_tensors_share_part_of_their_memory(mine):
    one, base = tensor(64 * KB), 1024 * KB
    assert answer(one, tensor(base)) == csgs.OK
    for theirs in SPAN:
        at = getattr(one, theirs)
        for address in (at, at + SPAN[theirs] - 4, at + 4 - SPAN[mine], at + (SPAN[theirs] - SPAN[mine]) // 8 * 4):
            want = csgs.EINVAL if mine in WRITTEN or theirs in WRITTEN else csgs.OK
            assert answer(one, tensor(base, **{mine: address})) == want and answer(tensor(base, **{mine: address}), one) == want, (theirs, address - at)
        for address in (at + SPAN[theirs], at - SPAN[mine]):
            assert answer(one, tensor(base, **{mine: address})) == csgs.OK, (theirs, address - at)


def test_tensors_whose_own_memory_meets():
    for a, b in (("p", "copy"), ("p", "m"), ("m", "v"), ("copy", "v"), ("p", "g"), ("m", "g"), ("p", "ids"), ("v", "n_dev")):
        one = tensor(64 * KB)
        assert answer(tensor(64 * KB, **{b: getattr(one, a) + 600})) == csgs.EINVAL, (a, b)


def test_lists_over_the_columns_of_one_buffer():
    """Parts of one matrix, of its copy and of its gradient; the same gradient and the same count for several."""
    base, L = 1 << 30, csgs.lib()
    cut = lambda i, first, **kw: tensor(base * (i + 2), p=base + 2 * first, ldp=900, g=4 * KB, n_dev=2 * KB, **kw)  # noqa: E731
    assert answer(cut(0, 0), cut(1, 300), cut(2, 600)) == csgs.OK
    assert answer(cut(0, 0), cut(1, 299), cut(2, 600)) == csgs.EINVAL
    assert answer(cut(0, 0), cut(1, 300), cut(2, 601)) == csgs.EINVAL
    assert answer(cut(0, 0), tensor(base * 9, g=base + 600, ldg=900)) == csgs.OK and answer(cut(0, 0), tensor(base * 9, g=base + 598, ldg=900)) == csgs.EINVAL
    # many tensors with one count; more interleaved ones than are compared in pairs
    n = 100_000
    ts = (csgs.AdamwTensor * n)(*[tensor((i + 2) << 20, n_dev=4096) for i in range(n)])
    assert L.csgs_adamw_list_bytes(ts, n) > 0
    n = 12_000
    ts = (csgs.AdamwTensor * n)(*[tensor((i + 2) << 40, p=base + 2 * i, cols=1, ldp=n, ldg=1, copy=0) for i in range(n)])
    assert L.csgs_adamw_list_bytes(ts, n) == 0 and L.csgs_adamw_list_init(C.byref(csgs.AdamwList(4096, 1 << 40, 0, 0, 0)), ts, n, None) == csgs.EUNSUPPORTED
    assert L.csgs_adamw_list_bytes(ts, 3000) > 0
    assert answer(tensor(base, ldp=1 << 50)) == csgs.EUNSUPPORTED


def test_states_on_their_values():
    L = csgs.lib()
    codes, exps, values = 64 * KB, 128 * KB, 256 * KB          # 40 x 300
    for c, e, v in ((values + 47_996, exps, values), (values - 11_999, exps, values), (codes, values + 100, values), (codes, codes + 11_999, values), (codes, codes - 79, values)):
        assert L.csgs_state_read(c, e, 0, 40, 300, v, 300, None) == csgs.EINVAL and L.csgs_state_write(v, 300, 0, 40, 300, c, e, None) == csgs.EINVAL
    assert L.csgs_state_read(codes, exps, 0, 40, 300, values, 1 << 50, None) == csgs.EUNSUPPORTED


def test_binding_sees_exponents_on_their_tensor():
    import torch
    p, both = torch.zeros(4, 300), torch.zeros(4 * 300 + 16, dtype=torch.uint8)
    s = csgs.adamw_states(p, 8)
    csgs.adamw_entry(p, p.clone(), **s)
    for k in ("m_exp", "v_exp"):
        for bad in (s["m"].view(-1)[8:16].view(4, 2), p.view(torch.uint8).view(-1)[100:108].view(4, 2), both[1196:1204].view(4, 2)):
            with pytest.raises(AssertionError):
                csgs.adamw_entry(p, p.clone(), **{**s, "v": both[:1200].view(4, 300), k: bad})
    csgs.adamw_entry(p, p.clone(), **{**s, "v": both[:1200].view(4, 300), "m_exp": both[1200:1208].view(4, 2), "v_exp": both[1208:].view(4, 2)})
