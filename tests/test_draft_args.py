"""What the proposer's operators refuse, and that the binding is the header's (no GPU needed: everything is refused before the device is touched)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2502_01662_b200 as pkg
from paper_2502_01662_b200 import build, draft

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    with open(os.path.join(ROOT, "include", "cos_draft.h")) as f:
        return re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)


def test_every_declared_symbol_is_exported_and_bound():
    names = set(re.findall(r"\bcos_status (cos_\w+)\s*\(", _header()))
    assert names == set(draft.EXPORTS)
    lib = pkg.load_library()
    for name in names:
        assert hasattr(lib, name), name


def test_structures_are_the_headers():
    for struct in (draft.cos_sample_args, draft.cos_top_args, draft.cos_distill_args):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % struct.__name__, _header()).group(1)
        fields = []
        for decl in body.split(";"):
            decl = re.sub(r"\[\w+\]", "", decl).strip()
            if decl:
                fields += [re.search(r"(\w+)\s*$", part).group(1) for part in decl.split(",")]
        assert fields == [f[0] for f in struct._fields_], struct.__name__
    assert re.search(r"#define COS_TOP_MAX (\d+)", _header()).group(1) == str(pkg.COS_TOP_MAX)


def test_a_change_of_any_header_makes_the_library_stale():
    assert os.path.join(build.INCLUDE, "cos_draft.h") in build.dependencies()


A = 1 << 20     # an address that is aligned; nothing reads it


def _sample(**kw):
    a = draft.cos_sample_args(logits=A, stride_row=100, rows=4, vocab=100, dtype=0, device=0, uniforms=A, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, tokens=A)
    return draft._library().cos_sample, a, kw


def _top(**kw):
    a = draft.cos_top_args(logits=A, stride_row=100, rows=4, vocab=100, dtype=0, device=0, k=5, temperature=1.0, values=A, ids=A, lse=A)
    return draft._library().cos_top_logits, a, kw


def _distill(name, **kw):
    a = draft.cos_distill_args(student=A, stride_student=100, rows=4, vocab=100, dtype=1, device=0, lists=1, k=5, ids=A, values=A, temperature=1.0, row_weights=A, loss=A, statistics=A, grad=A,
                               stride_grad=100)
    a.weights[0] = 1.0
    return getattr(draft._library(), name), a, kw


NAN, INF = float("nan"), float("inf")
CASES = [
    *[(_sample(**kw), st) for kw, st in (
        (dict(logits=None), 1), (dict(uniforms=None), 1), (dict(tokens=None), 1), (dict(rows=0), 1), (dict(vocab=0), 1), (dict(rows=-1), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1),
        (dict(stride_row=99), 1), (dict(stride_row=-100), 1), (dict(temperature=-1.0), 1), (dict(temperature=NAN), 1), (dict(top_p=0.0), 1), (dict(top_p=NAN), 1), (dict(min_p=-0.1), 1),
        (dict(min_p=1.1), 1), (dict(min_p=NAN), 1), (dict(filtered=A + (1 << 19), stride_filtered=50), 1), (dict(filtered=A, stride_filtered=200), 1), (dict(stride_row=0, filtered=A, stride_filtered=100), 1), (dict(logits=A + 2), 3), (dict(uniforms=A + 1), 3),
        (dict(row_top_k=A + 2), 3), (dict(prob=A + 2), 3), (dict(filtered=A + 1, stride_filtered=100), 3))],
    *[(_top(**kw), st) for kw, st in (
        (dict(logits=None), 1), (dict(values=None), 1), (dict(ids=None), 1), (dict(lse=None), 1), (dict(k=0), 1), (dict(k=101), 1), (dict(vocab=5000, stride_row=5000, k=1025), 1), (dict(temperature=0.0), 1),
        (dict(temperature=NAN), 1), (dict(rows=0), 1), (dict(stride_row=10), 1), (dict(logits=A + 1), 3), (dict(values=A + 2), 3))],
    *[(_distill(name, **kw), st) for name in ("cos_distill_loss", "cos_distill_grad", "cos_distill_step") for kw, st in (
        (dict(student=None), 1), (dict(ids=None), 1), (dict(values=None), 1), (dict(rows=0), 1), (dict(vocab=0), 1), (dict(dtype=9), 1), (dict(lists=0), 1), (dict(lists=9), 1), (dict(k=0), 1), (dict(k=1025), 1),
        (dict(lists=8, k=129), 1), (dict(temperature=0.0), 1), (dict(temperature=INF), 1), (dict(temperature=NAN), 1), (dict(stride_student=99), 1), (dict(student=A + 1), 3), (dict(ids=A + 1), 3), (dict(values=A + 2), 3),
        (dict(lse=A + 2), 3))],
    *[(_distill(name, **kw), st) for name, kw, st in (
        ("cos_distill_loss", dict(loss=None), 1), ("cos_distill_loss", dict(statistics=None), 1), ("cos_distill_loss", dict(statistics=A + 4), 3), ("cos_distill_grad", dict(statistics=None), 1),
        ("cos_distill_step", dict(stride_student=0, grad=A), 1), ("cos_distill_grad", dict(row_weights=None), 1), ("cos_distill_grad", dict(grad=None), 1), ("cos_distill_grad", dict(grad=A + 1), 3), ("cos_distill_step", dict(loss=None), 1),
        ("cos_distill_step", dict(grad=None), 1), ("cos_distill_step", dict(stride_grad=99), 1), ("cos_distill_step", dict(grad=A, stride_grad=101), 1))],
]


@pytest.mark.parametrize("call,status", CASES)
def test_the_library_refuses(call, status):
    fn, a, kw = call
    for name, v in kw.items():
        setattr(a, name, v)
    assert fn(ctypes.byref(a), None) == status, kw
    assert pkg.load_library().cos_verify_last_error(None)


def test_weights_and_null_arguments_are_refused():
    fn, a, _ = _distill("cos_distill_loss")
    for w in (-1.0, NAN, INF):
        a.weights[0] = w
        assert fn(ctypes.byref(a), None) == 1
    lib = draft._library()
    for name in draft.EXPORTS:
        assert getattr(lib, name)(None, None) == 1


def test_host_tensors_and_shapes_are_refused():
    x, u = torch.zeros(2, 10), torch.zeros(2)
    ids, values = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    for call in (lambda: pkg.sample(x, u), lambda: pkg.top_logits(x, 3), lambda: pkg.distill_loss(x, ids, values), lambda: pkg.distill_step(x, ids, values, u), lambda: pkg.sample(x[0], u),
                 lambda: pkg.top_logits(x[None], 3)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_the_binding_refuses():
    x, u = torch.zeros(4, 10, device="cuda"), torch.zeros(4, device="cuda")
    ids, values = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    bad = [lambda: pkg.sample(x.t(), u), lambda: pkg.sample(x, u[:3]), lambda: pkg.sample(x, u.double()), lambda: pkg.sample(x.double(), u), lambda: pkg.sample(x, u, temperature=u.double()),
           lambda: pkg.sample(x, u, top_k=u), lambda: pkg.sample(x, u, filtered=x[:, :9]), lambda: pkg.sample(x, u, filtered=x.half()), lambda: pkg.sample(x, u.cpu()),
           lambda: pkg.sample(x[:0], u[:0]), lambda: pkg.top_logits(x, 0), lambda: pkg.top_logits(x, 11), lambda: pkg.top_logits(x[:, ::2], 2), lambda: pkg.distill_loss(x, ids.long(), values),
           lambda: pkg.distill_loss(x, ids, values[:, :2]), lambda: pkg.distill_loss(x, ids, values, lse=u[:3]), lambda: pkg.distill_loss(x, ids, values, weights=[0.5, 0.5]),
           lambda: pkg.distill_step(x, ids, values, u[:2]), lambda: pkg.distill_step(x, ids, values, u, grad=x.half()), lambda: pkg.distill_loss(x, ids[0], values[0])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print(i)
    for call in (lambda: pkg.sample(x, u, temperature=-1.0), lambda: pkg.sample(x, u, top_p=0.0), lambda: pkg.sample(x, u, min_p=2.0), lambda: pkg.top_logits(x, 3, temperature=0.0),
                 lambda: pkg.distill_loss(x, ids, values, temperature=0.0), lambda: pkg.distill_loss(x, ids, values, weights=[-1.0])):
        with pytest.raises(pkg.CosVerifyError):
            call()


@pytest.mark.parametrize("rows,stride,out,stride_out,refused", [
    (1, 100, 99, 100, True), (1, 100, 100, 100, False), (1, 100, -100, 100, False), (1, 100, -99, 100, True), (4, 100, 100, 100, True), (4, 100, 400, 100, False), (4, 100, -400, 100, False),
    (4, 100, -399, 100, True), (4, 220, 100, 220, False), (4, 220, 120, 220, False), (4, 220, 121, 220, True), (4, 220, 99, 220, True), (4, 220, -100, 220, False), (4, 220, -121, 220, True),
    (4, 220, 540, 220, False), (4, 220, 100, 221, True), (4, 0, 50, 100, True), (4, 0, 100, 100, False), (4, 0, -300, 100, True), (4, 0, -400, 100, False)])
def test_outputs_that_overlap_inputs(rows, stride, out, stride_out, refused):
    """Columns of one buffer are apart or not by their distance in a row; what is refused is refused by reason of that, the others for a device that is not there."""
    for (fn, a, _), of in ((_sample(), "filtered"), (_distill("cos_distill_grad"), "grad"), (_distill("cos_distill_step"), "grad")):
        size = 4 if a.dtype == 0 else 2
        a.rows, a.device = rows, 1 << 20
        setattr(a, "stride_row" if of == "filtered" else "stride_student", stride)
        setattr(a, of, A + out * size)
        setattr(a, "stride_" + of, stride_out)
        st = fn(ctypes.byref(a), None)
        assert (st == 1) == refused and st != 0 and (b"overlaps" in pkg.load_library().cos_verify_last_error(None)) == refused
