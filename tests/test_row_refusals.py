"""What the calls on rows refuse, and what they say: every argument is checked on the host, before anything is enqueued, so this
needs no GPU."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2102_08124_amd import binding as tm      # noqa: E402

A = 1 << 20                                         # an address that nothing may follow


def norm(**k):
    return tm.tmask_norm_desc(**{**dict(x=A, ld_x=64, y=A, ld_y=64, rows=4, cols=64), **k})


def norm_grad(**k):
    return tm.tmask_norm_grad_desc(**{**dict(dy=A, ld_dy=64, x=A, ld_x=64, mean=A, rstd=A, dx=A, ld_dx=64, rows=4, cols=64), **k})


def gelu(**k):
    return tm.tmask_gelu_desc(**{**dict(x=A, ld_x=64, y=A, ld_y=64, rows=4, cols=64), **k})


def gelu_grad(**k):
    return tm.tmask_gelu_grad_desc(**{**dict(dy=A, ld_dy=64, x=A, ld_x=64, dx=A, ld_dx=64, rows=4, cols=64), **k})


def distill(**k):
    return tm.tmask_distill_desc(**{**dict(logits=A, ld_logits=64, teacher=A, ld_teacher=8, index=A, ld_index=8, loss=A, row_max=A, row_sum=A,
                                           dlogits=A, ld_dlogits=64, rows=4, vocab=64, k=8), **k})


CALLS = {
    "norm": lambda L, d, dt=0, pdt=0, eps=1e-5: L.tmask_layer_norm(d, dt, pdt, eps, None),
    "norm_grad": lambda L, d, dt=0, pdt=0, ws=A, n=1 << 30: L.tmask_layer_norm_backward(d, dt, pdt, ws, n, None),
    "gelu": lambda L, d, dt=0, pdt=0, form=0: L.tmask_bias_gelu(d, dt, pdt, form, None),
    "gelu_grad": lambda L, d, dt=0, pdt=0, form=0, ws=A, n=1 << 30: L.tmask_bias_gelu_backward(d, dt, pdt, form, ws, n, None),
    "distill": lambda L, d, dt=0, pdt=0, bits=32, T=1.0, ws=A, n=1 << 30: L.tmask_distill(d, dt, pdt, bits, T, ws, n, None),
    "distill_grad": lambda L, d, dt=0, pdt=0, bits=32, T=1.0: L.tmask_distill_backward(d, dt, pdt, bits, T, None),
}
DESCS = {"norm": norm, "norm_grad": norm_grad, "gelu": gelu, "gelu_grad": gelu_grad, "distill": distill, "distill_grad": distill}
NULL, SHAPE, DTYPE, WORKSPACE, ALIGN = (tm.TMASK_ERR_NULL, tm.TMASK_ERR_SHAPE, tm.TMASK_ERR_DTYPE, tm.TMASK_ERR_WORKSPACE, tm.TMASK_ERR_ALIGN)

WIDE = 1 << 31
REFUSED = [
    ("norm", dict(x=None), {}, NULL), ("norm", dict(y=None), {}, NULL), ("norm", dict(total=A, ld_total=64), {}, NULL),
    ("norm", dict(mean=A), {}, NULL), ("norm", dict(rstd=A), {}, NULL), ("norm", dict(rows=-1), {}, SHAPE), ("norm", dict(cols=0), {}, SHAPE),
    ("norm", dict(ld_x=63), {}, SHAPE), ("norm", dict(ld_y=0), {}, SHAPE), ("norm", dict(residual=A, ld_residual=63), {}, SHAPE),
    ("norm", dict(residual=A, ld_residual=64, total=A, ld_total=1), {}, SHAPE), ("norm", dict(ld_x=WIDE), {}, SHAPE), ("norm", dict(cols=WIDE), {}, SHAPE),
    ("norm", dict(rows=WIDE), {}, SHAPE), ("norm", {}, dict(eps=-1.0), SHAPE), ("norm", {}, dict(eps=float("nan")), SHAPE),
    ("norm", {}, dict(eps=float("inf")), SHAPE), ("norm", {}, dict(dt=2), DTYPE), ("norm", {}, dict(pdt=-1), DTYPE), ("norm", dict(x=A + 2), {}, ALIGN),
    ("norm", dict(y=A + 1), dict(dt=1), ALIGN), ("norm", dict(weight=A + 2), dict(dt=1), ALIGN), ("norm", dict(mean=A + 2, rstd=A), dict(dt=1), ALIGN),
    ("norm_grad", dict(dy=None), {}, NULL), ("norm_grad", dict(x=None), {}, NULL), ("norm_grad", dict(dx=None), {}, NULL),
    ("norm_grad", dict(mean=None), {}, NULL), ("norm_grad", dict(rstd=None), {}, NULL), ("norm_grad", dict(ld_dy=63), {}, SHAPE),
    ("norm_grad", dict(dtotal=A, ld_dtotal=63), {}, SHAPE), ("norm_grad", dict(ld_dx=-64), {}, SHAPE), ("norm_grad", dict(dweight=A), dict(ws=None), WORKSPACE),
    ("norm_grad", dict(dbias=A), dict(n=1), WORKSPACE), ("norm_grad", dict(dbias=A), dict(ws=A + 4), WORKSPACE), ("norm_grad", dict(dbias=A + 2), {}, ALIGN),
    ("norm_grad", {}, dict(dt=7), DTYPE), ("norm_grad", dict(rows=-3), {}, SHAPE),
    ("gelu", dict(x=None), {}, NULL), ("gelu", dict(y=None), {}, NULL), ("gelu", dict(ld_x=3), {}, SHAPE), ("gelu", {}, dict(form=2), DTYPE),
    ("gelu", {}, dict(pdt=3), DTYPE), ("gelu", dict(bias=A + 2), {}, ALIGN), ("gelu", dict(cols=-1), {}, SHAPE),
    ("gelu_grad", dict(dy=None), {}, NULL), ("gelu_grad", dict(x=None), {}, NULL), ("gelu_grad", dict(dx=None), {}, NULL), ("gelu_grad", dict(ld_dx=3), {}, SHAPE),
    ("gelu_grad", dict(dbias=A), dict(ws=None), WORKSPACE), ("gelu_grad", dict(dbias=A), dict(n=255), WORKSPACE),
    ("gelu_grad", dict(dbias=A + 1), dict(pdt=1), ALIGN), ("gelu_grad", {}, dict(form=-1), DTYPE),
]
for name in ("distill", "distill_grad"):
    REFUSED += [(name, *r) for r in [
        (dict(logits=None), {}, NULL), (dict(teacher=None), {}, NULL), (dict(index=None), {}, NULL), (dict(vocab=0), {}, SHAPE), (dict(rows=-1), {}, SHAPE),
        (dict(k=-1), {}, SHAPE), (dict(k=1025, ld_teacher=2000, ld_index=2000), {}, SHAPE), (dict(ld_logits=63), {}, SHAPE), (dict(ld_teacher=7), {}, SHAPE),
        (dict(ld_index=7), {}, SHAPE), (dict(ld_dlogits=63), {}, SHAPE), ({}, dict(T=0.0), SHAPE), ({}, dict(T=-1.0), SHAPE),
        ({}, dict(T=float("nan")), SHAPE), ({}, dict(T=float("inf")), SHAPE), ({}, dict(T=1e-19), SHAPE), ({}, dict(T=1e19), SHAPE), ({}, dict(bits=16), DTYPE), ({}, dict(dt=5), DTYPE), ({}, dict(pdt=5), DTYPE),
        (dict(logits=A + 2), {}, ALIGN), (dict(index=A + 4), dict(bits=64), ALIGN), (dict(row_weight=A + 2), {}, ALIGN), (dict(dlogits=A + 1), dict(dt=1), ALIGN)]]
REFUSED += [("distill", dict(loss=None), {}, NULL), ("distill", dict(row_max=None), {}, NULL), ("distill", dict(row_sum=None), {}, NULL),
            ("distill", dict(loss=A + 2), {}, ALIGN), ("distill_grad", dict(row_max=None), {}, NULL), ("distill_grad", dict(row_sum=None), {}, NULL),
            ("distill_grad", dict(dlogits=None), {}, NULL)]


@pytest.mark.parametrize("case", range(len(REFUSED)))
def test_refused(case):
    name, desc, args, code = REFUSED[case]
    L = tm.load_library()
    assert CALLS[name](L, DESCS[name](**desc), **args) == code
    assert L.tmask_last_error()


@pytest.mark.parametrize("name", sorted(CALLS))
def test_no_descriptor(name):
    assert CALLS[name](tm.load_library(), None) == NULL


def test_no_rows_need_no_tensors():
    L = tm.load_library()
    nothing = dict(x=None, y=None, dy=None, dx=None, mean=None, rstd=None, logits=None, teacher=None, index=None, loss=None, row_max=None, row_sum=None, dlogits=None)
    for name, call in CALLS.items():
        fields = {f for f, _ in type(DESCS[name]())._fields_}
        assert call(L, DESCS[name](**{k: v for k, v in nothing.items() if k in fields}, rows=0)) == 0


def test_layouts_match_the_header():
    assert [C.sizeof(t) for t in (tm.tmask_norm_desc, tm.tmask_norm_grad_desc, tm.tmask_gelu_desc, tm.tmask_gelu_grad_desc, tm.tmask_distill_desc)] == \
        [112, 120, 56, 80, 120]


@pytest.mark.parametrize("f", ["tmask_layer_norm_workspace_bytes", "tmask_bias_gelu_workspace_bytes", "tmask_distill_workspace_bytes"])
def test_workspace_sizes(f):
    size = getattr(tm.load_library(), f)
    assert size(-1, 64) == 0 and size(4, 0) == 0 and size(4, 1 << 31) == 0
    if "distill" not in f:
        assert size(1, 64) >= 256 and size(1 << 20, 1024) <= 64 << 20


# around the numbers of rows and columns at which calls are cut otherwise
BATCHES = [0, 1, 2, 4, 15, 16, 17, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 384, 385, 700, 1000, 1024, 1025, 2000, 2048, 2049, 4096, 4104, 5000,
           8192, 8200, 10000, 12288, 30000, 1 << 20, 1 << 30]


@pytest.mark.parametrize("f", ["tmask_layer_norm_workspace_bytes", "tmask_bias_gelu_workspace_bytes", "tmask_distill_workspace_bytes"])
def test_workspace_sizes_grow_with_both_arguments(f):
    """So that a program allocates once, for its longest batch and widest rows."""
    size = getattr(tm.load_library(), f)
    widths = sorted({max(1, (1 << b) + d) for b in range(21) for d in (-1, 0, 1, 7)} | {1000, 12000, 20000, 40000, 70001, 131072, 200003})
    table = [[size(r, c) for c in widths] for r in BATCHES]
    for a, b in zip(table, table[1:]):
        assert all(x <= y for x, y in zip(a, b))
    for row in table:
        assert all(x <= y for x, y in zip(row, row[1:]))


def test_tensors_that_do_not_fit():
    """Types and shapes are the binding's to check; host tensors are no tensors of a call."""
    x = torch.zeros((4, 64))
    for f in (lambda: tm.tmask_layer_norm(x, x), lambda: tm.tmask_bias_gelu(x, x), lambda: tm.tmask_bias_gelu_backward(x, x, x),
              lambda: tm.tmask_layer_norm_backward(x, x, x[:, 0], x[:, 0], x),
              lambda: tm.tmask_distill(x, x[:, :3], torch.zeros((4, 3), dtype=torch.int32), 1.0, x[:, 0])):
        with pytest.raises(ValueError, match="CUDA|device"):
            f()
    h = x.half()
    for f in (lambda: tm.tmask_layer_norm(h, h), lambda: tm.tmask_bias_gelu(h, h), lambda: tm.tmask_distill(h, x, x, 1.0, x)):
        with pytest.raises(TypeError, match="float32 or bfloat16"):
            f()
