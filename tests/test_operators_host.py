"""What dropout, the RMS norm and the head loss refuse, without a GPU: every check of the arguments comes before the first CUDA
call, so it answers here as it does on a device."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2510_09103_b200 as A

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EALIGN, ERANGE, ECUDA, ENOWORKSPACE, EUNSUPPORTED = -1, -2, -3, -4, -5, -6
P = 1 << 20            # an address that is never read: nothing is launched


def _code(f, *args):
    try:
        f(*args)
    except A.AdapmError as e:
        return e.code
    return 0


def _no_device():
    import torch
    return not torch.cuda.is_available()


def _dropout(**kw):
    a = dict(x=P, residual=None, y=2 * P, dtype=A.TYPE_BF16, rows=4, cols=16, p=0.1, seed=1, offset=0, step=None, x_ld=None,
             residual_ld=None, y_ld=None, stream=0)
    a.update(kw)
    return _code(lambda: A.adapm_dropout(**a))


def test_dropout_refusals():
    assert _dropout(dtype=2) == EINVAL
    assert _dropout(rows=-1) == EINVAL
    assert _dropout(x=None) == EINVAL and _dropout(y=None) == EINVAL
    assert _dropout(x_ld=15) == EINVAL and _dropout(y_ld=15) == EINVAL and _dropout(residual=3 * P, residual_ld=1) == EINVAL
    assert _dropout(p=-0.1) == ERANGE and _dropout(p=1.5) == ERANGE and _dropout(p=float("nan")) == ERANGE
    assert _dropout(rows=1 << 40, cols=1 << 40) == ERANGE
    assert _dropout(x=P + 1) == EALIGN and _dropout(step=P + 4) == EALIGN
    assert _dropout(y=P + 16) == EINVAL and _dropout(y=P, y_ld=24) == EINVAL          # over x, but not element on element
    assert _dropout(residual=3 * P, y=3 * P + 32) == EINVAL
    assert _dropout(rows=0) == 0 and _dropout(cols=0, x=None, y=None) == 0


def _norm(d=None, **kw):
    a = dict(x=P, residual=None, weight=2 * P, sum=None, y=3 * P, y8=None, y8_scales=None, rstd=None, stream=0)
    a.update(kw)
    return _code(lambda: A.adapm_rmsnorm_forward(d or A.rmsnorm_desc(4, 64), **a))


def test_rmsnorm_refusals():
    desc = A.rmsnorm_desc
    assert _norm(desc(-1, 64)) == EINVAL and _norm(desc(4, 0)) == EINVAL
    assert _norm(desc(4, 32769)) == ERANGE and _norm(desc(1 << 31, 8)) == ERANGE
    assert _norm(desc(4, 64, dtype=5)) == EINVAL and _norm(desc(4, 64, weight_dtype=-1)) == EINVAL
    assert _norm(desc(4, 64, q8_group=64)) == EINVAL
    assert _norm(desc(4, 64, eps=-1.0)) == ERANGE and _norm(desc(4, 64, eps=float("inf"))) == ERANGE
    assert _norm(desc(4, 64, drop_p=2.0)) == ERANGE
    assert _norm(desc(4, 64, x_ld=63)) == EINVAL and _norm(desc(4, 64, y_ld=1)) == EINVAL
    assert _norm(x=None) == EINVAL and _norm(weight=None) == EINVAL and _norm(y=None) == EINVAL
    assert _norm(y8=4 * P) == EINVAL                               # no room for its scales
    assert _norm(x=P + 1) == EALIGN and _norm(weight=P + 1) == EALIGN and _norm(rstd=P + 2) == EALIGN
    assert _norm(sum=3 * P + 16) == EINVAL                         # over y
    assert _norm(y=P + 16) == EINVAL and _norm(desc(4, 64, y_ld=72), y=P) == EINVAL     # over x, but not element on element
    assert _norm(sum=P + 128, y=3 * P) == EINVAL and _norm(y=2 * P) == EINVAL           # over x, over the weight
    assert _norm(y8=P, y8_scales=5 * P) == EINVAL
    assert _norm(desc(0, 64), x=None) == 0
    assert A.load().adapm_rmsnorm_forward(None, P, None, P, None, P, None, None, None, 0) == EINVAL


class _Scratch:
    """A buffer that says how long it is."""

    def __init__(self, n, at=16 * P):
        self.n, self.at = n, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 1


def _norm_grad(d=None, **kw):
    d = d or A.rmsnorm_desc(4, 64)
    a = dict(dy=P, dsum=None, sum=2 * P, rstd=3 * P, weight=4 * P, dresidual=5 * P, dx=None, dweight=6 * P, dweight_dtype=A.TYPE_F32,
             accumulate=False, scratch=_Scratch(A.adapm_rmsnorm_backward_scratch_bytes(d)), stream=0)
    a.update(kw)
    return _code(lambda: A.adapm_rmsnorm_backward(d, **a))


def test_rmsnorm_gradient_refusals():
    assert _norm_grad(dy=None) == EINVAL and _norm_grad(sum=None) == EINVAL and _norm_grad(rstd=None) == EINVAL and _norm_grad(weight=None) == EINVAL
    assert _norm_grad(dresidual=None, dweight=None) == EINVAL
    assert _norm_grad(dweight_dtype=7) == EINVAL
    assert _norm_grad(scratch=None) == EINVAL and _norm_grad(scratch=_Scratch(16)) == ENOWORKSPACE
    assert _norm_grad(scratch=_Scratch(1 << 30, 16 * P + 16)) == EALIGN
    assert _norm_grad(dweight=6 * P + 2) == EALIGN and _norm_grad(rstd=3 * P + 1) == EALIGN
    assert _norm_grad(dx=5 * P) == EINVAL                           # both gradients in one place
    assert _norm_grad(dresidual=P + 32) == EINVAL and _norm_grad(dresidual=4 * P) == EINVAL and _norm_grad(dresidual=6 * P) == EINVAL
    assert _norm_grad(dresidual=None, dx=2 * P + 2) == EINVAL
    assert _norm_grad(A.rmsnorm_desc(4, 64, residual_ld=3)) == EINVAL
    assert _norm_grad(A.rmsnorm_desc(0, 64), accumulate=True) == 0
    assert A.adapm_rmsnorm_backward_scratch_bytes(A.rmsnorm_desc(4, 1 << 20)) == 0
    assert A.load().adapm_rmsnorm_backward_scratch_bytes(None) == 0


def _head(d=None, **kw):
    d = d or A.head_loss_desc(4, 100, 64)
    a = dict(hidden=P, weight=2 * P, targets=3 * P, loss=4 * P, lse=5 * P, scratch=_Scratch(A.adapm_head_loss_scratch_bytes(d, False)), stream=0)
    a.update(kw)
    return _code(lambda: A.adapm_head_loss_forward(d, **a))


def _head_grad(d=None, **kw):
    d = d or A.head_loss_desc(4, 100, 64)
    a = dict(hidden=P, weight=2 * P, targets=3 * P, lse=5 * P, dloss=None, scale=1.0, dhidden=6 * P, dweight=7 * P,
             scratch=_Scratch(A.adapm_head_loss_scratch_bytes(d, True)), stream=0)
    a.update(kw)
    return _code(lambda: A.adapm_head_loss_backward(d, **a))


def test_head_loss_refusals():
    desc = A.head_loss_desc
    for f in (_head, _head_grad):
        assert f(desc(-1, 100, 64)) == EINVAL and f(desc(4, 0, 64)) == EINVAL and f(desc(4, 100, 0)) == EINVAL
        assert f(desc(1 << 25, 100, 64)) == ERANGE and f(desc(4, 1 << 25, 64)) == ERANGE and f(desc(4, 100, 1 << 17)) == ERANGE
        assert f(desc(1 << 24, 1 << 24, 64)) == ERANGE
        assert f(desc(4, 100, 60)) == EUNSUPPORTED
        assert f(desc(4, 100, 64, hidden_ld=56)) == EINVAL and f(desc(4, 100, 64, weight_ld=8)) == EINVAL
        assert f(desc(4, 100, 64, hidden_ld=68)) == EALIGN and f(desc(4, 100, 64, weight_ld=66)) == EALIGN
        assert f(desc(4, 100, 64, weight_ld=1 << 39)) == ERANGE
        assert f(desc(4, 100, 64, label_smoothing=1.5)) == ERANGE and f(desc(4, 100, 64, label_smoothing=float("nan"))) == ERANGE
        assert f(desc(4, 100, 64, z_loss=-1.0)) == ERANGE and f(desc(4, 100, 64, z_loss=float("inf"))) == ERANGE
        for name in ("hidden", "weight", "targets", "lse", "scratch"):
            assert f(**{name: None}) == EINVAL, name
        assert f(hidden=P + 8) == EALIGN and f(weight=P + 2) == EALIGN and f(targets=P + 4) == EALIGN
        assert f(scratch=_Scratch(1 << 30, 16 * P + 128)) == EALIGN
        assert f(scratch=_Scratch(64)) == ENOWORKSPACE
    assert _head(loss=None) == EINVAL
    assert _head(desc(0, 100, 64), hidden=None, targets=None) == 0
    assert _head_grad(dhidden=None, dweight=None) == EINVAL
    assert _head_grad(desc(4, 100, 64, dhidden_dtype=3)) == EINVAL and _head_grad(desc(4, 100, 64, dweight_dtype=-1)) == EINVAL
    assert _head_grad(dhidden=P) == EINVAL and _head_grad(dweight=2 * P + 128) == EINVAL and _head_grad(dweight=6 * P) == EINVAL
    assert _head(lse=4 * P) == EINVAL and _head(loss=3 * P + 8) == EINVAL
    assert _head_grad(dhidden=5 * P) == EINVAL and _head_grad(dweight=3 * P) == EINVAL and _head_grad(dloss=9 * P, dweight=9 * P) == EINVAL
    assert _head_grad(desc(0, 100, 64, accumulate=1), hidden=None) == 0
    assert A.load().adapm_head_loss_scratch_bytes(None, 0) == 0 and A.adapm_head_loss_scratch_bytes(desc(4, 100, 60), True) == 0
    st = C.c_int32()
    assert A.load().adapm_head_loss_status(None, 0, C.byref(st)) == EINVAL
    assert A.load().adapm_head_loss_forward(None, P, P, P, P, P, P, 1 << 30, 0) == EINVAL


def test_good_arguments_need_a_device():
    if not _no_device():
        pytest.skip("a CUDA device is present")
    assert _dropout() == ECUDA and _norm() == ECUDA and _norm_grad() == ECUDA and _head() == ECUDA and _head_grad() == ECUDA


def test_scratch_holds_two_pieces_and_no_more():
    """The gradient's scratch stays near two pieces of 64 M elements however large the vocabulary is."""
    for tokens, vocab in ((8192, 50257), (8192, 128256), (100, 128256)):
        n = A.adapm_head_loss_scratch_bytes(A.head_loss_desc(tokens, vocab, 1600), True)
        fixed = tokens * 1600 * 6 + (1 << 22)
        assert n <= 2 * 2 * (64 << 20) + fixed
    assert A.adapm_head_loss_scratch_bytes(A.head_loss_desc(8192, 50257, 1600), False) < (1 << 26)


@pytest.mark.parametrize("struct,first", [("adapm_rmsnorm", "int64_t rows, cols;      /* cols"), ("adapm_head_loss", "int64_t tokens")])
def test_descriptors_match_the_header(struct, first, tmp_path):
    """Field by field, with the compiler's own offsets."""
    cls = getattr(A, struct)
    src = tmp_path / "offsets.c"
    src.write_text('#include <stdio.h>\n#include "adapm.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu ", offsetof({struct}, {f}));\n' for f, _ in cls._fields_) +
                   f'  printf("%zu\\n", sizeof({struct}));\n  return 0;\n}}\n')
    exe = str(tmp_path / "offsets")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    want = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert want == [getattr(cls, f).offset for f, _ in cls._fields_] + [C.sizeof(cls)]
