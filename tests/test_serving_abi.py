"""Refusals of the 8-bit products, the exit logits and sampling, without a GPU:
pointers are fake device addresses that validation only compares and aligns."""

import os

import pytest
import torch

from paper_2402_00518_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH),
                                reason="libeetune.so not built (run __graft_entry__.build())")

GB = 1 << 30
A, BB, C, X, WS = (i << 40 for i in range(1, 6))


def expect(status, code, needle):
    assert status == code, (status, B.ee_last_error())
    assert needle in B.ee_last_error(), B.ee_last_error()


def mat(base, rows=100, cols=256, block_rows=1, dtype=B.EE_E4M3, ld=None, scale_ld=None, **kw):
    m = B.make_scaled(base, base + GB, block_rows, dtype, rows=rows, cols=cols, ld=-(-cols // 16) * 16 if ld is None else ld,
                      scale_ld=-(-rows // max(block_rows, 1)) if scale_ld is None else scale_ld)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


BAD_MATRIX = [
    (dict(dtype=B.EE_BF16), B.EE_ERR_DTYPE, "8-bit"),
    (dict(dtype=9), B.EE_ERR_DTYPE, "8-bit"),
    (dict(block_rows=64), B.EE_ERR_SHAPE, "block_rows"),
    (dict(block_rows=0), B.EE_ERR_SHAPE, "block_rows"),
    (dict(rows=0), B.EE_ERR_SHAPE, "rows"),
    (dict(rows=(1 << 20) + 1), B.EE_ERR_SHAPE, "rows"),
    (dict(cols=-1), B.EE_ERR_SHAPE, "cols"),
    (dict(ld=255), B.EE_ERR_SHAPE, "ld"),
    (dict(ld=264), B.EE_ERR_SHAPE, "ld"),
    (dict(ld=240), B.EE_ERR_SHAPE, "ld"),
    (dict(ld=1 << 23), B.EE_ERR_SHAPE, "ld"),
    (dict(scale_ld=0), B.EE_ERR_SHAPE, "scale_ld"),
    (dict(data=None), B.EE_ERR_NULL, "NULL"),
    (dict(scale=None), B.EE_ERR_NULL, "NULL"),
    (dict(data=A + 8), B.EE_ERR_ALIGN, "aligned"),
    (dict(scale=A + GB + 4), B.EE_ERR_ALIGN, "aligned"),
]


@pytest.mark.parametrize("kw,code,needle", BAD_MATRIX)
def test_bad_matrices(kw, code, needle):
    expect(B.ee_scaled_matmul(mat(A, **kw), mat(BB), C, B.EE_F32, 4096, 0, None, check=False), code, needle)
    expect(B.ee_scaled_matmul(mat(BB), mat(A, **kw), C, B.EE_F32, 4096, 0, None, check=False), code, needle)
    expect(B.ee_quantize_blocks(X, B.EE_F32, 100, 256, 256, mat(A, **kw), None, None, check=False), code, needle)
    expect(B.ee_quantize_blocks(X, B.EE_F32, 256, 100, 100, None, mat(A, **kw), None, check=False), code, needle)


@pytest.mark.parametrize("kw,code,needle", [
    (dict(a=None), B.EE_ERR_NULL, "a is NULL"),
    (dict(b=None), B.EE_ERR_NULL, "b is NULL"),
    (dict(b=mat(BB, dtype=B.EE_E5M2)), B.EE_ERR_DTYPE, "b must be"),
    (dict(b=mat(BB, cols=272)), B.EE_ERR_SHAPE, "columns"),
    (dict(c_dtype=B.EE_E4M3), B.EE_ERR_DTYPE, "c_dtype"),
    (dict(accumulate=2), B.EE_ERR_SHAPE, "accumulate"),
    (dict(accumulate=1, c_dtype=B.EE_BF16), B.EE_ERR_UNSUPPORTED, "accumulate"),
    (dict(ldc=99), B.EE_ERR_SHAPE, "ldc"),
    (dict(c=None), B.EE_ERR_NULL, "c is NULL"),
    (dict(c=C + 4), B.EE_ERR_ALIGN, "c is not"),
    (dict(c=A + 4096), B.EE_ERR_ALIAS, "codes"),
    (dict(c=BB + GB), B.EE_ERR_ALIAS, "scales"),
])
def test_bad_products(kw, code, needle):
    a = dict(a=mat(A), b=mat(BB), c=C, c_dtype=B.EE_F32, ldc=100, accumulate=0, stream=None)
    a.update(kw)
    expect(B.ee_scaled_matmul(check=False, **a), code, needle)


@pytest.mark.parametrize("kw,code,needle", [
    (dict(x_dtype=B.EE_E4M3), B.EE_ERR_DTYPE, "x_dtype"),
    (dict(rows=0), B.EE_ERR_SHAPE, "rows"),
    (dict(cols=(1 << 20) + 1), B.EE_ERR_SHAPE, "cols"),
    (dict(ldx=199), B.EE_ERR_SHAPE, "ldx"),
    (dict(x=None), B.EE_ERR_NULL, "x is NULL"),
    (dict(x=X + 2), B.EE_ERR_ALIGN, "x is not"),
    (dict(q=None, qt=None), B.EE_ERR_NULL, "both"),
    (dict(q=mat(A, 99, 200)), B.EE_ERR_SHAPE, "q is"),
    (dict(q=mat(A, 100, 199)), B.EE_ERR_SHAPE, "q is"),
    (dict(q=mat(A, 100, 209)), B.EE_ERR_SHAPE, "q is"),
    (dict(qt=mat(BB, 100, 200)), B.EE_ERR_SHAPE, "qt is"),
    (dict(qt=mat(BB, 200, 113)), B.EE_ERR_SHAPE, "qt is"),
    (dict(x=A + 64), B.EE_ERR_ALIAS, "x"),
    (dict(qt=mat(A + 4096, 200, 100)), B.EE_ERR_ALIAS, "codes"),
])
def test_bad_quantizing(kw, code, needle):
    a = dict(x=X, x_dtype=B.EE_BF16, rows=100, cols=200, ldx=200, q=mat(A, 100, 200), qt=mat(BB, 200, 100), stream=None)
    a.update(kw)
    expect(B.ee_quantize_blocks(check=False, **a), code, needle)


def norm_exit(h=256, V=1000, w_out=A, kind=B.EE_EXIT_NORM, I=0):
    return B.make_exit(kind, B.EE_BF16, h, V, I, 1e-5, w_out=w_out, gamma=A + 2 * GB, gamma_mlp=A + 3 * GB, w_gate=A + 4 * GB,
                       w_up=A + 5 * GB, w_down=A + 6 * GB)


def exit_logits(**kw):
    a = dict(e=norm_exit(), w_out=None, hidden=X, n_rows=10, logits=C, logits_dtype=B.EE_F32, ld=1000, ws=WS, ws_bytes=GB, stream=None)
    a.update(kw)
    return B.ee_exit_logits(check=False, **a)


@pytest.mark.parametrize("kw,code,needle", [
    (dict(e=None), B.EE_ERR_NULL, "descriptor"),
    (dict(e=norm_exit(w_out=None)), B.EE_ERR_NULL, "w_out"),
    (dict(e=norm_exit(h=100)), B.EE_ERR_SHAPE, "hidden"),
    (dict(e=norm_exit(kind=B.EE_EXIT_LAYER)), B.EE_ERR_UNSUPPORTED, "Layer"),
    (dict(w_out=mat(BB, 1000, 256, 128, dtype=B.EE_E5M2)), B.EE_ERR_DTYPE, "E4M3"),
    (dict(w_out=mat(BB, 999, 256, 128)), B.EE_ERR_SHAPE, "the exit's is"),
    (dict(w_out=mat(BB, 1000, 320, 128)), B.EE_ERR_SHAPE, "the exit's is"),
    (dict(w_out=mat(BB, 1000, 256, 128, data=BB + 1)), B.EE_ERR_ALIGN, "w_out"),
    (dict(n_rows=0), B.EE_ERR_SHAPE, "n_rows"),
    (dict(logits_dtype=B.EE_E5M2), B.EE_ERR_DTYPE, "logits_dtype"),
    (dict(ld=999), B.EE_ERR_SHAPE, "ld"),
    (dict(hidden=None), B.EE_ERR_NULL, "hidden"),
    (dict(logits=None), B.EE_ERR_NULL, "logits"),
    (dict(logits=C + 8), B.EE_ERR_ALIGN, "logits"),
    (dict(ws=None), B.EE_ERR_NULL, "workspace"),
    (dict(ws_bytes=16), B.EE_ERR_WORKSPACE, "workspace"),
    (dict(logits=X), B.EE_ERR_ALIAS, "hidden"),
    (dict(logits=A), B.EE_ERR_ALIAS, "w_out"),
    (dict(ws=C), B.EE_ERR_ALIAS, "workspace"),
    (dict(e=norm_exit(w_out=None), w_out=mat(BB, 1000, 256, 128), logits=BB), B.EE_ERR_ALIAS, "codes"),
])
def test_bad_logits(kw, code, needle):
    expect(exit_logits(**kw), code, needle)


def test_logits_workspace():
    e, w = norm_exit(), mat(BB, 1000, 256, 128)
    assert B.ee_logits_workspace_bytes(e, None, 10) < B.ee_logits_workspace_bytes(e, None, 1000)
    assert B.ee_logits_workspace_bytes(norm_exit(w_out=None), w, 100) >= 100 * (256 + 8)
    m = norm_exit(kind=B.EE_EXIT_MLP, I=512)
    assert B.ee_logits_workspace_bytes(m, w, 10) > B.ee_logits_workspace_bytes(m, None, 10)
    for n in (0, (1 << 20) + 1):
        with pytest.raises(B.EEError, match="n_rows"):
            B.ee_logits_workspace_bytes(e, None, n)
    # no workspace byte is needed past what is asked for: one less is refused, that much is not
    need = B.ee_logits_workspace_bytes(e, w, 10)
    expect(exit_logits(w_out=w, ws_bytes=need - 1), B.EE_ERR_WORKSPACE, "workspace")


def sample(**kw):
    a = dict(logits=X, dtype=B.EE_F32, n_rows=10, vocab=1000, ld=1000, allowed=None, allowed_ld=0, sampling=None, uniform=A, threshold=0.5,
             token=C, prob=C + GB, confidence=C + 2 * GB, exit_flag=C + 3 * GB, ws=WS, ws_bytes=GB, stream=None)
    a.update(kw)
    return B.ee_sample(check=False, **a)


@pytest.mark.parametrize("kw,code,needle", [
    (dict(dtype=B.EE_E4M3), B.EE_ERR_DTYPE, "dtype"),
    (dict(n_rows=0), B.EE_ERR_SHAPE, "n_rows"),
    (dict(vocab=0), B.EE_ERR_SHAPE, "vocab"),
    (dict(vocab=(1 << 20) + 1), B.EE_ERR_SHAPE, "vocab"),
    (dict(ld=999), B.EE_ERR_SHAPE, "ld"),
    (dict(allowed=BB, allowed_ld=31), B.EE_ERR_SHAPE, "allowed_ld"),
    (dict(allowed=BB + 4, allowed_ld=32), B.EE_ERR_ALIGN, "allowed"),
    (dict(threshold=float("nan")), B.EE_ERR_SHAPE, "threshold"),
    (dict(logits=None), B.EE_ERR_NULL, "logits"),
    (dict(uniform=None), B.EE_ERR_NULL, "uniform"),
    (dict(token=None), B.EE_ERR_NULL, "token"),
    (dict(logits=X + 4), B.EE_ERR_ALIGN, "logits"),
    (dict(prob=C + GB + 4), B.EE_ERR_ALIGN, "prob"),
    (dict(sampling=B.make_sampling(top_p=BB + 8)), B.EE_ERR_ALIGN, "top_p"),
    (dict(ws=None), B.EE_ERR_NULL, "workspace"),
    (dict(ws_bytes=0), B.EE_ERR_WORKSPACE, "workspace"),
    (dict(prob=C), B.EE_ERR_ALIAS, "token"),
    (dict(token=X + 64), B.EE_ERR_ALIAS, "logits"),
    (dict(exit_flag=A), B.EE_ERR_ALIAS, "uniform"),
    (dict(sampling=B.make_sampling(temperature=C)), B.EE_ERR_ALIAS, "temperature"),
    (dict(allowed=C + GB, allowed_ld=32), B.EE_ERR_ALIAS, "allowed"),
])
def test_bad_sampling(kw, code, needle):
    expect(sample(**kw), code, needle)


def test_sample_workspace():
    assert B.ee_sample_workspace_bytes(1, 1) > 0
    for n, v in ((0, 10), (10, 0), (10, (1 << 20) + 1)):
        with pytest.raises(B.EEError):
            B.ee_sample_workspace_bytes(n, v)


def test_strided_tensors_are_refused():
    q, s = torch.zeros(32, 64, dtype=torch.uint8), torch.zeros(2, 4)
    assert B.make_scaled(q, s).ld == 64
    for data, scale in ((q.t(), s), (q[:, ::2], s), (q, s.t())):
        with pytest.raises(ValueError):
            B.make_scaled(data, scale)
