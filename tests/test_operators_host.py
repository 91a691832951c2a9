"""What the calls around the vocabulary (verification of drafts, embedding, 8-bit values) refuse, on the host.  No device call is made:
every argument list below is rejected, or a no-op, before one."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def e3():
    from paper_2505_18573_b200 import build, binding
    build.build()
    binding.lib()
    return binding


P = 1 << 20  # an aligned address that nothing reads


def _verify(e3, **change):
    a = dict(logits=P, dt=e3.E3_F32, n_seq=2, max_draft=3, V=1000, row_stride=1000, temps=P, draft_tok=P, draft_len=None, draft_logits=None,
             draft_stride=0, draft_temps=None, draft_logp=None, uniforms=P, uniform_stride=8, out_tok=P, out_kept=P, out_logp=P, out_ent=P,
             workspace=P, workspace_bytes=1 << 20, stream=None)
    assert set(change) <= set(a)
    return e3.lib().e3_verify_drafts(*{**a, **change}.values())


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), "DTYPE"), (dict(n_seq=-1), "INVALID_ARG"), (dict(max_draft=-1), "INVALID_ARG"), (dict(V=0), "INVALID_ARG"),
    (dict(V=1 << 31, row_stride=1 << 31), "INVALID_ARG"), (dict(row_stride=999), "INVALID_ARG"), (dict(logits=None), "INVALID_ARG"),
    (dict(temps=None), "INVALID_ARG"), (dict(uniforms=None), "INVALID_ARG"), (dict(uniform_stride=7), "INVALID_ARG"),
    (dict(out_tok=None), "INVALID_ARG"), (dict(out_kept=None), "INVALID_ARG"), (dict(draft_tok=None), "INVALID_ARG"),
    (dict(draft_logits=P, draft_stride=999, draft_logp=P), "INVALID_ARG"), (dict(draft_logits=P, draft_stride=1000), "INVALID_ARG"),
    (dict(n_seq=1 << 25), "INVALID_ARG"), (dict(logits=P + 2), "ALIGNMENT"), (dict(uniforms=P + 4), "ALIGNMENT"),
    (dict(draft_tok=P + 1), "ALIGNMENT"), (dict(out_logp=P + 2), "ALIGNMENT"), (dict(workspace=P + 8), "ALIGNMENT"),
    (dict(workspace=None), "WORKSPACE"), (dict(workspace_bytes=64), "WORKSPACE"), (dict(n_seq=0, logits=None), None)])
def test_verify_drafts_refuses(e3, change, status):
    assert _verify(e3, **change) == (0 if status is None else getattr(e3, "E3_ERR_" + status))


def test_verify_workspace_grows_with_the_rows(e3):
    size = [e3.e3_workspace_bytes(e3.E3_CALL_VERIFY_DRAFTS, n, 1000) for n in (0, 1, 5, 2560)]
    assert size == sorted(size) and size[-1] >= 2560 * 8


@pytest.mark.parametrize("change, status", [
    (dict(dt=7), "DTYPE"), (dict(n=-1), "INVALID_ARG"), (dict(V=0), "INVALID_ARG"), (dict(D=0), "INVALID_ARG"), (dict(table_stride=15), "INVALID_ARG"),
    (dict(out_stride=15), "INVALID_ARG"), (dict(tok=None), "INVALID_ARG"), (dict(table=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"),
    (dict(tok=P + 2), "ALIGNMENT"), (dict(table=P + 1), "ALIGNMENT"), (dict(out=P + 1), "ALIGNMENT"), (dict(n=0, tok=None), None)])
def test_embed_refuses(e3, change, status):
    a = dict(tok=P, n=4, table=P, dt=e3.E3_BF16, V=10, D=16, table_stride=16, scale=C.c_float(1.0), out=P, out_stride=16, stream=None)
    assert e3.lib().e3_embed_tokens(*{**a, **change}.values()) == (0 if status is None else getattr(e3, "E3_ERR_" + status))


@pytest.mark.parametrize("change, status", [
    (dict(dt=7), "DTYPE"), (dict(table_dt=7), "DTYPE"), (dict(n=-1), "INVALID_ARG"), (dict(n=1 << 31), "INVALID_ARG"), (dict(V=0), "INVALID_ARG"),
    (dict(V=(1 << 22) + 1), "INVALID_ARG"), (dict(D=0), "INVALID_ARG"), (dict(D=64 * 65535 + 1, g_stride=1 << 22, dtable_stride=1 << 22), "INVALID_ARG"),
    (dict(D=1 << 22, g_stride=1 << 22, dtable_stride=1 << 22), "INVALID_ARG"),
    (dict(g_stride=15), "INVALID_ARG"), (dict(dtable_stride=15), "INVALID_ARG"), (dict(tok=None), "INVALID_ARG"), (dict(g=None), "INVALID_ARG"),
    (dict(dtable=None), "INVALID_ARG"), (dict(g=P + 1), "ALIGNMENT"), (dict(dtable=P + 2), "ALIGNMENT"), (dict(workspace=P + 4), "ALIGNMENT"),
    (dict(workspace=None), "WORKSPACE"), (dict(workspace_bytes=16), "WORKSPACE"), (dict(n=0, accumulate=1, dtable=None), None)])
def test_embed_backward_refuses(e3, change, status):
    a = dict(tok=P, n=4, g=P, dt=e3.E3_BF16, V=10, D=16, g_stride=16, scale=C.c_float(1.0), dtable=P, table_dt=e3.E3_F32, dtable_stride=16,
             accumulate=0, workspace=P, workspace_bytes=1 << 20, stream=None)
    assert e3.lib().e3_embed_tokens_backward(*{**a, **change}.values()) == (0 if status is None else getattr(e3, "E3_ERR_" + status))


def test_embed_workspace(e3):
    assert e3.e3_embed_workspace_bytes(0, 10, 16) == 0 and e3.e3_embed_workspace_bytes(4, (1 << 22) + 1, 16) == 0
    # keys and places of every token, first places of the vocabulary
    assert e3.e3_embed_workspace_bytes(131072, 151936, 1536) >= 16 * 131072 + 4 * 151937


@pytest.mark.parametrize("change, status", [
    (dict(dt=7), "DTYPE"), (dict(rows=-1), "INVALID_ARG"), (dict(cols=0), "INVALID_ARG"), (dict(row_stride=299), "INVALID_ARG"),
    (dict(block_rows=2), "INVALID_ARG"), (dict(q_stride=299), "INVALID_ARG"), (dict(scale_stride=2), "INVALID_ARG"), (dict(x=None), "INVALID_ARG"),
    (dict(q=None), "INVALID_ARG"), (dict(scale=None), "INVALID_ARG"), (dict(x=P + 2), "ALIGNMENT"), (dict(scale=P + 2), "ALIGNMENT"),
    (dict(rows=0, x=None), None)])
def test_quantize_refuses(e3, change, status):
    a = dict(x=P, dt=e3.E3_F32, rows=4, cols=300, row_stride=300, block_rows=1, q=P, q_stride=304, scale=P, scale_stride=3, stream=None)
    assert e3.lib().e3_quantize(*{**a, **change}.values()) == (0 if status is None else getattr(e3, "E3_ERR_" + status))


@pytest.mark.parametrize("change, status", [
    (dict(dt=7), "DTYPE"), (dict(rows=-1), "INVALID_ARG"), (dict(V=0), "INVALID_ARG"), (dict(D=0), "INVALID_ARG"), (dict(x_stride=192), "INVALID_ARG"),
    (dict(w_stride=192), "INVALID_ARG"), (dict(x_scale_stride=1), "INVALID_ARG"), (dict(w_scale_stride=1), "INVALID_ARG"),
    (dict(row_stride=499), "INVALID_ARG"), (dict(V=1 << 31, row_stride=1 << 31), "INVALID_ARG"), (dict(x=None), "INVALID_ARG"),
    (dict(x_scale=None), "INVALID_ARG"), (dict(w=None), "INVALID_ARG"), (dict(w_scale=None), "INVALID_ARG"), (dict(logits=None), "INVALID_ARG"),
    (dict(x=P + 8), "ALIGNMENT"), (dict(w=P + 8), "ALIGNMENT"), (dict(x_stride=216), "ALIGNMENT"), (dict(w_stride=216), "ALIGNMENT"),
    (dict(x_scale=P + 2), "ALIGNMENT"), (dict(logits=P + 1), "ALIGNMENT"), (dict(out_status=P + 2), "ALIGNMENT"), (dict(rows=0, x=None), None)])
def test_project_refuses(e3, change, status):
    a = dict(x=P, x_scale=P, rows=3, x_stride=208, x_scale_stride=2, w=P, w_scale=P, V=500, w_stride=208, w_scale_stride=2, D=200, logits=P,
             dt=e3.E3_BF16, row_stride=500, out_status=None, stream=None)
    assert e3.lib().e3_project_vocab(*{**a, **change}.values()) == (0 if status is None else getattr(e3, "E3_ERR_" + status))
