"""Refusals of the rotary and attention calls: host-side checks, no device is touched."""
import ctypes as C

import pytest

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
PTR = 1 << 20            # an aligned address that a refused call never reads


@pytest.fixture(scope="module")
def B():
    import __graft_entry__ as ge
    ge.build()
    from paper_2404_15159_b200 import binding
    return binding


def test_struct_layouts(B):
    assert C.sizeof(B.mixlora_rope_shape_t) == 40 + 32
    assert C.sizeof(B.mixlora_attention_shape_t) == 56 + 32
    assert C.sizeof(B.mixlora_attention_mask_t) == 40


def rope(B, q=PTR, k=PTR, pos=PTR, w=PTR, qo=2 * PTR, ko=2 * PTR, **edit):
    s = B.make_rope_shape(edit.pop("tokens", 4), 4, 2, 64, 32)
    for n, v in edit.items():
        setattr(s, n, v)
    return [f(C.byref(s), q, k, pos, w, qo, ko, None) for f in (B.lib.mixlora_rope_forward, B.lib.mixlora_rope_backward)]


@pytest.mark.parametrize("edit,status", [
    (dict(struct_size=3), INVALID), (dict(tokens=-1), INVALID), (dict(q_heads=0), INVALID), (dict(k_heads=-1), INVALID),
    (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=520), UNSUPPORTED), (dict(rotary_dim=31), INVALID),
    (dict(rotary_dim=0), INVALID), (dict(rotary_dim=66), INVALID), (dict(layout=2), INVALID), (dict(dtype=5), INVALID),
    (dict(amplitude=float("nan")), INVALID), (dict(reserved=1), INVALID), (dict(q_stride=8), INVALID),
    (dict(k_stride=132), UNSUPPORTED), (dict(q_out_stride=-256), INVALID), (dict(q=None), INVALID), (dict(q=PTR + 8), INVALID),
    (dict(k=None), INVALID), (dict(ko=None), INVALID), (dict(w=None), INVALID), (dict(w=PTR + 4), INVALID),
    (dict(pos=PTR + 2), INVALID), (dict(qo=PTR, q_stride=512), INVALID)])
def test_rope_refusals(B, edit, status):
    assert rope(B, **edit) == [status] * 2


def test_rope_without_tokens_needs_no_device(B):
    assert rope(B, tokens=0) == [OK] * 2
    assert rope(B, tokens=0, k=None, ko=None, k_heads=0) == [OK] * 2


@pytest.mark.parametrize("args", [(3, 1e4, 0, 1, 0, 0, 0, PTR), (0, 1e4, 0, 1, 0, 0, 0, PTR), (64, 0.0, 0, 1, 0, 0, 0, PTR),
                                  (64, 1e4, 0, 0.0, 0, 0, 0, PTR), (64, 1e4, 4, 1, 0, 0, 0, PTR), (64, 1e4, 0, 1, 0, 0, 0, None),
                                  (64, 1e4, 3, 2, 4, 4, 8192, PTR), (64, 1e4, 3, 2, 1, 4, 0, PTR),
                                  (64, float("inf"), 0, 1, 0, 0, 0, PTR), (64, 1e4, 3, 2, float("nan"), 4, 8192, PTR)])
def test_frequency_refusals(B, args):
    assert B.lib.mixlora_rope_frequencies(*args, None) == INVALID
    assert B.lib.mixlora_rope_frequencies(514, 1e4, 0, 1, 0, 0, 0, PTR, None) == UNSUPPORTED


def attention(B, drop=(), ws=PTR, ws_bytes=1 << 40, mask_edit=None, at=None, **edit):
    s = B.make_attention_shape(2, 16, 16, 4, 2, 64)
    for n, v in edit.items():
        setattr(s, n, v)
    m = B.make_attention_mask(PTR, PTR)
    for n, v in (mask_edit or {}).items():
        setattr(m, n, v)
    p = {n: PTR for n in ("q", "k", "v", "o", "lse", "d_o", "d_q", "d_k", "d_v")}
    p.update({n: None for n in drop})
    p.update(at or {})
    f = B.lib.mixlora_attention_forward(C.byref(s), C.byref(m), p["q"], p["k"], p["v"], p["o"], p["lse"], ws, ws_bytes, None)
    b = B.lib.mixlora_attention_backward(C.byref(s), C.byref(m), p["q"], p["k"], p["v"], p["o"], p["lse"], p["d_o"], ws,
                                         ws_bytes, p["d_q"], p["d_k"], p["d_v"], None)
    return f, b, B.lib.mixlora_attention_workspace_bytes(C.byref(s), 0), B.lib.mixlora_attention_workspace_bytes(C.byref(s), 1)


@pytest.mark.parametrize("edit,status", [
    (dict(struct_size=1), INVALID), (dict(n_seqs=-1), INVALID), (dict(q_rows=-1), INVALID), (dict(k_rows=-1), INVALID),
    (dict(max_q_len=-1), INVALID), (dict(max_k_len=-1), INVALID), (dict(q_heads=0), INVALID), (dict(kv_heads=0), INVALID),
    (dict(q_heads=3), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED),
    (dict(dtype=2), INVALID), (dict(causal=2), INVALID), (dict(window=-1), INVALID), (dict(scale=0.0), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(softcap=-1.0), INVALID),
    (dict(softcap=float("nan")), INVALID), (dict(softcap=1e-42, scale=1e3), INVALID), (dict(q_stride=8), INVALID), (dict(k_stride=-128), INVALID),
    (dict(v_stride=132), UNSUPPORTED), (dict(o_stride=260), UNSUPPORTED), (dict(q_rows=2 ** 30 + 1), UNSUPPORTED),
    (dict(k_rows=2 ** 30 + 1), UNSUPPORTED)])
def test_attention_shape_refusals(B, edit, status):
    f, b, wf, wb = attention(B, **edit)
    assert (f, b, wf, wb) == (status, status, 0, 0)


def test_attention_pointer_and_workspace_refusals(B):
    for n in ("q", "k", "v", "o"):
        assert attention(B, drop=[n])[:2] == (INVALID, INVALID)
        assert attention(B, at={n: PTR + 8})[:2] == (INVALID, INVALID)
    for n in ("d_o", "d_q", "d_k", "d_v"):
        s = B.make_attention_shape(2, 16, 16, 4, 2, 64)
        m = B.make_attention_mask(PTR, PTR)
        p = {x: PTR for x in ("d_o", "d_q", "d_k", "d_v")}
        p[n] = None
        assert B.lib.mixlora_attention_backward(C.byref(s), C.byref(m), PTR, PTR, PTR, PTR, PTR, p["d_o"], PTR, 1 << 40,
                                                p["d_q"], p["d_k"], p["d_v"], None) == INVALID
        assert B.lib.mixlora_attention_backward(C.byref(s), C.byref(m), PTR, PTR, PTR, PTR, None, PTR, PTR, 1 << 40,
                                                PTR, PTR, PTR, None) == INVALID
    for edit in (dict(q_off=None), dict(k_off=None), dict(k_len=PTR + 2), dict(prefix=PTR + 1), dict(slopes=PTR + 2)):
        assert attention(B, mask_edit=edit)[:2] == (INVALID, INVALID)
    need_f, need_b = attention(B, ws=None)[2:]
    assert 0 < need_f <= need_b
    assert attention(B, ws=None)[:2] == (WORKSPACE, WORKSPACE)
    assert attention(B, ws=PTR + 16)[:2] == (WORKSPACE, WORKSPACE)
    assert attention(B, ws_bytes=need_f - 1)[:2] == (WORKSPACE, WORKSPACE)


def test_decoding_workspace_holds_the_partials_of_a_split(B):
    s = B.make_attention_shape(1, 1, 100000, 8, 1, 128, max_q_len=1)
    plain = B.make_attention_shape(1, 1, 100000, 8, 1, 128)
    size = lambda x: B.lib.mixlora_attention_workspace_bytes(C.byref(x), 0)  # noqa: E731
    assert size(s) > size(plain) > 0
