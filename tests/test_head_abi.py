"""Refusals of the head's losses: host-side checks, no device is touched."""
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


def call(B, top=0, x=PTR, w=2 * PTR, target=3 * PTR, logit=4 * PTR, t_lse=None, weights=None, norm=None, loss=5 * PTR,
         lse=None, totals=None, d_x=6 * PTR, ws=7 * PTR, ws_bytes=None, **edit):
    s = B.make_head_shape(edit.pop("tokens", 4), edit.pop("d_model", 64), edit.pop("vocab", 100), teacher_top=top)
    for n, v in edit.items():
        setattr(s, n, v)
    need = B.lib.mixlora_head_workspace_bytes(C.byref(s), 1)
    tail = [weights, norm, loss, lse, totals, d_x, ws, 1 << 40 if ws_bytes is None else ws_bytes(need), None]
    if top or edit.get("teacher_top"):
        return B.lib.mixlora_head_distill(C.byref(s), x, w, target, logit, t_lse, *tail)
    return B.lib.mixlora_head_loss(C.byref(s), x, w, target, *tail)


def test_struct_layout(B):
    assert C.sizeof(B.mixlora_head_shape_t) == 72


BAD = [
    (dict(struct_size=3), INVALID), (dict(tokens=-1), INVALID), (dict(d_model=0), INVALID), (dict(vocab=0), INVALID),
    (dict(vocab=-5), INVALID), (dict(dtype=2), INVALID), (dict(reserved=1), INVALID), (dict(scale=0.0), INVALID),
    (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(softcap=-1.0), INVALID), (dict(softcap=float("inf")), INVALID), (dict(temperature=0.0), INVALID),
    (dict(temperature=float("nan")), INVALID), (dict(z_loss=-1.0), INVALID), (dict(z_loss=float("inf")), INVALID), (dict(z_loss=2e6), INVALID), (dict(z_loss=float("nan")), INVALID),
    (dict(scale=1e-30, temperature=1e20), INVALID), (dict(scale=1e30, temperature=1e-20), INVALID),
    (dict(softcap=1e-30, scale=1e20), INVALID), (dict(softcap=1e30, temperature=1e-20), INVALID),
    (dict(x_stride=32), INVALID), (dict(w_stride=-64), INVALID), (dict(d_x_stride=8), INVALID),
    (dict(x_stride=68), UNSUPPORTED), (dict(d_model=60), UNSUPPORTED), (dict(d_model=65544), UNSUPPORTED),
    (dict(vocab=(1 << 20) + 1), UNSUPPORTED), (dict(tokens=(1 << 24) + 1), UNSUPPORTED),
    (dict(w_stride=(1 << 32) + 8), UNSUPPORTED),
    (dict(x=None), INVALID), (dict(x=PTR + 8), INVALID), (dict(w=None), INVALID), (dict(w=PTR + 2), INVALID),
    (dict(target=None), INVALID), (dict(target=PTR + 2), INVALID), (dict(weights=PTR + 2), INVALID),
    (dict(norm=PTR + 1), INVALID), (dict(loss=None), INVALID), (dict(loss=PTR + 2), INVALID), (dict(lse=PTR + 2), INVALID),
    (dict(totals=PTR + 2), INVALID), (dict(d_x=PTR + 4), INVALID), (dict(d_x=PTR), INVALID),
    (dict(ws=None), WORKSPACE), (dict(ws=PTR + 128), WORKSPACE), (dict(ws_bytes=lambda n: n - 1), WORKSPACE)]


@pytest.mark.parametrize("edit,status", BAD)
def test_refusals_of_both(B, edit, status):
    assert call(B, **edit) == status
    assert call(B, top=3, **edit) == status


def test_refusals_of_lists(B):
    assert call(B, top=-1) == INVALID
    assert call(B, top=257) == UNSUPPORTED
    assert call(B, top=3, logit=None) == INVALID
    assert call(B, top=3, logit=PTR + 2) == INVALID
    assert call(B, top=3, t_lse=PTR + 2) == INVALID
    s = B.make_head_shape(4, 64, 100, teacher_top=3)          # lists given to the form for labels, and the other way round
    assert B.lib.mixlora_head_loss(C.byref(s), PTR, PTR, PTR, None, None, PTR, None, None, None, PTR, 1 << 40, None) == INVALID
    s = B.make_head_shape(4, 64, 100)
    assert B.lib.mixlora_head_distill(C.byref(s), PTR, PTR, PTR, PTR, None, None, None, PTR, None, None, None, PTR, 1 << 40,
                                      None) == INVALID
    assert B.lib.mixlora_head_loss(None, PTR, PTR, PTR, None, None, PTR, None, None, None, PTR, 1 << 40, None) == INVALID


def test_workspace_is_bounded_by_the_piece(B):
    size = lambda s, g: B.lib.mixlora_head_workspace_bytes(C.byref(s), g)  # noqa: E731
    assert size(B.make_head_shape(4, 60, 100), 1) == 0
    for dtype in (B.MIXLORA_DTYPE_BF16, B.MIXLORA_DTYPE_FP32):
        for vocab in (1, 32000, 131072, 1 << 20):
            few, many = (size(B.make_head_shape(t, 1024, vocab, dtype), 1) for t in (1 << 19, 1 << 20))
            parts = 0 if dtype == B.MIXLORA_DTYPE_BF16 else 6 * vocab * 1024      # the fp32 head taken apart
            assert few - parts < 2.7e9 and many - few <= 32 * (1 << 19)      # a few numbers a token
    # a teacher's entries and their probabilities, 12 bytes each, are what grows with them
    lists = B.make_head_shape(1 << 20, 64, 2, teacher_top=256)
    assert size(lists, 1) < 12.1 * (256 << 20) + 2e9
    assert size(B.make_head_shape(8192, 4096, 32000), 0) < size(B.make_head_shape(8192, 4096, 32000), 1)


@pytest.mark.parametrize("d", [8, 512, 520, 4096, 65536])
@pytest.mark.parametrize("vocab", [1, 512, 520, 2048, 32000, 1 << 20])
@pytest.mark.parametrize("top", [0, 64, 256])
def test_workspace_is_what_the_header_says(B, d, vocab, top):
    # rows of x, exponentials and listed logits may each come to 512 MiB, where a row of each has about the same size
    t = 1 << 22
    for dtype, most in ((B.MIXLORA_DTYPE_BF16, 1.7e9), (B.MIXLORA_DTYPE_FP32, 1.8e9 + 6 * vocab * d)):
        for grad in (0, 1):
            got = B.lib.mixlora_head_workspace_bytes(C.byref(B.make_head_shape(t, d, vocab, dtype, teacher_top=top)), grad)
            assert 0 < got <= most + 9 * t + (12 * top + 12 if top else 0) * t


def test_the_binding_raises(B):
    import torch
    with pytest.raises(B.MixLoraError) as e:
        B.alloc_head_workspace(B.make_head_shape(4, 60, 100), True, device="cpu")
    assert e.value.status == 1
    s = B.make_head_shape(4, 64, 100)
    x = torch.zeros(4, 64)
    with pytest.raises(B.MixLoraError) as e:
        B.mixlora_head_loss(s, x, x, None, None, None, x, None, None, None, None, stream=0)
    assert e.value.status == INVALID
    with pytest.raises(B.MixLoraError) as e:
        B.mixlora_head_distill(s, x, x, x, x, None, None, None, x, None, None, None, None, stream=0)
    assert e.value.status == INVALID
