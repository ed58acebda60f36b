"""The paged calls refuse tensors of another type, size or density than the one whose address they pass on.  (Host tensors and
a stand-in for the library, which takes every call: nothing is launched.)"""
import pytest
import torch

import paper_2606_04511_amd.sparda as sp

BF, I32, I16 = torch.bfloat16, torch.int32, torch.int16
B, H, G, K, N = 2, 3, 4, 5, 7


class Takes:
    """A library whose calls succeed."""

    def __getattr__(self, name):
        return lambda *args: sp.SPARDA_OK


@pytest.fixture(autouse=True)
def stand_in(monkeypatch):
    monkeypatch.setattr(sp, "load", Takes)
    monkeypatch.setattr(sp, "_stream", lambda *a: 0)
    monkeypatch.setattr(sp, "_present", lambda: -1)  # the current device is the host


def shape():
    return sp.SpardaShape(batch=B, n_kv_heads=H, group_size=G, k_total=K, t_cap=128, nc_cap=0)


def pages():
    k = torch.zeros(4, H, 64, 128, dtype=BF)
    return sp.SpardaPages(64, torch.zeros(B, 2, dtype=I32), k, k.clone(), torch.zeros(4, H, 1, 128, dtype=BF))


def refused(fn, args, name, bad):
    """Each of `bad` in the place of argument `name` is refused by that name; the arguments as they are, and an address, are taken."""
    fn(**args)
    fn(**{**args, name: 0x7F0000000000, **({"ws_bytes": 1024} if name == "ws" else {})})
    for x in bad:
        with pytest.raises(ValueError, match=f"^{name}:"):
            fn(**{**args, name: x})


def lengths():
    return [torch.zeros(B, dtype=torch.int64), torch.zeros(B, dtype=torch.float32), torch.zeros(B - 1, dtype=I32),
            torch.zeros(2 * B, dtype=I32)[::2], torch.zeros(1, dtype=I32).expand(B)]


def wrong(good):
    """Tensors of another type, one element short, and not dense."""
    return [good.float() if good.dtype != torch.float32 else good.int(), good.flatten()[:-1],
            torch.stack((good, good), -1)[..., 0], good.flatten()[:1].expand(good.numel())]


def test_rotate_positions():
    x, rope = torch.zeros(B, H, N, 128), sp.SpardaRope(0, sp.SPARDA_ROPE_HALF, None)
    args = dict(rope=rope, type=sp.SPARDA_F32, batch=B, n_heads=H, n_tok=N, x=x, pos=torch.zeros(B, N, dtype=I32), pos_ld=N, y=x.clone())
    wide = torch.zeros(B, 3 * N, dtype=I32)
    refused(sp.sparda_rotate, args, "pos", [
        torch.arange(N), torch.zeros(B, N), torch.zeros(B * N - 1, dtype=I32), wide[:, ::3], wide[:, :N], torch.zeros(N, B, dtype=I32).t(),
        torch.zeros(N, dtype=I32)])
    refused(sp.sparda_rotate, {**args, "pos_ld": 0}, "pos", [torch.zeros(N - 1, dtype=I32), wide[0, ::3][:N], torch.zeros(N)])
    # rows that lie pos_ld apart, one row for all sequences, a slice of a longer row
    refused(sp.sparda_rotate, {**args, "pos": wide[:, 4:4 + N], "pos_ld": 3 * N}, "pos", [wide[:, 4:3 + N], wide[:1, :N - 1]])
    refused(sp.sparda_rotate, {**args, "pos": torch.zeros(N, dtype=I32).expand(B, N), "pos_ld": 0}, "pos", [wide[:, :N - 1]])
    refused(sp.sparda_rotate, {**args, "pos": wide[0, 3:3 + N], "pos_ld": 0}, "pos", [wide[0, 3:2 + N]])


def test_append_lengths():
    rows = lambda h: torch.zeros(B, h, N, 128, dtype=BF)  # noqa: E731
    args = dict(shape=shape(), pages=pages(), rope=None, n_max=N, n_new=torch.zeros(B, dtype=I32), t_ctx=torch.zeros(B, dtype=I32),
                k_new=rows(H), v_new=rows(H), q=rows(H * G), q_out=rows(H * G), f=rows(H), f_out=rows(H),
                t_new=torch.zeros(B, dtype=I32))
    for name in ("n_new", "t_ctx", "t_new"):
        refused(sp.sparda_paged_append, args, name, lengths())


def test_select_tensors():
    args = dict(shape=shape(), pages=pages(), f=torch.zeros(B, H, 1, 128, dtype=BF), t_ctx=torch.zeros(B, dtype=I32), t_max=100,
                sel=torch.zeros(B, H, 1, K, dtype=I16), cnt=torch.zeros(B, H, 1, dtype=I16), ws=torch.zeros(1024, dtype=torch.uint8))
    refused(sp.sparda_paged_select, args, "t_ctx", lengths())
    refused(sp.sparda_paged_select, args, "f", wrong(args["f"]) + [torch.zeros(B, H, N, 128, dtype=BF)[:, :, -1:]])
    for name in ("sel", "cnt"):
        refused(sp.sparda_paged_select, args, name, wrong(args[name]))
    refused(sp.sparda_paged_select, args, "ws", [torch.zeros(2048, dtype=torch.uint8)[::2]])
    refused(sp.sparda_paged_select, {**args, "ws_bytes": 1024}, "ws", [torch.zeros(1023, dtype=torch.uint8), torch.zeros(255)])


@pytest.mark.parametrize("listed", [False, True])
def test_attention_tensors(listed):
    args = dict(shape=shape(), pages=pages(), q=torch.zeros(B, H * G, 1, 128, dtype=BF), t_ctx=torch.zeros(B, dtype=I32), t_max=100,
                sel=torch.zeros(B, H, 1, K, dtype=I16) if listed else None, cnt=torch.zeros(B, H, 1, dtype=I16) if listed else None,
                sm_scale=0.1, o=torch.zeros(B, H * G, 1, 128, dtype=BF), ws=torch.zeros(1024, dtype=torch.uint8))
    refused(sp.sparda_paged_attn, args, "t_ctx", lengths())
    for name in ("q", "o"):
        # the newest tokens' rows of a chunk's queries lie N rows apart
        refused(sp.sparda_paged_attn, args, name, wrong(args[name]) + [torch.zeros(B, H * G, N, 128, dtype=BF)[:, :, -1:]])
    if listed:
        for name in ("sel", "cnt"):
            refused(sp.sparda_paged_attn, args, name, wrong(args[name]))
    refused(sp.sparda_paged_attn, args, "ws", [torch.zeros(2048, dtype=torch.uint8)[::2]])
    refused(sp.sparda_paged_attn, {**args, "ws_bytes": 1024}, "ws", [torch.zeros(1023, dtype=torch.uint8)])
