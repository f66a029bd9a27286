"""Refusals of the paged-cache entry points: bad arguments come back with their
status and a message before any device work (no GPU needed)."""

import ctypes

import pytest
import torch

from paper_2607_00501_amd import binding as B

P = ctypes.c_void_p(0x50000)
ODD = ctypes.c_void_p(0x50002)
FOUR = ctypes.c_void_p(0x50004)
EINVAL, ESHAPE, EALIGN, EWORKSPACE = 1, 2, 3, 6


def _call(name, defaults, **changed):
    args = dict(defaults, **changed)
    assert set(changed) <= set(defaults)
    status = getattr(B.lib(), name)(*args.values())
    if status:
        assert name in B.qm_last_error()
    return status


PLAN = dict(lens=P, new_lens=P, n_req=4, page_size=16, tables=P, max_pages=8, prefix_pages=0, free_ring=P,
            ring=ctypes.c_void_p(0x60000), n_pages=100, max_tokens=10, lens_out=ctypes.c_void_p(0x70000), kv_lens=P,
            offsets=P, positions=P, slots=P, ring_out=ctypes.c_void_p(0x80000), refused=P, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(page_size=0), ESHAPE), (dict(page_size=8), ESHAPE), (dict(page_size=48), ESHAPE),
    (dict(page_size=512), ESHAPE), (dict(page_size=-16), ESHAPE), (dict(n_pages=0), ESHAPE),
    (dict(n_pages=1 << 31), ESHAPE), (dict(n_req=0), ESHAPE), (dict(n_req=1025), ESHAPE), (dict(max_pages=0), ESHAPE),
    (dict(max_pages=(1 << 20) + 1), ESHAPE), (dict(prefix_pages=-1), ESHAPE), (dict(prefix_pages=9), ESHAPE),
    (dict(max_tokens=-1), ESHAPE), (dict(max_tokens=65537), ESHAPE),
    (dict(lens_out=P), EINVAL), (dict(ring_out=ctypes.c_void_p(0x60000)), EINVAL),
    *[({k: None}, EINVAL) for k, v in PLAN.items() if isinstance(v, ctypes.c_void_p)],
    *[({k: ODD}, EALIGN) for k, v in PLAN.items() if isinstance(v, ctypes.c_void_p)],
    (dict(slots=FOUR), EALIGN)])
def test_plan_refusals(change, status):
    assert _call("qkv_plan", PLAN, **change) == status


APPEND = dict(q=P, k=P, v=P, hq=4, hkv=2, d=64, tokens=3, positions=P, slots=P, interleaved=0, q_norm=P, k_norm=P,
              eps=1e-6, table=P, table_len=10, q_out=P, k_pages=P, v_pages=P, n_pages=4, page_size=16, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(page_size=24), ESHAPE), (dict(n_pages=0), ESHAPE), (dict(d=80), ESHAPE), (dict(hq=0), ESHAPE),
    (dict(hkv=1025), ESHAPE), (dict(tokens=-1), ESHAPE), (dict(tokens=65537), ESHAPE), (dict(table_len=0), ESHAPE),
    (dict(interleaved=2), EINVAL), (dict(q_norm=None), EINVAL), (dict(k_norm=None), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL),
    *[({k: None}, EINVAL) for k in ("q", "k", "v", "positions", "slots", "table", "q_out", "k_pages", "v_pages")],
    *[({k: FOUR}, EALIGN) for k in ("q", "k", "v", "slots", "table", "q_out", "k_pages", "v_pages")],
    (dict(positions=ODD), EALIGN)])
def test_append_refusals(change, status):
    assert _call("qkv_rope_append", APPEND, **change) == status


ATTEND = dict(q=P, k_pages=P, v_pages=P, n_pages=10, page_size=16, tables=P, max_pages=4, prefix=P, prefix_pages=1,
              offsets=P, kv_lens=P, n_req=2, tokens=2, hq=4, hkv=2, d=64, scale=0.1, out=ctypes.c_void_p(0x60000), workspace=P,
              ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(page_size=100), ESHAPE), (dict(n_pages=0), ESHAPE), (dict(n_pages=1 << 31), ESHAPE),
    (dict(max_pages=0), ESHAPE), (dict(prefix_pages=5), ESHAPE), (dict(prefix_pages=-1), ESHAPE),
    (dict(n_req=0), ESHAPE), (dict(n_req=2000), ESHAPE), (dict(tokens=-1), ESHAPE), (dict(tokens=65537), ESHAPE),
    (dict(hq=3), ESHAPE), (dict(hq=0), ESHAPE), (dict(hkv=0), ESHAPE), (dict(hq=129, hkv=129), ESHAPE),
    (dict(hq=1026), ESHAPE), (dict(hq=258), ESHAPE), (dict(out=P), EINVAL), (dict(d=96), ESHAPE), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    *[({k: None}, EINVAL) for k in ("q", "k_pages", "v_pages", "tables", "prefix", "offsets", "kv_lens", "out")],
    *[({k: FOUR}, EALIGN) for k in ("q", "k_pages", "v_pages", "out", "workspace")],
    *[({k: ODD}, EALIGN) for k in ("tables", "prefix", "offsets", "kv_lens")]])
def test_attention_refusals(change, status):
    assert _call("qattn_paged_f16", ATTEND, **change) == status


def test_row_argmax_refusals():
    args = dict(logits=P, rows=3, n=10, tokens=P, workspace=P, ws_bytes=3 * 2048, stream=None)
    for change, status in [(dict(rows=-1), ESHAPE), (dict(rows=32769), ESHAPE), (dict(n=0), ESHAPE),
                           (dict(n=(1 << 31) - 1), ESHAPE), (dict(logits=None), EINVAL), (dict(tokens=None), EINVAL),
                           (dict(workspace=None), EWORKSPACE), (dict(ws_bytes=3 * 2048 - 1), EWORKSPACE),
                           (dict(logits=ODD), EALIGN), (dict(tokens=ODD), EALIGN), (dict(workspace=ODD), EALIGN)]:
        assert _call("qdec_argmax_rows", args, **change) == status
    assert B.qdec_argmax_rows_workspace_bytes(7) == 7 * B.ARGMAX_WORKSPACE_BYTES
    assert B.qdec_argmax_rows_workspace_bytes(0) == 0
    with pytest.raises(B.QmError):
        B.qdec_argmax_rows_workspace_bytes(-1)


def test_batch_decoder_leaves_its_state_at_a_refusal():
    """Tokens of a wrong type or place are refused before anything is counted."""
    from paper_2607_00501_amd.decoder import BatchDecoder
    dec = BatchDecoder.__new__(BatchDecoder)
    dec.max_tokens, dec.emb, dec.turn, dec.cfg = 8, torch.zeros(4, 4), 0, None
    for tokens in (torch.zeros(9, dtype=torch.int32), torch.zeros(0, dtype=torch.int32), torch.zeros(3),
                   torch.zeros((8, 2), dtype=torch.int32)[:, 0], torch.zeros(3, dtype=torch.int32, device="meta")):
        with pytest.raises(ValueError):
            dec.step(tokens, None)
        assert dec.turn == 0


def test_nothing_to_do_is_no_error():
    assert _call("qkv_rope_append", APPEND, tokens=0) == 0
    assert _call("qattn_paged_f16", ATTEND, tokens=0) == 0
    assert _call("qdec_argmax_rows", dict(logits=None, rows=0, n=10, tokens=None, workspace=None, ws_bytes=0,
                                          stream=None)) == 0


def test_workspace_query_refusals():
    for args in ((3, 2, 64, 1, 1, 0), (4, 2, 80, 1, 1, 0), (4, 2, 64, 0, 1, 0), (4, 2, 64, 1, -1, 0),
                 (4, 2, 64, 1, 65537, 0), (4, 2, 64, 1, 1, -1)):
        with pytest.raises(B.QmError) as e:
            B.qattn_paged_workspace_bytes(*args)
        assert e.value.status == ESHAPE


def test_binding_refuses_wrong_tensors(monkeypatch):
    """Types, shapes and strides are checked before the library is called (CPU
    tensors: the device check comes last)."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    f16 = torch.zeros((2, 2, 16, 64), dtype=torch.float16)
    ints = torch.zeros(2, dtype=torch.int32)
    good = dict(q=torch.zeros((3, 4, 64), dtype=torch.float16), k_pages=f16, v_pages=f16, tables=ints.view(1, 2),
                offsets=ints, kv_lens=ints[:1], scale=0.1, out=torch.zeros((3, 256), dtype=torch.float16),
                workspace=torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(ValueError, match="current device"):
        B.qattn_paged_f16(**good)
    for name, bad in [("q", good["q"].float()), ("q", torch.zeros((3, 64, 4), dtype=torch.float16).transpose(1, 2)),
                      ("v_pages", f16[:1]), ("tables", ints.view(1, 2).long()), ("offsets", ints[:1]),
                      ("kv_lens", ints), ("out", good["out"][:2]), ("workspace", ints)]:
        with pytest.raises(ValueError, match=name):
            B.qattn_paged_f16(**dict(good, **{name: bad}))
