"""What the calls of the 8-bit cache and of draft verification refuse, without a launch (this runs without a GPU)."""
import pytest
import torch

import paper_2602_00182_amd as d

EINVAL, ESHAPE, EALIGN, EWORKSPACE = 1, 2, 3, 4
P = 4096  # a 16-byte aligned address that is never read: every call below ends before a launch


def lib():
    return d.api.lib()


APPEND = dict(qkv=P, ldqkv=1024, qbuf=P, pool=P, table=P, n_pages=4, n_slots=2, max_pages=2, positions=P, slots=0, cos=P, sin=P, R=1, Hq=4,
              Hkv=2, D=128, Lrope=8, stream=0)
READ = dict(pool=P, table=P, n_pages=4, n_slots=2, max_pages=2, positions=P, slots=0, k=P, v=P, R=1, Hkv=2, D=128, stream=0)
COPY = dict(pool=P, n_layers=1, n_pages=4, Hkv=2, D=128, src=P, dst=P, n=1, stream=0)
ATTN = dict(q=P, pool=P, table=P, n_pages=4, n_slots=2, max_pages=2, seqlens=P, slots=0, out=P, ws=P, ws_bytes=1 << 40, R=1, Hq=4, Hkv=2, D=128,
            scale=0.1, stream=0)
VERIFY = dict(p=P, q=P, drafts=P, n_drafts=P, u=P, accepted=P, tokens=P, ws=P, ws_bytes=1 << 40, B=1, N=2, V=100, stream=0)

CASES = [("det_kv8_rope_append", APPEND, change, code) for change, code in [
    (dict(qkv=0), EINVAL), (dict(qbuf=0), EINVAL), (dict(pool=0), EINVAL), (dict(table=0), EINVAL), (dict(positions=0), EINVAL), (dict(cos=0), EINVAL),
    (dict(R=0), EINVAL), (dict(Hq=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(n_pages=0), EINVAL), (dict(n_slots=0), EINVAL), (dict(max_pages=0), EINVAL),
    (dict(Lrope=0), EINVAL), (dict(ldqkv=1016), EINVAL), (dict(ldqkv=1028), EALIGN), (dict(D=64), ESHAPE), (dict(max_pages=131073), ESHAPE),
    (dict(qkv=P + 2), EALIGN), (dict(qbuf=P + 8), EALIGN), (dict(pool=P + 8), EALIGN), (dict(cos=P + 4), EALIGN)]]
CASES += [("det_kv8_read", READ, change, code) for change, code in [
    (dict(k=0), EINVAL), (dict(v=0), EINVAL), (dict(positions=0), EINVAL), (dict(pool=0), EINVAL), (dict(R=0), EINVAL), (dict(D=96), ESHAPE),
    (dict(k=P + 2), EALIGN), (dict(pool=P + 4), EALIGN)]]
CASES += [("det_kv8_copy_pages", COPY, change, code) for change, code in [
    (dict(pool=0), EINVAL), (dict(src=0), EINVAL), (dict(dst=0), EINVAL), (dict(n=0), EINVAL), (dict(n_layers=0), EINVAL), (dict(n_pages=0), EINVAL),
    (dict(Hkv=0), EINVAL), (dict(D=64), ESHAPE), (dict(n_layers=65536), ESHAPE), (dict(pool=P + 8), EALIGN)]]
CASES += [("det_attn_decode_kv8", ATTN, change, code) for change, code in [
    (dict(q=0), EINVAL), (dict(pool=0), EINVAL), (dict(table=0), EINVAL), (dict(seqlens=0), EINVAL), (dict(out=0), EINVAL), (dict(ws=0), EINVAL),
    (dict(R=0), EINVAL), (dict(Hq=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(max_pages=-1), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=-0.1), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(D=64), ESHAPE), (dict(Hq=5), ESHAPE),
    (dict(Hq=34), ESHAPE), (dict(R=3), ESHAPE), (dict(max_pages=131073), ESHAPE), (dict(q=P + 2), EALIGN), (dict(out=P + 4), EALIGN),
    (dict(ws=P + 8), EALIGN), (dict(ws_bytes=0), EWORKSPACE)]]
CASES += [("det_verify_drafts", VERIFY, change, code) for change, code in [
    (dict(p=0), EINVAL), (dict(drafts=0), EINVAL), (dict(u=0), EINVAL), (dict(accepted=0), EINVAL), (dict(tokens=0), EINVAL), (dict(B=0), EINVAL),
    (dict(N=0), EINVAL), (dict(V=0), EINVAL), (dict(N=64), ESHAPE), (dict(V=(1 << 30) + 1), ESHAPE), (dict(B=65536), ESHAPE),
    (dict(ws=0), EINVAL), (dict(ws=P + 8), EALIGN), (dict(ws_bytes=15), EWORKSPACE), (dict(p=P + 4), EALIGN), (dict(q=P + 4), EALIGN)]]


@pytest.mark.parametrize("name,args,change,code", CASES, ids=lambda x: str(x) if isinstance(x, dict) and len(x) == 1 else "")
def test_a_call_that_is_refused_says_why(name, args, change, code):
    call = {**args, **change}
    assert getattr(lib(), name)(*[None if isinstance(v, int) and v == 0 and k in POINTERS else v for k, v in call.items()]) == code


POINTERS = {"qkv", "qbuf", "pool", "table", "positions", "slots", "cos", "sin", "k", "v", "src", "dst", "q", "seqlens", "out", "ws", "p", "drafts",
            "n_drafts", "u", "accepted", "tokens", "stream"}


def test_sizes():
    assert d.det_verify_drafts_workspace_bytes(3, 2049) == 3 * 2 * 16 and d.det_verify_drafts_workspace_bytes(1, 0) == 0
    assert d.det_kv8_pool_bytes(10, 8) == 10 * 8 * d.KV8_RECORD
    assert d.det_kv8_pool_bytes(0, 8) == 0 and d.det_kv8_pool_bytes(1, 8, 64) == 0
    assert d.det_attn_decode_kv8_workspace_bytes(1, 32, 8, 64, 4) == 0
    assert d.det_attn_decode_kv8_workspace_bytes(1, 32, 7, 128, 4) == 0
    assert d.det_attn_decode_kv8_workspace_bytes(1, 32, 8, 128, 131073) == 0
    assert d.det_attn_decode_kv8_workspace_bytes(1, 32, 8, 128, 131072) > 0
    with pytest.raises(d.api.DetError):
        d.kv8_pool(1, 4, 2, 96, device="cpu")
    assert d.kv8_pool(2, 4, 3, device="cpu").shape == (2, 4, 3, d.KV8_RECORD)


def test_the_binding_refuses_what_does_not_fit():
    pool, table = d.kv8_pool(1, 4, 2, device="cpu"), torch.zeros((3, 2), dtype=torch.int32)
    bf, i32 = dict(dtype=torch.bfloat16), dict(dtype=torch.int32)
    q, out, lens = torch.zeros((3, 4, 128), **bf), torch.zeros((3, 4, 128), **bf), torch.zeros(3, **i32)
    ws = torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(ValueError):
        d.det_attn_decode_kv8(q, pool, table, lens, None, out, ws, 0.1)                # all layers' pools instead of one
    with pytest.raises(ValueError):
        d.det_attn_decode_kv8(q, pool[0], table, lens[:2], None, out, ws, 0.1)
    with pytest.raises(ValueError):
        d.det_attn_decode_kv8(q, pool[0], table[:2], lens, None, out, ws, 0.1)         # fewer slots than rows
    with pytest.raises(ValueError):
        d.det_attn_decode_kv8(q, pool[0], table, lens, lens[:2], out, ws, 0.1)
    with pytest.raises(ValueError):
        d.det_attn_decode_kv8(q, pool[0], table, lens, None, out, ws, 0.1)             # host tensors
    with pytest.raises(ValueError):
        d.det_kv8_rope_append(torch.zeros((3, 100), **bf), q, pool[0], table, lens, None, torch.zeros(8, 64), torch.zeros(8, 64))
    with pytest.raises(ValueError):
        d.det_kv8_copy_pages(pool[0], lens, lens)
    with pytest.raises(ValueError):
        d.det_kv8_copy_pages(pool, lens, lens[:2])
    with pytest.raises(ValueError):
        d.det_kv8_read(pool[0], table, lens, None, torch.zeros((3, 1, 128), **bf), torch.zeros((3, 1, 128), **bf))
    with pytest.raises(ValueError):
        d.det_verify_drafts(torch.zeros(2, 3, 9), torch.zeros(2, 3, 9), torch.zeros((2, 2), **i32), None, torch.zeros(2, 3), lens[:2], torch.zeros((2, 3), **i32))
