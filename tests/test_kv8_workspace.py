"""Workspaces of calls over the 8-bit cache whose rows name slots: as much as the chunk-by-chunk form needs, no more for rows that walk."""
import numpy as np
import pytest
import torch

import paper_2602_00182_amd as d
from paper_2602_00182_amd import api

PARTIAL = 528  # bytes of a chunk of one (row, head)


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (16, 4), (8, 1), (16, 1), (15, 5), (8, 8), (1, 1), (1000, 1000)])
@pytest.mark.parametrize("pages", [1, 5, 512])
def test_sizes(Hq, Hkv, pages):
    tile, chunks = 16 // (Hq // Hkv), -(-pages // 4)
    last = 0
    for R in (1, 2, 15, 16, 17, 447, 448, 449, 895, 896, 1000, 5000, 32768, 65536):
        size = d.det_attn_decode_kv8_rows_workspace_bytes(R, Hq, Hkv, 128, pages)
        if -(-R // tile) * Hkv < 896:
            assert size == R * Hq * chunks * PARTIAL == d.det_attn_decode_kv8_workspace_bytes(R, Hq, Hkv, 128, pages)
        assert max(last, 16) <= size <= max(16, 895 * 16 * chunks * PARTIAL)  # enough for fewer rows too
        last = size
    assert d.det_attn_decode_kv8_workspace_bytes(32768, Hq, Hkv, 128, pages) == 32768 * Hq * chunks * PARTIAL  # rows that are their slots


def test_refusals():
    size = d.det_attn_decode_kv8_rows_workspace_bytes
    assert size(0, 4, 2, 128, 1) == size(1, 4, 3, 128, 1) == size(1, 4, 2, 64, 1) == size(1, 4, 2, 128, 131073) == size(1, 17, 1, 128, 1) == 0
    cfg = d.layer_cfg(512, 4, 2, 128, 1024, 256, 1e-5, 0.1)
    for name in ("det_decoder_layer_kv8", "det_qdecoder_layer_kv8"):
        assert getattr(d, name + "_rows_workspace_bytes")(cfg, 0, 4) == 0 and getattr(d, name + "_rows_workspace_bytes")(cfg, 5, 0) == 0
        few, same = (getattr(d, name + end)(cfg, 100, 512) for end in ("_rows_workspace_bytes", "_workspace_bytes"))
        assert few == same
        many, rows, more = (getattr(d, name + "_rows_workspace_bytes")(cfg, R, 512) for R in (4000, 20000, 40000))
        attention = 447 * 8 * 4 * 128 * PARTIAL
        assert attention < many < getattr(d, name + "_workspace_bytes")(cfg, 4000, 512) and more - rows < 20000 * 40000 and rows - attention < 20000 * 40000
    P = 4096  # never read: the call ends before a launch
    call = lambda R, ws_bytes: api.lib().det_attn_decode_kv8(P, P, P, 4, 2, 2, P, P, P, P, ws_bytes, R, 4, 2, 128, 0.1, None)
    assert call(100, 100 * 4 * PARTIAL - 1) == 4 and call(3, 16) == 4


def test_a_models_prompt_needs_no_partials_for_every_row():
    from paper_2602_00182_amd import decode
    model = decode.DecodeModel.__new__(decode.DecodeModel)
    cfg = d.layer_cfg(2048, 16, 4, 128, 5632, 32768, 1e-5, 0.1)
    for model.quantized in (False, True):
        model.cache8 = True
        assert model.layer_workspace_bytes(cfg, 32768, named=True) < 4 << 30 < 32 << 30 < model.layer_workspace_bytes(cfg, 32768)
        model.cache8 = False
        assert model.layer_workspace_bytes(cfg, 64, named=True) == model.layer_workspace_bytes(cfg, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("R", [1700, 1000])
def test_many_rows_with_just_that(R):
    """Rows that walk, with a workspace of sixteen bytes: the call leaves what lies behind it, and gives the bytes it gives with a large one."""
    import detsynth as ds
    from gpu_util import DEV, step, up, up_bf16
    from kv8_ref import SCALE, Cache

    Hq, Hkv, n = 16, 4, R
    cache = Cache(7900, [n], Hkv)
    q = up_bf16(ds.normal_bf16(7901, (R, Hq, 128)))
    pool, table, lens, slots = up(cache.pool), up(cache.table), up(np.arange(1, n + 1, dtype=np.int32)), torch.zeros(R, dtype=torch.int32, device=DEV)
    size = d.det_attn_decode_kv8_rows_workspace_bytes(R, Hq, Hkv, 128, table.shape[1])
    full = d.det_attn_decode_kv8_workspace_bytes(R, Hq, Hkv, 128, table.shape[1])
    assert size < full
    outs = []
    for held in (16, size, full):
        ws = torch.full((held + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
        out = torch.empty_like(q)
        step(f"{R} rows, workspace of {held}")
        d.det_attn_decode_kv8(q, pool, table, lens, slots, out, ws[:held], SCALE)
        torch.cuda.synchronize()
        assert (ws == 0x5A).all()
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.gpu
@pytest.mark.parametrize("quantized", [False, True])
def test_layers_of_many_rows_in_their_workspace(quantized):
    import detsynth as ds
    from gpu_util import DEV, step, up
    from paper_2602_00182_amd import decode

    R, H, Hq, Hkv, F = 3700, 256, 4, 2, 512  # 463 tiles of eight rows, 926 with both KV heads
    g = lambda i, shape, std=0.05, mean=0.0: ds.normal_bf16_torch(7950 + i, shape, std, mean, DEV)
    layer = dict(norm1=g(1, (H,), 0.1, 1.0), wqkv=g(2, (H, (Hq + 2 * Hkv) * 128)), wo=g(3, (Hq * 128, H)), norm2=g(4, (H,), 0.1, 1.0), wgu=g(5, (H, 2 * F)),
                 wdown=g(6, (F, H)))
    w = dict(embed=g(7, (512, H), 1.0), lm_head=g(8, (H, 512)), final_norm=g(9, (H,)), layers=[layer])
    m = decode.DecodeModel(decode.ModelCfg(H=H, Hq=Hq, Hkv=Hkv, D=128, F=F, V=512, n_layers=1), w, quantized=quantized, cache8=True)
    pages, lc = -(-R // 64), d.layer_cfg(H, Hq, Hkv, 128, F, R, 1e-5, 0.08)
    cos, sin = (up(t) for t in ds.rope_tables(R, 128))
    table = up(np.arange(pages, dtype=np.int32)[None])
    pos, slots = torch.arange(R, dtype=torch.int32, device=DEV), torch.zeros(R, dtype=torch.int32, device=DEV)
    x0 = g(10, (R, H), 1.0)
    out = []
    sizes = [m.layer_workspace_bytes(lc, R, named=True), m.layer_workspace_bytes(lc, R)]
    assert sizes[0] < sizes[1]
    for held in sizes:
        ws = torch.full((held + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
        x, pool = x0.clone(), d.kv8_pool(1, pages, Hkv)[0]
        step(f"layer of {R} rows, quantized {quantized}, workspace of {held}")
        m.layer(m.layers[0][1], lc, x, pool, table, pos, slots, cos, sin, ws[:held])
        torch.cuda.synchronize()
        assert (ws[held:] == 0x5A).all()
        out.append((x, pool))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    with pytest.raises(d.api.DetError):
        m.layer(m.layers[0][1], lc, x0, pool, table, pos, slots, cos, sin, ws[:sizes[0] - 256])
