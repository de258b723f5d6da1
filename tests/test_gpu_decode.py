"""Decoding behind a fused layer (pipeline.paged_layer, decode_step) against the oracle's chain: projection, rotation, causal
attention over the patched context and the tokens decoded so far."""
import numpy as np
import pytest
import torch

from oracle import qcf_oracle as orc
from paper_2604_08585_amd import inputs, pipeline
from gpu_util import DEV, quantizer, to_np

pytestmark = pytest.mark.gpu


def _decode(cfg, new, steps, accepted, **kw):
    wl = inputs.make_config(cfg, orc.PlantOps())
    sh = wl.shape
    L = pipeline.upload(wl, DEV)
    pipeline.fuse_layer(L)
    P = pipeline.paged_layer(L, more=new * steps, new=new, **kw)
    dt, quant = inputs.torch_dtype(sh.dtype), quantizer(sh.dtype)
    rng = np.random.default_rng(30 + cfg)
    k_ctx, v_ctx = to_np(L.k_fused), to_np(L.v_fused)
    off = np.concatenate([[0], np.cumsum(L.ctx_lens)])
    keys = [list(k_ctx[off[b]:off[b + 1]]) for b in range(L.B)]
    values = [list(v_ctx[off[b]:off[b + 1]]) for b in range(L.B)]
    tol = 2e-2 if sh.dtype == "bf16" else 1e-4
    w = np.asarray(wl.w_qkv, dtype=np.float64)
    H, Hkv, D = sh.n_q_heads, sh.n_kv_heads, sh.head_dim
    for step in range(steps):
        x = quant(rng.standard_normal((L.B * new, sh.d_model)))
        o = to_np(pipeline.decode_step(P, torch.from_numpy(x).to(device=DEV, dtype=dt), L.w_qkv))
        y = quant(x @ w.T).reshape(L.B, new, H + 2 * Hkv, D)
        for b in range(L.B):
            n = len(keys[b])
            pos = n + np.arange(new)
            q = quant(orc.rope_at(y[b, :, :H], pos, sh.rope_base, sh.rope_style))
            k = keys[b] + list(quant(orc.rope_at(y[b, :, H:H + Hkv], pos, sh.rope_base, sh.rope_style)))
            v = values[b] + list(y[b, :, H + Hkv:])
            ref, _ = orc.recompute_attn(q, pos, np.stack(k), np.stack(v))
            print(f"cfg {cfg} step {step} request {b}: {n} + {new} tokens, worst {np.abs(o[b] - ref).max():.2e}", flush=True)
            if not P.keep:
                assert np.abs(o[b] - ref).max() <= tol
            else:
                # the same pages, attended to by the oracle
                pages = P.pages[b].cpu().numpy()
                for i in range(new):
                    count = -(-(n + i + 1) // P.cache.desc.page_size)
                    assert all(p[0] == 0 and p[p >= 0][-1] == count - 1 for p in pages[i])
                    for h in range(H):
                        p = pages[i, h // (H // Hkv)]
                        rows = [t for j in p[p >= 0] for t in range(16 * j, min(16 * j + 16, n + i + 1))]
                        z = np.stack(k)[rows, h // (H // Hkv)] @ q[i, h] / np.sqrt(D)
                        e = np.exp(z - z.max())
                        assert np.abs(o[b, i, h] - e @ np.stack(v)[rows, h // (H // Hkv)] / e.sum()).max() <= tol
            keys[b], values[b] = k[:n + accepted], v[:n + accepted]
        pipeline.advance(P, accepted)
    assert P.held.tolist() == [n + steps * accepted for n in L.ctx_lens]


@pytest.mark.parametrize("new,steps,accepted,keep", [(1, 4, 1, 0), (3, 3, 2, 0), (1, 3, 1, 9), (2, 2, 1, 6)])
def test_decoding_behind_a_fused_layer(new, steps, accepted, keep):
    """float32, 512 tokens of context; drafts of which some are taken back, and attention cut down to a few pages."""
    _decode(0, new, steps, accepted, keep=keep)


def test_decoding_behind_a_fused_layer_in_bf16():
    _decode(1, 1, 2, 1)
    _decode(1, 1, 1, 1, keep=40, last=2)
