"""Models whose matrices are in microscaled 4-bit floating point (EC_MXFP4W): whole generations under teacher forcing against the oracle,
which decodes the same codes exactly.  The tolerance is that of the bfloat16 path, which the arithmetic is."""
import numpy as np
import pytest
import torch

import ec_inputs
import paper_2603_18489_amd as ec
from oracle import entropycache as eco
from tests.gpu_harness import run_teacher_forced, run_teacher_forced_batch

pytestmark = pytest.mark.gpu
TOL = 2e-2


def small_cfg(hq, hkv, hd, d, f, vocab=4096, layers=2, scale=16.0):
    return ec_inputs.ModelCfg(n_layers=layers, d_model=d, n_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ffn=f, vocab=vocab,
                              mask_id=vocab - 1, rms_eps=1e-5, rope_base=10000.0, logit_scale=scale, dtype="mxfp4w")


@pytest.mark.parametrize("hq,hkv,hd,f,P,N,block,k,n,tau", [
    (4, 4, 64, 768, 64, 64, 32, 2, 1, 3.0),
    (4, 2, 128, 1280, 50, 70, 32, 4, 2, 2.5),     # grouped queries, ragged last block
    (8, 2, 64, 768, 100, 33, 32, 2, 3, 1e9),      # 133 rows in full steps: the tiled kernels on the bf16 expansion
    (4, 2, 64, 6272, 40, 128, 32, 64, 1, 1e9),    # up to 96 rows; 784 gate/up tiles in groups of three
    (2, 2, 64, 128, 20, 90, 32, 40, 1, 1e9),      # one step of 128 k, five row tiles
])
def test_whole_generation(hq, hkv, hd, f, P, N, block, k, n, tau):
    cfg = small_cfg(hq, hkv, hd, d=hq * hd if hq * hd >= 256 else 256 if f > 128 else 128, f=f)
    w = ec_inputs.make_weights(cfg, 7, gain_jitter=0.1)
    dec = ec_inputs.DecodeCfg(gen_len=N, block=block, k_recent=k, tokens_per_step=n, tau=tau)
    s = run_teacher_forced(cfg, w, dec, ec_inputs.make_prompt(cfg.vocab, P, 3), TOL)
    print(s)
    assert s["modes"][eco.PARTIAL] >= 1 and s["tokens_exact"] > 0 and s["modes_exact"] > 0


@pytest.mark.parametrize("rows,f,vocab", [(9, 8192, 4096), (20, 12288, 16400), (40, 12416, 32784), (60, 24704, 4096), (96, 24704, 4096)])
def test_group_sizes_and_row_tiles(rows, f, vocab):
    """Gate/up matrices of two, three and six tiles to a block, LM heads of two, four and eight, one to six row tiles (and a down projection
    whose K is split over blocks)."""
    cfg = small_cfg(2, 2, 64, 128, f, vocab=vocab, layers=1)
    w = ec_inputs.make_weights(cfg, 11, gain_jitter=0.1)
    dec = ec_inputs.DecodeCfg(gen_len=128, block=min(rows, 32), k_recent=max(rows - 32, 0), tau=1e9)
    s = run_teacher_forced(cfg, w, dec, ec_inputs.make_prompt(cfg.vocab, 30, 5), TOL, max_steps=72 if rows > 32 else 4)
    assert s["modes"][eco.PARTIAL] >= 3 and s["tokens_exact"] > 0


def test_batch():
    cfg = small_cfg(4, 2, 128, 512, 768)
    w = ec_inputs.make_weights(cfg, 13, gain_jitter=0.1)
    dec = ec_inputs.DecodeCfg(gen_len=36, block=32, k_recent=3, tokens_per_step=1, tau=2.5, batch=4)
    prompts = [ec_inputs.make_prompt(cfg.vocab, P, 20 + i) for i, P in enumerate((70, 9, 33, 150))]
    s = run_teacher_forced_batch(cfg, w, dec, prompts, TOL, max_steps=12)
    assert s["modes"][eco.PARTIAL] >= 1 and s["tokens_exact"] > 0


@pytest.mark.timeout(900)
def test_two_layer_twin():
    wl = ec_inputs.WORKLOADS["llada8b_mxfp4_l2"]
    cfg = wl.model.replace(logit_scale=8.0)
    w = ec_inputs.make_weights(cfg, wl.seed, threads=16)
    prompt = ec_inputs.make_prompt(cfg.vocab, wl.prompt_len, wl.seed)
    eco.enable_f64_cache(True)
    try:
        s = run_teacher_forced(cfg, w, wl.decode, prompt, TOL, max_steps=14, check_cache_every=6,
                               mode_fn=lambda i: eco.FULL if i % 12 == 0 else eco.PARTIAL, verbose=True)
    finally:
        eco.enable_f64_cache(False)
    assert s["steps"] == 14 and s["tokens_exact"] > 0 and s["rows_decided"] > 0


def test_matrices_quantised_on_the_device_and_the_model_of_their_values():
    """weights_to_device brings bfloat16 matrices to 4 bits on the device, to the codes that the host's encoder gives; and a full step of
    more than 96 rows gives the bits of the bfloat16 model that holds the same values."""
    cfg = small_cfg(4, 2, 64, 256, 768)
    plain = ec_inputs.make_weights(cfg.replace(dtype="bf16"), 3, gain_jitter=0.1)
    host = {}
    for name, v in plain.items():
        f32 = lambda x: eco.to_f64(x).astype(np.float32)
        is_matrix = name in ec.binding.QUANT_MATRICES or name == "lm_head"
        host[name] = v if not is_matrix else ([ec_inputs.quantize_blocks_e2m1(f32(x)) for x in v] if isinstance(v, list)
                                              else ec_inputs.quantize_blocks_e2m1(f32(v)))
    dev, up = ec.weights_to_device(cfg, plain), ec.weights_to_device(cfg, host)
    for name in ("lm_head", "lm_head_mx"):
        assert torch.equal(dev[name], up[name])
    for name in ec.binding.QUANT_MATRICES:
        for l in range(2):
            assert torch.equal(dev[name][l], up[name][l]) and torch.equal(dev[name + "_mx"][l], up[name + "_mx"][l])
    # the values as a bfloat16 model: every one is a bfloat16 number
    values = {}
    for name, v in plain.items():
        back = lambda n, x: ec.mxfp4_dequantize(ec.Mxfp4(n, x), torch.bfloat16)
        if name == "lm_head":
            values[name] = back(dev[name], dev[name + "_mx"])
        elif name in ec.binding.QUANT_MATRICES:
            values[name] = [back(c, s) for c, s in zip(dev[name], dev[name + "_mx"])]
        else:
            values[name] = dev[name]
    dec = ec_inputs.DecodeCfg(gen_len=64, block=32, k_recent=2, tau=3.0)
    prompt = ec_inputs.make_prompt(cfg.vocab, 90, 1)
    logits = []
    for c, w in ((cfg, dev), (cfg.replace(dtype="bf16"), values)):
        g = ec.EntropyCache(c, w, dec, prompt)
        g.keep_logits(True)
        g.step(ec.EC_FULL)
        kv = g.debug_read(ec.EC_DBG_KCACHE, 1)
        logits.append((kv, g.debug_read(ec.EC_DBG_LOGITS, count=32)))
        g.close()
    assert np.array_equal(logits[0][0], logits[1][0])     # 154 rows: the tiled kernels on the same fragments
    # The LM head's 32 rows come from codes here and from bfloat16 there: the same 256 products, sums of another order, so 2 * 256 additions
    # off by at most 2^-24 of the products' magnitudes, which sum to no more than sqrt(256) times what random signs leave of them.
    assert np.abs(logits[0][1] - logits[1][1]).max() <= 2 * 256 * 2.0 ** -24 * 16 * np.abs(logits[1][1]).max()
