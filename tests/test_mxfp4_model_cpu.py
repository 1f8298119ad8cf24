"""Models in microscaled 4-bit floating point, without a GPU: the oracle's decoder, the encoder of the inputs, the model that both give,
and the configurations and weights that ec_init refuses."""
import ctypes as C

import numpy as np
import pytest

import ec_inputs
import paper_2603_18489_amd as ec
from oracle import entropycache as eco


def test_decoder_has_the_values_of_the_format():
    assert eco.e2m1_values().tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6]
    codes = np.arange(256, dtype=np.uint8).reshape(4, 64)
    scales = np.array([[0, 127, 128, 254]] * 4, dtype=np.uint8)
    v = eco.to_f64(ec_inputs.MxMatrix(codes, scales))
    assert v.shape == (4, 128)
    for r in range(4):
        for k in (0, 1, 31, 32, 63, 64, 100, 127):
            c = codes[r, k // 2] >> (4 * (k % 2)) & 15
            assert v[r, k] == eco.e2m1_values()[c] * 2.0 ** (float(scales[r, k // 32]) - 127)


@pytest.mark.parametrize("spread", [0.0, 3.0])
def test_encoder_takes_the_nearest_value(spread):
    rng = np.random.default_rng(3)
    w = (rng.standard_normal((50, 96)) * np.exp(spread * rng.standard_normal((50, 96)))).astype(np.float32)
    w[0] = 0.0
    w[1, :32] = np.float32(2.0 ** -149)
    w[2, :32] = 2.0 ** 127
    w[3, :18] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, -7]   # ties go to the even code
    q = ec_inputs.quantize_blocks_e2m1(w)
    assert q.shape == w.shape and q.codes.shape == (50, 48) and q.scales.shape == (50, 3)
    assert eco.to_f64(q)[3, :18].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 6, 6, 0, -1, -1, -2, -2, -4, -4, -6]
    step = np.repeat(2.0 ** (q.scales.astype(np.float64) - 127), 32, axis=1)
    x, got = w.astype(np.float64), eco.to_f64(q)
    grid = np.array([v * s for s in (1, -1) for v in (0, 0.5, 1, 1.5, 2, 3, 4, 6)])
    near = np.abs(x[..., None] - grid * step[..., None]).min(axis=-1)
    assert (np.abs(got - x) == near).all()
    top = np.abs(x).reshape(50, 3, 32).max(axis=2) / step[:, ::32]
    assert ((top < 8) & ((top >= 4) | (q.scales == 0))).all()


def test_a_model_in_4_bits_is_the_model_of_its_values():
    cfg = ec_inputs.ModelCfg(n_layers=2, d_model=128, n_heads=2, n_kv_heads=1, head_dim=64, d_ffn=256, vocab=96, mask_id=95,
                             logit_scale=3.0, dtype="mxfp4w")
    w = ec_inputs.make_weights(cfg, 5, gain_jitter=0.1)
    assert w["w_down"][1].shape == (128, 256) and w["lm_head"].shape == (96, 128)
    full = {k: ([eco.to_f64(x) for x in v] if isinstance(v, list) else eco.to_f64(v)) for k, v in w.items()}
    dec = ec_inputs.DecodeCfg(gen_len=12, block=8, k_recent=2, tau=1e9)
    prompt = ec_inputs.make_prompt(cfg.vocab + 96, 9, 1) % 90
    a, b = (eco.eco_init(eco.OracleModel(cfg, x), dec, prompt) for x in (w, full))
    for _ in range(4):
        ra, rb = eco.eco_step(a, eco.AUTO), eco.eco_step(b, eco.AUTO)
        assert np.array_equal(ra["logits"], rb["logits"]) and ra["tokens"] == rb["tokens"]


def test_what_ec_init_refuses():
    lib = ec.load_library()
    wl = ec_inputs.WORKLOADS["llada8b_mxfp4_l2"]
    dec, plen = ec.binding.decode_cfg_struct(wl.decode), (C.c_int32 * 1)(64)
    good = ec.model_cfg_struct(wl.model)
    need = lib.ec_workspace_bytes(C.byref(good), C.byref(dec), plen)
    # the bf16 expansion and the 4.25 bits an element beside it
    assert need > ec_inputs.weight_bytes(wl.model) * (1 + 32 / 8.5) * 0.99
    for change in (dict(d_model=4096 - 64), dict(d_ffn=12288 + 64), dict(n_heads=1, n_kv_heads=1, head_dim=64)):
        bad = ec.model_cfg_struct(wl.model.replace(**change))
        assert lib.ec_workspace_bytes(C.byref(bad), C.byref(dec), plen) == 0
    # scales that are missing, codes that are not aligned: before anything touches the device
    L = wl.model.n_layers
    keep = []

    def weights(**over):
        w = ec.ec_weights()
        for name, kind in ec.ec_weights._fields_:
            if kind is C.c_void_p:
                setattr(w, name, over.get(name, 1 << 20))
            else:
                arr = (C.c_void_p * L)(*[over.get(name, 1 << 20)] * L)
                keep.append(arr)
                setattr(w, name, C.cast(arr, C.POINTER(C.c_void_p)))
        return w
    prompt = (C.c_int32 * 64)()
    for over in (dict(lm_head_mx=None), dict(wq_mx=None), dict(w_down_mx=None), dict(w_up=(1 << 20) + 8), dict(lm_head=(1 << 20) + 4)):
        ctx = C.c_void_p()
        rc = lib.ec_init(C.byref(ctx), C.byref(good), C.byref(weights(**over)), C.byref(dec), prompt, plen, 1 << 20, need, None)
        assert rc == ec.EC_ERR_ARG and not ctx and b"EC_MXFP4W" in lib.ec_last_error(None)
