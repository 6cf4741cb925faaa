"""Which buffers of precc_rms_norm may share memory (no GPU: a call is refused before the device is looked at, and
one that is not ends there)."""
import ctypes

import pytest

from paper_2609_34054_b200 import binding

ROWS, WIDTH = 6, 64
BF16, E4M3, SCALES, GAIN = 2 * ROWS * WIDTH, ROWS * WIDTH, 4 * ROWS, 2 * WIDTH
AT = dict(x=0x10000, residual=0x20000, gain=0x30000, residual_out=0x40000, out=0x50000, out_e4m3=0x60000, out_scale=0x70000)


@pytest.fixture(scope="module")
def call():
    from paper_2609_34054_b200 import build
    build.build()
    lib = binding.load_library()
    # a context's memory, of a device -1 that is never the current one: nothing is launched where there is a GPU either, and a refusal writes its message
    ctx = (ctypes.c_ubyte * (1 << 16))(*[255] * (1 << 16))

    def run(**moved):
        a = {**AT, **moved}
        rc = lib.precc_rms_norm(ctx, a["x"], a["residual"], a["gain"], ROWS, WIDTH, 1e-5, a["residual_out"], a["out"], a["out_e4m3"], a["out_scale"], None)
        return rc, lib.precc_last_error(ctx).decode()
    return run


def _refused(answer):
    return "overlap" in answer[1] and answer[0] != 0


@pytest.mark.parametrize("moved", [
    {}, dict(out=AT["x"]), dict(out=AT["residual"]), dict(residual_out=AT["residual"]), dict(residual_out=AT["x"]), dict(out=AT["x"], residual_out=AT["residual"]),
    dict(out=AT["residual"], residual_out=AT["x"]), dict(out=None), dict(residual=None, residual_out=None), dict(residual=AT["x"]), dict(residual=AT["x"], out=AT["x"]),
    dict(out_e4m3=AT["x"] + BF16), dict(out_e4m3=AT["x"] - E4M3), dict(out_scale=AT["x"] + BF16), dict(out_scale=AT["gain"] - SCALES), dict(out=AT["x"] + BF16),
    dict(out=None, out_e4m3=AT["x"] + BF16), dict(residual_out=AT["gain"] + GAIN), dict(out_e4m3=AT["out"] + BF16)])
def test_allowed(call, moved):
    rc, message = call(**moved)
    assert rc != 0 and "overlap" not in message          # (no GPU, or not the context's)


@pytest.mark.parametrize("moved", [
    dict(out_e4m3=AT["x"]), dict(out_e4m3=AT["residual"]), dict(out_e4m3=AT["x"] + BF16 - 16), dict(out_e4m3=AT["x"] - E4M3 + 16), dict(out_e4m3=AT["gain"]),
    dict(out_scale=AT["x"]), dict(out_scale=AT["x"] + BF16 - 4), dict(out_scale=AT["gain"] + GAIN - 4), dict(out_scale=AT["residual"] - SCALES + 4),
    dict(out=AT["x"] + 16), dict(out=AT["x"] - 16), dict(out=AT["residual"] + 128), dict(residual_out=AT["x"] + 16), dict(out=AT["gain"]), dict(residual_out=AT["gain"]),
    dict(out=AT["residual_out"]), dict(out=AT["residual_out"] + 32), dict(out_e4m3=AT["out"]), dict(out_e4m3=AT["residual_out"]), dict(out_scale=AT["out_e4m3"]),
    dict(out_scale=AT["out"] + 64), dict(out=AT["x"], residual_out=AT["x"]), dict(residual=None, residual_out=None, out_e4m3=AT["x"]),
    dict(residual=None, residual_out=None, out=None, out_e4m3=AT["x"])])
def test_refused(call, moved):
    assert _refused(call(**moved))
