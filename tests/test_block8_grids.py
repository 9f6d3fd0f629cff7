"""Launches of the 8-bit format at the largest sizes: a launch holds fewer than 2^32 work-items along x, while the entry
points take up to 2^31 - 1 blocks of 16 lanes each.  On the CPU by launch_recorder.c, and one such call on the GPU."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

from paper_2512_14080_amd import binding as B
from test_block8_cpu import built
from test_gpu_parity import _torch

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def _record(calls, tmp_path):
    so = os.path.join(str(tmp_path), "launch_recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "launch_recorder.c")], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), so], input=json.dumps(calls), text=True,
                       capture_output=True, cwd=ROOT, timeout=60, env={**os.environ, "PYTHONPATH": ROOT + os.pathsep + HERE})
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


def _main():
    rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    rec.rec_name.restype = ctypes.c_char_p
    from launch_recorder import _routing
    L, p, ws, out = B.lib(), 0x20000000, (0x30000000, 1 << 62), []

    def ok(rc):
        assert rc == B.MOE_OK, B.moe_last_error()

    for c in json.load(sys.stdin):
        rec.rec_clear()
        if "rows" in c:
            ok(L.moe_quantize_rows(*c["rows"], p, p, p, None))
            ok(L.moe_dequantize_rows(*c["rows"], p, p, p, None))
        else:
            D = B.dims(*c["dims"])
            r = _routing(B, D, D.T * D.K)
            ok(L.moe_route(D, p, p, None, 0, ctypes.byref(r), None))
            q, k = B.MoeQExperts(), B.MoeCkpt()
            ok(L.moe_qexperts_init(D, p, L.moe_qexperts_bytes(D), ctypes.byref(q)))
            ok(L.moe_ckpt_init(D, r.capacity, B.MOE_CKPT_X, p, L.moe_ckpt_bytes(D, r.capacity, B.MOE_CKPT_X),
                               ctypes.byref(k)))
            q.state = B.MOE_HELD_WRITTEN
            rec.rec_clear()
            ok(L.moe_fwd_quant(D, p, ctypes.byref(q), None, ctypes.byref(r), None, p, *ws, None))
            ok(L.moe_fwd_ckpt(D, p, p, p, None, ctypes.byref(r), ctypes.byref(k), p, *ws, None))
            ok(L.moe_bwd_ckpt(D, p, None, ctypes.byref(k), p, p, None, p, ctypes.byref(r), p, p, p, p, p, None, *ws, None))
        out.append([(rec.rec_name(i).decode(), rec.rec_grid(i, 0) & 0xFFFFFFFF) for i in range(rec.rec_count())])
    print(json.dumps(out))


@built
@pytest.mark.parametrize("rows,cols", [(1 << 28, 8), ((1 << 31) - 1, 128), (1 << 26, 4096 // 8), (1 << 20, 1 << 17),
                                       (127, (1 << 31) - 8)])
def test_rows_grids(tmp_path, rows, cols):
    l, = _record([{"rows": (rows, cols)}], tmp_path)
    blocks = -(-cols // 128)
    for kernel in ("20quantize_rows_kernel", "22dequantize_rows_kernel"):
        groups = [x for name, x in l if kernel in name]
        assert max(groups) * 256 < 1 << 32
        assert sum(16 * x for x in groups) >= rows * blocks > sum(16 * (x - 1) for x in groups)


@built
def test_layer_grids(tmp_path):
    """X of 2^28 blocks, 64 GB."""
    l, = _record([{"dims": (1 << 23, 4096, 64, 8, 1)}], tmp_path)
    found = [(name, x) for name, x in l if "quant_prepare" in name or "bwd_lists" in name]
    assert len(found) == 3
    for name, x in found:
        assert 1024 * x < 1 << 32, (name, x)
    # and the rest of X: three times the half that such a launch does not hold
    rest = [(name, x) for name, x in l if "quantize_rows_kernel" in name]
    assert len(rest) == 3 and all(16 * x == 1 << 27 for _, x in rest), rest


@pytest.mark.gpu
def test_rows_past_a_launchs_work_items():
    """2^28 + 5 rows of one short block: codes, scales and values are those of the same rows in a small call."""
    torch = _torch()
    base, rows, cols = 65537, (1 << 28) + 5, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    small = torch.randn((base, cols), generator=g, device="cuda")
    small = (small * torch.exp2(torch.randint(-30, 30, (base, 1), generator=g, device="cuda").float())).to(torch.bfloat16)

    def through(x):
        n = x.shape[0]
        q = torch.full((n, cols), 0xAB, dtype=torch.uint8, device="cuda")
        s = torch.full((n, 4), 0xCD, dtype=torch.uint8, device="cuda")
        back = torch.full((n, cols), 7.0, dtype=torch.bfloat16, device="cuda")
        B.moe_quantize_rows(n, cols, x, q, s)
        B.moe_dequantize_rows(n, cols, q, s, back)
        return q, s, back

    want = through(small)
    X = small.repeat(-(-rows // base), 1)[:rows]
    for got, w in zip(through(X), want):
        whole = rows // base
        assert (got[:whole * base].view(whole, base, -1) == w).all()
        assert torch.equal(got[whole * base:], w[:rows - whole * base])


@pytest.mark.gpu
def test_one_row_of_the_most_columns():
    """2^31 - 8 columns: blocks of the last columns as of the first."""
    torch = _torch()
    base, cols = 128 * 1021, (1 << 31) - 8
    g = torch.Generator(device="cuda").manual_seed(2)
    small = torch.randn((base,), generator=g, device="cuda")
    small = (small * torch.exp2(torch.randint(-30, 30, (base,), generator=g, device="cuda").float())).to(torch.bfloat16)

    def through(x):
        n = x.shape[0]
        q = torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda")
        s = torch.full((B.scale_stride(n),), 0xCD, dtype=torch.uint8, device="cuda")
        back = torch.full((n,), 7.0, dtype=torch.bfloat16, device="cuda")
        B.moe_quantize_rows(1, n, x, q, s)
        B.moe_dequantize_rows(1, n, q, s, back)
        return q, s[:-(-n // 128)], back

    X = small.repeat(-(-cols // base))[:cols]
    whole = cols // base
    want, tail = through(small), through(X[whole * base:].clone())
    for got, w, t, per in zip(through(X), want, tail, (1, 128, 1)):
        n = whole * base // per
        assert (got[:n].view(whole, -1) == w).all() and torch.equal(got[n:], t)


if __name__ == "__main__":
    _main()
