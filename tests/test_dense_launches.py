"""Which kernels moe_decode, moe_decode_quant and the dense products launch, without a GPU: launch_recorder.c takes the
place of the HIP launches in a process of its own (as launch_recorder.py does for the other calls)."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

from paper_2512_14080_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libsonicmoe.so not built")
HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def launches(calls, tmp_path):
    """calls: ["decode" | "quant", dims] or ["fwd" | "bwd", T, k, n, act]; a list of (name, grid x, y, z) each."""
    so = os.path.join(str(tmp_path), "launch_recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "launch_recorder.c")], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), so], input=json.dumps(calls), text=True,
                       capture_output=True, cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT + os.pathsep + HERE})
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


def _main():
    rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    rec.rec_name.restype = ctypes.c_char_p
    L, at, out = B.lib(), [1 << 44], []
    ref = ctypes.byref

    def new():  # (addresses that nothing reads, each with room for the largest operand)
        at[0] += 1 << 48
        return at[0]

    def ok(rc):
        assert rc == B.MOE_OK, B.moe_last_error()

    for kind, *sizes in json.load(sys.stdin):
        rec.rec_clear()
        at[0] = 1 << 44
        if kind in ("decode", "quant"):
            D = B.dims(*sizes[0])
            q = B.MoeQExperts()
            ok(L.moe_qexperts_init(D, new(), L.moe_qexperts_bytes(D), ref(q)))
            q.state = B.MOE_HELD_WRITTEN
            X, Wr, W1, W2, O = (new() for _ in range(5))
            if kind == "quant":
                ok(L.moe_decode_quant(D, X, Wr, None, ref(q), None, None, O, None, None, new(), 1 << 46, None))
            else:
                ok(L.moe_decode(D, X, Wr, None, W1, W2, None, None, O, None, None, new(), 1 << 46, None))
        else:
            l = B.linear_dims(*sizes)
            a = [new() for _ in range(7)]
            if kind == "fwd":
                ok(L.moe_linear_fwd(l, a[0], a[1], None, None, None, a[2], a[3], 1 << 46, None))
            else:
                ok(L.moe_linear_bwd(l, a[0], a[1], a[2], a[3], None, a[4], a[5], a[6], new(), 1 << 46, None))
        out.append([(rec.rec_name(i).decode(), *(rec.rec_grid(i, x) for x in range(3))) for i in range(rec.rec_count())])
    print(json.dumps(out))


@pytest.mark.parametrize("kind", ["decode", "quant"])
def test_decode_is_two_launches(kind, tmp_path):
    dims = [(T, d, n, E, K) for T in (1, 2, 8, 9, 17, 64) for d, n, E, K in ((128, 64, 8, 1), (1536, 256, 128, 8),
                                                                           (4096, 512, 1024, 16))]
    for got in launches([[kind, D] for D in dims], tmp_path):
        assert len(got) == 2
        assert "decode_router" in got[0][0] and "decode_kernel" in got[1][0]
        assert got[1][1] <= 256


def test_linear_streams_or_tiles(tmp_path):
    """Streamed in groups of rows while the workgroups are about one round, in tiles beyond."""
    sizes = [(1, 1024, 1536), (45, 1000, 2824), (512, 512, 512), (512, 1000, 2824), (40, 4096, 14336)]
    got = launches([["fwd", *s, "gelu"] for s in sizes], tmp_path)
    assert ["linear_few" in g[0][0] for g in got] == [True, True, True, False, False]
    assert got[1][0][1:] == [23, 1, 3]


def test_linear_whole_rounds(tmp_path):
    """784 tiles of 256 x 256 are three rounds of 256 CUs and 16 more, whose columns have a launch of their own."""
    split, whole = launches([["fwd", 1777, 4096, 14336, "swiglu"], ["fwd", 2048, 4096, 8192, "none"]], tmp_path)
    assert len(split) == 2 and split[0] != split[1]
    assert len(whole) == 1


@pytest.mark.parametrize("act", B.ACTIVATIONS)
def test_linear_grids_fit(act, tmp_path):
    """The largest sizes that are not refused: every launch within 2^31 blocks in x and 65535 in y and z, and its
    workgroups of 256 threads (the streaming one has 512 and small grids) within 2^32 threads."""
    N = 2 if act == "swiglu" else 1
    sizes = [(1 << 28, 8, 8), (1 << 28, 512, 8), (1 << 28, 8, 512 // N), ((1 << 28) - 7, 8, 504 // N // 8 * 8),
             (1 << 22, 1 << 15, (1 << 15) // N), (1 << 13, (1 << 24) - 8, (1 << 13) // N),
             (1 << 13, (1 << 13) // N, ((1 << 24) // N) - 8), (1, (1 << 24) - 8, 8), (1, 8, (1 << 24) - 8), (64, 8, (1 << 24) - 8)]
    for got in launches([[k, *s, act] for s in sizes for k in ("fwd", "bwd")], tmp_path):
        assert got
        for name, x, y, z in got:
            assert 1 <= x and 256 * x * y * z < 1 << 32 and y <= 65535 and z <= 65535, (name, x, y, z)


if __name__ == "__main__":
    _main()
