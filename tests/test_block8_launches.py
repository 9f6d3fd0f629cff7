"""Which kernels the 8-bit calls choose, without a GPU: the rules on sizes.  A process of its own runs each call with
launch_recorder.c in the place of the HIP launches (as launch_recorder.py does for the 16-bit calls)."""
import ctypes
import json
import os
import re
import subprocess
import sys

import pytest

from launch_recorder import record
from paper_2512_14080_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libsonicmoe.so not built")
HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def launches(calls, tmp_path):
    """calls: (dims, "quant" | "kept" | "ckpt" | "bwd", m_tile of a rounding up or 0, whether X is kept)."""
    so = os.path.join(str(tmp_path), "launch_recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "launch_recorder.c")], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), so], input=json.dumps(calls), text=True,
                       capture_output=True, cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT + os.pathsep + HERE})
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


def _main():
    rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    rec.rec_name.restype = ctypes.c_char_p
    from launch_recorder import _routing
    L, p, ws = B.lib(), 0x20000000, (0x30000000, 1 << 62)
    ref, out = ctypes.byref, []

    def ok(rc):
        assert rc == B.MOE_OK, B.moe_last_error()

    for dims, kind, m_tile, keep_x in json.load(sys.stdin):
        D = B.dims(*dims)
        r = _routing(B, D, D.T * D.K)
        ok(L.moe_route(D, p, p, None, 0, ref(r), None))
        if m_tile:
            tc, r = r, _routing(B, D, B.moe_round_capacity(D, m_tile))
            r.mask = tc.mask + 64
            ok(L.moe_round_tokens(D, m_tile, B.ROUND_MODES["up"], None, ref(tc), ref(r), None))
        q, c, flags = B.MoeQExperts(), B.MoeCkpt(), B.MOE_CKPT_X if keep_x else 0
        ok(L.moe_qexperts_init(D, p, L.moe_qexperts_bytes(D), ref(q)))
        ok(L.moe_ckpt_init(D, r.capacity, flags, p, L.moe_ckpt_bytes(D, r.capacity, flags), ref(c)))
        q.state = B.MOE_HELD_WRITTEN
        rec.rec_clear()
        if kind in ("quant", "kept"):
            ok(L.moe_fwd_quant(D, p, ref(q), None, ref(r), ref(c) if kind == "kept" else None, p, *ws, None))
        else:
            ok(L.moe_fwd_ckpt(D, p, p, p, None, ref(r), ref(c), p, *ws, None))
        if kind == "bwd":
            rec.rec_clear()
            ok(L.moe_bwd_ckpt(D, p, None if keep_x else p, ref(c), p, p, None, p, ref(r), p, p, p, p, p, None, *ws, None))
        out.append([(rec.rec_name(i).decode(), rec.rec_grid(i, 0), rec.rec_grid(i, 1)) for i in range(rec.rec_count())])
    print(json.dumps(out))


def _names(l):
    return " ".join(x[0] for x in l)


@pytest.mark.parametrize("dims,m_tile,stream", [
    ((1, 1536, 256, 128, 8), 0, True), ((16, 768, 256, 8, 8), 0, True), ((17, 768, 256, 8, 8), 0, False),
    ((80, 1024, 256, 64, 8), 0, True), ((88, 1024, 256, 64, 8), 0, False),   # 10 and 11 rows an expert
    ((256, 4096, 512, 128, 8), 0, True), ((257, 4096, 512, 128, 8), 0, False),  # 16 and 17 at a long k
    ((64, 4096, 14336, 8, 2), 0, False),
    ((64, 1024, 256, 64, 8), 8, True), ((64, 1024, 256, 64, 8), 16, False),  # rounded up to m_tile rows each
])
def test_few_rows_stream(tmp_path, dims, m_tile, stream):
    l, kept = launches([(dims, "quant", m_tile, False), (dims, "kept", m_tile, False)], tmp_path)
    assert ("stream8" in _names(l)) == stream
    assert ("quant_prepare" in _names(l)) != stream  # (rows quantised as they are loaded, no m-tile list)
    # what is kept is written by the tiled projections
    assert "stream8" not in _names(kept) and "OpUp8" in _names(kept)


@pytest.mark.parametrize("dims,tiles", [
    ((1, 1536, 256, 128, 8), 16), ((2, 1536, 256, 128, 8), 16), ((3, 1536, 256, 128, 8), 8), ((8, 1536, 256, 128, 8), 8),
    ((1, 4096, 14336, 8, 2), 448), ((32, 768, 512, 64, 1), 16), ((9, 1536, 256, 128, 8), 8),  # 85 MB of weights
    ((16, 1536, 256, 128, 8), 0), ((9, 1024, 256, 64, 8), 0), ((8, 2048, 1024, 32, 4), 0),
])
def test_few_tokens_by_row_and_token(tmp_path, dims, tiles):
    """Two launches up to E / 2 rows, or E of few weights; three where there are more, with a rounding, or with a checkpoint."""
    T, d, _, _, K = dims
    l, rounded, kept = launches([(dims, "quant", 0, False), (dims, "quant", 8, False), (dims, "kept", 0, False)], tmp_path)
    if tiles:
        assert [(re.search("stream8_(row_up|token_down)", name).group(1), x, y) for name, x, y in l] == [
            ("row_up", tiles, T * K), ("token_down", d // 32, T)]
    for x in (rounded, kept) if tiles else (l, rounded, kept):
        assert not re.search("stream8_(row_up|token_down)", _names(x)) and "agg_o" in _names(x)


def test_grids_of_the_most_tokens_that_stream(tmp_path):
    """16 rows of each of 4096 experts: no grid past 65535 workgroups but along x."""
    l, = launches([((65536, 4096, 64, 4096, 1), "quant", 0, False)], tmp_path)
    assert "stream8" in _names(l) and "agg_o_f32" in _names(l)
    assert all(y <= 65535 for _, _, y in l), l


@pytest.mark.parametrize("T,E,K,rows", [(40, 512, 8, 16), (100, 128, 8, 32), (300, 2048, 8, 16), (9, 8, 8, 16)])
def test_streaming_grid_holds_a_hot_experts_groups(tmp_path, T, E, K, rows):
    l, = launches([((T, 1536, 256, E, K), "quant", 0, False)], tmp_path)
    for name, _, y in l[:2]:
        assert "stream8" in name and E + K * ((T - 1) // rows) <= y <= E + T * K // rows


@pytest.mark.parametrize("dims,up,down", [
    ((800, 1536, 512, 64, 4), 128, 128), ((1777, 1536, 512, 64, 4), 256, 128), ((8000, 1536, 512, 64, 4), 256, 256),
    ((1000, 1024, 256, 64, 8), 128, 256), ((2000, 1024, 256, 64, 8), 256, 128), ((16384, 1024, 256, 64, 8), 256, 256),
    ((1000, 4096, 512, 128, 8), 128, 128), ((4000, 4096, 512, 128, 8), 256, 256), ((4096, 4096, 14336, 8, 2), 256, 256),
])
def test_tile_rows(tmp_path, dims, up, down):
    l, = launches([(dims, "quant", 0, False)], tmp_path)
    names = _names(l)
    assert int(re.search(r"OpUp8INS_7GemmCfgILi(\d+)E", names).group(1)) == up
    assert int(re.search(r"OpDown8INS_7GemmCfgILi(\d+)E", names).group(1)) == down
    # a second list where the two differ: a workgroup more beside those that quantise X
    per = 64
    assert l[0][1] == 1 + (up != down) + -(-dims[0] * (dims[1] // 128) // per)


@pytest.mark.parametrize("dims,quarters", [
    ((4096, 4096, 14336, 8, 2), True), ((4096, 4096, 4096, 16, 2), True), ((4096, 4096, 4032, 16, 2), False),
    ((300, 4096, 14336, 8, 2), False),  # in tiles of 128 rows
])
def test_the_last_round_of_a_long_k_in_quarters(tmp_path, dims, quarters):
    l, = launches([(dims, "quant", 0, False)], tmp_path)
    down = [(re.search(r"OpDown8INS_7GemmCfgILi(\d+)E.*EELi(\d)E", name).groups(), x) for name, x, _ in l if "OpDown8" in name]
    if quarters:  # (a round may leave half of its workgroups' tiles, each four quarters)
        assert [g for g, _ in down] == [("256", "1"), ("128", "2")] and [x for _, x in down] == [256, 512]
    else:
        assert len(down) == 1 and down[0][0][1] == "0"


def test_kept_x_needs_no_launch_of_its_own(tmp_path):
    dims = (5003, 896, 192, 40, 3)
    fwd, fwd_x, bwd, bwd_x = launches([(dims, k, 0, x) for k in ("ckpt", "bwd") for x in (False, True)], tmp_path)
    assert len(fwd) == len(fwd_x) and len(bwd) == len(bwd_x)
    assert "quant_prepare" in _names(fwd_x) and "OpUpCkpt" in _names(fwd)
    lists, lists_x = (next(x for x in l if "bwd_lists" in x[0]) for l in (bwd, bwd_x))
    assert lists_x[1] - lists[1] == -(-5003 * 7 // 64)
    for l in (bwd, bwd_x):  # dH from 8-bit H: the last template argument
        assert re.search(r"OpDHINS_7GemmCfg.*?EELb[01]ELb1E", _names(l))


@pytest.mark.parametrize("dims", [(32768, 1536, 256, 128, 8), (1777, 1536, 512, 64, 4), (64, 1024, 256, 64, 8)])
@pytest.mark.parametrize("which", [B.MOE_WS_FWD_QUANT, B.MOE_WS_FWD_CKPT, B.MOE_WS_BWD_CKPT])
def test_workspace_size_does_not_depend_on_the_device(tmp_path, dims, which):
    sizes = [record([{"call": "ws", "dims": dims, "which": which, "cus": c}], tmp_path)[0] for c in (256, 32, 64, 304)]
    assert len(set(sizes)) == 1, sizes


def test_workspace_of_a_rounding_that_streams_in_wider_groups(tmp_path):
    """A capacity whose groups of 16 rows pass the grid's 65535 and whose groups of 32 do not: an A in fp32 is there."""
    D = B.dims(1024, 128, 64, 4096, 8)
    cap = 1 << 20
    assert D.E + cap // 16 > 65535 >= D.E + cap // 32
    n = B.lib().moe_workspace_bytes(D, cap, B.MOE_WS_FWD_QUANT)
    parts = cap * (4 * D.n + 128 + 4 + 2 * D.d) + D.T * (D.d + 4)  # A32, A8, their scales, Y; X and its scales
    assert n >= parts


if __name__ == "__main__":
    _main()
