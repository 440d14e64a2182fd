"""The four-bit operators where no GPU is needed: layout, encoding and tiles (tests/mx_check.cpp), what the calls refuse before they touch the
device, and the checks of the binding."""
import ctypes
import os
import subprocess

import pytest
import torch

import mx_reference as ref
from paper_2504_12526_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_12526_amd", "csrc")
HEADER = os.path.join(CSRC, "mom_mx.h")
vp = ctypes.c_void_p
OK, NULL, SHAPE, ALIGN, ALIAS, WORKSPACE = (binding.MOM_OK, binding.MOM_ERR_NULL, binding.MOM_ERR_SHAPE, binding.MOM_ERR_ALIGN,
                                            binding.MOM_ERR_ALIAS, binding.MOM_ERR_WORKSPACE)


def _check(tmp_path, include):
    exe = os.path.join(str(tmp_path), "mx_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", include, "-o", exe, os.path.join(ROOT, "tests", "mx_check.cpp")], check=True)
    return subprocess.run([exe], capture_output=True, text=True)


def test_layout_encoding_tiles_and_shares(tmp_path):
    r = _check(tmp_path, CSRC)
    assert r.returncode == 0 and ": ok" in r.stdout, r.stdout


@pytest.mark.parametrize("old,new,says", [
    ("P * (D / 2 + D / 32) + quad * 2 * D", "P * (D / 2 + D / 32) + quad * D", "filled"),
    ("P * (D + D / 32) + quad * (D / 8)", "P * (D + D / 16) + quad * (D / 8)", "append"),
    ("if (back != x) b |= 1;", "", "code"),
    ("b -= 1;", "b -= 0;", "code"),
    ("- 127 - 2 + ((top", "- 127 - 3 + ((top", "scale"),
    ("> (3u << 21) ? 1 : 0", ">= (3u << 21) ? 1 : 0", "scale"),
    ("{ return (m * group + rows - 1) / rows; }", "{ return (m * group + rows) / rows; }", "number"),
    ("{ return T * group / rows + B; }", "{ return T * group / rows; }", "number"),
    ("if (b >= B || tile >=", "if (tile >=", "sequence"),
    ("tile >= tiles_of(m, group, rows))", "tile > tiles_of(m, group, rows))", "sequence"),
    ("checked_tile(b, number - b * tiles,", "checked_tile(b, number,", "tile"),
    ("checked_tile(b, number - before,", "checked_tile(b, number,", "number"),
    ("/ group) + 1;", "/ group);", "divided"),
    ("hi = p1 + 1;", "hi = p1;", "taken"),
    ("const int base = s.lo / kStep * kStep,", "const int base = s.lo / kStep * kStep + kStep,", "taken"),
    ("const int64_t r = window + rows / group + 2 + kStep;", "const int64_t r = window;", "taken"),
])
def test_a_planted_mistake_is_caught(tmp_path, old, new, says):
    """Planted in a copy of the header, on the CPU."""
    text = open(HEADER).read()
    assert text.count(old) == 1, old
    with open(os.path.join(str(tmp_path), "mom_mx.h"), "w") as f:
        f.write(text.replace(old, new))
    r = _check(tmp_path, str(tmp_path))
    assert r.returncode != 0 and says in r.stdout, r.stdout


def test_reference_encoding_by_hand():
    x = torch.zeros(4, 32, dtype=torch.float64)
    x[0, :8] = torch.tensor([6, -0.25, 0.75, 1.25, 2.5, 3.5, 5, 0.3])
    x[1, 0] = 7.0
    x[2, 0] = 7.0 + 1e-9
    x[3, 5] = float("nan")
    codes, scales = ref.encode(x)
    assert codes[0, :8].tolist() == [7, 8, 2, 2, 4, 6, 6, 1] and scales[:, 0].tolist() == [127, 127, 128, 255]
    assert codes[1, 0] == 7 and codes[2, 0] == 6
    v = ref.decode(codes, scales)
    assert v[0, :8].tolist() == [6, 0, 1, 1, 2, 4, 4, 0.5] and v[2, 0] == 8 and v[3].isnan().all()
    assert torch.equal(ref.unpack(ref.pack(codes)), codes)


def test_block_bytes():
    for P in (16, 32, 64, 128, 256):
        for D in (64, 128, 256):
            assert binding.mom_mx_block_bytes(D, P) == ref.block_bytes(P, D)
    for D, P in ((32, 16), (96, 16), (128, 8), (128, 24), (128, 512), (0, 16), (128, 0), (-128, 16)):
        assert binding.mom_mx_block_bytes(D, P) == 0


# fake addresses, far apart and never dereferenced
A = [0x10000000 * (i + 1) for i in range(16)]


def _append(q=A[0], qs=32 * 128, k=A[1], ks=8 * 128, v=A[2], vs=8 * 128, slots=A[3], positions=A[4], freq=A[5], rot=128, T=4, Hq=32, Hkv=8, D=128,
            q_out=A[6], cache=A[7], pages=10, P=16):
    return binding.lib().mom_mx_kv_append(vp(q), qs, vp(k), ks, vp(v), vs, vp(slots), vp(positions), vp(freq), rot, 0, T, Hq, Hkv, D, vp(q_out), vp(cache), pages, P, None)


def test_append_refuses_before_any_launch():
    for bad in (dict(T=-1), dict(D=96), dict(P=24), dict(pages=0), dict(pages=1 << 31), dict(Hkv=0), dict(Hq=0), dict(rot=8), dict(rot=144), dict(rot=-16),
                dict(ks=8 * 128 - 8), dict(vs=8 * 128 + 4), dict(qs=31 * 128), dict(ks=1 << 32)):
        assert _append(**bad) == SHAPE, bad
    for bad in (dict(k=0), dict(v=0), dict(slots=0), dict(cache=0), dict(q_out=0), dict(positions=0), dict(freq=0)):
        assert _append(**bad) == NULL, bad
    for bad in (dict(k=A[1] + 8), dict(v=A[2] + 2), dict(q=A[0] + 4), dict(q_out=A[6] + 8), dict(cache=A[7] + 8), dict(slots=A[3] + 4), dict(positions=A[4] + 2), dict(freq=A[5] + 1)):
        assert _append(**bad) == ALIGN, bad
    block = 8 * ref.block_bytes(16, 128)
    for bad in (dict(cache=A[1]), dict(q_out=A[2]), dict(cache=A[3] - 10 * block + 16), dict(q_out=A[7] + 10 * block - 16), dict(q_out=A[0], qs=33 * 128), dict(q_out=A[0] + 16)):
        assert _append(**bad) == ALIAS, bad
    assert _append(T=0, q=0, k=0, v=0, slots=0, cache=0) == OK


def _read(cache=A[0], pages=10, P=16, slots=A[1], T=4, Hkv=8, D=128, k=A[2], v=A[3]):
    return binding.lib().mom_mx_kv_read(vp(cache), pages, P, vp(slots), T, Hkv, D, vp(k), vp(v), None)


def test_read_refuses_before_any_launch():
    for bad in (dict(T=-1), dict(pages=0), dict(P=17), dict(D=32), dict(Hkv=0)):
        assert _read(**bad) == SHAPE, bad
    for bad in (dict(cache=0), dict(slots=0), dict(k=0), dict(v=0)):
        assert _read(**bad) == NULL, bad
    for bad in (dict(cache=A[0] + 8), dict(slots=A[1] + 4), dict(k=A[2] + 2), dict(v=A[3] + 8)):
        assert _read(**bad) == ALIGN, bad
    for bad in (dict(k=A[0]), dict(v=A[2]), dict(k=A[1] + 16)):
        assert _read(**bad) == ALIAS, bad
    assert _read(T=0, cache=0, slots=0, k=0, v=0) == OK


def _attend(q=A[0], qs=32 * 128, starts=A[1], T=4, B=2, Hq=32, Hkv=8, D=128, cache=A[2], pages=10, P=16, table=A[3], stride=5, lens=A[4], max_kv=80, scale=1.0,
            window=0, out=A[5], lse=A[6], ws=A[7], wsb=None):
    wsb = 1 << 30 if wsb is None else wsb
    return binding.lib().mom_mx_attention(vp(q), qs, vp(starts), T, B, Hq, Hkv, D, vp(cache), pages, P, vp(table), stride, vp(lens), max_kv, scale, window, vp(out),
                                          vp(lse), vp(ws), wsb, None)


def test_attention_refuses_before_any_launch():
    for bad in (dict(T=-1), dict(B=-1), dict(B=0), dict(Hq=30), dict(Hkv=0), dict(D=80), dict(P=20), dict(pages=0), dict(qs=32 * 128 - 8), dict(qs=32 * 128 + 4),
                dict(stride=-1), dict(max_kv=-1), dict(window=-1), dict(starts=0, T=5), dict(max_kv=1 << 31)):
        assert _attend(**bad) == SHAPE, bad
    for bad in (dict(q=0), dict(cache=0), dict(table=0), dict(lens=0), dict(out=0)):
        assert _attend(**bad) == NULL, bad
    for bad in (dict(q=A[0] + 2), dict(cache=A[2] + 8), dict(out=A[5] + 8), dict(table=A[3] + 2), dict(lens=A[4] + 1), dict(starts=A[1] + 2), dict(lse=A[6] + 2)):
        assert _attend(**bad) == ALIGN, bad
    for bad in (dict(out=A[0]), dict(out=A[2] + 16), dict(lse=A[5] + 4), dict(out=A[3]), dict(lse=A[4]), dict(lse=A[1] + 8)):
        assert _attend(**bad) == ALIAS, bad
    # long sequences of few rows are shared out, and take the workspace that the query says
    long = dict(T=1, B=1, starts=0, stride=4096, max_kv=65536, pages=4096, cache=1 << 40)
    need = binding.mom_mx_attention_workspace_bytes(1, 1, 32, 8, 128, 65536)
    assert need > 0
    assert _attend(**long, ws=0) == NULL and _attend(**long, ws=A[7] + 4) == ALIGN and _attend(**long, wsb=1024) == WORKSPACE
    assert _attend(**long, ws=A[5] - need + 64, wsb=need) == ALIAS
    assert _attend(T=0, q=0, cache=0, table=0, lens=0, out=0) == OK


def test_attention_workspace():
    wb = binding.mom_mx_attention_workspace_bytes
    assert wb(1, 1, 32, 8, 128, 256) == 0 and wb(0, 0, 32, 8, 128, 4096) == 0 and wb(1, 1, 30, 8, 128, 4096) == 0 and wb(1, 1, 32, 8, 96, 4096) == 0
    assert wb(8192, 1, 32, 8, 128, 131072) == 0                       # rows enough for every compute unit: nothing is shared out
    sizes = [wb(1, 1, 32, 8, 128, n) for n in (512, 4096, 32768, 131072, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[-1] < 64 << 20           # however long


def test_products_refuse_before_any_launch():
    L = binding.lib()

    def mv(x=A[0], M=2, c=A[1], s=A[2], N=48, K=64, out=A[3], fp32=0, res=A[4]):
        return L.mom_mx_matvec(vp(x), M, vp(c), vp(s), N, K, vp(out), fp32, vp(res), None)

    def gu(x=A[0], M=2, gc=A[1], gs=A[2], uc=A[3], us=A[4], N=48, K=64, out=A[5]):
        return L.mom_mx_gateup(vp(x), M, vp(gc), vp(gs), vp(uc), vp(us), N, K, vp(out), None)

    def qu(w=A[0], N=48, K=64, c=A[1], s=A[2]):
        return L.mom_mx_quantize(vp(w), N, K, vp(c), vp(s), None)

    for call in (mv, gu):
        for bad in (dict(M=-1), dict(M=binding.MOM_MX_MAX_ROWS + 1), dict(N=-1), dict(K=0), dict(K=48), dict(K=32768 + 32)):
            assert call(**bad) == SHAPE, bad
        assert call(M=0) == OK and call(N=0) == OK
        for bad in (dict(x=0), dict(out=0)):
            assert call(**bad) == NULL, bad
        for bad in (dict(x=A[0] + 8), dict(out=A[3] + 2)):
            assert call(**bad) == ALIGN, bad
        for bad in (dict(out=A[0]), dict(out=A[1]), dict(out=A[2])):
            assert call(**bad) == ALIAS, bad
    assert mv(fp32=1) == SHAPE and mv(c=0) == NULL and mv(s=0) == NULL and mv(c=A[1] + 8) == ALIGN and mv(res=A[4] + 8) == ALIGN and mv(res=A[3] + 16) == ALIAS
    assert gu(gc=0) == NULL and gu(us=0) == NULL and gu(uc=A[3] + 4) == ALIGN and gu(out=A[3] + 16) == ALIAS and gu(out=A[4] + 16) == ALIAS
    assert qu(N=-1) == SHAPE and qu(K=33) == SHAPE and qu(K=32800) == SHAPE and qu(N=0) == OK
    assert qu(w=0) == NULL and qu(c=0) == NULL and qu(s=0) == NULL and qu(w=A[0] + 2) == ALIGN and qu(c=A[1] + 4) == ALIGN
    assert qu(c=A[0] + 16) == ALIAS and qu(s=A[1] + 16) == ALIAS


def test_binding_checks_shapes_and_types():
    bf = dict(dtype=torch.bfloat16)
    k = torch.zeros(3, 2, 64, **bf)
    cache = torch.zeros(4, 2, ref.block_bytes(16, 64), dtype=torch.uint8)
    slots, lens, table = torch.zeros(3, dtype=torch.int64), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)
    ap, at, mv = binding.mom_mx_kv_append, binding.mom_mx_attention, binding.mom_mx_matvec
    for call in (lambda: ap(k, k[:2], slots, cache, 16), lambda: ap(k.float(), k, slots, cache, 16), lambda: ap(k, k, slots.int(), cache, 16),
                 lambda: ap(k, k, slots, cache[:, :, :-1], 16), lambda: ap(k, k, slots, cache, 32), lambda: ap(k, k, slots, cache, 16, q=k),
                 lambda: ap(k, k, slots, cache, 16, positions=slots.int()), lambda: ap(k.transpose(0, 1).contiguous().transpose(0, 1), k, slots, cache, 16),
                 lambda: binding.mom_mx_kv_read(cache, 16, slots, k, k.float()), lambda: at(k, cache, 16, table.long(), lens, 9, k, None),
                 lambda: at(k, cache, 16, table, lens.long(), 9, k, None), lambda: at(k, cache, 16, table, lens, 9, k.float(), None),
                 lambda: at(k, cache, 16, table, lens, 9, k.clone(), None, q_starts=lens), lambda: at(k, cache, 16, table, lens, 9, k.clone(), None, lse=k),
                 lambda: mv(torch.zeros(1, 64, **bf), cache[0, :, :32].contiguous(), cache[0, :, :1].contiguous(), torch.zeros(1, 2, **bf)),
                 lambda: mv(torch.zeros(1, 64), cache[0, :, :32].contiguous(), cache[0, :, :2].contiguous(), torch.zeros(1, 2, **bf)),
                 lambda: binding.mom_mx_quantize(torch.zeros(2, 64, **bf), cache[0, :, :32].contiguous(), cache[0, :, :3].contiguous())):
        with pytest.raises(ValueError):
            call()
