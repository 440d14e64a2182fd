"""Drafted tokens in a tree where no GPU is needed: what rows see, shares, powers and workspaces (tests/draft_check.cpp), the reference by hand, what the calls refuse before
they touch the device, and the checks of the binding."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import draft_reference as dref
import mx_reference as ref
from paper_2504_12526_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_12526_amd", "csrc")
HEADER = os.path.join(CSRC, "mom_draft.h")
vp = ctypes.c_void_p
OK, NULL, SHAPE, ALIGN, ALIAS, WORKSPACE = (binding.MOM_OK, binding.MOM_ERR_NULL, binding.MOM_ERR_SHAPE, binding.MOM_ERR_ALIGN,
                                            binding.MOM_ERR_ALIAS, binding.MOM_ERR_WORKSPACE)


def _check(tmp_path, include):
    exe = os.path.join(str(tmp_path), "draft_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", include, "-o", exe, os.path.join(ROOT, "tests", "draft_check.cpp")], check=True)
    return subprocess.run([exe], capture_output=True, text=True, timeout=60)


def test_what_rows_see_shares_powers_and_workspaces(tmp_path):
    r = _check(tmp_path, CSRC)
    assert r.returncode == 0 and ": ok" in r.stdout, r.stdout


@pytest.mark.parametrize("old,new,says", [
    ("if (hi > 32) hi = 32;", "if (hi > 31) hi = 31;", "bits"),
    ("if (hi <= lo) return 0;", "if (hi < lo) return 0;", "bits"),
    ("w + 1 < words ? mask[w + 1]", "w + 2 < words ? mask[w + 1]", "mask bit"),
    ("high << (32 - s)", "high << (31 - s)", "mask bit"),
    ("return p >= 0 && p < j ? p : -1;", "return p >= 0 ? p : -1;", "above"),
    ("for (int i = left; i < count; ++i) x &= x - 1;", "", "sight"),
    ("return {base, 32 * w", "return {0, 32 * w", "sight"),
    ("left -= count;", "", "sight"),
    ("return {base > left ? base - left : 0, lowest};", "return {0, lowest};", "sight"),
    ("n - m > window ? n - m - window : 0;", "n - m > window ? n - m - window + 1 : 0;", "span"),
    ("base - window + (m < window ? m : window) : 0;", "base - window : 0;", "whole"),
    ("    q += q * share < steps;\n    q += q * share < steps;\n", "", "shares"),
    ("<= workgroups) hi = mid;", "<= 2 * workgroups) hi = mid;", "plan share"),
    ("(size_t)p.workgroups * Hkv * p.rows", "(size_t)p.numbers * Hkv * p.rows", "plan"),
    ("y = fma(y, f, c3);", "", "power"),
    ("c10 = c9 * kLn2 / 10;", "c10 = 0;", "power"),
    ("t = t > -1100.0 ? t : -1100.0;", "", "power"),
    ("{ return (V + kChunk - 1) / kChunk; }", "{ return V / kChunk + 1; }", "chunks"),
    ("l.lists = l.rows + 2 * (size_t)T * sizeof(Row);", "l.lists = l.rows + (size_t)T * sizeof(Row);", "layout"),
])
def test_a_planted_mistake_is_caught(tmp_path, old, new, says):
    """Planted in a copy of the header, on the CPU."""
    text = open(HEADER).read()
    assert text.count(old) == 1, old
    shutil.copy(os.path.join(CSRC, "mom_mx.h"), str(tmp_path))
    with open(os.path.join(str(tmp_path), "mom_draft.h"), "w") as f:
        f.write(text.replace(old, new))
    r = _check(tmp_path, str(tmp_path))
    assert r.returncode != 0 and says in r.stdout, r.stdout


def test_reference_by_hand():
    assert dref.tree(torch.tensor([-1, 0, 0, 1, 7]), [0, 5], 5, [9], 1)[:2] == ([[1], [3], [5], [11], [16]], [4, 5, 5, 6, 4])
    p = torch.log(torch.tensor([[0.5, 0.3, 0.2], [0.1, 0.1, 0.8], [0.6, 0.2, 0.2]]))
    q = torch.log(torch.tensor([[0.2, 0.7, 0.1], [1 / 3, 1 / 3, 1 / 3], [0.1, 0.1, 0.8]]))
    go = lambda u, **k: dref.verify(p, k.get("q", q), [0, 1, 0], k.get("parents", [-1, 0, 0]), k.get("children", 2), [0, 3], [k.get("t", 1.0)], u)
    # the first child has 0.3 of the 0.7 it was drawn with; what is left then is (0.3, 0, 0.1) / 0.4, and the second 0.75 of 0.2
    assert go([0.95, 0.42, 0.0]) == ([0, 1, -1], [1, 2, -1], [2])
    assert go([0.15, 0.43, 0.9]) == ([0, 2, -1], [0, 0, -1], [2])
    # one child alone: what is left is drawn from, token 0 up to 0.75
    assert go([0.74, 0.43, 0.0], children=1) == ([0, -1, -1], [0, -1, -1], [1]) and go([0.76, 0.43, 0.0], children=1)[1][0] == 2
    # without q the refused token alone goes: (0.5, 0, 0.2) / 0.7
    assert go([0.5, 0.31, 0.71], q=None)[0] == [0, 2, -1] and go([0.72, 0.31, 0.72], q=None) == ([0, -1, -1], [2, -1, -1], [1])
    assert go([0.0, 0.9, 0.9], t=0.0) == ([0, 2, -1], [0, 0, -1], [2])
    assert go([0.05, 0.42, 0.0], parents=[-1, 0, 1])[0] == [0, 1, 2]
    cache = torch.arange(2 * ref.block_bytes(16, 64), dtype=torch.int64).to(torch.uint8).view(2, 1, -1)
    moved, lens = dref.keep(cache, 16, 64, torch.tensor([[1, 0]]), [20], [0, 6], [0, 2, 5, -1, -1, -1], [3])
    assert lens == [17]
    for to, source in ((15, 16), (16, 19)):
        for x, y in zip(ref.get(moved, 16, 64, 1 - to // 16, to % 16), ref.get(cache, 16, 64, 1 - source // 16, source % 16)):
            assert torch.equal(torch.nan_to_num(x, nan=-1e9), torch.nan_to_num(y, nan=-1e9))


# fake addresses, far apart and never dereferenced
A = [0x10000000 * (i + 1) for i in range(20)]


def _tree(parents=A[0], starts=A[1], T=6, B=2, lens=A[2], table=A[3], stride=4, P=16, max_kv=64, masks=A[4], words=1, positions=A[5], slots=A[6]):
    return binding.lib().mom_mx_tree(vp(parents), vp(starts), T, B, vp(lens), vp(table), stride, P, max_kv, vp(masks), words, vp(positions), vp(slots), None)


def test_tree_refuses_before_any_launch():
    for bad in (dict(T=-1), dict(T=(1 << 29) + 1), dict(B=-1), dict(B=0), dict(words=0), dict(words=17), dict(P=24), dict(stride=-1), dict(max_kv=-1), dict(starts=0, T=7)):
        assert _tree(**bad) == SHAPE, bad
    for bad in (dict(lens=0), dict(table=0)):
        assert _tree(**bad) == NULL, bad
    for bad in (dict(parents=A[0] + 2), dict(starts=A[1] + 1), dict(lens=A[2] + 2), dict(table=A[3] + 2), dict(masks=A[4] + 2), dict(positions=A[5] + 1), dict(slots=A[6] + 4)):
        assert _tree(**bad) == ALIGN, bad
    for bad in (dict(masks=A[0]), dict(positions=A[1] + 8), dict(slots=A[2]), dict(slots=A[3] + 24), dict(masks=A[5] + 20), dict(positions=A[6])):
        assert _tree(**bad) == ALIAS, bad
    assert _tree(T=0, lens=0, table=0) == OK and _tree(masks=0, positions=0, slots=0) == OK


def _attend(q=A[0], qs=32 * 128, starts=A[1], T=4, B=2, Hq=32, Hkv=8, D=128, cache=A[2], pages=10, P=16, table=A[3], stride=5, lens=A[4], max_kv=80, scale=1.0,
            window=0, masks=A[8], words=2, out=A[5], lse=A[6], ws=A[7], wsb=1 << 30):
    return binding.lib().mom_mx_tree_attention(vp(q), qs, vp(starts), T, B, Hq, Hkv, D, vp(cache), pages, P, vp(table), stride, vp(lens), max_kv, scale, window, vp(masks), words,
                                               vp(out), vp(lse), vp(ws), wsb, None)


def test_attention_refuses_before_any_launch():
    for bad in (dict(T=-1), dict(B=-1), dict(B=0), dict(Hq=30), dict(Hkv=0), dict(D=80), dict(P=20), dict(pages=0), dict(qs=32 * 128 - 8), dict(qs=32 * 128 + 4),
                dict(stride=-1), dict(max_kv=-1), dict(window=-1), dict(starts=0, T=5), dict(max_kv=1 << 31), dict(words=0), dict(words=17)):
        assert _attend(**bad) == SHAPE, bad
    for bad in (dict(q=0), dict(cache=0), dict(table=0), dict(lens=0), dict(out=0), dict(masks=0)):
        assert _attend(**bad) == NULL, bad
    for bad in (dict(q=A[0] + 2), dict(cache=A[2] + 8), dict(out=A[5] + 8), dict(table=A[3] + 2), dict(lens=A[4] + 1), dict(starts=A[1] + 2), dict(lse=A[6] + 2), dict(masks=A[8] + 1)):
        assert _attend(**bad) == ALIGN, bad
    for bad in (dict(out=A[0]), dict(out=A[2] + 16), dict(lse=A[5] + 4), dict(out=A[3]), dict(lse=A[4]), dict(lse=A[1] + 8), dict(lse=A[8] + 28), dict(out=A[8])):
        assert _attend(**bad) == ALIAS, bad
    long = dict(T=1, B=1, starts=0, stride=4096, max_kv=65536, pages=4096, cache=1 << 40)
    need = binding.mom_mx_tree_attention_workspace_bytes(1, 1, 32, 8, 128, 65536)
    assert need > 0
    assert _attend(**long, ws=0) == NULL and _attend(**long, ws=A[7] + 4) == ALIGN and _attend(**long, wsb=1024) == WORKSPACE
    assert _attend(**long, ws=A[5] - need + 64, wsb=need) == ALIAS
    assert _attend(T=0, q=0, cache=0, table=0, lens=0, out=0, masks=0) == OK
    wb = binding.mom_mx_tree_attention_workspace_bytes
    assert wb(1, 1, 32, 8, 128, 256) == 0 and wb(0, 0, 32, 8, 128, 4096) == 0 and wb(1, 1, 30, 8, 128, 4096) == 0 and wb(1, 1, 32, 8, 96, 4096) == 0
    for args in ((16, 1, 32, 8, 128), (256, 32, 32, 8, 128), (300, 5, 28, 4, 128), (64, 4, 16, 1, 64), (80, 1, 8, 2, 256)):
        sizes = [wb(*args, n) for n in [*range(0, 9000, 37), *range(9000, 1 << 20, 7001)]]
        assert sizes == sorted(sizes), args


def _verify(target=1 << 40, ts=5000, draft=1 << 41, ds=5000, bf16=0, V=5000, tokens=A[0], parents=A[1], children=2, starts=A[2], T=6, B=2, temps=A[3], u=A[4], rows=A[5], out=A[6],
            counts=A[7], ws=A[8], wsb=1 << 30):
    return binding.lib().mom_verify_drafts(vp(target), ts, vp(draft), ds, bf16, V, vp(tokens), vp(parents), children, vp(starts), T, B, vp(temps), vp(u), vp(rows), vp(out), vp(counts),
                                           vp(ws), wsb, None)


def test_verify_refuses_before_any_launch():
    for bad in (dict(T=-1), dict(B=-1), dict(B=0), dict(V=0), dict(V=(1 << 30) + 1), dict(children=0), dict(ts=4999), dict(ds=4999), dict(ts=1 << 32), dict(starts=0, T=7),
                dict(T=1 << 29), dict(T=1 << 24, ts=1 << 20, ds=1 << 20, V=1 << 20), dict(T=1 << 25, B=1 << 25, draft=0)):
        assert _verify(**bad) == SHAPE, bad
    for bad in (dict(target=0), dict(tokens=0), dict(u=0), dict(rows=0), dict(out=0), dict(counts=0), dict(ws=0)):
        assert _verify(**bad) == NULL, bad
    for bad in (dict(target=(1 << 40) + 2), dict(draft=(1 << 41) + 1), dict(draft=(1 << 41) + 1, bf16=1), dict(tokens=A[0] + 1), dict(parents=A[1] + 2), dict(starts=A[2] + 2), dict(temps=A[3] + 2),
                dict(u=A[4] + 1), dict(rows=A[5] + 2), dict(out=A[6] + 1), dict(counts=A[7] + 2), dict(ws=A[8] + 8)):
        assert _verify(**bad) == ALIGN, bad
    need = binding.mom_verify_drafts_workspace_bytes(6, 2, 5000)
    assert _verify(wsb=need - 1) == WORKSPACE
    for bad in (dict(rows=A[0]), dict(out=A[1] + 4), dict(counts=A[2]), dict(rows=A[6] + 20), dict(counts=A[4] + 20), dict(ws=A[5] - need + 16, wsb=need), dict(ws=(1 << 40) + 6 * 5000 * 4 - 16),
                dict(rows=(1 << 41) + 64), dict(counts=A[3])):
        assert _verify(**bad) == ALIAS, bad
    assert _verify(T=0, target=0, tokens=0, u=0, rows=0, out=0, counts=0, ws=0) == OK
    wb = binding.mom_verify_drafts_workspace_bytes
    assert wb(0, 1, 5) == 0 and wb(1, 0, 5) == 0 and wb(1, 1, 0) == 0 and wb(1, 1, 5) > 0


def _keep(cache=1 << 40, pages=10, P=16, Hkv=8, D=128, table=A[0], stride=4, max_kv=64, lens=A[1], starts=A[2], T=6, B=2, rows=A[3], counts=A[4], new=A[5]):
    return binding.lib().mom_mx_kv_keep(vp(cache), pages, P, Hkv, D, vp(table), stride, max_kv, vp(lens), vp(starts), T, B, vp(rows), vp(counts), vp(new), None)


def test_keep_refuses_before_any_launch():
    for bad in (dict(T=-1), dict(B=-1), dict(B=0), dict(pages=0), dict(P=24), dict(Hkv=0), dict(D=96), dict(stride=-1), dict(max_kv=-1), dict(starts=0, T=7), dict(B=1 << 27)):
        assert _keep(**bad) == SHAPE, bad
    for bad in (dict(cache=0), dict(table=0), dict(lens=0), dict(rows=0), dict(counts=0), dict(new=0)):
        assert _keep(**bad) == NULL, bad
    for bad in (dict(cache=(1 << 40) + 8), dict(table=A[0] + 2), dict(lens=A[1] + 1), dict(starts=A[2] + 2), dict(rows=A[3] + 1), dict(counts=A[4] + 2), dict(new=A[5] + 1)):
        assert _keep(**bad) == ALIGN, bad
    for bad in (dict(new=A[1]), dict(new=A[4] + 4), dict(new=A[3] + 20), dict(table=(1 << 40) + 64), dict(new=A[0] + 28), dict(rows=(1 << 40) + 8)):
        assert _keep(**bad) == ALIAS, bad
    assert _keep(T=0, B=0, cache=0, rows=0) == OK


def test_binding_checks_shapes_and_types():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    lens, table, rows, lg, ws = i32(2), i32(2, 4), i32(6), torch.zeros(6, 50), torch.zeros(9, dtype=torch.uint8)
    q = torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    cache = torch.zeros(4, 2, ref.block_bytes(16, 64), dtype=torch.uint8)
    tr, at, ve, ke = binding.mom_mx_tree, binding.mom_mx_tree_attention, binding.mom_verify_drafts, binding.mom_mx_kv_keep
    u = torch.zeros(6)
    for call in (lambda: tr(lens), lambda: tr(lens, masks=rows.long().view(6, 1)), lambda: tr(lens, positions=rows, parents=rows[:5]), lambda: tr(lens.long(), positions=rows),
                 lambda: tr(lens, positions=i32(7)), lambda: tr(lens, slots=rows), lambda: tr(lens, slots=rows.long(), page_table=table[:1], page_tokens=16),
                 lambda: tr(lens, slots=rows.long(), page_table=table.long(), page_tokens=16), lambda: tr(lens, positions=rows, q_starts=i32(2)),
                 lambda: at(q, cache, 16, table, lens, 9, rows, q, None), lambda: at(q, cache, 16, table, lens, 9, i32(5, 1), q, None), lambda: at(q, cache, 16, table, lens, 9, i32(6, 2)[:, :1], q, None),
                 lambda: at(q, cache, 16, table, lens.long(), 9, i32(6, 1), q, None), lambda: at(q, cache, 16, table, lens, 9, i32(6, 1), q.float(), None),
                 lambda: ve(lg.double(), rows, u, rows, rows, lens, ws), lambda: ve(lg, rows.long(), u, rows, rows, lens, ws), lambda: ve(lg, rows, u.double(), rows, rows, lens, ws),
                 lambda: ve(lg, rows, u, rows, rows, lens, ws, draft=lg.bfloat16()), lambda: ve(lg, rows, u, rows, rows, lens, ws, draft=lg[:5]), lambda: ve(lg.t().contiguous().t(), rows, u, rows, rows, lens, ws),
                 lambda: ve(lg, rows, u, rows, rows, i32(4), ws), lambda: ve(lg, rows, u, rows, rows, lens, ws, temperatures=u), lambda: ve(lg, rows, u, rows, rows, lens, ws, parents=lens),
                 lambda: ke(cache, 16, 128, table, lens, rows, lens, lens), lambda: ke(cache, 16, 64, table, lens, rows.long(), lens, lens), lambda: ke(cache, 16, 64, table, lens, rows, i32(3), lens),
                 lambda: ke(cache, 16, 64, table, lens, i32(7), lens, lens)):
        with pytest.raises((ValueError, AttributeError)):
            call()
