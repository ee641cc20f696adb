"""What the calls on rotated rows and drafted trees refuse before any GPU work, and the registers of their kernels (CPU: nothing is run)."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2406_05317_amd import binding as lb
from paper_2406_05317_amd import build as lib_build
from test_pages_cpu import BAD_PAGES, FAKE, pages, requests, tensor

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = lb.LOCOCO_OK, lb.LOCOCO_EINVAL, lb.LOCOCO_EUNSUPPORTED, lb.LOCOCO_EWORKSPACE


def rotation(**over):
    kw = dict(struct_size=C.sizeof(lb.lococo_rotation), dtype=lb.LOCOCO_BF16, n_q_heads=8, n_kv_heads=2, head_dim=128, rotary_dim=128, pairing=0,
              norm=1, norm_eps=0.0, freqs=FAKE[11], q_weight=FAKE[12], k_weight=FAKE[13], q_weight_stride=0, k_weight_stride=0)
    kw.update(over)
    return lb.lococo_rotation(*(kw[n] for n, _ in lb.lococo_rotation._fields_))


Q, K, QO, KO = (tensor(FAKE[i]) for i in (6, 7, 8, 9))
DQO, DKO, DQ, DK, DQW, DKW = (0x900000 + 0x10000 * i for i in range(6))


def rotate(rot=None, q=Q, k=K, qo=QO, ko=KO, per=3, tokens=3, positions=FAKE[10]):
    r = rotation() if rot is None else rot
    ref = lambda x: x and C.byref(x)
    return lb.lib().lococo_rows_rotate(C.byref(r), ref(q), ref(k), ref(qo), ref(ko), per, tokens, positions, None)


def back(rot=None, q=Q, k=K, per=3, tokens=3, positions=FAKE[10], gqo=DQO, gko=DKO, gq=DQ, gk=DK, gqw=DQW, gkw=DKW, ws=None, size=0):
    r = rotation() if rot is None else rot
    ref = lambda x: x and C.byref(x)
    return lb.lib().lococo_rows_rotate_backward(C.byref(r), ref(q), ref(k), per, tokens, positions, gqo, gko, gq, gk, gqw, gkw, ws, size, None)


def append(pg=None, rot=None, q=Q, k=K, v=KO, qo=QO, per=3, tokens=3, slots=FAKE[10], positions=FAKE[14]):
    p, r = pages() if pg is None else pg, rotation() if rot is None else rot
    ref = lambda x: x and C.byref(x)
    return lb.lib().lococo_pages_append(C.byref(p), C.byref(r), ref(q), ref(k), ref(v), ref(qo), per, tokens, slots, positions, None)


BAD_ROTATIONS = [(dict(struct_size=8), EINVAL), (dict(dtype=5), EINVAL), (dict(n_q_heads=0), EINVAL), (dict(n_kv_heads=-1), EINVAL),
                 (dict(n_q_heads=65536), EUNSUPPORTED), (dict(head_dim=0), EINVAL), (dict(head_dim=100), EUNSUPPORTED),
                 (dict(head_dim=264), EUNSUPPORTED), (dict(rotary_dim=130), EINVAL), (dict(rotary_dim=-2), EINVAL), (dict(rotary_dim=63), EINVAL),
                 (dict(pairing=2), EINVAL), (dict(norm=2), EINVAL), (dict(norm=0, rotary_dim=0, q_weight=None, k_weight=None), EINVAL),
                 (dict(norm_eps=-1.0), EINVAL), (dict(norm_eps=float("inf")), EINVAL), (dict(norm_eps=float("nan")), EINVAL),
                 (dict(freqs=None), EINVAL), (dict(freqs=FAKE[11] + 2), EINVAL), (dict(norm=0), EINVAL), (dict(q_weight=FAKE[12] + 8), EINVAL),
                 (dict(k_weight=None, k_weight_stride=128), EINVAL), (dict(k_weight_stride=64), EINVAL), (dict(q_weight_stride=132), EINVAL),
                 (dict(dtype=lb.LOCOCO_F32, q_weight=FAKE[12] + 2), EINVAL)]


@pytest.mark.parametrize("over,want", BAD_ROTATIONS)
def test_rotations_are_checked_by_every_call(over, want):
    r, out = rotation(**over), C.c_size_t(0)
    assert rotate(r) == back(r) == append(rot=r) == want
    assert lb.lib().lococo_rows_rotate_backward_workspace_bytes(C.byref(r), 3, C.byref(out)) == want
    assert len(lb.lib().lococo_last_error()) > 0


def test_rotation_of_rows_checks_its_arguments():
    L, r = lb.lib(), rotation()
    assert L.lococo_rows_rotate(None, C.byref(Q), C.byref(K), C.byref(QO), C.byref(KO), 3, 3, None, None) == EINVAL
    assert rotate(q=None, k=None, qo=None, ko=None) == rotate(q=None) == rotate(k=None) == rotate(qo=None) == rotate(ko=None) == EINVAL
    assert rotate(per=0) == rotate(tokens=-1) == rotate(positions=FAKE[10] + 1) == EINVAL
    assert rotate(per=2 ** 30, tokens=2 ** 30) == EUNSUPPORTED
    for bad in (tensor(None), tensor(FAKE[6] + 8), tensor(st=64), tensor(st=132), tensor(sh=-8)):
        assert rotate(q=bad) == rotate(k=bad) == rotate(qo=bad) == rotate(ko=bad) == EINVAL
    # in place with other strides; onto the other's rows
    assert rotate(qo=tensor(FAKE[6], sh=2048)) == rotate(ko=tensor(FAKE[7], st=256)) == EINVAL
    assert rotate(qo=KO) == rotate(qo=K) == rotate(ko=Q) == EINVAL
    # 16 rows at a time, two blocks of heads: fewer than 2^24 workgroups
    few = rotation(n_q_heads=8, n_kv_heads=8)
    fit = 16 * (2 ** 23 - 1)
    assert rotate(few, per=fit + 1, tokens=fit + 1) == EUNSUPPORTED
    assert rotate(tokens=0, q=tensor(None), k=tensor(None), qo=tensor(None), ko=tensor(None)) == OK


def test_the_way_back_checks_its_arguments():
    L, out = lb.lib(), C.c_size_t(0)
    assert back(q=None, k=None) == back(q=None) == back(k=None) == EINVAL            # a weight's gradient without its rows
    plain = rotation(q_weight=None, k_weight=None)
    assert back(plain) == back(plain, gkw=None) == EINVAL
    for name in ("gqo", "gko", "gq", "gk"):
        assert back(**{name: None}) == EINVAL, name
        assert back(**{name: DQ + 2}) == EINVAL, name
    for name in ("gqw", "gkw"):
        assert back(**{name: DQW + 1}) == EINVAL
        for other in (FAKE[6], FAKE[7], FAKE[11], FAKE[12], FAKE[10], DQO, DKO, DQ):
            assert back(**{name: other}) == EINVAL, (name, hex(other))
    assert back(gq=FAKE[6]) == back(gq=FAKE[7]) == back(gk=DQ) == back(gq=DKO) == back(gk=DQO) == back(gq=FAKE[10]) == EINVAL
    assert back(per=0) == back(tokens=-1) == EINVAL
    assert back(per=2 ** 30, tokens=2 ** 30) == EUNSUPPORTED
    r = rotation()
    assert L.lococo_rows_rotate_backward_workspace_bytes(C.byref(r), 3, None) == EINVAL
    assert L.lococo_rows_rotate_backward_workspace_bytes(C.byref(r), -1, C.byref(out)) == EINVAL
    assert L.lococo_rows_rotate_backward_workspace_bytes(C.byref(r), 2 ** 30, C.byref(out)) == EUNSUPPORTED
    assert L.lococo_rows_rotate_backward_workspace_bytes(C.byref(plain), 3, C.byref(out)) == OK and out.value == 0
    assert L.lococo_rows_rotate_backward_workspace_bytes(C.byref(r), 3, C.byref(out)) == OK and out.value > 0
    need = out.value
    for ws, size in ((None, 0), (None, need), (0xa00000, need - 1), (0xa00000 + 64, need)):
        assert back(ws=ws, size=size) == back(ws=ws, size=size, gqw=None) == EWORKSPACE
    assert back(tokens=0, q=tensor(None), k=tensor(None), gqo=None, gko=None, gq=None, gk=None, ws=None) == OK


@pytest.mark.parametrize("hq,hkv,strides", [(32, 8, 0), (1, 1, 0), (32, 8, 128), (5, 3, 0), (64, 64, 128)])
def test_workspace_of_the_way_back_is_bounded(hq, hkv, strides):
    """A row of head_dim floats for each workgroup: sixteen to a compute unit, or one to a block of heads where those are more."""
    out = C.c_size_t(0)
    for tokens in (0, 1, 17, 1000, 10 ** 5, 2 ** 30 - 2):
        r = rotation(n_q_heads=hq, n_kv_heads=hkv, q_weight_stride=strides, k_weight_stride=strides)
        assert lb.lib().lococo_rows_rotate_backward_workspace_bytes(C.byref(r), tokens, C.byref(out)) == OK
        assert 0 < out.value <= max(16 * 256, hq + hkv) * 128 * 4 + 256


@pytest.mark.parametrize("over,want", BAD_PAGES)
def test_pages_are_checked(over, want):
    p = pages(**over)
    assert append(pg=p) == want
    m = FAKE[12]
    r = requests()
    assert lb.lib().lococo_pages_attn_tree(C.byref(p), C.byref(r), C.byref(Q), C.byref(QO), 3, m, 1, None, 0, None) == want
    assert lb.lib().lococo_pages_move(C.byref(p), 2, 3, FAKE[4], FAKE[5], FAKE[6], None) == want


def test_append_checks_its_arguments():
    for over in (dict(dtype=lb.LOCOCO_F32), dict(n_q_heads=4), dict(n_kv_heads=1), dict(head_dim=64, rotary_dim=64)):
        assert append(rot=rotation(**over)) == EINVAL, over
    for name in ("q", "k", "v", "qo"):
        for bad in (None, tensor(None), tensor(FAKE[6] + 8), tensor(st=64), tensor(sb=12)):
            assert append(**{name: bad}) == EINVAL, name
    assert append(qo=K) == append(qo=KO) == append(qo=tensor(FAKE[6], sh=2048)) == EINVAL
    assert append(slots=None) == append(positions=None) == append(slots=FAKE[10] + 2) == append(positions=FAKE[10] + 1) == EINVAL
    assert append(per=0) == append(tokens=-1) == EINVAL
    assert append(per=2 ** 30, tokens=2 ** 30) == EUNSUPPORTED
    none = tensor(None)
    assert append(q=none, k=none, v=none, qo=none, tokens=0, slots=None, positions=None) == OK


def test_trees_check_their_arguments():
    L = lb.lib()
    names = ["starts", "held", "bases", "parents", "masks", "positions"]

    def tree(n=3, tokens=4, words=2, **over):
        a = {**dict(zip(names, FAKE)), **over}
        return L.lococo_pages_tree(n, tokens, a["starts"], a["held"], a["bases"], a["parents"], words, a["masks"], a["positions"], None)

    for name in names:
        if name != "bases":
            assert tree(**{name: None}) == EINVAL, name
        assert tree(**{name: FAKE[9] + 2}) == EINVAL, name
    for out in ("masks", "positions"):
        for src in names[:4]:
            assert tree(**{out: FAKE[names.index(src)]}) == EINVAL, (out, src)
    assert tree(masks=FAKE[5]) == EINVAL
    assert tree(n=0) == tree(tokens=-1) == tree(words=0) == EINVAL
    assert tree(n=4097) == tree(tokens=2 ** 30) == tree(words=9) == EUNSUPPORTED
    assert L.lococo_pages_tree(1, 0, None, None, None, None, 1, None, None, None) == OK


def test_attention_under_masks_checks_its_arguments():
    L, p, r = lb.lib(), pages(), requests()

    def attn(q=Q, o=QO, per=3, masks=FAKE[12], words=1, rq=r, ws=None, size=0):
        return L.lococo_pages_attn_tree(C.byref(p), C.byref(rq), q and C.byref(q), o and C.byref(o), per, masks, words, ws, size, None)

    assert attn(masks=None) == attn(masks=FAKE[12] + 2) == attn(words=0) == attn(words=-1) == EINVAL
    assert attn(words=9) == EUNSUPPORTED
    assert attn(o=Q) == attn(q=None) == attn(o=None) == attn(per=0) == EINVAL
    for bad in (tensor(None), tensor(FAKE[7] + 8), tensor(st=64)):
        assert attn(q=bad) == attn(o=bad) == EINVAL
    for over in (dict(n=0), dict(max_new=1), dict(tables=None), dict(starts=FAKE[5] + 2), dict(held=None)):
        assert attn(rq=requests(**over)) == EINVAL, over
    long = requests(n=1, tokens=1, max_new=1, max_held=100000, table_pages=2000)
    assert attn(per=1, rq=long) == EWORKSPACE
    assert L.lococo_pages_attn_tree(C.byref(p), C.byref(requests(tokens=0, max_new=0)), C.byref(tensor(None)), C.byref(tensor(None)), 1, None, 0, None, 0,
                                    None) == OK


def test_workspace_under_masks_does_not_shrink_with_more_keys():
    """A workspace for a larger max_held serves calls with a smaller one, whichever way either is dealt out."""
    L, out = lb.lib(), C.c_size_t(0)
    for p in (pages(), pages(n_q_heads=32, n_kv_heads=8), pages(dtype=lb.LOCOCO_F32, head_dim=64)):
        for n, new in ((1, 1), (3, 9), (70, 1), (32, 60), (5, 250)):
            last = 0
            for held in sorted([1, 511, 768, 769, 1000, 2048, 2049, 5000, 30000, 65536, 10 ** 6, 2 ** 31 - 1]):
                r = requests(n=n, tokens=n * new, max_new=new, max_held=held, table_pages=2 ** 23)
                assert L.lococo_pages_attn_tree_workspace_bytes(C.byref(p), C.byref(r), C.byref(out)) == OK
                assert out.value >= last
                last = out.value
    assert L.lococo_pages_attn_tree_workspace_bytes(C.byref(pages()), C.byref(requests()), None) == EINVAL


def test_keeping_and_moving_check_their_arguments():
    L, p = lb.lib(), pages(k_codes=None, dtype=9)                       # keeping reads neither the arrays nor the heads
    names = ["tables", "starts", "held", "slots", "kept", "ring", "ends", "held_after", "ends_after", "sources", "targets", "totals"]
    good = dict(zip(names, FAKE))

    def keep(n=3, tokens=4, width=5, pg=p, **over):
        a = dict(good, **over)
        return L.lococo_pages_keep(C.byref(pg), n, tokens, width, *(a[k] for k in names), None)

    for name in names:
        assert keep(**{name: None}) == EINVAL, name
        assert keep(**{name: FAKE[13] + 2}) == EINVAL, name
    assert keep(ends=FAKE[6] + 4) == keep(ends_after=FAKE[6] + 4) == EINVAL
    for out in ("ring", "held_after", "ends_after", "sources", "targets", "totals"):
        for src in ("tables", "starts", "held", "slots", "kept", "ends"):
            assert keep(**{out: good[src]}) == EINVAL, (out, src)
    assert keep(sources=good["targets"]) == keep(totals=good["held_after"]) == EINVAL
    assert keep(n=0) == keep(tokens=-1) == keep(width=0) == EINVAL
    assert keep(n=4097) == keep(tokens=2 ** 30) == keep(width=2 ** 25) == EUNSUPPORTED
    assert keep(pg=pages(page_rows=24)) == EUNSUPPORTED
    q = pages()
    move = lambda n=2, tokens=3, starts=FAKE[4], a=FAKE[5], b=FAKE[6]: L.lococo_pages_move(C.byref(q), n, tokens, starts, a, b, None)
    assert move(n=0) == move(tokens=-1) == move(starts=None) == move(a=None) == move(b=FAKE[6] + 2) == EINVAL
    assert move(n=4097) == EUNSUPPORTED
    assert move(tokens=0, starts=None, a=None, b=None) == OK


def test_struct_of_the_header():
    assert C.sizeof(lb.lococo_rotation) == 80


def test_the_binding_refuses_what_does_not_fit():
    """Host tensors, other types and shapes raise before the library is called."""
    f = torch.ones(32)
    with pytest.raises(TypeError):
        lb.Rotation(dtype=torch.bfloat16, n_q_heads=2, n_kv_heads=1, head_dim=64, freqs=f)
    with pytest.raises(TypeError):
        lb.Rotation(dtype=torch.bfloat16, n_q_heads=2, n_kv_heads=1, head_dim=64, norm=True, q_weight=torch.ones(64))
    rot = lb.Rotation(dtype=torch.bfloat16, n_q_heads=2, n_kv_heads=1, head_dim=64, norm=True)
    x = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lb.lococo_rows_rotate(rot, None, None, None, None)
    with pytest.raises((TypeError, RuntimeError, AssertionError)):
        lb.lococo_rows_rotate(rot, x, None, x, None)
    with pytest.raises(TypeError):
        lb.lococo_rows_rotate(rot, x.float(), None, x.float(), None)


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source,kernel,builds", [("pages_attn_tree.hip", "pages_tree_tile_k", 6), ("rows_rotate.hip", "rows_rotate_back_k", 6),
                                                  ("pages_append.hip", "pages_append_k", 6), ("pages_tree.hip", "pages_tree_k", 4)])
def test_kernels_keep_everything_in_registers(tmp_path, source, kernel, builds):
    r = subprocess.run(["hipcc", "-x", "hip", *lib_build.FLAGS, *lib_build.EXTRA.get(source, []), "--cuda-device-only", "-c",
                        os.path.join(lib_build.CSRC, source), "-o", str(tmp_path / "a.o"), "-Rpass-analysis=kernel-resource-usage"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    spilled = [int(n) for n in re.findall(r"VGPRs Spill: (\d+)", r.stderr)]
    scratch = [int(n) for n in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    assert sum(kernel in n for n in names) == builds and len(names) == len(spilled) == len(scratch)
    assert not any(spilled) and not any(scratch), dict(zip(names, zip(spilled, scratch)))
