"""What lococo_pages_* refuse before any GPU work, and the registers of their kernels (CPU: nothing is run)."""
import ctypes as C
import os
import re
import shutil
import subprocess
import sys

import pytest

from paper_2406_05317_amd import binding as lb
from paper_2406_05317_amd import build as lib_build

FAKE = [0x10000 * (i + 1) for i in range(16)]              # never read: the calls fail, or do nothing, before


def pages(**over):
    kw = dict(struct_size=C.sizeof(lb.lococo_pages), dtype=lb.LOCOCO_BF16, n_q_heads=8, n_kv_heads=2, head_dim=128, page_rows=64, n_pages=10,
              attn_scale=0.0, k_codes=FAKE[0], k_scales=FAKE[1], v_codes=FAKE[2], v_scales=FAKE[3])
    kw.update(over)
    return lb.lococo_pages(*(kw[n] for n, _ in lb.lococo_pages._fields_))


def requests(**over):
    kw = dict(n=2, tokens=3, table_pages=5, max_new=2, max_held=300, tables=FAKE[4], starts=FAKE[5], held=FAKE[6])
    kw.update(over)
    return lb.lococo_requests(*(kw[n] for n, _ in lb.lococo_requests._fields_))


def tensor(p=FAKE[7], sb=4096, sh=1024, st=128):
    return lb.lococo_tensor(p, sb, sh, st)


BAD_PAGES = [(dict(struct_size=8), lb.LOCOCO_EINVAL), (dict(dtype=5), lb.LOCOCO_EINVAL), (dict(n_q_heads=7), lb.LOCOCO_EINVAL),
             (dict(n_kv_heads=0), lb.LOCOCO_EINVAL), (dict(head_dim=100), lb.LOCOCO_EUNSUPPORTED), (dict(head_dim=512), lb.LOCOCO_EUNSUPPORTED),
             (dict(head_dim=0), lb.LOCOCO_EINVAL), (dict(page_rows=8), lb.LOCOCO_EUNSUPPORTED), (dict(page_rows=48), lb.LOCOCO_EUNSUPPORTED),
             (dict(page_rows=0), lb.LOCOCO_EINVAL), (dict(n_pages=0), lb.LOCOCO_EINVAL), (dict(n_pages=2 ** 24), lb.LOCOCO_EUNSUPPORTED),
             (dict(n_pages=2 ** 31 - 1), lb.LOCOCO_EUNSUPPORTED), (dict(attn_scale=float("inf")), lb.LOCOCO_EINVAL),
             (dict(n_q_heads=131072, n_kv_heads=65536), lb.LOCOCO_EUNSUPPORTED), (dict(v_scales=None), lb.LOCOCO_EINVAL),
             (dict(k_scales=FAKE[1] + 4), lb.LOCOCO_EINVAL), (dict(v_codes=FAKE[0]), lb.LOCOCO_EINVAL)]


@pytest.mark.parametrize("over,want", BAD_PAGES)
def test_pages_are_checked_by_every_call(over, want):
    L, p, t, out = lb.lib(), pages(**over), tensor(), C.c_size_t(0)
    assert L.lococo_pages_workspace_bytes(C.byref(p), C.byref(requests()), C.byref(out)) == want
    assert len(L.lococo_last_error()) > 0
    assert L.lococo_pages_store(C.byref(p), C.byref(t), C.byref(t), 3, 3, FAKE[8], None) == want
    assert L.lococo_pages_load(C.byref(p), FAKE[8], 3, 3, C.byref(t), C.byref(tensor(FAKE[9])), None) == want
    assert L.lococo_pages_attn(C.byref(p), C.byref(requests()), C.byref(t), C.byref(tensor(FAKE[9])), 3, None, 0, None) == want


@pytest.mark.parametrize("over,want", [
    (dict(n=0), lb.LOCOCO_EINVAL), (dict(n=4097, max_new=1), lb.LOCOCO_EUNSUPPORTED), (dict(tokens=-1), lb.LOCOCO_EINVAL),
    (dict(tokens=2 ** 30, max_new=2 ** 30), lb.LOCOCO_EUNSUPPORTED), (dict(tokens=2 ** 30 - 2, max_new=2 ** 30), lb.LOCOCO_EUNSUPPORTED),
    (dict(table_pages=0), lb.LOCOCO_EINVAL), (dict(table_pages=2 ** 24), lb.LOCOCO_EUNSUPPORTED), (dict(max_new=1), lb.LOCOCO_EINVAL),
    (dict(max_held=-1), lb.LOCOCO_EINVAL)])
def test_requests_are_checked(over, want):
    L, out = lb.lib(), C.c_size_t(0)
    r, p, t = requests(**over), pages(), tensor()
    assert L.lococo_pages_workspace_bytes(C.byref(p), C.byref(r), C.byref(out)) == want
    assert L.lococo_pages_attn(C.byref(p), C.byref(r), C.byref(t), C.byref(tensor(FAKE[9])), 3, None, 0, None) == want


@pytest.mark.parametrize("n,tokens,least", [(32, 32, 1), (32, 40, 2), (32, 64, 2), (32, 65, 3), (1, 77, 77)])
def test_max_new_covers_every_row_of_a_call(n, tokens, least):
    """Rows that no request has count among those max_new * n has to cover."""
    L, p, out = lb.lib(), pages(), C.c_size_t(0)
    size = lambda most: L.lococo_pages_workspace_bytes(C.byref(p), C.byref(requests(n=n, tokens=tokens, max_new=most)), C.byref(out))
    assert size(least) == lb.LOCOCO_OK and size(least - 1) == lb.LOCOCO_EINVAL
    assert size(least - 1) == lb.LOCOCO_EINVAL and b"max_new" in L.lococo_last_error()


def test_call_arguments_are_checked():
    L, p, t, u, out = lb.lib(), pages(), tensor(), tensor(FAKE[9]), C.c_size_t(0)
    ok = dict(tables=FAKE[4], starts=FAKE[5], held=FAKE[6])
    for name in ok:
        for bad in (None, FAKE[5] + 2):
            assert L.lococo_pages_attn(C.byref(p), C.byref(requests(**{name: bad})), C.byref(t), C.byref(u), 3, None, 0, None) == lb.LOCOCO_EINVAL
    r = requests()
    attn = lambda q, o, per=3, pg=p, rq=r: L.lococo_pages_attn(pg and C.byref(pg), rq and C.byref(rq), q and C.byref(q), o and C.byref(o), per, None, 0, None)
    assert attn(t, t) == attn(None, u) == attn(t, None) == attn(t, u, 0) == attn(t, u, pg=None) == attn(t, u, rq=None) == lb.LOCOCO_EINVAL
    for bad in (tensor(None), tensor(FAKE[7] + 8), tensor(st=64), tensor(st=132), tensor(sh=-8), tensor(sb=12)):
        assert attn(bad, u) == attn(t, bad) == lb.LOCOCO_EINVAL
        assert L.lococo_pages_store(C.byref(p), C.byref(bad), C.byref(u), 3, 3, FAKE[8], None) == lb.LOCOCO_EINVAL
        assert L.lococo_pages_load(C.byref(p), FAKE[8], 3, 3, C.byref(t), C.byref(bad), None) == lb.LOCOCO_EINVAL
    assert L.lococo_pages_store(C.byref(p), C.byref(t), C.byref(u), 3, 3, None, None) == lb.LOCOCO_EINVAL
    assert L.lococo_pages_store(C.byref(p), C.byref(t), C.byref(u), 3, -1, FAKE[8], None) == lb.LOCOCO_EINVAL
    assert L.lococo_pages_load(C.byref(p), FAKE[8], 3, 3, C.byref(t), C.byref(t), None) == lb.LOCOCO_EINVAL
    assert L.lococo_pages_store(C.byref(p), C.byref(t), C.byref(u), 3, 2 ** 30, FAKE[8], None) == lb.LOCOCO_EUNSUPPORTED
    assert L.lococo_pages_workspace_bytes(C.byref(p), C.byref(r), None) == lb.LOCOCO_EINVAL
    # parts of a long request need a workspace; nothing is launched without it
    long = requests(n=1, tokens=1, max_new=1, max_held=320, table_pages=2000)
    assert L.lococo_pages_workspace_bytes(C.byref(p), C.byref(long), C.byref(out)) == lb.LOCOCO_OK and out.value == 0
    long.max_held = 100000
    assert L.lococo_pages_workspace_bytes(C.byref(p), C.byref(long), C.byref(out)) == lb.LOCOCO_OK and out.value > 0
    need = out.value
    for ws, size in ((None, 0), (None, need), (FAKE[10], need - 1), (FAKE[10] + 64, need)):
        assert L.lococo_pages_attn(C.byref(p), C.byref(long), C.byref(t), C.byref(u), 1, ws, size, None) == lb.LOCOCO_EWORKSPACE
    assert b"workspace" in L.lococo_last_error()


def test_calls_of_no_rows_do_nothing():
    L, p, none = lb.lib(), pages(), tensor(None)
    assert L.lococo_pages_store(C.byref(p), C.byref(none), C.byref(none), 1, 0, None, None) == lb.LOCOCO_OK
    assert L.lococo_pages_load(C.byref(p), None, 1, 0, C.byref(none), C.byref(none), None) == lb.LOCOCO_OK
    assert L.lococo_pages_attn(C.byref(p), C.byref(requests(tokens=0, max_new=0)), C.byref(none), C.byref(none), 1, None, 0, None) == lb.LOCOCO_OK


IDLE = """
import ctypes as C, sys
sys.path.insert(0, sys.argv[1])
from test_pages_cpu import FAKE, lb, pages, requests, tensor
L, none, out = lb.lib(), tensor(None), C.c_size_t(0)
for dtype in (lb.LOCOCO_F32, lb.LOCOCO_BF16):
    for d in (64, 96, 128):
        for max_new in (0, 1, 9, 77):
            for max_held in (0, 300, 769, 4096, 131072):
                p, r = pages(dtype=dtype, head_dim=d), requests(tokens=0, max_new=max_new, max_held=max_held, table_pages=3000)
                st = L.lococo_pages_workspace_bytes(C.byref(p), C.byref(r), C.byref(out))
                st |= L.lococo_pages_attn(C.byref(p), C.byref(r), C.byref(none), C.byref(none), 1, None, 0, None)
                assert st == lb.LOCOCO_OK, (dtype, d, max_new, max_held, st)
print("every idle turn returned")
"""


def test_idle_turns_do_nothing_whatever_they_promise():
    """No rows, with max_new and max_held as a server's busier turns have them (in a process of its own: an arithmetic trap would end it)."""
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", IDLE, here], capture_output=True, text=True, timeout=300, cwd=os.path.dirname(here))
    assert r.returncode == 0 and "every idle turn returned" in r.stdout, (r.returncode, r.stderr[-2000:])


def test_workspace_does_not_shrink_with_more_keys():
    """A workspace for a larger max_held serves calls with a smaller one."""
    L, p, out = lb.lib(), pages(), C.c_size_t(0)
    for n, new in ((1, 1), (3, 1), (70, 1), (2, 9), (5, 300)):
        last = 0
        for held in sorted([1, 255, 256, 257, 768, 769, 1000, 2048, 2049, 5000, 65536, 10 ** 6, 2 ** 31 - 1]):
            r = requests(n=n, tokens=n * new, max_new=new, max_held=held)
            assert L.lococo_pages_workspace_bytes(C.byref(p), C.byref(r), C.byref(out)) == lb.LOCOCO_OK
            assert out.value >= last
            last = out.value


@pytest.mark.parametrize("n,tokens,max_new", [(512, 40, 33), (4096, 64, 64), (4096, 4, 9), (4096, 4, 33), (300, 1055, 1024), (64, 127, 64),
                                              (4096, 4096, 2), (700, 50, 17), (1, 77, 77), (32, 32, 1)])
@pytest.mark.parametrize("kv,group", [(8, 4), (32, 1), (1, 1), (4, 8), (1, 64)])
@pytest.mark.parametrize("dtype,d", [(lb.LOCOCO_BF16, 128), (lb.LOCOCO_F32, 128), (lb.LOCOCO_BF16, 64)])
def test_workspace_is_bounded_by_what_is_resident(n, tokens, max_new, kv, group, dtype, d):
    """Parts of the keys are for calls that leave the device idle.  Two workgroups to each of 256 compute units are resident: however many
    requests of a call are idle, the parts of eight times as many tiles of 32 rows are room enough."""
    L, out = lb.lib(), C.c_size_t(0)
    p = pages(dtype=dtype, n_q_heads=kv * group, n_kv_heads=kv, head_dim=d)
    for held in (1000, 5000, 131072, 2 ** 30):
        r = requests(n=n, tokens=tokens, max_new=max_new, max_held=held)
        assert L.lococo_pages_workspace_bytes(C.byref(p), C.byref(r), C.byref(out)) == lb.LOCOCO_OK
        assert out.value <= 8 * 512 * 32 * (d + 2) * 4, held


def test_plan_arguments_are_checked():
    L, p = lb.lib(), pages(k_codes=None, dtype=9)                       # the plan reads neither the arrays nor the heads
    names = ["new", "held", "tables", "ring", "ends", "held_after", "ends_after", "starts", "slots", "positions", "totals"]
    good = dict(zip(names, FAKE))

    def plan(n=3, tokens=4, width=5, pg=p, **over):
        a = dict(good, **over)
        return L.lococo_pages_plan(C.byref(pg), n, tokens, width, *(a[k] for k in names), None)

    for name in names:
        assert plan(**{name: None}) == lb.LOCOCO_EINVAL, name
        assert plan(**{name: FAKE[12] + 2}) == lb.LOCOCO_EINVAL, name
    assert plan(ends=FAKE[4] + 4) == plan(ends_after=FAKE[4] + 4) == lb.LOCOCO_EINVAL
    for out in ("held_after", "ends_after", "starts", "slots", "positions", "totals"):
        for src in ("new", "held", "tables", "ring", "ends"):
            assert plan(**{out: good[src]}) == lb.LOCOCO_EINVAL, (out, src)
    assert plan(n=0) == plan(tokens=-1) == plan(width=0) == lb.LOCOCO_EINVAL
    assert plan(n=4097) == plan(tokens=2 ** 30) == plan(width=2 ** 25) == lb.LOCOCO_EUNSUPPORTED
    assert plan(pg=pages(page_rows=24)) == lb.LOCOCO_EUNSUPPORTED


@pytest.mark.parametrize("over,fit", [                                   # a launch's dimension has fewer than 2^32 threads: 2^24 workgroups of 256
    (dict(head_dim=128, n_q_heads=32, n_kv_heads=32), 32 * (2 ** 19 - 2) + 31),               # 32 rows a workgroup, 32 kv heads, one spare tile
    (dict(head_dim=64, n_q_heads=32, n_kv_heads=32, dtype=lb.LOCOCO_F32), 16 * (2 ** 19 - 2) + 15),
    (dict(head_dim=128, n_q_heads=128, n_kv_heads=64), 16 * (2 ** 18 - 2) + 15),              # two rows a token
    (dict(head_dim=96, n_q_heads=1, n_kv_heads=1), 4 * (2 ** 24 - 1)),                        # 4 rows a workgroup
    (dict(head_dim=256, n_q_heads=8, n_kv_heads=2), 4 * (2 ** 24 - 1))])
def test_attention_takes_what_a_launch_takes(over, fit):
    L, p, out = lb.lib(), pages(**over), C.c_size_t(0)
    size = lambda tokens: L.lococo_pages_workspace_bytes(C.byref(p), C.byref(requests(n=1, tokens=tokens, max_new=tokens)), C.byref(out))
    assert size(fit) == lb.LOCOCO_OK and size(fit + 1) == lb.LOCOCO_EUNSUPPORTED
    assert L.lococo_pages_attn(C.byref(p), C.byref(requests(n=1, tokens=fit + 1, max_new=fit + 1)), C.byref(tensor()), C.byref(tensor(FAKE[9])),
                               fit + 1, None, 0, None) == lb.LOCOCO_EUNSUPPORTED


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_attention_kernels_keep_everything_in_registers(tmp_path):
    """A reload from scratch memory waits for every load on its way: the codes requested a tile ahead (with 6 registers there the kernel of
    32 rows took a tenth longer)."""
    r = subprocess.run(["hipcc", "-x", "hip", *lib_build.FLAGS, *lib_build.EXTRA["pages_attn.hip"], "--cuda-device-only", "-c",
                        os.path.join(lib_build.CSRC, "pages_attn.hip"), "-o", str(tmp_path / "a.o"), "-Rpass-analysis=kernel-resource-usage"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    spilled = [int(n) for n in re.findall(r"VGPRs Spill: (\d+)", r.stderr)]
    scratch = [int(n) for n in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    waves = [int(n) for n in re.findall(r"Occupancy \[waves/SIMD\]: (\d+)", r.stderr)]
    assert sum("pages_attn_tile_k" in n for n in names) == 6 and len(names) == len(spilled) == len(scratch) == len(waves)
    assert not any(spilled) and not any(scratch), dict(zip(names, zip(spilled, scratch)))
    assert all(w >= 2 for w in waves)                                  # two workgroups of four waves to a compute unit
