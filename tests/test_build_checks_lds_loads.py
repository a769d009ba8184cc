"""The build-time check of loads into LDS that are waited for by counts (csrc/check_lds_loads.py): small hand-written listings, a
loop whose last steps ask for nothing among them, and the kernel as it is compiled."""
import importlib.util
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2410_03065_amd", "csrc")
spec = importlib.util.spec_from_file_location("check_lds_loads", os.path.join(CSRC, "check_lds_loads.py"))
chk = importlib.util.module_from_spec(spec)
spec.loader.exec_module(chk)

BRING = "\tbuffer_load_dwordx4 v35, s[0:3], s49 offen lds\n\tbuffer_load_dwordx4 v35, s[0:3], s49 offen offset:1024 lds\n"      # half a step: two loads
CODES = "\tglobal_load_dwordx4 v[2:5], v1, s[8:9]\n\tbuffer_load_ushort v9, v1, s[0:3], 0 offen\n"
BARRIER = "\ts_barrier\n"
END = "\ts_waitcnt vmcnt(0)\n\ts_endpgm\n"


def wait(n):
    return "\ts_waitcnt vmcnt(%d)\n" % n


def problems(body):
    return chk.check_kernel("k", body.split("\n"), 2)[1]


#: three half steps, four steps' codes; the first must have come
BEGIN = BRING * 3 + CODES * 4 + wait(8 + 4) + BARRIER


def half(n):
    return wait(n) + BARRIER + BRING


def test_a_beginning_in_its_order():
    assert not problems(BEGIN + END)
    assert problems(CODES * 4 + BRING * 3 + wait(8 + 4) + BARRIER + END)          # the codes first: the count covers nothing
    assert problems(BRING * 3 + CODES * 4 + wait(8 + 5) + BARRIER + END)


def test_steps_that_ask_for_codes_and_last_steps_that_do_not():
    step, last = half(4) + half(4) + CODES, half(2) + half(2)
    loop = "\ts_cbranch_scc1 .LBB0_2\n.LBB0_1:\n" + step * 4 + "\ts_cbranch_scc1 .LBB0_1\n.LBB0_2:\n"
    assert not problems(BEGIN + loop + last * 3 + END)
    assert not problems(BEGIN + loop + (half(4) + half(4)) + END)                 # one last step: the loop's codes are still between
    found = problems(BEGIN + loop + (half(4) + half(4)) * 3 + END)                # the loop's count where nothing is asked for
    assert found and all("a later barrier" in p for p in found)


def test_a_path_that_skips_the_loop():
    loop = "\ts_cbranch_scc1 .LBB0_2\n.LBB0_1:\n" + half(4) * 2 + CODES + "\ts_cbranch_scc1 .LBB0_1\n.LBB0_2:\n"
    assert not problems(BEGIN + loop + END)
    assert problems(BEGIN + "\ts_cbranch_scc1 .LBB0_9\n" + half(2) * 2 + ".LBB0_9:\n" + half(8 + 4) + END)


def test_stores_do_not_count_as_loads_behind():
    assert not problems(BRING * 3 + CODES + wait(2 + 4) + BARRIER + END)
    assert problems(BRING * 3 + "\tglobal_store_dword v1, v2, s[8:9]\n" * 2 + wait(2 + 4) + BARRIER + END)


def test_what_is_outstanding_at_the_end():
    assert problems(BRING + "\ts_endpgm\n") and not problems(BRING + END)


def test_a_second_tile_begins_anew():
    tile = BEGIN + half(2) + half(2) + wait(0)
    assert not problems(tile + "\ts_cbranch_scc1 .LBB0_5\n\ts_endpgm\n.LBB0_5:\n" + tile + END)


@pytest.mark.parametrize("line", ["s_waitcnt 0x3f70", "s_setpc_b64 s[30:31]"])
def test_what_is_not_understood_is_refused(line):
    with pytest.raises(ValueError):
        problems(BRING + "\t%s\n" % line + END)


def test_the_kernel_as_it_is_compiled(tmp_path):
    """Every instance, on every path; and with one count that is too large by a load, in a copy of the listing, the check speaks."""
    sys.path.insert(0, ROOT)
    import __graft_entry__ as entry
    listing = str(tmp_path / "kernels_w4.s")
    if not os.path.exists(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")):
        pytest.skip("no compiler")
    entry._run(entry._compile("kernels_w4.hip", listing, ["-S", "--cuda-device-only"]))
    check = [sys.executable, os.path.join(CSRC, "check_lds_loads.py")]
    p = subprocess.run(check + [listing, "w4_wide_kernel"], stdout=subprocess.PIPE, text=True)
    assert p.returncode == 0 and p.stdout.count("0 problem(s)") == 8, p.stdout
    name, lines = next(chk.kernels(open(listing).read(), "w4_wide_kernelILb0ELi4"))
    at = max(i for i, l in enumerate(lines) if "s_barrier" in l)
    while "vmcnt(2)" not in lines[at]:
        at -= 1
    assert chk.check_kernel(name, lines[:at] + [lines[at].replace("vmcnt(2)", "vmcnt(3)")] + lines[at + 1:], 2)[1]
