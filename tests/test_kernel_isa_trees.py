"""Static checks of the machine code of the tree attention and of the eviction's move (no GPU needed: hipcc cross-compiles): the hand-written parts of
their synchronisation, which the compiler does not know the meaning of.

  steps       a step of the page loop is handed over through LDS behind a barrier with a wait for LDS alone, so that requests for later steps
              stay on their way: nothing may touch LDS between that wait and its barrier
  hand-over   a work item publishes its state with device-coherent stores (sc1), waits until all of them are acknowledged (`s_waitcnt vmcnt(0)`),
              passes a barrier and only then raises the arrival counter (a returning atomic add); whoever arrives last reads the states
              with device-coherent loads
  in place    a piece's tokens are all in registers (`s_waitcnt vmcnt(0)`, then a barrier) before any of them is written
"""
import os
import re
import shutil
import subprocess
import tempfile

import pytest

from paper_2506_09397_amd import build as B


def kernels(text, name):
    """{kernel: instructions, with "asm{" and "}asm" around what the source writes itself}"""
    out, cur = {}, None
    for line in text.split("\n"):
        m = re.match(r"^(_Z\S+):", line)
        if m:
            cur = out.setdefault(m.group(1), []) if name in m.group(1) else None
            continue
        t = line.strip()
        if cur is None or not t:
            continue
        if t.startswith(";;#ASM"):
            cur.append("asm{" if t.startswith(";;#ASMSTART") else "}asm")
        elif t[0] not in ";.":
            cur.append(t.split(" ;")[0].strip())
    return out


def own_waits(ins, what):
    """indices of waits for `what` alone that the source has written itself"""
    return [k for k, t in enumerate(ins) if re.fullmatch(rf"s_waitcnt {what}\(0\)", t) and ins[k - 1] == "asm{"]


def before_barrier(ins, k):
    """what is issued between instruction k and the next barrier"""
    b = next((j for j in range(k + 1, len(ins)) if ins[j] == "s_barrier"), len(ins))
    return [t for t in ins[k + 1:b] if not t.endswith("asm") and t != "asm{"], b


def check_attention(ins, bodies=3):
    bad = []
    waits = own_waits(ins, "lgkmcnt")
    if len(waits) < 2 * bodies:
        bad.append(f"only {len(waits)} waits for LDS of the page loop's own")
    for k in waits:
        between, b = before_barrier(ins, k)
        if b == len(ins) or any(t.startswith(("ds_", "s_cbranch", "s_branch", "s_endpgm")) for t in between):
            bad.append(f"between a step's wait and its barrier: {between[:3]}")
    adds = [k for k, t in enumerate(ins) if t.startswith("global_atomic_add") and t.endswith(" sc0")]
    if len(adds) != bodies:
        bad.append(f"{len(adds)} arrival counters in place of {bodies}")
    for a in adds:
        b = max((k for k in range(a) if ins[k] == "s_barrier"), default=-1)
        w = max((k for k in range(max(b, 0)) if ins[k].startswith("s_waitcnt") and "vmcnt(0)" in ins[k]), default=-1)
        first = max((k for k in range(max(w, 0)) if ins[k] == "s_barrier"), default=0)
        state = [k for k in range(first, max(b, 0)) if ins[k].startswith("global_store")]
        if len(state) < 6:
            bad.append(f"only {len(state)} stores of a state before its counter")
        if any(k > w for k in state):
            bad.append("a store of a state is issued behind the wait for the acknowledgements")
        bad += [f"`{ins[k]}` publishes a state without device coherence" for k in state if not ins[k].endswith(" sc1")]
        after = next((k for k in range(a, len(ins)) if ins[k] == "s_barrier"), len(ins))
        loads = [t for t in ins[after:] if t.startswith("global_load")][:20]
        bad += [f"`{t}` reads a state without device coherence" for t in loads if not t.endswith(" sc1")]
        if len(loads) < 20:
            bad.append("the loads of the stored states were not found")
    return bad


def check_in_place(ins):
    bad = []
    waits = own_waits(ins, "vmcnt")
    if len(waits) != 1:
        return [f"{len(waits)} waits for a piece's loads in place of one"]
    w = waits[0]
    between, b = before_barrier(ins, w)
    if b == len(ins) or any(t.startswith(("global_", "s_cbranch", "s_branch")) for t in between):
        bad.append(f"between a piece's wait and its barrier: {between[:3]}")
    if any(t.startswith("global_store") for t in ins[:w]):
        bad.append("a token is written before all of its piece have been read")
    if not any(t.startswith("global_store") for t in ins[b:]) or not any(t.startswith("global_load_dwordx4") for t in ins[:w]):
        bad.append("a piece's loads or stores were not found")
    # (the loop goes back to the front: what is read behind the barrier may be page numbers only)
    if any(t.startswith("global_load_dwordx") for t in ins[b:]):
        bad.append("part of a piece is read behind the barrier")
    return bad


STEP = "\t;;#ASMSTART\n\ts_waitcnt lgkmcnt(0)\n\t;;#ASMEND\n\ts_barrier\n"
GOOD = "_Z21tree_attention_kernelv:\n" + 2 * STEP + 8 * "\tglobal_store_dword v1, v2, s[4:5] sc1\n" + \
    "\ts_waitcnt vmcnt(0) expcnt(0) lgkmcnt(0)\n\ts_barrier\n\tglobal_atomic_add v3, v3, v4, s[4:5] sc0\n\ts_barrier\n" + \
    24 * "\tglobal_load_dword v1, v2, s[4:5] sc1\n" + "\ts_endpgm\n"
MOVE = "_Z17evict_move_kernelv:\n\ts_barrier\n" + 4 * "\tglobal_load_dwordx4 v[0:3], v[8:9], off\n" + "\t;;#ASMSTART\n\ts_waitcnt vmcnt(0)\n\t;;#ASMEND\n\ts_barrier\n" + \
    "\tglobal_load_dword v9, v[8:9], off\n\tglobal_store_dwordx4 v[8:9], v[0:3], off\n\ts_endpgm\n"


def attention(text):
    return check_attention(kernels(text, "tree_attention")["_Z21tree_attention_kernelv"], bodies=1)


def test_planted_mistakes_of_the_attention_are_found():
    assert attention(GOOD) == []
    for a, b, what in [("\t;;#ASMEND\n\ts_barrier\n", "\t;;#ASMEND\n\tds_write_b32 v0, v1\n\ts_barrier\n", "wait and its barrier"),
                       (STEP, "\ts_barrier\n", "waits for LDS"),
                       ("v2, s[4:5] sc1\n\tglobal_store", "v2, s[4:5]\n\tglobal_store", "without device coherence"),
                       ("\ts_waitcnt vmcnt(0) expcnt(0) lgkmcnt(0)\n", "", "a state"),
                       ("lgkmcnt(0)\n\ts_barrier\n\tglobal_atomic", "lgkmcnt(0)\n\tglobal_store_dword v1, v2, s[4:5] sc1\n\ts_barrier\n\tglobal_atomic", "behind the wait"),
                       ("\ts_barrier\n\tglobal_load_dword v1, v2, s[4:5] sc1", "\ts_barrier\n\tglobal_load_dword v1, v2, s[4:5]", "without device coherence")]:
        assert a in GOOD
        assert any(what in x for x in attention(GOOD.replace(a, b, 1))), (a, attention(GOOD.replace(a, b, 1)))


def test_planted_mistakes_of_the_move_are_found():
    move = lambda text: check_in_place(kernels(text, "evict_move")["_Z17evict_move_kernelv"])
    assert move(MOVE) == []
    store, load = "\tglobal_store_dwordx4 v[8:9], v[0:3], off\n", "\tglobal_load_dwordx4 v[0:3], v[8:9], off\n"
    assert move(MOVE.replace("\ts_barrier\n" + load, "\ts_barrier\n" + store + load, 1))
    assert move(MOVE.replace(store, load + store, 1))
    assert move(MOVE.replace("\t;;#ASMSTART\n\ts_waitcnt vmcnt(0)\n\t;;#ASMEND\n", "", 1))


def assembly(source):
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "a.s")
        cmd = ["hipcc", *[f for f in B.FLAGS if f != "-fPIC"], "--cuda-device-only", "-S", os.path.join(B.CSRC, source), "-o", out]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        return open(out).read()


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_tree_attention_keeps_its_hand_written_synchronisation():
    found = kernels(assembly("tree.hip"), "tree_attention_kernel")
    assert len(found) == 4, list(found)       # bf16 as the caller's rows and within a step, float32 with heads of 64 and of 128
    for name, ins in found.items():
        assert not check_attention(ins), (name, check_attention(ins)[:5])


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_evictions_in_place_read_a_piece_before_they_write_it():
    found = {k: v for k, v in kernels(assembly("evict.hip"), "evict_move_kernel").items() if re.search(r"ILi\d+ELb[01]ELb1E", k)}
    assert len(found) == 3, list(found)
    for name, ins in found.items():
        assert not check_in_place(ins), (name, check_in_place(ins))
