"""Checks on the gfx950 assembly of the layers' products (built here, host only,
no GPU).  Their operands come into LDS by hand-written DMA, waited for by hand:

1. m0, which the DMA sets without being able to name it as clobbered, has no
   other use, and nothing is spilled (a spill is a memory operation in a loop
   that counts them).
2. At every barrier no LDS read is in flight: behind it other waves write what
   was being read.
3. Counted waits (vmcnt(N), N > 0) stand in the forms of four stages alone: c,
   the loads of one K tile, inside the loop (the tile behind the next may be on
   its way), and 2 c before it.  A load added to the loop, or one taken away,
   changes c and fails the check."""

import re
import subprocess

import pytest

from test_lds_read_asm import HAVE_HIPCC, VMEM, basic_blocks, functions, loops

READ = re.compile(r"^ds_read|^ds_load")
COUNT = re.compile(r"vmcnt\((\d+)\)")
DMA = re.compile(r"^buffer_load_dwordx4 .*\blds\b")


def products(funcs):
    return {n: b for n, b in funcs.items()
            if re.search(r"k_(gemm|backward)(_direct)?I", n) and "join" not in n}


def m0_problems(body):
    """m0 outside the DMA's own three instructions; scratch accesses."""
    lines = [t for t in (ln.split(";")[0].strip() for ln in body) if t and not t.startswith(".")]
    bad = []
    for i, t in enumerate(lines):
        if t.startswith("scratch_"):
            bad.append(t)
        if re.search(r"\bm0\b", t):
            ok = (re.match(r"s_mov_b32 m0, s\d+$", t) and lines[i + 1] == "s_nop 0"
                  and DMA.match(lines[i + 2]))
            if not ok:
                bad.append(t)
    return bad


def reads_at_barriers(body):
    """Barriers that some path reaches with an LDS read in flight."""
    blocks, succ = basic_blocks(body)
    bad, entry, todo = set(), {0: False}, [0]
    while todo:
        b = todo.pop()
        flying = entry[b]
        for i, t in enumerate(blocks[b][1]):
            if READ.match(t):
                flying = True
            elif t.startswith("s_waitcnt") and "lgkmcnt(0)" in t:
                flying = False
            elif t.startswith("s_barrier") and flying:
                bad.add((b, i))
        for s in succ[b]:
            if s not in entry or (flying and not entry[s]):
                entry[s] = flying or entry.get(s, False)
                todo.append(s)
    return bad


def counted_waits(body):
    """(N of hand-written counted waits in loops with the loads of an iteration,
    N of those outside loops)"""
    blocks, succ = basic_blocks(body)
    preds = [[] for _ in blocks]
    for v, ws in enumerate(succ):
        for w in ws:
            preds[w].append(v)

    def waits(b):
        ins, out, inside = blocks[b][1], [], False
        for t in ins:
            inside = t.startswith(";;#ASMSTART") or (inside and not t.startswith(";;#ASMEND"))
            m = COUNT.search(t) if inside and t.startswith("s_waitcnt") else None
            if m and int(m.group(1)):
                out.append(int(m.group(1)))
        return out

    # innermost loops that issue DMA
    found = [c for c in loops(set(range(len(blocks))), succ, preds)
             if any(DMA.match(t) for b in c for t in blocks[b][1])]
    found = [c for c in found if not any(o < c for o in found)]
    in_loops, covered = [], set()
    for c in found:
        covered |= c
        n = sum(1 for b in c for t in blocks[b][1] if VMEM.match(t))
        in_loops += [(w, n) for b in sorted(c) for w in waits(b)]
    outside = [w for b in range(len(blocks)) if b not in covered for w in waits(b)]
    return in_loops, outside


def test_checks_flag_what_they_look_for():
    dma = ["s_mov_b32 m0, s3", "s_nop 0", "buffer_load_dwordx4 v1, s[0:3], 0 offen lds"]
    assert m0_problems(dma) == []
    assert m0_problems(dma[:1] + ["v_readlane_b32 s5, v0, m0"] + dma[1:])
    assert m0_problems(["scratch_load_dword v9, off, s32"])
    body = ["ds_read_b128 v[0:3], v9", "s_waitcnt lgkmcnt(0)", "s_barrier", "s_endpgm"]
    assert reads_at_barriers(body) == set()
    assert reads_at_barriers(body[:1] + body[2:])
    # round a loop: the read of one iteration meets the barrier of the next
    loop = [".LBB0_1:", "s_barrier", "ds_read_b128 v[0:3], v9", "s_cbranch_scc1 .LBB0_1", "s_endpgm"]
    assert reads_at_barriers(loop)
    wait = [";;#ASMSTART", "s_waitcnt vmcnt(2) lgkmcnt(0)", "s_barrier", ";;#ASMEND"]
    first = [";;#ASMSTART", "s_waitcnt vmcnt(4)", "s_barrier", ";;#ASMEND"]
    body = first + [".LBB0_1:"] + wait + dma + dma + ["s_cbranch_scc1 .LBB0_1", "s_endpgm"]
    assert counted_waits(body) == ([(2, 2)], [4])
    assert counted_waits(first + [".LBB0_1:"] + wait + dma + body[-2:])[0] == [(2, 1)]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    from paper_2301_09830_amd import build
    out = tmp_path_factory.mktemp("asm") / "stage_ops.s"
    cmd = build.compile_command(str(out), "stage_ops.hip")
    cmd = [c for c in cmd if c not in ("-fPIC", "-shared")] + ["--cuda-device-only", "-S"]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr[-2000:]
    found = products(functions(open(out).read().split("\n")))
    assert len(found) >= 30
    return found


@pytest.mark.skipif(not HAVE_HIPCC, reason="hipcc not available")
def test_m0_belongs_to_the_dma(kernels):
    bad = {n: p for n, p in ((n, m0_problems(b)) for n, b in kernels.items()) if p}
    assert bad == {}
    assert sum(any(DMA.match(t.strip()) for t in b) for b in kernels.values()) >= 20


@pytest.mark.skipif(not HAVE_HIPCC, reason="hipcc not available")
def test_no_lds_read_is_in_flight_at_a_barrier(kernels):
    bad = {n: p for n, p in ((n, reads_at_barriers(b)) for n, b in kernels.items()) if p}
    assert bad == {}


@pytest.mark.skipif(not HAVE_HIPCC, reason="hipcc not available")
def test_counted_waits_match_the_loads(kernels):
    """Of a Form<WM, WN, FA, FB, S>: only S = 4 counts its loads."""
    counted = 0
    for name, body in kernels.items():
        inside, outside = counted_waits(body)
        form = re.search(r"4FormILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E", name)
        if not form or form.group(5) != "4":
            assert inside == [] and outside == [], name
            continue
        wm, wn, fa, fb = (int(form.group(i)) for i in range(1, 5))
        c = (wm * fa + wn * fb) * 16 * 128 // 1024 // (wm * wn)   # 1024 bytes an instruction
        assert inside and all(w == c and n == c for w, n in inside), (name, inside)
        assert outside and all(w == 2 * c for w in outside), (name, outside)
        counted += 1
    assert counted >= 12
