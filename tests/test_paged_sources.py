"""Rules of the paged cache's kernel sources that a compiler does not check."""
import glob
import os
import re
import subprocess

from paper_2502_14477_amd import build
from test_pending_loads import functions

WAIT = "s_waitcnt lgkmcnt(8)"


def asm_statements():
    for path in sorted(glob.glob(os.path.join(build.PAGED, "*.hip")) + glob.glob(os.path.join(build.PAGED, "*.h"))):
        for m in re.finditer(r"\basm\s*(?:volatile)?\s*\((.*?)\)\s*;", open(path).read(), re.S):
            yield os.path.basename(path), m.group(1)


def test_inline_assembly_neither_loads_nor_touches_m0():
    """A load in a statement of its own would be taken as done when the statement ends."""
    found = list(asm_statements())
    assert found
    for f, s in found:
        assert not re.search(r"load|store|ds_|buffer_|atomic|\bm0\b", s.split(":")[0]), (f, s)


def fewest_reads_behind_a_write(code):
    """[(index, reads)]: at every counted wait, the LDS reads that lie behind the last LDS write on the path that has the fewest of them."""
    labels = {c[0]: i for i, c in enumerate(code) if len(c) == 1}
    starts = sorted({0} | set(labels.values()) | {i + 1 for i, c in enumerate(code) if c[0].startswith(("s_branch", "s_cbranch", "s_endpgm"))})
    end_of = dict(zip(starts, starts[1:] + [len(code)]))
    most, entry, todo, found = 64, {0: 64}, [0], {}
    while todo:
        at = todo.pop()
        reads, following = entry[at], [end_of[at]]
        for i in range(at, end_of[at]):
            if len(code[i]) == 1:
                continue
            op, operands = code[i]
            if op.startswith("ds_read"):
                reads = min(reads + 1, most)
            elif op.startswith("ds_write"):
                reads = 0
            elif "%s %s" % (op, operands) == WAIT and code[i + 1][0] == "s_barrier":
                found[i] = min(reads, found.get(i, most))
            elif op.startswith(("s_branch", "s_cbranch")):
                following = [labels[operands]] + ([] if op == "s_branch" else [i + 1])
            elif op == "s_endpgm":
                following = []
        for to in following:
            if to < len(code) and reads < entry.get(to, most + 1):
                entry[to] = reads
                todo.append(to)
    return sorted(found.items())


def test_the_walk_sees_what_it_looks_for():
    code = """_Zk:
	ds_write_b128 v0, v[4:7]
	s_cbranch_scc1 .LBB0_2
%s.LBB0_2:
%s	s_waitcnt lgkmcnt(8)
	s_barrier
	s_endpgm
.Lfunc_end0:
"""
    read = "\tds_read_b128 v[8:11], v0\n"
    walk = lambda a, b: fewest_reads_behind_a_write(functions(code % (a * read, b * read))["_Zk"])
    assert [n for _, n in walk(9, 8)] == [8] and [n for _, n in walk(9, 3)] == [3]


def test_writes_are_done_where_the_waves_meet():
    """LDS operations are done in order: where at most eight are under way, a write with eight reads and more behind it is not among them."""
    cmd = [build._hipcc(), *build.FLAGS, *build.PAGED_FLAGS["attend_many.hip"], "--cuda-device-only", "-S", os.path.join(build.PAGED, "attend_many.hip"), "-o", "-"]
    listing = subprocess.run(cmd, check=True, stdout=subprocess.PIPE, stderr=subprocess.DEVNULL, text=True).stdout
    found = {name: fewest_reads_behind_a_write(code) for name, code in functions(listing).items() if "attend_many" in name}
    assert len(found) == 8 and all(found.values())
    assert all(n >= 8 for waits in found.values() for _, n in waits), found
