"""Static check of the compiled softmax kernels (no GPU needed): no instruction reads a register that a
matrix instruction still writes.  The hardware does not wait for such a result; the compiler counts the
wait states in between, but not always across the end of a loop, where the kernels therefore wait
themselves.  Every path of the generated assembly is followed from each matrix instruction until its
result is due: passes + 4 wait states (an instruction is one, s_nop n is n + 1); another matrix
instruction may take the result as its own accumulator without a wait."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2401_08281_amd", "csrc")

PASSES = {"32x32x16": 8, "16x16x32": 4, "16x16x4_f32": 8}    # of four cycles each


def registers(token):
    """('v' or 'a', number) of every vector register that an operand names."""
    out = set()
    for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", token):
        out |= {(kind, n) for n in range(int(a), int(b) + 1)}
    for kind, a in re.findall(r"\b([va])(\d+)\b", token):
        out.add((kind, int(a)))
    return out


def split(line):
    body = line.split(";")[0].strip()
    name, _, rest = body.partition(" ")
    name = name.split("\t")[0]
    rest = body[len(name):]
    ops = [o.strip() for o in re.split(r",\s*(?![^\[]*\])", rest)] if rest.strip() else []
    return name, ops


class Function:
    def __init__(self, lines):
        self.code, self.labels = [], {}
        for line in lines:
            m = re.match(r"^(\.LBB\w+):", line)
            if m:
                self.labels[m.group(1)] = len(self.code)
                continue
            s = line.strip()
            if not s or s.startswith((";", ".", "//")) or s.endswith(":"):
                continue
            self.code.append(split(line))

    def next(self, i):
        name, ops = self.code[i]
        if name == "s_endpgm":
            return []
        if name == "s_branch":
            return [self.labels[ops[0]]]
        out = [i + 1] if i + 1 < len(self.code) else []
        if name.startswith("s_cbranch"):
            out.append(self.labels[ops[0]])
        return out

    def faults(self):
        found = []
        for i, (name, ops) in enumerate(self.code):
            if not name.startswith("v_mfma"):
                continue
            due = next(p for shape, p in PASSES.items() if shape in name) + 4
            dst = registers(ops[0])
            work, seen = [(j, 0) for j in self.next(i)], {}
            while work:
                j, waited = work.pop()
                if waited >= due or seen.get(j, 1 << 30) <= waited:
                    continue
                seen[j] = waited
                n, o = self.code[j]
                store = n.startswith(("global_store", "ds_write", "buffer_store", "flat_store", "global_atomic", "ds_add"))
                reads = o if store else o[1:]
                if n.startswith("v_mfma"):
                    reads = o[1:3] + ([o[3]] if registers(o[3]) != registers(ops[0]) else [])
                if any(registers(r) & dst for r in reads):
                    found.append((i, name, j, n, o, waited))
                    continue
                if registers(o[0] if o else "") >= dst and not store:
                    continue                                   # overwritten (the next product of a chain)
                step = int(o[0], 0) + 1 if n == "s_nop" else 1
                work += [(k, waited + step) for k in self.next(j)]
        return found


@pytest.mark.parametrize("source", ["kernels_logprob.hip", "kernels_attend.hip"])
def test_no_read_of_a_pending_matrix_result(source, tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    from paper_2401_08281_amd import build as b
    out = str(tmp_path / "kernels.s")
    flags = [f for f in b.FLAGS if f != "-fPIC"]
    subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only", os.path.join(CSRC, source), "-o", out], check=True,
                   stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    cur, name, seen = None, None, 0
    bad = []
    for line in open(out).read().splitlines() + ["\t.section end"]:
        m = re.match(r"^(_ZN\S*kernel\S*):", line)
        if m:
            name, cur = m.group(1), []
        elif cur is not None and line.strip().startswith(".section"):
            f = Function(cur)
            seen += sum(n.startswith("v_mfma") for n, _ in f.code)
            bad += [(name,) + x for x in f.faults()]
            cur = None
        elif cur is not None:
            cur.append(line)
    assert seen > 0
    assert not bad, bad[:5]
