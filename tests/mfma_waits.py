"""Waits after matrix instructions in the assembly of the built library.

A matrix instruction writes its result some wait states after it was issued, and the hardware does not hold back an ordinary
vector or memory instruction that touches the result's registers earlier.  The compiler puts the waits in for instructions of
its own; those inside inline assembly it does not know.  `too_early` follows every path through a kernel and finds the
instructions that touch a result before it is there.
"""
import collections
import re
import struct
import subprocess
import tempfile

from tests.kernel_resources import _MAGIC

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# v_mfma_*_16x16x128_f8f6f4 takes 8 passes of 4 cycles; 12 wait states have to lie before another use of its result
WAIT = 12
_REG = re.compile(r"\b([av])(?:(\d+)\b|\[(\d+):(\d+)\])")


def code_objects(lib_path):
    """The gfx950 ELFs of the library's offload bundles."""
    blob = open(lib_path, "rb").read()
    at = blob.find(_MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", blob, at + len(_MAGIC))
        pos = at + len(_MAGIC) + 8
        for _ in range(count):
            off, size, idlen = struct.unpack_from("<QQQ", blob, pos)
            if size and b"gfx950" in blob[pos + 24:pos + 24 + idlen]:
                yield blob[at + off:at + off + size]
            pos += 24 + idlen
        at = blob.find(_MAGIC, at + 1)


def listings(elf):
    """{kernel: [(address, text, branch target or None)]} of the functions in an ELF's text."""
    with tempfile.NamedTemporaryFile(suffix=".o") as f:
        f.write(elf)
        f.flush()
        text = subprocess.run([OBJDUMP, "-d", f.name], check=True, capture_output=True, text=True).stdout
    return parse(text)


def parse(text):
    found, body, first = {}, None, 0
    for line in text.splitlines():
        if line.endswith(">:"):
            m = re.match(r"([0-9a-f]+) <(.*)>:", line)
            first, body = int(m.group(1), 16), found.setdefault(m.group(2), [])
        elif body is not None and "//" in line:
            words, tail = line.split("//", 1)
            to = re.search(r"<[^>]*?(?:\+0x([0-9a-f]+))?>", tail) if "<" in tail else None
            body.append((int(tail.split(":")[0], 16), words.strip(), first + int(to.group(1) or "0", 16) if to else None))
    return found


def _registers(text):
    out = set()
    for kind, one, lo, hi in _REG.findall(text):
        out.update((kind, i) for i in ([int(one)] if one else range(int(lo), int(hi) + 1)))
    return out


def _successors(body):
    at = {a: i for i, (a, _, _) in enumerate(body)}
    out = []
    for i, (_, text, to) in enumerate(body):
        op = text.split()[0]
        assert op not in ("s_swappc_b64", "s_call_b64"), "kernels call no functions"
        to_there = []
        if op == "s_setpc_b64":  # a far branch: s_getpc, the distance added, s_setpc
            (pc, lo, hi) = (body[i - j][1].split() for j in (3, 2, 1))
            assert (pc[0], lo[0], hi[0]) == ("s_getpc_b64", "s_add_u32", "s_addc_u32"), (pc, lo, hi)
            away = (int(hi[-1], 0) & 0xffffffff) << 32 | int(lo[-1], 0) & 0xffffffff
            to_there = [at[body[i - 2][0] + (away - (1 << 64) if away >> 63 else away)]]
        elif op == "s_branch" or op.startswith("s_cbranch"):
            to_there = [at[to]]
        if op not in ("s_endpgm", "s_branch", "s_setpc_b64") and i + 1 < len(body):
            to_there.append(i + 1)
        out.append(to_there)
    return out


def too_early(body):
    """[(instruction, wait states between the matrix instruction and it)] of one listing."""
    next_of = _successors(body)
    steps = []  # (the registers it begins to write, wait states it counts for)
    for _, text, _ in body:
        op, _, rest = text.partition(" ")
        steps.append((_registers(rest.split(",")[0]) if op.startswith("v_mfma") else None, int(rest.split()[0], 0) + 1 if op == "s_nop" else 1))
    since = [None] * len(body)  # on the way there with the fewest: {register: wait states}
    since[0], todo, bad = {}, collections.deque([0]), {}
    while todo:
        i = todo.popleft()
        begins, states = steps[i]
        if begins is None and since[i]:
            early = [since[i][r] for r in _registers(body[i][1].partition(" ")[2]) if r in since[i]]
            if early:
                bad[i] = min(early)
        after = {r: s + states for r, s in since[i].items() if s + states < WAIT}
        if begins is not None:
            after.update(dict.fromkeys(begins, 0))
        for j in next_of[i]:
            if since[j] is None:
                since[j] = dict(after)
            else:
                fewer = {r: s for r, s in after.items() if s < since[j].get(r, WAIT)}
                if not fewer:
                    continue
                since[j].update(fewer)
            todo.append(j)
    return [(body[i][1], s) for i, s in sorted(bad.items())]
