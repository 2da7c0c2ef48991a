"""Whether a vector memory load can still be writing a register that an inline assembly statement reads or writes.

The compiler waits for its own loads (of spilled values among them) in front of what uses their registers, inline assembly included, but for statements
that pin registers and say that they touch memory: of those it does not look at the pinned ones.  A spilled value that was loaded for another path can
then arrive on top of a statement's results.  This reads the assembly of a kernel and follows every path through it."""
import re

_REG = re.compile(r"\bv(?:\[(\d+):(\d+)\]|(\d+)\b)")
_VMEM = re.compile(r"(global|scratch|buffer|flat)_(load|store|atomic)")


def _registers(text):
    for first, last, one in _REG.findall(text):
        yield from ([int(one)] if one else range(int(first), int(last) + 1))


def kernels(assembly):
    """name and lines of every function"""
    name, body = None, None
    for line in assembly.split("\n"):
        m = re.match(r"(_Z\w+):", line)
        if m:
            name, body = m.group(1), []
        elif line.startswith(".Lfunc_end") and body is not None:
            yield name, body
            body = None
        elif body is not None:
            body.append(line)


def _instructions(lines):
    """[(text, in a statement)] and the labels' places; what statements put into another subsection stands behind the function"""
    main, other, into = [], [], 0
    for line in lines:
        if line.strip().startswith(".subsection"):
            into = int(line.split()[1])
            other.append(";;#ASMSTART" if into else ";;#ASMEND")
        else:
            (other if into else main).append(line)
    found, labels, inside = [], {}, False
    for line in main + other:
        if ";;#ASMSTART" in line or ";;#ASMEND" in line:
            inside = ";;#ASMSTART" in line
            continue
        text = line.split(";")[0].strip()
        m = re.match(r"([\w.$]+):$", text)
        if m:
            labels[m.group(1)] = len(found)
        elif text and not text.startswith("."):
            found.append((text, inside))
    return found, labels


def conflicts(lines):
    """[(instruction in a statement, register)] where a load may be in flight.  A state is, for every register that a load writes, how many vector
    memory operations were issued after it (stores count too, results come in order); vmcnt(N) leaves the N youngest."""
    ins, labels = _instructions(lines)
    starts = sorted({0} | set(labels.values()) | {i + 1 for i, (t, _) in enumerate(ins) if re.match(r"s_c?branch|s_endpgm", t)})
    starts = [s for s in starts if s < len(ins)]
    end = dict(zip(starts, starts[1:] + [len(ins)]))
    states, todo, found = {0: {}}, [0], set()
    while todo:
        start = todo.pop()
        pending = dict(states[start])
        for text, inside in ins[start:end[start]]:
            if text.startswith("s_waitcnt"):
                m = re.search(r"vmcnt\((\d+)\)", text)
                if m:
                    pending = {r: age for r, age in pending.items() if age < int(m.group(1))}
                continue
            if inside:
                found.update((text, r) for r in _registers(text) if r in pending)
            if _VMEM.match(text):
                pending = {r: age + 1 for r, age in pending.items() if age < 62}  # (the counter holds 63)
                if "_load" in text.split()[0] and "lds" not in text.split()[0]:
                    pending.update((r, 0) for r in _registers(text.split(",")[0]))
        last = ins[end[start] - 1][0]
        after = []
        if re.match(r"s_c?branch", last):
            after.append(labels[last.split()[1]])
        if not re.match(r"s_branch|s_endpgm", last):
            after.append(end[start])
        for s in after:
            if s not in end:
                continue
            old = states.get(s)
            new = dict(old or {})
            for r, age in pending.items():
                new[r] = min(age, new.get(r, age))
            if old is None or new != old:
                states[s] = new
                todo.append(s)
    reached = sum(end[s] - s for s in states)
    return sorted(found), reached / max(len(ins), 1)
