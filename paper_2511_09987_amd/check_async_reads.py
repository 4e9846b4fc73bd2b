"""Static check of the assembly of kernels that issue LDS reads from inline asm and wait for them later.

Such a read names its destination registers as an asm output, so the compiler believes they hold the data as soon as
the asm statement ends; they do only after the `s_waitcnt lgkmcnt(n)` that covers the read.  The kernels are written
so that every use comes after that wait, but nothing stops the register allocator from placing a copy of such a
register between the read and the wait, which would silently copy stale data.  This check follows every path through every
kernel of an assembly listing, keeps the LDS operations that are still outstanding (they return in order, so a
wait for n leaves the newest n), and reports every instruction that reads or writes a register an outstanding read
is going to write (a later LDS read into the same registers excepted: it simply wins).  The build runs it on the
compiler's output and fails on any finding."""
import re

COUNTED = 15                              # the most operations that a wait can leave outstanding

_REG = re.compile(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b")


def _regs(text):
    out = set()
    for m in _REG.finditer(text):
        if m.group(1):
            out.update(range(int(m.group(1)), int(m.group(2)) + 1))
        else:
            out.add(int(m.group(3)))
    return out


def kernels(asm_text):
    """(name, index of the first line, index behind the last line) of every function in the listing."""
    lines = asm_text.split("\n")
    out = []
    i = 0
    while i < len(lines):
        m = re.match(r"^(_Z\w+):", lines[i])
        i += 1
        if m:
            first = i - 1
            while i < len(lines) and not re.match(r"^(\.Lfunc_end|_Z)\w*:", lines[i]):
                i += 1
            out.append((m.group(1), first, i))
    return out


def _instructions(lines, first, last):
    """[(line index, operation, text)] of a function, and where its labels point in that list."""
    code, labels = [], {}
    for i in range(first + 1, last):
        text = lines[i].split(";")[0].strip()
        if text.endswith(":"):
            labels[text[:-1]] = len(code)
        elif text and not text.startswith("."):
            code.append((i, text.split()[0], text))
    return code, labels


def violations(asm_text):
    """Findings as strings; empty when every register of an outstanding LDS read is left alone until its wait."""
    lines = asm_text.split("\n")
    found = {}                                # findings in the order in which they were met, each once
    for name, first, last in kernels(asm_text):
        code, labels = _instructions(lines, first, last)
        targets = set(labels.values())
        todo, seen = [(0, ())], set()         # where a path goes on, with what is outstanding there
        while todo:
            at, pending = todo.pop()          # pending: (line index, destination registers), oldest first
            while at < len(code):
                while pending and not pending[0][1]:
                    pending = pending[1:]     # nothing older hides behind these: any wait that counts them is as good
                if at in targets:
                    if (at, pending) in seen:
                        break
                    seen.add((at, pending))
                i, op, text = code[at]
                at += 1
                if op.startswith("s_waitcnt"):
                    m = re.search(r"lgkmcnt\((\d+)\)", text)
                    if m:
                        n = int(m.group(1))
                        pending = pending[max(len(pending) - n, 0):] if n else ()
                    continue
                if op == "s_endpgm":
                    break
                if op == "s_branch" or op.startswith("s_cbranch"):
                    todo.append((labels[text.split()[1]], pending))
                    if op == "s_branch":
                        break
                    continue
                read = op.startswith("ds_read") or op.startswith("ds_load")
                # another read into the same registers is harmless (LDS reads return in order: the later one wins);
                # only its address must not come from a register that is still to be delivered
                touched = _regs(text) if not read else _regs(text.split(",", 1)[1]) if "," in text else set()
                for since, dst in pending:
                    if touched & dst:
                        found[f"{name}: line {i + 1} '{text}' touches v{sorted(touched & dst)} that the read at "
                              f"line {since + 1} '{lines[since].strip()}' has yet to deliver"] = None
                if read:
                    pending += ((i, frozenset(_regs(text.split(",")[0]))),)
                elif op.startswith("ds_") or op.startswith("s_load") or op.startswith("s_buffer_load"):
                    pending += ((i, frozenset()),)      # counts towards lgkmcnt, delivers no vector register
                if len(pending) > COUNTED:    # no wait tells those before the newest apart
                    before = pending[:-COUNTED]
                    pending = ((before[0][0], frozenset().union(*(dst for _, dst in before))),) + pending[-COUNTED:]
    return list(found)


if __name__ == "__main__":
    import sys
    bad = violations(open(sys.argv[1]).read())
    print("\n".join(bad) if bad else "no finding")
    sys.exit(1 if bad else 0)
