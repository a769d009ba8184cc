"""Build-time check for the kernel whose loads into LDS are waited for by hand-counted waits (products with 4-bit weights, many rows).

Loads that go from memory straight into LDS fill no register, so the compiler waits for none of them.  w4_wide_kernel brings its activations
in half steps, a ring of four, and before a barrier waits until at most so many loads are outstanding that the half step read behind the barrier
must have come.  Which loads those are depends on how many others the compiler keeps between them, and in what order.  This script reads the
compiler's assembly listing of the kernel source (produced by the build; nothing is disassembled), follows every path, and fails if

  * at a tile's first barrier more than two half steps' loads into LDS may be outstanding, or more than one at a later barrier, or
  * any is when the kernel ends.

A barrier is a tile's first until loads into LDS have been outstanding at one; where none is any more, the next is a first again (a kernel
holds tiles of two widths).

Vector loads return in the order they were issued; stores are not counted on (a wait for n operations may leave the last n loads).
A half step is MB / 2 loads a wave, MB being the kernel's second template argument.

    python check_lds_loads.py listing.s w4_wide_kernel
"""
import re
import sys

AT_FIRST, LATER = 2, 1                   # half steps that may be outstanding


def parse_kernel(lines):
    """-> blocks {label: ([item, ...], [label of a successor, ...])}, the first label.  Items: "lds", "load", ("wait", n), "barrier", "end"."""
    blocks, label, items = {}, "entry", []
    after = {}
    order = ["entry"]

    def close(successors, falls):
        blocks[label] = (items, successors)
        after[label] = falls
    successors = []
    for raw in lines:
        line = raw.split(";")[0].strip()
        m = re.match(r"^(\.LBB\d+_\d+):", line)
        if m:
            close(successors, True)
            label, items, successors = m.group(1), [], []
            order.append(label)
            continue
        if not line or line.startswith(".") or line.endswith(":"):
            continue
        op, _, rest = line.partition(" ")
        if re.match(r"(buffer|global|flat|scratch)_load", op):
            items.append("lds" if re.search(r"\blds\b", rest) or "_lds_" in op else "load")
        elif op == "s_waitcnt":
            n = re.search(r"vmcnt\((\d+)\)", rest)
            if n:
                items.append(("wait", int(n.group(1))))
            elif not re.search(r"cnt\(", rest):
                raise ValueError("a wait that is not understood: " + line)
        elif op == "s_barrier":
            items.append("barrier")
        elif op == "s_endpgm":
            items.append("end")
        elif re.match(r"s_(cbranch\w*|branch)$", op):
            # a block of its own behind every branch
            close(successors + [rest.strip()], op != "s_branch")
            label, items, successors = "%s+%d" % (label.split("+")[0], len(order)), [], []
            order.append(label)
        elif re.match(r"s_(setpc|swappc|call)", op):
            raise ValueError("a jump that is not understood: " + line)
    close(successors, False)
    for a, b in zip(order, order[1:]):
        if after[a] and "end" not in blocks[a][0]:
            blocks[a][1].append(b)
    return blocks, "entry"


def check_kernel(name, lines, half_step):
    """-> (number of loads into LDS, problems).  A state is the outstanding loads from the oldest into LDS on, and whether there was a barrier."""
    blocks, first = parse_kernel(lines)
    problems, seen, todo = set(), set(), [(first, (), False)]
    while todo:
        at = todo.pop()
        if at in seen:
            continue
        seen.add(at)
        label, queue, barrier = at
        items, successors = blocks[label]
        queue, ended = list(queue), False
        for item in items:
            if item in ("lds", "load"):
                queue.append(item)
                while queue and queue[0] != "lds":      # what is older than the oldest into LDS does not matter
                    queue.pop(0)
                del queue[:-64]                          # no counter says more
            elif item == "barrier":
                most = half_step * (LATER if barrier else AT_FIRST)
                if queue.count("lds") > most:
                    problems.add("%s: %d loads into LDS may be outstanding at %s barrier in %s, %d are allowed" % (
                        name, queue.count("lds"), "a later" if barrier else "a first", label, most))
                barrier = "lds" in queue
            elif item == "end":
                if "lds" in queue:
                    problems.add("%s: loads into LDS may be outstanding at its end in %s" % (name, label))
                ended = True
                break
            else:
                queue = queue[len(queue) - item[1]:] if item[1] < len(queue) else queue
                while queue and queue[0] != "lds":
                    queue.pop(0)
                barrier = barrier and bool(queue)
        if not ended:
            todo += [(s, tuple(queue), barrier) for s in successors]
    return sum(items.count("lds") for items, _ in blocks.values()), sorted(problems)


def kernels(text, pattern):
    """(symbol, its lines) of the kernels whose names hold `pattern`."""
    lines = text.split("\n")
    for s in (i for i, l in enumerate(lines) if re.match(r"^_Z\w*%s\w*:" % re.escape(pattern), l)):
        e = s
        while e < len(lines) and not lines[e].startswith(".Lfunc_end"):
            e += 1
        yield lines[s].split(":")[0], lines[s + 1:e]


def main(argv):
    if len(argv) != 3:
        sys.exit(__doc__)
    bad, found = 0, 0
    for name, lines in kernels(open(argv[1]).read(), argv[2]):
        found += 1
        n, problems = check_kernel(name, lines, int(re.search(r"ILb\dELi(\d+)E", name).group(1)) // 2)
        print("check_lds_loads: %s: %d loads into LDS, %d problem(s)" % (name, n, len(problems)))
        for p in problems[:20]:
            print("  " + p)
        bad += len(problems) + (n == 0)
    if not found:
        sys.exit("check_lds_loads: no kernel matching %r in %s" % (argv[2], argv[1]))
    sys.exit(1 if bad else 0)


if __name__ == "__main__":
    main(sys.argv)
