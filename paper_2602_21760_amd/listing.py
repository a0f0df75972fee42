"""Checks of the compiler's listings of kernels that hold inline asm.

For the compiler an LDS read written in asm has filled its registers when the statement ends; in truth the data arrives at a later wait.  The sources pass every such register
through the statement that waits, so nothing that uses it can come earlier, but a copy, a spill or another value in the same register could.  Whether the code that was made has one
depends on the compiler and on every edit, so build() looks.

And a vector instruction that takes the result of an MFMA has to come some wait states behind it.  The compiler puts them before its own instructions, not before those in asm.
"""
import re

_REGISTERS = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)")
_BRANCH = re.compile(r"s_(c?branch\w*)\s+(\.LBB\w+)")
_LGKM = re.compile(r"lgkmcnt\((\d+)\)")


def _registers(text):
    """{(file, number)} of the vector registers named in an operand list."""
    found = set()
    for file, first, last, one in _REGISTERS.findall(text):
        found.update((file, i) for i in range(int(first or one), int(last or one) + 1))
    return found


def _functions(listing):
    """{name: [(label or None, instruction or None, in asm, line)]}"""
    functions, code, asm = {}, None, False
    for number, line in enumerate(listing.split("\n"), 1):
        text = line.strip()
        if re.match(r"_Z\w+:", line):
            code = functions.setdefault(line.split(":")[0], [])
        elif code is None or text.startswith(".Lfunc_end"):
            code = None
        elif text.startswith(";;#ASM"):
            asm = text.startswith(";;#ASMSTART")
        elif re.match(r"\.LBB\w+:", text):
            code.append((text.split(":")[0], None, asm, number))
        else:
            text = text.split(";")[0].strip()
            if text and not text.startswith("."):
                code.append((None, text, asm, number))
    return functions


def _walk(code, labels, start, advance, stop, most=64):
    """Follows all paths from the instruction behind `start` with a count: stop(instruction, in asm, line, count) -> True ends a path, advance(instruction) is added to the count."""
    seen, todo = set(), [(start + 1, 0)]
    while todo:
        i, count = todo.pop()
        while i < len(code) and (i, count) not in seen:
            seen.add((i, count))
            label, text, asm, line = code[i]
            i += 1
            if label is not None:
                continue
            if stop(text, asm, line, count) or text.startswith("s_endpgm"):
                break
            count = min(count + advance(text), most)
            branch = _BRANCH.match(text)
            if branch and branch.group(1) == "branch":
                i = labels[branch.group(2)]
            elif branch:
                todo.append((labels[branch.group(2)], count))


def reads_in_flight(listing):
    """(number of LDS reads in asm, [what touches the registers of one before its wait]).  A read has arrived at a wait that leaves at most as many requests outstanding as
    LDS instructions came after it; they complete in order."""
    reads, faults = 0, set()
    for name, code in _functions(listing).items():
        labels = {label: i for i, (label, *_) in enumerate(code) if label is not None}
        for i, (_, text, asm, line) in enumerate(code):
            if not asm or text is None or not text.startswith("ds_read"):
                continue
            reads += 1
            filled = _registers(text.split(",")[0])

            def stop(other, _, at, younger):
                wait = _LGKM.search(other) if other.startswith("s_waitcnt") else None
                if wait and int(wait.group(1)) <= younger:
                    return True
                if filled & _registers(other) or other.startswith("s_endpgm"):
                    faults.add("%s: '%s' (line %d) before the data of '%s' (line %d) has arrived" % (name, other, at, text, line))
                    return True
                return False
            _walk(code, labels, i, lambda other: 1 if other.startswith("ds_") else 0, stop)
    return reads, sorted(faults)


def mfma_wait_states(mfma):
    """Wait states between an MFMA and a vector instruction that touches its result: the passes it takes (four rows of the result each, and in fp32 twice as many) and 4."""
    if "_16x16x32_" in mfma:
        return 8
    return 12 if "_16x16x4_" in mfma else 20


def early_uses_of_mfma_results(listing):
    """[asm instructions that touch an MFMA's result too early]"""
    found = set()
    for name, code in _functions(listing).items():
        labels = {label: i for i, (label, *_) in enumerate(code) if label is not None}
        for i, (_, text, asm, line) in enumerate(code):
            if text is None or not text.startswith("v_mfma"):
                continue
            need, result = mfma_wait_states(text), _registers(text.split(",")[0])

            def stop(other, in_asm, at, states):
                if states >= need:
                    return True
                # (what an LDS read fills arrives long after the MFMA's result)
                used = other.split(",", 1)[-1] if other.startswith("ds_read") else other
                if in_asm and other.startswith(("v_", "ds_")) and result & _registers(used):
                    found.add("%s: '%s' (line %d) %d wait states after '%s' (line %d), not %d" % (name, other, at, states, text, line, need))
                    return True
                return False
            _walk(code, labels, i, lambda other: int(other.split()[1], 0) + 1 if other.startswith("s_nop") else 1, stop)
    return sorted(found)


def faults(listing):
    return reads_in_flight(listing)[1] + early_uses_of_mfma_results(listing)
