"""Reads the compiler's listing of this repository's own kernels: how many wait states lie between a matrix product and an LDS write of its result,
along every path through branches."""
import re


def registers(text):
    found = set()
    for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        found |= {(kind, i) for i in range(int(a), int(b) + 1)}
    return found | {(kind, int(a)) for kind, a in re.findall(r"\b([va])(\d+)\b", text)}


def functions(listing):
    """{name: ([(line, instruction)], {label: index})}"""
    res, name = {}, None
    for number, line in enumerate(listing.splitlines(), 1):
        text = line.split(";")[0].strip()
        start = re.match(r"^(_Z\w+):", line)
        if start:
            name = start.group(1)
            res[name] = ([], {})
        elif name and line.startswith(".Lfunc_end"):
            name = None
        elif name and re.match(r"^\.LBB\w+:", text):
            res[name][1][text[:-1]] = len(res[name][0])
        elif name and text and not text.startswith("."):
            res[name][0].append((number, text))
    return res


def early_lds_writes(program, labels, states):
    """[(line of a product, line of the LDS write, states between)] with fewer than states[product] between them."""
    early = []
    for i, (line, text) in enumerate(program):
        if not text.startswith("v_mfma"):
            continue
        result, needed = registers(text.split(",")[0]), states[text.split()[0]]
        paths, seen = [(i + 1, 0, result)], set()
        while paths:
            at, waited, live = paths.pop()
            while at < len(program) and waited < needed and live and (at, waited) not in seen:
                seen.add((at, waited))
                number, now = program[at]
                op, _, rest = now.partition(" ")
                if op.startswith("ds_write") and registers(rest.split(",", 1)[1]) & live:
                    early.append((line, number, waited))
                    break
                if op.startswith("s_cbranch"):
                    paths.append((labels[rest.split()[0]], waited + 1, live))
                elif op == "s_branch":
                    at, waited = labels[rest.split()[0]], waited + 1
                    continue
                elif op == "s_endpgm":
                    break
                elif op.startswith(("v_", "ds_read", "buffer_load", "global_load")) and "lds" not in now:
                    live = live - registers(rest.split(",")[0])      # (a product that adds to this one's result is looked at by itself)
                waited += int(rest.split()[0], 0) + 1 if op == "s_nop" else 1
                at += 1
    return early
