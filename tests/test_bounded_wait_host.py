"""The bounded wait of the tensor-core kernels, run step by step on the host: its instructions as they stand in the source,
against a barrier and a clock that the test moves."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SECOND = 2_000_000_000   # cycles, about; a wait has two
WORD = 1 << 32


def source():
    """The instructions and labels of the wait, and the values of its immediate operands."""
    text = open(os.path.join(ROOT, "paper_2605_26660_b200", "csrc", "tcgen05.cuh")).read()
    body = text[text.index("void mbar_wait("):]
    end = body.index('::"r"')
    asm = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', body[:end]))
    constants = {}
    for x in re.findall(r"constexpr (?:unsigned|long long) ([^;]*);", text):
        for name, value in re.findall(r"(k\w+Cycles) = ([^,]*)", x):
            constants[name] = eval(re.sub(r"(?<=\d)(ull|ll|u)", "", value))
    operands = re.findall(r'"(r|n)"\((\w+)\)', body[end: body.index(': "memory"')])
    immediate = {"%%%d" % i: constants[name] for i, (kind, name) in enumerate(operands) if kind == "n"}
    code = []
    for line in asm.replace("\\n\\t", "\n").replace("\\n", "\n").replace("%%", "%").split("\n"):
        line = line.strip("{} \t")
        while re.match(r"\w+:", line):
            label, line = line.split(":", 1)
            code.append(("label", label))
            line = line.strip("{} \t")
        code += [("op", x.strip()) for x in line.split(";") if x.strip() and not x.strip().startswith(".reg")]
    return code, immediate


def run(complete, clock, dead=0, steps=100_000):
    """complete(n): whether the n-th look finds the barrier complete; clock(n): its n-th reading.  Returns (dead, looks)."""
    code, immediate = source()
    labels = {x: i for i, (kind, x) in enumerate(code) if kind == "label"}
    reg, at, looks, reads = {}, 0, 0, 0
    value = lambda x: immediate[x] if x in immediate else int(x) if re.fullmatch(r"\d+", x) else reg[x]  # noqa: E731
    for _ in range(steps):
        if at == len(code):
            return dead, looks
        kind, op = code[at]
        at += 1
        if kind == "label":
            continue
        if op.startswith("@"):
            guard, op = op[1:].split(" ", 1)
            if not reg[guard]:
                continue
        name, _, rest = op.partition(" ")
        args = [x.strip() for x in rest.split(",")]
        wide = WORD if name.endswith(".u32") else 1 << 64
        if name.startswith("mbarrier.try_wait.parity"):
            reg[args[0]] = complete(looks)
            looks += 1
        elif name == "bra":
            at = labels[args[0]]
        elif name == "ld.volatile.shared.u32":
            reg[args[0]] = dead
        elif name == "st.volatile.shared.u32":
            dead = int(args[1])
        elif args[-1] in ("%clock", "%clock64"):
            reg[args[0]] = (7 * SECOND + clock(reads)) % wide
            reads += 1
        elif name.startswith("mov."):
            reg[args[0]] = value(args[1])
        else:
            a, b = value(args[1]), value(args[2])
            kind = name.rsplit(".", 1)[0]
            reg[args[0]] = {"add": lambda: (a + b) % wide, "sub": lambda: (a - b) % wide, "min": lambda: min(a, b),
                            "setp.ne": lambda: a != b, "setp.lt": lambda: a < b}[kind]()
    raise AssertionError("the wait does not end")


def test_a_complete_barrier_is_seen_at_once():
    assert run(lambda n: True, lambda n: 0) == (0, 1)
    assert run(lambda n: n >= 3, lambda n: 100 * n) == (0, 4)


@pytest.mark.parametrize("step", [1_000_000, 60_000_000])
def test_a_barrier_that_never_completes_raises_the_flag_after_about_two_seconds(step):
    asked = []
    dead, looks = run(lambda n: False, lambda n: asked.append(n * step) or asked[-1])
    assert dead == 1 and looks >= 5 and 1.9 * SECOND <= asked[-1] <= 2.2 * SECOND


def test_another_wait_that_gave_up_ends_this_one():
    dead, looks = run(lambda n: False, lambda n: 0, dead=1)
    assert dead == 1 and looks <= 2


@pytest.mark.parametrize("away", [1, 2, 7])
@pytest.mark.parametrize("seconds", [1, 2, 3, 60])
def test_a_context_that_was_switched_out_looks_again_and_has_time_left(seconds, away):
    # between a look and the clock, or anywhere; the barrier completes meanwhile, or some time after the return
    clock = lambda n: 1000 * n if n < away else seconds * SECOND + SECOND // 2 + 1000 * n  # noqa: E731
    for complete in (away + 1, away + 60):
        assert run(lambda n: n >= complete, clock)[0] == 0
    assert run(lambda n: n >= 60, lambda n: seconds * SECOND * (1 + n // 20) + 1000 * n)[0] == 0   # three times
