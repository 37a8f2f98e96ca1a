"""The order of the streamed distillation's accesses to what its row warps hand to
a teacher's warp, on the CPU: the steps of both as the source has them, taken in every
order that its barriers allow, for clusters of one CTA (no exchange between rows)."""
import os
import re

import paper_2607_19331_gb300 as iso

TEACHERS, ROWS = 4, 13


def _kernel():
    path = os.path.join(os.path.dirname(iso.__file__), "csrc", "iso_distill.cu")
    with open(path) as f:
        src = re.sub(r"//[^\n]*", "", f.read())
    body = src[src.index("k_distill_stream(const"):]
    body = body[:body.index("k_distill_long(const")]
    rows, teacher = body.split("Top t = top_of(", 1)
    return rows, teacher


def _steps(text, steps):
    """The named steps in the order of their last occurrence."""
    at = {name: [m.start() for m in re.finditer(pattern, text)] for name, pattern in steps.items()}
    assert all(at.values()), at
    return sorted(at, key=lambda name: at[name][-1])


def _stale_reads(row_steps, teacher_steps):
    """(row read for, row found) of every read that can meet another row's value.
    A state: position of the row warps, of each teacher, and whose value each slot holds."""
    start = ((0, 0), ((0, 0),) * TEACHERS, (None,) * TEACHERS)
    seen, todo, wrong = {start}, [start], set()
    place = lambda p, steps: (p[0], p[1] + 1) if p[1] + 1 < len(steps) else (p[0] + 1, 0)        # noqa: E731
    done = lambda p, steps, name: p[0] + (1 if p[1] > steps.index(name) else 0)                   # noqa: E731
    while todo:
        rows, teachers, held = todo.pop()
        after = []
        if rows[0] < ROWS:
            slot, phase, name = rows[0] % TEACHERS, rows[0] // TEACHERS, row_steps[rows[1]]
            if name != "wait prepared" or done(teachers[slot], teacher_steps, "arrive prepared") > phase:
                now = held[:slot] + (rows[0],) + held[slot + 1:] if name == "write" else held
                after.append((place(rows, row_steps), teachers, now))
        for slot, p in enumerate(teachers):
            row, name = slot + p[0] * TEACHERS, teacher_steps[p[1]]
            if row >= ROWS:
                continue
            if name == "wait written" and done(rows, row_steps, "arrive written") <= row:
                continue
            if name == "read" and held[slot] != row:
                wrong.add((row, held[slot]))
            after.append((rows, teachers[:slot] + (place(p, teacher_steps),) + teachers[slot + 1:], held))
        for state in after:
            if state not in seen:
                seen.add(state)
                todo.append(state)
    return wrong


def test_a_teachers_warp_meets_its_own_rows_sums():
    rows, teacher = _kernel()
    row_steps = _steps(rows, {"write": r"\bof_row\[slot\]\s*=", "wait prepared": r"wait\S*\(smem_u32\(&prepared\[slot\]\)",
                              "arrive written": r"mbar_arrive\(smem_u32\(&written\[slot\]\)\)"})
    teacher_steps = _steps(teacher, {"arrive prepared": r"arrive_warp\(smem_u32\(&prepared\[slot\]\)\)",
                                     "wait written": r"wait\S*\(smem_u32\(&written\[slot\]\)", "read": r"=\s*of_row\[slot\]"})
    assert teacher_steps == ["arrive prepared", "wait written", "read"]
    assert not _stale_reads(row_steps, teacher_steps)


def test_the_model_finds_a_write_before_its_wait():
    teacher_steps = ["arrive prepared", "wait written", "read"]
    assert _stale_reads(["write", "wait prepared", "arrive written"], teacher_steps)
    assert _stale_reads(["wait prepared", "arrive written", "write"], teacher_steps)
    assert not _stale_reads(["wait prepared", "write", "arrive written"], teacher_steps)
