"""Build-time check of the device assembly of the sources whose kernels issue global loads by hand.

A load written in inline asm (`global_load_dwordx4 v[a:b], ...`) returns at once; its destination
registers hold the data only after an `s_waitcnt vmcnt(N)` that the load is old enough for.  Until then
no instruction may read or write them: a copy would take the old contents, and an overwritten register
would be overwritten again when the data lands.  The kernels keep that rule in their source (every
register filled by such a load passes through an await_*() before its first use), but the compiler is
free to move or copy a variable between the two asm statements - it cannot know the register is not
ready - and it does so where a loop closes with the variable in another register than it opened with.

The check follows every path of a kernel's control-flow graph.  State = the registers that may still be
in flight, each with the least number of vector-memory loads issued after it on any path (loads return
in order, so `s_waitcnt vmcnt(N)` retires exactly the entries with at least N younger loads; stores are
not counted as younger: they may complete out of order with loads, so counting them would be
optimistic).  Every instruction that names an in-flight register and is neither the wait that retires it
nor a later load into it is reported.  Waits and loads of the compiler's own count like the hand-written
ones: the hardware does not tell them apart.
"""
import re

_LABEL = re.compile(r"^([.\w$]+):")
_BRANCH = re.compile(r"^(s_cbranch_\w+|s_branch)\s+([.\w$]+)")
_VRANGE = re.compile(r"\bv\[(\d+):(\d+)\]")
_VONE = re.compile(r"\bv(\d+)\b")
_VMCNT = re.compile(r"vmcnt\((\d+)\)")
_DRAINED = "; ring drained"   # left by a source where none of its hand-issued loads is in flight any more
_CAP = 64   # the counter has six bits: nothing is ever younger than that


def _vregs(text):
    out = set()
    for a, b in _VRANGE.findall(text):
        out.update(range(int(a), int(b) + 1))
    out.update(int(a) for a in _VONE.findall(text))
    return out


def _is_vmem_load(t):
    op = t.split()[0]
    return op.startswith(("global_load", "buffer_load", "flat_load", "scratch_load")) or \
        (op.startswith(("global_atomic", "buffer_atomic", "flat_atomic")) and " glc" in t)


class _Ins:
    __slots__ = ("line", "text", "hand")

    def __init__(self, line, text, hand):
        self.line, self.text, self.hand = line, text, hand


def _functions(asm_text):
    """(name, [(line number, text, inside inline asm) | label]) for every function of the file."""
    funcs, cur, name, in_asm = [], None, None, False
    types = set(re.findall(r"\.type\s+([.\w$]+),@function", asm_text))
    if not types:   # a piece of a listing
        cur = []
        funcs.append(("", cur))
    for i, raw in enumerate(asm_text.split("\n"), 1):
        t = raw.strip() if raw.strip().startswith((";;#", _DRAINED)) else raw.split(";")[0].strip()
        if t.startswith(";;#ASMSTART"):
            in_asm = True
            continue
        if t.startswith(";;#ASMEND"):
            in_asm = False
            continue
        if not t:
            continue
        m = _LABEL.match(t)
        if m:
            if m.group(1) in types:
                name, cur = m.group(1), []
                funcs.append((name, cur))
            elif cur is not None:
                cur.append(m.group(1))
            continue
        if t.startswith("."):
            if t.startswith(".Lfunc_end") or t.startswith(".section") or t.startswith(".size"):
                cur = None if t.startswith((".size", ".section")) else cur
            continue
        if cur is not None:
            cur.append(_Ins(i, t, in_asm))
    return funcs


def _blocks(items):
    """Basic blocks: list of (labels, instructions, successor labels, falls through)."""
    blocks, labels, ins = [], [], []

    def close(succ, fall):
        nonlocal labels, ins
        if labels or ins:
            blocks.append((labels, ins, succ, fall))
        labels, ins = [], []

    for it in items:
        if isinstance(it, str):
            if ins:
                close([], True)
            labels.append(it)
            continue
        ins.append(it)
        m = _BRANCH.match(it.text)
        if m:
            close([m.group(2)], m.group(1) != "s_branch")
        elif it.text.startswith(("s_endpgm", "s_setpc", "s_trap")):
            close([], False)
    close([], False)
    return blocks


def _step(state, it, report):
    """Advance `state` (register -> (younger loads, line of the load)) over one instruction."""
    t = it.text
    if t.startswith("s_waitcnt"):
        m = _VMCNT.search(t)
        if m:
            n = int(m.group(1))
            for r in [r for r, (y, _) in state.items() if y >= n]:
                del state[r]
        return
    regs = _vregs(t)
    if _is_vmem_load(t):
        dst = _vregs(t.split(",")[0]) if "_lds_" not in t.split()[0] else set()
        hit = (regs - dst) & state.keys()   # an address taken from a register in flight
        if hit and report is not None:
            report(it, hit, state)
        for r in state:
            y, ln = state[r]
            state[r] = (min(y + 1, _CAP), ln)
        if it.hand:
            for r in dst:
                state[r] = (0, it.line)
        else:
            for r in dst:          # the compiler's own load: it waits for it itself
                state.pop(r, None)
        return
    hit = regs & state.keys()
    if hit and report is not None:
        report(it, hit, state)


def _entry_states(blocks, start, step, merge):
    """State before every block (None where no path leads): step(state, instruction) changes a state in place, merge(into, state) takes another
    path's in and says whether that changed anything.  A branch to a label that is not in the listing counts as falling through."""
    index = {lab: b for b, (labels, _, _, _) in enumerate(blocks) for lab in labels}
    entry = [None] * len(blocks)
    if blocks:
        entry[0] = dict(start)
    work = [0] if blocks else []
    while work:
        b = work.pop()
        _, ins, targets, fall = blocks[b]
        state = dict(entry[b])
        for it in ins:
            step(state, it)
        to = [index[x] for x in targets if x in index]
        if (fall or len(to) < len(targets)) and b + 1 < len(blocks):
            to.append(b + 1)
        for t in to:
            if entry[t] is None:
                entry[t] = dict(state)
                work.append(t)
            elif merge(entry[t], state):
                work.append(t)
    return entry


def _merge_least(into, state):
    """Least number per key; a key that one side lacks counts as far away."""
    changed = False
    for r, v in state.items():
        if r not in into or into[r] > v:
            into[r] = v
            changed = True
    return changed


def check_hand_issued_loads(asm_text, name):
    """Raise RuntimeError when a path through a kernel of `asm_text` touches the destination of a
    hand-issued load before a wait has retired it."""
    bad = []
    for fname, items in _functions(asm_text):
        blocks = _blocks(items)
        for (_, ins, _, _), state in zip(blocks, _entry_states(blocks, {}, lambda st, it: _step(st, it, None), _merge_least)):
            if state is None:
                continue

            def report(it, hit, st):
                r = min(hit)
                bad.append(f"{name}: {fname[:80]}: line {it.line}: `{it.text[:70]}` touches v{sorted(hit)[:8]}, "
                           f"loaded by hand at line {st[r][1]} with {st[r][0]} younger loads and no wait that covers it")

            for it in ins:
                _step(state, it, report)
    if bad:
        raise RuntimeError(f"{len(bad)} uses of registers whose hand-issued loads may still be in flight:\n  " + "\n  ".join(bad[:12]))


_SREG = re.compile(r"\bs(\d+)\b|\bs\[(\d+):(\d+)\]|\b(vcc)(_lo|_hi)?\b")
# scalar instructions whose first operand is not (or not always) written
_SCALAR_NO_WRITE = ("s_cmp", "s_bitcmp", "s_cbranch", "s_branch", "s_waitcnt", "s_nop", "s_barrier", "s_setprio", "s_sleep", "s_endpgm", "s_setreg",
                    "s_sendmsg", "s_setpc", "s_cmov", "s_trap", "s_sethalt", "s_set_gpr")
SCALAR_WAIT = 5   # wait states between a vector instruction that writes a scalar register and a vector-memory one that reads it


def _sregs(text):
    out = set()
    for one, a, b, vcc, half in _SREG.findall(text):
        if one:
            out.add(int(one))
        elif vcc:
            out |= {106, 107} if not half else {106 if half == "_lo" else 107}
        else:
            out |= set(range(int(a), int(b) + 1))
    return out


def _scalar_step(state, it):
    """Advance `state` (scalar register -> wait states since a vector instruction wrote it, while fewer than SCALAR_WAIT)."""
    t = it.text
    if t.startswith(";"):
        return
    passed = 1 + (int(t.split()[1], 0) if t.startswith("s_nop") else 0)
    for r in list(state):
        state[r] += passed
        if state[r] >= SCALAR_WAIT:
            del state[r]
    ops = t.split(None, 1)[1].split(",") if " " in t or "\t" in t else []
    if t.startswith("v_"):
        dst = _sregs(ops[0]) if ops else set()
        if len(ops) > 1 and ("_co_" in t.split()[0] or t.startswith(("v_div_scale", "v_mad_u64", "v_mad_i64"))):
            dst |= _sregs(ops[1])   # the carry
        state.update(dict.fromkeys(dst, 0))
    elif t.startswith("s_") and not t.startswith(_SCALAR_NO_WRITE) and ops:
        for r in _sregs(ops[0]):
            state.pop(r, None)


def check_scalar_bases(asm_text, name):
    """A scalar register written by a vector instruction - a lane read, the reload of a scalar spilled to a vector register's lanes, a
    comparison - may be read by a vector-memory instruction only SCALAR_WAIT wait states later.  The compiler fills them in in front of
    its own loads, but not in front of one inside an asm statement, whose base is then a stale address.  Raise RuntimeError when any
    path of the control-flow graph comes to a hand-issued load too soon."""
    bad = []
    for fname, items in _functions(asm_text):
        blocks = _blocks(items)
        for (_, ins, _, _), state in zip(blocks, _entry_states(blocks, {}, _scalar_step, _merge_least)):
            if state is None:
                continue
            for it in ins:
                if it.hand and it.text.startswith("global_load_"):
                    close = _sregs(it.text) & state.keys()
                    if close:
                        bad.append(f"{name}.s:{it.line}: {fname[:60]} `{it.text[:70]}` reads s{sorted(close)}, written by a vector instruction less "
                                   f"than {SCALAR_WAIT} wait states before")
                _scalar_step(state, it)
    if bad:
        raise RuntimeError("hand-issued loads read scalar registers too early:\n  " + "\n  ".join(bad[:10]))


def _is_ring_load(it):
    """A load of a decode kernel's ring: weights (non-temporal), and their scales and zero points."""
    return it.hand and (re.match(r"global_load_dwordx4 .* nt$", it.text) is not None or it.text.startswith(("global_load_dwordx2", "global_load_ushort")))


def _ring_step(state, it):
    """Advance `state` (registers that a load of the ring was issued into and that may be part of it still: until the source says that
    the ring is drained)."""
    if _is_ring_load(it):
        state.update(dict.fromkeys(_vregs(it.text.split(",")[0]), 0))
    elif it.text.startswith(_DRAINED):
        state.clear()


def ring_copies(asm_text, kernel):
    """(function, copies) for every function with `kernel` in its name: its VGPR-to-VGPR copies that name a register of the ring, on
    any path on which a load of the ring was issued into it before and the ring was not drained since.  (The activation loads are
    consumed before the loop and their registers reused.)"""
    out = []
    for fname, items in _functions(asm_text):
        if kernel not in fname:
            continue
        blocks, n = _blocks(items), 0
        for (_, ins, _, _), state in zip(blocks, _entry_states(blocks, {}, _ring_step, _merge_least)):
            if state is None:
                continue
            for it in ins:
                if re.match(r"v_(mov_b(32|64)_e32|swap_b32) v[\[\d][^,]*, v[\[\d]", it.text) and _vregs(it.text) & state.keys():
                    n += 1
                _ring_step(state, it)
        out.append((fname, n))
    return out
