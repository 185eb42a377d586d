"""Where hipcc's assembly for gfx950 keeps vector registers in scratch memory, and with which lanes.

A vector register that is spilled behind an `if` of some lanes, in front of the instruction that switches the others on again, is stored for
those lanes only; what the others read back later is whatever lay in scratch.  hipcc has done so.  `partial_stores` finds such stores:
it follows the execution mask through a kernel as the conditions that lead to it, `()` for all lanes, None where it is not known.
"""
import re

_KERNEL = re.compile(r"^(_Z\w+):")
_LABEL = re.compile(r"^(\.L\w+):")
_JUMP = re.compile(r"^s_c?branch(?:_\w+)? (\.L\w+)")
_NO_RESULT = ("s_cmp", "s_bitcmp", "s_waitcnt", "s_barrier", "s_nop", "s_setprio", "s_sleep", "s_inst", "s_setreg", "s_endpgm", "s_cbranch", "s_branch",
              "s_dcache", "s_icache", "s_sethalt", "s_ttrace", "s_trap", "s_set_gpr")


def _kernels(assembly):
    name, body = None, []
    for line in assembly.splitlines():
        m = _KERNEL.match(line)
        if m:
            name, body = m[1], []
        elif name and line.startswith(".Lfunc_end"):
            yield name, body
            name = None
        elif name:
            body.append(line)


def _scalars(operand):
    """The scalar registers that an operand names, 32 bits each."""
    m = re.match(r"^s\[(\d+):(\d+)\]$", operand) or re.match(r"^s(\d+)()$", operand)
    if m:
        return ["s%d" % k for k in range(int(m[1]), int(m[2] or m[1]) + 1)]
    return {"vcc": ["vcc_lo", "vcc_hi"], "vcc_lo": ["vcc_lo"], "vcc_hi": ["vcc_hi"]}.get(operand, [])


def _vectors(operand):
    m = re.match(r"^v\[(\d+):(\d+)\]$", operand) or re.match(r"^v(\d+)()$", operand)
    return ["v%d" % k for k in range(int(m[1]), int(m[2] or m[1]) + 1)] if m else []


def _either(x, y):
    if () in (x, y):
        return ()
    if None in (x, y):
        return None
    if x == y[:len(x)]:
        return x
    if y == x[:len(y)]:
        return y
    if x[:-1] == y[:-1] and x[-1][0] == y[-1][0]:        # a condition and its opposite
        return x[:-1]
    return None


def _both(x, y):
    if None in (x, y):
        return None
    return y if x == y[:len(x)] else x if y == x[:len(y)] else None


def _without(x, y):
    """x and not y."""
    if None in (x, y):
        return None
    if len(y) == len(x) + 1 and y[:-1] == x:
        return x + ((y[-1][0], not y[-1][1]),)
    for a, b in zip(x, y):
        if a != b:
            return x if a[0] == b[0] else None           # nothing in common
    return None


def _exclusive(x, y):
    if None in (x, y):
        return None
    return _without(x, y) if len(y) > len(x) else _without(y, x) if len(x) > len(y) else None


class _State(dict):
    """Masks by the scalar register that holds half of them, or by (vector register, lane) where that register was put aside; "exec"."""

    def mask(self, operand):
        if operand == "exec":
            return self["exec"]
        if operand == "-1":
            return ()
        r = _scalars(operand)
        return self.get(r[0]) if len(r) == 2 and self.get(r[0]) == self.get(r[1]) else None

    def put(self, operand, mask):
        for r in _scalars(operand):
            if mask is None:
                self.pop(r, None)
            else:
                self[r] = mask

    def narrowed(self, here):
        """exec under a condition that the instruction at `here` has found, which may have been there before with another outcome."""
        for key in [k for k, mask in self.items() if mask and k != "exec" and any(c[0] == here for c in mask)]:
            del self[key]
        e = self["exec"]
        return None if e is None or any(c[0] == here for c in e) else e + ((here, True),)

    def step(self, ins, here):
        op, _, rest = ins.partition(" ")
        a = [x.strip() for x in rest.split(",")] if rest else [""]
        if op.endswith("saveexec_b64"):
            e, src = self["exec"], self.mask(a[1])
            if op == "s_and_saveexec_b64":
                new = _both(e, src) if src is not None else self.narrowed(here)
            else:
                new = {"s_or_saveexec_b64": _either, "s_andn2_saveexec_b64": lambda e, src: _without(src, e)}.get(op, lambda *_: None)(e, src)
            self.put(a[0], e)
            self["exec"] = new
        elif op.startswith("s_") and a[0] == "exec":
            x, y = self.mask(a[1]), self.mask(a[-1])
            if op == "s_mov_b64":
                self["exec"] = x
            elif op == "s_or_b64":
                self["exec"] = _either(x, y)
            elif op in ("s_and_b64", "s_andn2_b64") and a[1] == "exec" and y is None:
                self["exec"] = self.narrowed(here)
            else:
                self["exec"] = {"s_and_b64": _both, "s_andn2_b64": _without, "s_xor_b64": _exclusive}.get(op, lambda *_: None)(x, y)
        elif op.startswith("s_") and a[0] in ("exec_lo", "exec_hi") or op.startswith("v_cmpx"):
            self["exec"] = None
        elif op == "s_mov_b64":
            self.put(a[0], self.mask(a[1]))
        elif op in ("s_or_b64", "s_xor_b64"):
            self.put(a[0], (_either if op == "s_or_b64" else _exclusive)(self.mask(a[1]), self.mask(a[2])))
        elif op == "s_mov_b32":
            r = _scalars(a[1])
            self.put(a[0], self["exec"] if a[1] in ("exec_lo", "exec_hi") else self.get(r[0]) if r else None)
        elif op == "v_writelane_b32":
            r = _scalars(a[1])
            self.pop((a[0], a[2]), None)
            if r and r[0] in self:
                self[a[0], a[2]] = self[r[0]]
        elif op == "v_readlane_b32":
            self.put(a[0], self.get((a[1], a[2])))
        elif op.startswith("s_") and not op.startswith(_NO_RESULT):
            self.put(a[0], None)
        else:                                            # vector results, and the scalar ones of comparisons and carries
            self.put(a[0], None)
            if op.startswith("v_") and len(a) > 1:
                self.put(a[1], None)
            if "store" not in op:
                for v in _vectors(a[0]):
                    for key in [k for k in self if isinstance(k, tuple) and k[0] == v]:
                        del self[key]


def _stores(body):
    """{place: (mask, instruction)} of the instructions that spill a vector register."""
    blocks, order = {"": []}, [""]
    for line in body:
        m = _LABEL.match(line)
        if m:
            order.append(m[1])
            blocks[m[1]] = []
            continue
        text, _, comment = line.partition(";")
        text = " ".join(text.split())
        if text and not text.startswith("."):
            blocks[order[-1]].append((text, "Folded Spill" in comment))
    behind = dict(zip(order, order[1:]))
    start, work, found = {"": _State(exec=())}, [""], {}
    while work:
        name = work.pop()
        state = _State(start[name])

        def go(to):
            if to not in blocks:
                return
            if to not in start:
                start[to] = _State(state)
            else:
                old = start[to]
                met = _State((k, v) for k, v in old.items() if k != "exec" and state.get(k) == v)
                met["exec"] = old["exec"] if old["exec"] == state["exec"] else None
                if met == old:
                    return
                start[to] = met
            work.append(to)

        for i, (text, spill) in enumerate(blocks[name]):
            if spill:
                found[name, i] = state["exec"], text
            m = _JUMP.match(text)
            if m:
                go(m[1])
            if text.startswith(("s_branch", "s_endpgm")):
                break
            if not m:
                state.step(text, (name, i))
        else:
            go(behind.get(name))
    return found


def partial_stores(assembly):
    """[(kernel, instruction)] for vector registers that are spilled while lanes are off, or while it is not known that none are."""
    return [(name, text) for name, body in _kernels(assembly) if any("Folded Spill" in line for line in body)
            for mask, text in _stores(body).values() if mask != ()]
