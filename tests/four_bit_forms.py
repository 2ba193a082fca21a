"""Which instance of the 4-bit products' kernel a call runs: the rules, read from the sources of the two launchers, over the sizes of a call."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_02613_amd", "csrc")
LINE, POWERS, MOST_LDS = 256, 72, 160 * 1024


class Call:
    """What a launcher knows: m rows, n columns of the result, k; groups with sorted rows, None for dense ones."""

    def __init__(self, swiglu, m, n, k, groups=None):
        self.swiglu, self.m, self.n, self.k, self.offsets, self.groups = swiglu, m, n, k, groups is not None, groups or 1
        live = m if self.groups > 2 * m and m < self.groups else self.groups
        self.live, self.each = live, -(-m // live)

    def workgroups(self, cols, rows):
        tiles = -(-self.m // rows) if not self.offsets else min(max((self.each * 3 // 2 + rows - 1) // rows, 1), 8)
        return -(-self.n // cols) * self.live * tiles

    def lds(self, nw, kw, mt, wt, kc, direct):
        lt = 2 * wt if self.swiglu else wt
        x = mt * 32 * kc * (2 if self.k > kc else 1) if kc else min(self.m, mt * 16) * (-(-self.k // LINE) * LINE) * 2
        red = nw * kw * 16 * (lt * 16 + 4) * 4 if kw > 1 else 0
        return (0 if direct else nw * kw * lt * 16 * POWERS) + max(x, red)


def python_of(condition):
    """A launcher's condition as a Python expression over a Call `c`."""
    e = condition.replace("&&", " and ").replace("||", " or ").replace("!", " not ").replace("g.groups", "c.groups").replace("g.offsets", "c.offsets").replace("g.m", "c.m")
    e = re.sub(r"\beach\b", "c.each", e).replace("workgroups(g, ", "c.workgroups(").replace("kMostLds", str(MOST_LDS))
    e = re.sub(r"lds_of<(?:true|false), ([^>]*)>\(g\)", lambda m: "c.lds(" + m.group(1).replace("true", "True").replace("false", "False") + ")", e)
    return e.replace("/", "//")


def rules(swiglu):
    """The launcher's statements in order, as (depth of the braces, condition or None, form or None)."""
    text = open(os.path.join(CSRC, "k_four_swiglu.hip" if swiglu else "k_four_matmul.hip")).read()
    body = re.search(r"\nhipError_t launch\(const FourGemm &g, hipStream_t st\)\n\{\n(.*?)\n\}\n", text, re.S).group(1)
    out, depth = [], 0
    for line in body.splitlines():
        line = line.split("//")[0].strip()
        if not line:
            continue
        if line == "}":
            depth -= 1
            continue
        if line.startswith("const "):
            name, value = re.fullmatch(r"const (?:int|bool) (\w+) = (.*);", line).groups()
            out.append((depth, name, value))
            continue
        condition, rest = re.fullmatch(r"(?:if \((.*)\) )?(\{|return launch_as<[^;]*;)", line).groups()
        form = None
        if rest != "{":
            form = re.fullmatch(r"return launch_as<(true|false), (.*), TOut>\(g, row_tiles\(g, (\d+)\), st\);", rest)
            assert form and form.group(1) == ("true" if swiglu else "false") and int(form.group(2).split(", ")[2]) * 16 == int(form.group(3)), line
            form = form.group(2)
        out.append((depth, None, (condition, form)))
        depth += rest == "{"
    assert depth == 0
    return out


def form_of(c):
    """The template arguments NW, KW, MT, WT, D, KC, wavefronts, direct and whether k is whole lines, of the instance that the call runs."""
    names, skip = {}, None
    for depth, name, what in rules(c.swiglu):
        if skip is not None and depth > skip:
            continue
        skip = None
        if name is not None:
            if name != "each":
                value = re.sub(r"^(.*) \? (.*) : (.*)$", r"(\2) if (\1) else (\3)", what).replace("g.k", "c.k")
                names[name] = eval(python_of(value), {"c": c}, names)
            else:
                assert what == "rows_each(g)"
            continue
        condition, form = what
        true = condition is None or eval(python_of(condition), {"c": c}, names)
        if form is None:
            skip = None if true else depth
        elif true:
            return form + (", true" if c.k % LINE == 0 else ", false")
    raise AssertionError("no form")
