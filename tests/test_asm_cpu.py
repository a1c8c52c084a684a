"""Instructions written out in the kernels' sources keep what the compiler, which does not look into them, would have kept."""
import pathlib
import re

CSRC = pathlib.Path(__file__).resolve().parents[1] / "paper_2609_03844_amd" / "csrc"


def statements():
    """(file, instructions, what follows them) of each asm statement."""
    for path in sorted(CSRC.iterdir()):
        if path.suffix in (".hip", ".hpp", ".cpp"):
            for text in re.findall(r"\basm(?:\s+volatile)?\s*\((.*?)\);", path.read_text(), re.S):
                code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text[:text.index(":")]))
                yield path.name, code.replace("\\t", "").split("\\n"), text[text.index(":"):]


def test_accesses_wait_for_their_scalar_registers():
    """Five wait states between a vector instruction that writes a scalar register and an access to memory that reads it: within
    the statement, as the vector instruction may stand right in front of it."""
    accesses = 0
    for name, code, operands in statements():
        states = 0
        for instruction in code:
            if re.match(r"(buffer|global|flat|scratch)_", instruction):
                accesses += 1
                assert states >= 5 or '"s"' not in operands, (name, code)
            nop = re.match(r"s_nop (\d+)", instruction)
            states += int(nop[1]) + 1 if nop else 1
    assert accesses >= 3


def test_m0_is_written_by_the_compiler():
    """It may keep a value of its own there across a statement that does not say otherwise."""
    fetches = 0
    for name, code, operands in statements():
        for instruction in code:
            assert not re.match(r"s_\w+ m0\b", instruction), (name, code)
            if re.match(r"buffer_load.* lds$", instruction):
                fetches += 1
                assert '"{m0}"(' in operands, (name, code)
    assert fetches >= 3
