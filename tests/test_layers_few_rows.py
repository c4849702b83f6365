"""The number of rows up to which the binding asks for no workspace first is the library's (no GPU needed)."""
import paper_2312_08053_amd as kimad
from paper_2312_08053_amd import binding


def test_few_rows():
    """Operands off 16-byte addresses are read as they lie by the kernel of few rows, and laid out anew in a workspace for every other."""
    need = kimad.lib().kimad_linear_workspace_bytes
    at = 0x10002
    assert need(at, 9, at, 9, binding.FEW_ROWS, 16, 9) == 0 < need(at, 9, at, 9, binding.FEW_ROWS + 1, 16, 9)
