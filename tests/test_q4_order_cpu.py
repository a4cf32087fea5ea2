"""Order that the kernels of the 4-bit state need and that no result shows on one chip: read from their source."""
import re

from tests.test_dependent_launches_cpu import _code, _dependent_kernels


def _body(name, kernel):
    return {k: body for k, _, body in _dependent_kernels(_code(name))}[kernel]


def test_codes_pass_through_shared_memory_behind_a_barrier_of_the_warp():
    """A vote exchanges values and orders no memory."""
    body = _body("pack_q4.cu", "pack_q4_kernel")
    stores = [m.start() for m in re.finditer(r"\*reinterpret_cast<uint16_t\*>\(row \+", body)]
    loads = [m.start() for m in re.finditer(r"\*reinterpret_cast<const uint4\*>\(stage", body)]
    assert stores and loads and "unsigned char* row = stage[wid][t]" in body
    assert "__syncwarp();" in body[stores[-1]:loads[0]]


def _pos_stores(body, state):
    return [m.start() for m in re.finditer(re.escape(state) + r"pos\[[^;=]*\] = ", body)]


def test_positions_of_a_step_are_written_by_one_thread():
    """The incoming token's position and the release of a slot may meet in the same word (the incoming token goes at once)."""
    body = _body("decode_q4.cu", "decode_q4_kernel")
    last = body.index("else if (rank == 0) {")
    at = _pos_stores(body, "c.state.")
    assert at and all(x > last for x in at) and "if (write) {" in body[last:at[0]]


def test_positions_of_a_16_bit_step_are_written_by_one_thread():
    body = _body("decode_mma.cu", "decode_mma_kernel")
    last = body.rindex("if (rank == 0 && tid == 0) {")
    at = _pos_stores(body, "c.")
    assert at and all(x > last for x in at)
