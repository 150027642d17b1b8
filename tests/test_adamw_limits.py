"""What gas_sq_norms, gas_adamw_steps and gas_adamw_unpack refuse for its size alone, before anything is launched: a launch has less than 2^32 threads, a
wavefront of them for every 256 elements, and one that asks for more runs on a part of them without an error."""
import array

from paper_2106_05609_amd import binding as B

AT, LIMIT = 4096, 4 * (0xFFFFFFFF // 256) * 256           # an address that nothing reads; elements


def said(status):
    return status, B.lib().gas_last_error().decode()


def adamw(sizes):
    n = len(sizes)
    q = lambda v: array.array("q", v).tobytes()
    room = B.gas_adamw_elements(sizes)
    return said(B._calls().gas_adamw_steps(n, q([AT] * n), array.array("i", [0] * n).tobytes(), q(sizes), q([AT] * n), AT, AT, 0, 0, room, 32, 0.1, 0.1, 0.1, 1e-8,
                                           0, 1, 0, 0, 1.0, 0))


def test_a_tensor_of_more_elements_than_a_launch_takes():
    for sizes in ([LIMIT + 1], [5, LIMIT + 1], [1 << 40]):
        status, why = adamw(sizes)
        assert status == -1 and f"tensor {len(sizes) - 1} is too large" in why, (sizes, status, why)


def test_the_norm_and_the_unpacking_of_too_many_elements():
    n = (0xFFFFFFFF // 256) * 32768 + 1
    sizes = array.array("q", [n]).tobytes()
    status, why = said(B._calls().gas_sq_norms(1, array.array("q", [AT]).tobytes(), sizes, AT, 0, AT, 1 << 60, 0))
    assert status == -1 and "too many elements" in why
    status, why = said(B._calls().gas_adamw_unpack(AT, AT, AT, (0xFFFFFFFF // 256) * 4096 + 256, 0, AT, AT, 0))
    assert status == -1 and "too many elements" in why
