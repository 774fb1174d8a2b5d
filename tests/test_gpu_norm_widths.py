"""The norm's backward pass gives the same bits for a row width whatever widths were asked for before it, and on any thread: the
order of the sums of dweight and dbias follows from the grid, which is that of the width itself."""
import threading

import pytest

pytestmark = pytest.mark.gpu

WIDTHS = {"registers": [2560, 1024, 1536, 2048], "pairs": [1802, 514, 1026], "singles": [1001, 201, 65], "ring": [5120, 3584, 4096]}


def _on_a_new_thread(f):
    got = []

    def run():
        try:
            got.append(f())
        except BaseException as e:       # (raised again where the test sees it)
            got.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    if isinstance(got[0], BaseException):
        raise got[0]
    return got[0]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("io,res", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("kind", list(WIDTHS))
def test_gradients_do_not_depend_on_the_calls_before(kind, io, res, bias):
    import torch
    from paper_2312_00752_b200 import binding as K
    widths = [w // 2 for w in WIDTHS[kind]] if io == "f32" and kind in ("registers", "ring") else WIDTHS[kind]
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    rows, g = 3000, torch.Generator(device="cuda").manual_seed(1)
    args = {}
    for D in widths:
        s = torch.randn(rows, D, generator=g, device="cuda").to(types[res])
        dy = torch.randn(rows, D, generator=g, device="cuda").to(types[io])
        args[D] = (s, torch.ones(D, device="cuda"), dy, torch.ones(rows, 2, device="cuda"))
    torch.cuda.synchronize()

    def run(D):
        out = K.ssm_norm_bwd(*args[D], has_bias=bias)
        torch.cuda.synchronize()
        return [out["dweight"]] + ([out["dbias"]] if bias else [])

    alone = {D: _on_a_new_thread(lambda: run(D)) for D in widths}
    for order in (widths, widths[::-1], widths[1:] + widths[:1]):
        together = _on_a_new_thread(lambda: {D: run(D) for D in order})
        for D in widths:
            assert all(torch.equal(p, q) for p, q in zip(alone[D], together[D])), (order, D)
