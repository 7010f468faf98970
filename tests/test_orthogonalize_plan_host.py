"""Which kernels take the products of orthogonalisation (host only; ortho_probe.cpp, linked to the library): a matrix of a side that is no multiple
of 128 or 256 takes nobody else's kernel away, and the matrices of the tests on the GPU reach every kernel there is."""
import subprocess

import pytest

from test_plan_host import _compile

DEFAULT = (3.4445, -4.7750, 2.0315)
STAGED = "234"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    exe = _compile("ortho_probe.cpp", str(tmp_path_factory.mktemp("ortho") / "probe"))

    def ask(matrices, steps=5, coefficients=DEFAULT):
        """[(rows, cols[, copies])] -> (thin, [kernels of matrix 0 round by round, ...])"""
        text = "%d %r %r %r %d\n" % (steps, *coefficients, len(matrices)) + "\n".join("%d %d %d" % (*m, *((1,) if len(m) == 2 else ())) for m in matrices)
        out = subprocess.run([exe], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout.split()
        return out[0] == "1", ["".join(r[i] for r in out[2:]) for i in range(len(matrices))]

    return ask


LARGE = [(2048, 8192), (8192, 2048)]
GPT2 = [(768, 2304), (768, 768), (768, 3072), (3072, 768)] * 5


@pytest.mark.parametrize("beside", [(2048, 60), (2048, 320), (300, 300), (1, 20000), (2048, 64), (2048, 576), (1000, 40)])
def test_products_of_large_matrices_keep_their_kernels(kernels, beside):
    alone = kernels(LARGE)[1]
    thin, found = kernels(LARGE + [beside])
    assert not thin and found[:2] == alone and alone[0].count("3") == 3 and set(alone[0]) <= set("34")


def test_blocks_of_256_stay_beside_a_side_of_128(kernels):
    """The 640 x 640 shares the rounds on blocks of 128 (undivided where it is not symmetric), not the three on blocks of 256."""
    alone, found = kernels(LARGE)[1], kernels(LARGE + [(640, 640)])[1]
    assert [k == "3" for k in found[0]] == [k == "3" for k in alone[0]] and set("".join(found[:2])) <= set(STAGED)


@pytest.mark.parametrize("beside", [(768, 10), (768, 320), (64, 4000)])
def test_many_matrices_keep_their_kernels(kernels, beside):
    alone = kernels(GPT2)[1]
    found = kernels(GPT2 + [beside])[1]
    assert found[:20] == alone and all(set(k) <= set("." + STAGED) for k in alone)


def test_few_products_share_a_launch(kernels):
    """Where blocks of 128 would not pay for a launch of their own: straight from the caches with the odd one."""
    found = kernels([(1024, 1024)] * 4 + [(1024, 320)])[1]
    assert found[0][0] in "01" and found[4][0] == found[0][0]


def test_matrices_of_one_kind_share_every_round(kernels):
    for matrices in ([(768, 768, 12)], [(1024, 1024)] * 4, GPT2, LARGE, [(2305, 1002)], [(100, 260), (260, 100)], [(640, 640)] * 9):
        for r in zip(*kernels(matrices)[1]):
            assert len(set(r) - {"."}) == 1, (matrices, r)


def test_thin_matrices(kernels):
    assert kernels([(48, 900), (900, 48), (1, 5000)]) == (True, ["", "", ""])
    assert not kernels([(48, 900), (900, 65)])[0] and not kernels([(20, 16500)])[0] and not kernels([(64, 2048, 65)])[0]


# of tests on the GPU: the kernels that they are there for
@pytest.mark.parametrize("matrices,steps,has", [
    ([(2048, 3300)], 5, "4"), ([(1024, 1600, 8)], 5, "4"), ([(768, 768, 12)], 5, "2"), ([(130, 513)], 5, "0"), ([(1200, 2000, 5)], 5, "2"),
    ([(2048, 8192, 1)], 5, "34"), ([(8192, 2048, 1)], 5, "34"), ([(2000, 8190, 1)], 5, "34"), ([(2048, 2048, 7)], 5, "3"), ([(5376, 5400, 1)], 5, "3"),
    (LARGE, 5, "34"), ([(2304, 2304)], 5, "2"), ([(2048, 2048)] * 7, 5, "3")])
def test_kernels_that_tests_reach(kernels, matrices, steps, has):
    found = kernels(matrices, steps)[1]
    assert set(has) <= set("".join(found)), found


def test_two_steps_at_a_time_through_the_gram_matrix(kernels):
    """Seven products two steps, three the last of an odd number"""
    for rows, cols in ((520, 1000), (1900, 600), (1024, 1600)):
        for steps in (1, 2, 3, 4, 6, 7):
            assert len(kernels([(rows, cols)], steps)[1][0]) == steps // 2 * 7 + steps % 2 * 3
    assert len(kernels([(700, 1000)], 4)[1][0]) == 12
