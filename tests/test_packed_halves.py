"""The packed scan's tensor-core kernel with operands of two parts: the model of tests/test_packed_roles.py with the masked tile in two halves of 64
steps (both of their parts), each with a place of its own and products that start when it is there, two places for C H in turn, and three items' rows
of x; and the model of the launch that makes the sums of cut sequences: no outputs, no scores, a tile a block, rows of x given back by those who make
the parts of x'."""
import os
import random
import re

import pytest

from tests import test_packed_roles as roles


@pytest.fixture(autouse=True)
def rings(monkeypatch):
    monkeypatch.setattr(roles, "XS", 3)


def test_rings_are_the_kernels():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_19460_b200", "csrc", "ssd_packed_tc.cu")
    sizes = dict((m[0], int(m[1])) for m in re.findall(r"constexpr int (PT_\w+) = (\d+)", open(path).read()))
    assert (sizes["PT_SLOTS"], sizes["PT_VECS"], sizes["PT_PARTS"]) == (roles.SLOTS, roles.VECS, roles.PARTS)
    assert sizes["PT_XS"] == roles.XS


class Halves(roles.Model):
    def __init__(self, *a):
        super().__init__(*a)
        self.mfull, self.mempty, self.chdone, self.chfree = ([roles.Bar(1) for _ in range(2)] for _ in range(4))

    def products_y(self):
        yield from self.scores(0)
        for i in range(self.ni):
            c, j = divmod(i, self.nh)
            yield from self.wait(self.xready[i % roles.XS], i // roles.XS)
            if i:
                yield from self.wait(self.yfree, i - 1)
            for side in (0, 1):
                yield from self.wait(self.mfull[side], i)
                self.issue([("M%d" % side, i), ("X%d" % (i % roles.XS), i)], "Y", i if side else ("half", i))
                self.commit(self.mempty[side])
            self.commit(self.yfull)
            if j == self.nh - 1 and c + 1 < self.nb:
                yield from self.scores(c + 1)

    def mask(self):
        for i in range(self.ni):
            c, j = divmod(i, self.nh)
            yield from self.vectors(i)
            if j == 0:
                yield from self.wait(self.gfull, c)
            for side in (0, 1):
                if i:
                    yield from self.wait(self.mempty[side], i - 1)
                self.read("G", c)
                self.read("V%d" % (i % roles.VECS), i)
                yield
                self.read("G", c)
                self.write("M%d" % side, i)
                yield
                self.mfull[side].arrive()
            if j == self.nh - 1:
                self.gfree.arrive()
            self.vempty[i % roles.VECS].arrive()

    def products_s(self):
        for i in range(self.ni):
            c, j = divmod(i, self.nh)
            kb, kc = 2 * c, 2 * c + 1
            if j == 0:
                yield from self.wait_tile(kb)
            if i:
                yield from self.wait(self.sfree, i - 1)
            for k in range(4 * i, 4 * i + 4):
                yield from self.wait(self.xpfull[k % roles.PARTS], k // roles.PARTS)
                self.issue([("tile%d" % (kb % roles.SLOTS), kb), ("XP%d" % (k % roles.PARTS), k)], "S", i if k % 4 == 3 else ("part", k))
                self.commit(self.xpempty[k % roles.PARTS])
            self.commit(self.sdone)
            if j == self.nh - 1:
                self.commit(self.tempty[kb % roles.SLOTS])
            if j == 0:
                yield from self.wait_tile(kc)
            yield from self.wait(self.hfull, i)
            if i >= 2:
                yield from self.wait(self.chfree[i & 1], i // 2 - 1)
            self.issue([("tile%d" % (kc % roles.SLOTS), kc), ("H", i)], "CH%d" % (i & 1), i)
            self.commit(self.chdone[i & 1])
            if j == self.nh - 1:
                self.commit(self.tempty[kc % roles.SLOTS])

    def outputs(self):
        for i in range(self.ni):
            yield from self.vectors(i)
            self.vempty[i % roles.VECS].arrive()
            yield from self.wait(self.chdone[i & 1], i // 2)
            yield from self.wait(self.yfull, i)
            sums = ("Y", "CH%d" % (i & 1))
            for name in sums + ("X%d" % (i % roles.XS),):
                self.read(name, i)
            yield
            for name in sums:
                self.read(name, i)
            self.write("X%d" % (i % roles.XS), ("y", i))
            self.yfree.arrive()
            yield
            self.chfree[i & 1].arrive()
            if self.tail and i // self.nh == self.nb - 1:
                continue
            yield
            self.read("X%d" % (i % roles.XS), ("y", i))      # the copy to the rows of y
            self.xempty[i % roles.XS].arrive()

    def state(self):
        self.write("H", 0)
        yield
        self.hfull.arrive()
        for i in range(self.ni):
            yield from self.vectors(i)
            yield from self.wait(self.sdone, i)
            self.read("S", i)
            yield
            self.read("S", i)
            self.sfree.arrive()
            self.vempty[i % roles.VECS].arrive()
            if i + 1 < self.ni:
                yield from self.wait(self.chdone[i & 1], i // 2)
                self.write("H", i + 1)
                yield
                self.hfull.arrive()


class Sums(roles.Model):
    """All blocks are whole (a range that is not the last one)."""

    def __init__(self, *a):
        super().__init__(*a)
        assert not self.tail
        self.tempty = [roles.Bar(1) for _ in range(roles.SLOTS)]
        self.vempty = [roles.Bar(2) for _ in range(roles.VECS)]          # parts of x', states

    def nothing(self):
        return
        yield

    products_y = outputs = mask = nothing

    def products_s(self):
        for i in range(self.ni):
            c, j = divmod(i, self.nh)
            if j == 0:
                yield from self.wait_tile(c)
            if i:
                yield from self.wait(self.sfree, i - 1)
            for k in range(4 * i, 4 * i + 4):
                yield from self.wait(self.xpfull[k % roles.PARTS], k // roles.PARTS)
                self.issue([("tile%d" % (c % roles.SLOTS), c), ("XP%d" % (k % roles.PARTS), k)], "S", i if k % 4 == 3 else ("part", k))
                self.commit(self.xpempty[k % roles.PARTS])
            self.commit(self.sdone)
            if j == self.nh - 1:
                self.commit(self.tempty[c % roles.SLOTS])

    def loads(self):
        for c in range(self.nb):
            slot = c % roles.SLOTS
            if c >= roles.SLOTS:
                yield from self.wait(self.tempty[slot], c // roles.SLOTS - 1)
            self.flying.append(("tile%d" % slot, c, self.tfull[slot]))
            for i in range(c * self.nh, (c + 1) * self.nh):
                if i >= roles.XS:
                    yield from self.wait(self.xempty[i % roles.XS], i // roles.XS - 1)
                self.flying.append(("X%d" % (i % roles.XS), i, self.xfull[i % roles.XS]))

    def parts(self):
        for i in range(self.ni):
            yield from self.vectors(i)
            yield from self.wait(self.xfull[i % roles.XS], i // roles.XS)
            for k in range(4 * i, 4 * i + 4):
                self.read("X%d" % (i % roles.XS), i)
                if k >= roles.PARTS:
                    yield from self.wait(self.xpempty[k % roles.PARTS], k // roles.PARTS - 1)
                self.write("XP%d" % (k % roles.PARTS), k)
                yield
                self.xpfull[k % roles.PARTS].arrive()
            self.read("X%d" % (i % roles.XS), i)
            self.xempty[i % roles.XS].arrive()
            self.vempty[i % roles.VECS].arrive()

    def state(self):
        for i in range(self.ni):
            yield from self.vectors(i)
            yield from self.wait(self.sdone, i)
            self.read("S", i)
            yield
            self.read("S", i)
            self.sfree.arrive()
            self.vempty[i % roles.VECS].arrive()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("nb,nh", [(1, 1), (2, 1), (7, 1), (1, 2), (2, 2), (6, 2)])
def test_outputs(nb, nh, tail):
    for seed in range(40):
        Halves(nb, nh, tail, random.Random(seed)).run()


@pytest.mark.parametrize("nb,nh", [(1, 1), (2, 1), (7, 1), (13, 1), (1, 2), (2, 2), (9, 2)])
def test_sums(nb, nh):
    for seed in range(40):
        Sums(nb, nh, False, random.Random(seed)).run()
