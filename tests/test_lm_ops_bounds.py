"""CPU model of the bound that the alternatives of a row are listed by: few entries are not
below it, whatever the row's logits have in common."""

import numpy as np
import pytest

LISTED = {64: 512, 256: 2048, 512: 2048}   # candidates that a team's list holds


def bound_of_groups(groups, k, fine):
    """From the highest bit down; the lower half where too many groups reach the bound."""
    least, reach = 0, 256

    def take(bit, least, reach):
        t = least | 1 << bit
        n = int((groups >= t).sum())
        return (t, n) if n >= k else (least, reach)

    for bit in range(31, 15, -1):
        least, reach = take(bit, least, reach)
    if fine and reach > 2 * k:
        for bit in range(15, -1, -1):
            least, reach = take(bit, least, reach)
    return least


def order_of(x):
    u = (x.astype(np.float32) + 0).view(np.uint32)
    return np.where(u & 0x80000000, ~u, u | 0x80000000).astype(np.uint64)


def groups_of(order, nt):
    """Largest of each group: a wave's lanes have four, two or one lanes of a workgroup one."""
    V, ve = len(order), 4
    at = np.arange(V) // ve
    group = at % 64 * 4 + np.minimum(at // 64 * 4 // max(1, -(-V // (64 * ve))), 3) if nt == 64 else at % nt // (nt // 256)
    out = np.full(256, order_of(np.array([-np.inf]))[0], np.uint64)
    np.maximum.at(out, group, order)
    return out


@pytest.mark.parametrize("offset", [0.0, -40.0, 1000.0, -1000.0, 3000.0, 1.0e5])
@pytest.mark.parametrize("nt,V", [(64, 1000), (256, 4099), (512, 32003)])
def test_the_list_holds_rows_with_an_offset(nt, V, offset):
    for k in (1, 5, 20, 64):
        rng = np.random.default_rng(V + k)
        x = (rng.standard_normal(V) * 2.5 + offset).astype(np.float32)
        order = order_of(x)
        groups = groups_of(order, nt)
        least = bound_of_groups(groups, k, True)
        # The k largest are listed, and about 256 ln(256 / (256 - G)) entries where G groups
        # reach the bound; a float32 step at the offset may hold equal entries beside them.
        G = int((groups >= least).sum())
        n = int((order >= least).sum())
        ties = int(np.unique(x[np.argsort(-x)][:k + 1], return_counts=True)[1].max())
        assert n >= min(k, V) and G <= 2 * k + ties * 4
        assert n <= 256 * np.log(256 / (256 - min(G, 255))) * 1.5 + 20 + 4 * ties and n < LISTED[nt]
        assert (np.sort(order)[::-1][:k] >= least).all()


def test_sixteen_bits_alone_do_not_bound_them():
    """Why the lower bits are taken."""
    rng = np.random.default_rng(3)
    x = (rng.standard_normal(32003) * 2.5 + 3000).astype(np.float32)
    order = order_of(x)
    least = bound_of_groups(groups_of(order, 512), 64, False)
    assert (order >= least).sum() > LISTED[512]
