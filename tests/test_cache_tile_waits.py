"""Order of events in a CTA of the cache's tensor-memory kernel (hifa4_cache_attention.cu): behind the barrier of the whole CTA, O is
read from tensor memory, the K and V tiles are written over and the memory goes to another CTA, so every product has to be complete
and every arrival of a commit there.  The kernel's waits and arrivals, restated as a graph (an edge: happens before).  A product is
issued by a thread and complete some time later; a commit arrives when the products that its thread issued before are complete."""
import pytest

K_STAGES, RAW_STAGES = 3, 3


def events(n, tiles, alt, end="all"):
    """n pages of a CTA with two tiles, one thread of issue per tile.  tiles: those that have rows; alt: both take the same rows, tile h the
    pages h, h + 2, ..  end: what the issuers wait for before the barrier ("all", or only the stages of the last page)."""
    before, last, issued = {}, {}, {0: [], 1: []}

    def add(ev, after=(), thread=None):
        deps = list(after)
        if thread is not None:
            if thread in last:
                deps.append(last[thread])
            last[thread] = ev
        before.setdefault(ev, []).extend(deps)

    def product(ev, h, after=()):
        add(("issue",) + ev, after, ("issuer", h))
        add(("done",) + ev, [("issue",) + ev])
        issued[h].append(("done",) + ev)

    def commit(bar, h):
        add(bar, [last[("issuer", h)]] + issued[h])

    free_k = lambda j: [("KE", j, h) for h in (0, 1)] if j >= 0 else []      # both issuers arrive for every page
    free_v = lambda j: [("VE", j, h) for h in (0, 1)] if j >= 0 else []
    for j in range(n):
        add(("load", j), [("v tile", j - RAW_STAGES)] if j >= RAW_STAGES else [], "loader")
        add(("k tile", j), [("load", j)] + free_k(j - K_STAGES), "dequantize")
        add(("v tile", j), [("load", j)] + free_v(j - K_STAGES), "dequantize")
    own = [list(range(h, n, 2)) if alt else list(range(n)) if h < tiles else [] for h in (0, 1)]
    for h in (0, 1):
        for x in range(len(own[h])):
            add(("scores read", h, x), [("SF", h, x)], ("softmax", h))
            add(("P", h, x), [("OD", h, x - 1)] if x else [], ("softmax", h))
        behind = 2 if alt else 1
        for j in range(n + behind):
            if j < n:
                mine = j in own[h]
                x = own[h].index(j) if mine else None
                add(("k seen", j, h), [("k tile", j)] + ([("scores read", h, x - 1)] if x else []), ("issuer", h))
                if mine:
                    product(("S", h, x), h)
                    commit(("SF", h, x), h)
                    commit(("KE", j, h), h)
                else:
                    add(("KE", j, h), [last[("issuer", h)]])
            if j >= behind:
                i = j - behind
                mine = i in own[h]
                x = own[h].index(i) if mine else None
                add(("v seen", i, h), [("v tile", i)] + ([("P", h, x)] if mine else []), ("issuer", h))
                if mine:
                    product(("O", h, x), h)
                    commit(("OD", h, x), h)
                    commit(("VE", i, h), h)
                else:
                    add(("VE", i, h), [last[("issuer", h)]])
        waits = [e for i in range(max(n - K_STAGES, 0) if end == "all" else n - 1, n) for e in free_k(i) + free_v(i)]
        if end == "all" and own[h]:
            waits.append(("OD", h, len(own[h]) - 1))
        add(("end", h), waits, ("issuer", h))
    add("barrier", list(last.values()))
    return before


def missing(n, tiles, alt, **kw):
    """Products and arrivals that are not ordered before the barrier."""
    before = events(n, tiles, alt, **kw)
    seen, todo = set(), ["barrier"]
    while todo:
        for d in before[todo.pop()]:
            if d not in seen:
                seen.add(d)
                todo.append(d)
    return [e for e in before if e[0] in ("done", "SF", "KE", "OD", "VE") and e not in seen]


@pytest.mark.parametrize("tiles,alt", [(2, False), (1, True)])
def test_every_product_is_complete_before_the_barrier(tiles, alt):
    for n in range(1, 40):
        assert not missing(n, tiles, alt), n


def test_the_last_page_alone_leaves_a_product_out():
    """With both tiles on the same rows the last page is one tile's: the other tile's last product is that of the page before."""
    for n in range(2, 40):
        late = missing(n, 1, True, end="last page")
        h = n % 2                                                            # the tile that has not the last page
        assert ("done", "O", h, (n + 1 - h) // 2 - 1) in late
        assert not [e for e in missing(n, 2, False, end="last page") if e[0] == "done"]
