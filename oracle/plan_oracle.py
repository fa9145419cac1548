"""A step's page bookkeeping from its definition, in plain Python lists.  Shares no code with the GPU path."""


class Refused(Exception):
    pass


def plan(state, new, keep, max_rows, page):
    """state: dict of kv_len, seen, borrowed (lists), table (list of rows), free (list, its end the top).  Changes it and returns (cu_q, slots,
    pos) with max_rows entries, or raises Refused and changes nothing."""
    n = len(new)
    pages = lambda x: -(-x // page)
    back, todo = [], []
    for b in range(n):
        old, lent = state["kv_len"][b], state["borrowed"][b]
        k = old if keep is None else min(keep[b], old)
        to = k + new[b]
        if min(old, new[b], k, lent) < 0 or lent * page > old or to > page * len(state["table"][b]) or old > page * len(state["table"][b]):
            raise Refused(1)
        own = list(range(lent, pages(old)))                  # entries that hold pages of its own
        if k < lent * page:
            if k % page:
                raise Refused(1)
            stay, lent = [], k // page
        else:
            stay = [e for e in own if e < pages(to)]
        back += [(b, e) for e in own if e not in stay]
        have = lent + len(stay)
        todo.append((k, to, lent, list(range(have, pages(to)))))
    if sum(new) > max_rows:
        raise Refused(2)
    free = state["free"] + [state["table"][b][e] for b, e in reversed(back)]
    if len(free) > state["n_pages"]:
        raise Refused(3)
    if sum(len(t[3]) for t in todo) > len(free):
        raise Refused(4)
    cu, slots, pos = [0], [], []
    for b, (k, to, lent, take) in enumerate(todo):
        for e in take:
            state["table"][b][e] = free.pop()
        state["seen"][b] = (state["seen"][b] - (state["kv_len"][b] - k) if k else 0) + new[b]
        state["kv_len"][b], state["borrowed"][b] = to, lent
        cu.append(cu[-1] + new[b])
        for i in range(new[b]):
            slots.append(state["table"][b][(k + i) // page] * page + (k + i) % page)
            pos.append(state["seen"][b] - new[b] + i)
    state["free"] = free
    return cu, slots + [-1] * (max_rows - len(slots)), pos + [0] * (max_rows - len(pos))
