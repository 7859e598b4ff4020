"""Two threads, two caches, two streams: calls whose kernels need different amounts of shared memory do not disturb one another."""
import threading

import pytest
import torch

from paper_2609_35750_b200 import binding as B

pytestmark = pytest.mark.gpu


def together(*works):
    """Runs the functions in threads of their own, each on a stream of its own; the first error is raised here."""
    errors, start = [], threading.Barrier(len(works))

    def one(work):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(60)
                work()
                torch.cuda.current_stream().synchronize()
        except BaseException as e:  # noqa: BLE001
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=one, args=(w,)) for w in works]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if errors:
        raise errors[0]


def test_evictions_of_caches_of_different_sizes():
    def cache(pages, n, leave):
        g = torch.Generator(device="cuda").manual_seed(pages)
        table = torch.randperm(pages, generator=g, device="cuda").int().view(1, -1)
        weight = torch.rand((1, pages), generator=g, device="cuda")
        weight[:, n:] = 0
        free = torch.zeros(4 + pages, dtype=torch.int32, device="cuda")
        free[0] = pages - n
        lens = torch.tensor([n], dtype=torch.int32, device="cuda")
        kept = [x.clone() for x in (table, lens, free, weight)]

        def once():
            now = [x.clone() for x in kept]
            evicted, count = B.kvs_cache_evict_lowest(n - leave, 4, 16, 1, *now[:3], now[3])
            return (*now, evicted, count)

        want = once()
        assert int(want[-1]) == leave and int(want[2][1]) == B.KVS_OK

        def work():
            got = [once() for _ in range(150)]
            for one in got:
                assert all(torch.equal(x, y) for x, y in zip(one, want))
        return work

    together(cache(32768, 30000, 300), cache(130000, 120000, 1000))


def test_verifications_of_vocabularies_of_different_sizes():
    def vocabulary(V):
        g = torch.Generator(device="cuda").manual_seed(V)
        p = torch.rand((1, 1, V), generator=g, device="cuda")
        none = torch.zeros((1, 0), device="cuda")
        u = torch.rand(1, generator=g, device="cuda")
        once = lambda: B.kvs_verify_drafts(p, none.view(1, 0, 1).expand(1, 0, V).contiguous(), none.int(), none, u)  # noqa: E731
        want = once()

        def work():
            got = [once() for _ in range(200)]
            for one in got:
                assert all(torch.equal(x, y) for x, y in zip(one, want))
        return work

    together(vocabulary(11_000_000), vocabulary(1 << 24))


def test_evictions_by_ranges_of_tables_of_different_sizes():
    def cache(pages, calls=6000):
        one = B.PagedCache.__new__(B.PagedCache)
        free = torch.zeros(4 + pages, dtype=torch.int32, device="cuda")
        one.__dict__.update(num_pages=pages, page_size=1, num_seqs=1, max_pages=pages, token_weight=None, free_list=free,
                            block_table=torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1),
                            n_tokens=torch.tensor([pages], dtype=torch.int32, device="cuda"))
        ranges = torch.tensor([[0, 100, 1]], dtype=torch.int32, device="cuda")

        def work():
            stream = torch.cuda.current_stream()
            for _ in range(calls):                                # page after page leaves from slot 100
                one.evict(ranges, stream=stream)
            assert int(one.n_tokens) == pages - calls and free[:2].tolist() == [calls, B.KVS_OK]
            assert torch.equal(free[4:4 + calls].cpu(), torch.arange(100, 100 + calls, dtype=torch.int32))
        return work

    together(cache(13000), cache(51200))
