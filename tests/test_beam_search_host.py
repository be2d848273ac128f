"""Without a GPU: what a BeamSearch that cannot be made leaves behind.  torch's streams are replaced by names, the library's calls recorded."""
import pytest
import torch

from paper_2506_10470_amd.engine import BeamSearch


class Library:
    """Objects by number, those that there are in `alive`; the creations named in `failing` raise."""
    MAX_TOP = MAX_BEAMS = 32

    def __init__(self, *failing):
        self.failing, self.alive, self.made = failing, set(), 0

    def PagesConfig(self, *a):
        return a

    BeamsConfig = PagesConfig

    def _create(self, name):
        if name in self.failing:
            raise RuntimeError(name)
        self.made += 1
        self.alive.add((name, self.made))
        return self.made

    def tdp_pages_create(self, cfg):
        return self._create("pages")

    def tdp_beams_create(self, cfg):
        return self._create("beams")

    def tdp_pages_destroy(self, h):
        self.alive.remove(("pages", h))

    def tdp_beams_destroy(self, h):
        self.alive.remove(("beams", h))


class Stream:
    pass


@pytest.fixture(autouse=True)
def streams(monkeypatch):
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", Stream)


def search(library):
    return BeamSearch(library, 1, 2, 64, 100, 16, 4, 4, 40, 2)


@pytest.mark.parametrize("failing", ["pages", "beams"])
def test_a_search_that_cannot_be_made_keeps_nothing(failing):
    library = Library(failing)
    with pytest.raises(RuntimeError, match=failing):
        search(library)
    assert not library.alive


def test_a_search_gives_back_what_it_has():
    library = Library()
    with search(library) as s:
        assert len(library.alive) == 2
    assert not library.alive
    s.close()
