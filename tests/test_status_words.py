"""Status words of handles: each has one holder, is allocated with the others once a device, and goes to nobody else while work that
may write it could be in flight."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1805_07941_b200", "csrc")

PROGRAM = r"""
#include <set>
#include <thread>
#include <vector>
#include "status_words.cuh"

static int words[2][qc::StatusWords::kWords];
static int calls = 0;

int main() {
  qc::StatusWords pool;
  int wrong = 0;
  int* w = nullptr;
  // an allocation that fails is reported and tried again
  wrong += pool.take(0, &w, [](int**, size_t) { return 2; }) != 2 || w != nullptr;
  const auto from = [](int device) {
    return [device](int** base, size_t bytes) { ++calls; *base = words[device]; return bytes == sizeof(words[device]) ? 0 : 1; };
  };
  std::vector<int*> held;
  std::set<int*> all;
  for (int i = 0; i < qc::StatusWords::kWords; ++i) {
    wrong += pool.take(0, &w, from(0)) != 0 || !w || !all.insert(w).second;
    held.push_back(w);
  }
  wrong += pool.take(0, &w, from(0)) != 0 || w != nullptr;                       // none left
  wrong += pool.take(1, &w, from(1)) != 0 || w < words[1] || w >= words[1] + qc::StatusWords::kWords || calls != 2;
  // given back while something may be in flight: never handed out again; the next one is
  pool.give(0, held[7], false);
  wrong += pool.take(0, &w, from(0)) != 0 || w != nullptr;
  pool.give(0, held[9], true);
  wrong += pool.take(0, &w, from(0)) != 0 || w != held[9];
  for (int* h : held)
    if (h != held[7]) pool.give(0, h, true);
  std::set<int*> again;
  std::vector<std::thread> threads;
  std::mutex mu;
  for (int t = 0; t < 8; ++t)
    threads.emplace_back([&] {
      for (int i = 0; i < 100; ++i) {
        int* mine = nullptr;
        const int e = pool.take(0, &mine, from(0));
        std::lock_guard<std::mutex> lock(mu);
        wrong += e != 0 || !mine || mine == held[7] || !again.insert(mine).second;
      }
    });
  for (auto& t : threads) t.join();
  return wrong;
}
"""


def test_a_word_has_one_holder(tmp_path):
    source, binary = tmp_path / "words.cpp", tmp_path / "words"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-pthread", "-x", "c++", "-I", CSRC, "-o", str(binary), str(source)], check=True)
    assert subprocess.run([str(binary)], timeout=60).returncode == 0
