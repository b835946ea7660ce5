// Whose turn it is to enqueue kernels that use a stream's workspace.
#pragma once
#include <condition_variable>
#include <mutex>

namespace lqq {

// Calls on one stream can share a workspace, and they may come from several host threads.  Where a call enqueues two kernels and the
// second reads what the first has left in the workspace (the chunks of a large decode batch, the partial sums of K slices), no other
// call that writes there may get in between.  So every call that uses a workspace holds its stream's turn while it enqueues; calls on
// other streams do not wait.  The turns that are held are a list through their holders' own frames: nothing is allocated.
class WorkspaceTurn {
public:
    WorkspaceTurn(const void *workspace, const void *stream) : used(workspace != nullptr), stream(stream)
    {
        if (!used) return;
        Turns &t = turns();
        std::unique_lock<std::mutex> lock(t.mutex);
        while (t.held(stream)) {
            ++t.waiting;
            t.given_back.wait(lock);
            --t.waiting;
        }
        next = t.first;
        t.first = this;
    }
    ~WorkspaceTurn()
    {
        if (!used) return;
        Turns &t = turns();
        std::lock_guard<std::mutex> lock(t.mutex);
        WorkspaceTurn **at = &t.first;
        while (*at != this) at = &(*at)->next;
        *at = next;
        if (t.waiting) t.given_back.notify_all();
    }
    WorkspaceTurn(const WorkspaceTurn &) = delete;
    WorkspaceTurn &operator=(const WorkspaceTurn &) = delete;

private:
    struct Turns {
        std::mutex mutex;
        std::condition_variable given_back;
        WorkspaceTurn *first = nullptr;
        int waiting = 0;
        bool held(const void *stream) const
        {
            for (const WorkspaceTurn *h = first; h; h = h->next)
                if (h->stream == stream) return true;
            return false;
        }
    };
    static Turns &turns()
    {
        static Turns t;
        return t;
    }
    const bool used;
    const void *const stream;
    WorkspaceTurn *next = nullptr;
};

}  // namespace lqq
