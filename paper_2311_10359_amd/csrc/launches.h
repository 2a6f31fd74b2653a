// What the library's translation units share on the host.
#pragma once

namespace fikit {

// Counts a launch of this thread: how a waiting call waits goes by their number since the last wait.
void count_launch();

}  // namespace fikit
